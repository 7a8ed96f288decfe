"""The 64-bit references of tests/delta_reference.py against differences, and the forward one
against the oracle's prefill state (CPU)."""
import numpy as np

from oracle import oracle as orc
from tests import delta_reference as ref


def _case(lengths, HK, HV, dk, dv, seed):
    r = np.random.default_rng(seed)
    n = sum(lengths)
    q, k = r.normal(size=(n, HK, dk)), r.normal(size=(n, HK, dk))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    return (q, k, r.normal(size=(n, HV, dv)), -np.log1p(np.exp(r.normal(size=(n, HV)) - 1)),
            1 / (1 + np.exp(-r.normal(size=(n, HV))))), r


def test_gradient_matches_differences():
    """Central differences of sum(c o) + sum(d S_T): with a step of 1e-5 the formula is met
    to the differences' own error, a few 1e-10 of the third derivatives plus 1e-16 / 1e-5."""
    lengths = [4, 0, 3]
    x, r = _case(lengths, 2, 4, 5, 3, 0)
    s0, scale = r.normal(size=(3, 4, 3, 5)), 0.7
    do, ds = r.normal(size=(7, 4, 3)), r.normal(size=(3, 4, 3, 5))

    def loss(args, s):
        o, last, _ = ref.forward(lengths, *args, scale, s)
        return (do * o).sum() + (ds * last).sum()

    g = ref.backward(lengths, *x, scale, s0, do, ds)
    for i in range(6):
        for _ in range(12):
            args = [a.copy() for a in (*x, s0)]
            at = tuple(r.integers(0, m) for m in args[i].shape)
            h = 1e-5
            args[i][at] += h
            up = loss(args[:5], args[5])
            args[i][at] -= 2 * h
            down = loss(args[:5], args[5])
            assert abs((up - down) / (2 * h) - g[i][at]) < 1e-7


def test_norm_gradient_matches_differences():
    r = np.random.default_rng(1)
    x, w, dz = r.normal(size=(3, 2, 8)), r.normal(size=8), r.normal(size=(3, 2, 8))
    a = r.normal(size=(3, 2))
    cs = np.concatenate([np.cos(a), np.sin(a)], 1)
    for rms in (False, True):
        for pairs in (False, True):
            dx, dw = ref.norm_backward(x, w, dz, rms, 1e-3, 4, cs, pairs)
            for arr, grad in ((x, dx), (w, dw)):
                for _ in range(10):
                    at, h = tuple(r.integers(0, m) for m in arr.shape), 1e-5
                    keep = arr[at]
                    arr[at] = keep + h
                    up = (dz * ref.norm(x, w, rms, 1e-3, 4, cs, pairs)).sum()
                    arr[at] = keep - h
                    down = (dz * ref.norm(x, w, rms, 1e-3, 4, cs, pairs)).sum()
                    arr[at] = keep
                    assert abs((up - down) / (2 * h) - grad[at]) < 1e-7


def test_states_match_the_oracle():
    x, _ = _case([20], 2, 4, 8, 8, 2)
    q, k, v, la, beta = x
    _, last, _ = ref.forward([20], *x, 1.0)
    S = orc.prefill(k, v, np.exp(la), beta)
    assert np.max(np.abs(S - last[0])) < 1e-12
