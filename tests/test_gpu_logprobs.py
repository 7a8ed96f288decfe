"""Log probabilities of given tokens and of the best ones, entropy, and their gradient, through the
C ABI, against 64-bit references.

Bars.  The sum of exponentials: chains of 32 elements per chunk, 16 chunks, a wave's tree and the
workgroup's waves or parts, 64 more (120 roundings at most, 7e-6), each exponential |d| e^d 2^-23
(4e-8): its logarithm is off by 7.5e-6, logp and lse by that and 2^-23 of their size.
entropy: the quotient's sums by the same share of the terms, 1.5e-5 (1 + entropy + ln s).
Gradient: p by |z| + |lse| and the exponential's argument, 2^-23 each (|z| < 40 here: 1e-5), of
every term, and the sum over 256 given tokens 2e-5.  bf16: 2^-8 of the value on top.  Tokens are
exact."""
import numpy as np
import pytest

from paper_2609_12399_amd import onela as ab
from paper_2609_12399_amd import runner
from tests import model_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def same_or_near(got, want, bar):
    got = f64(got)
    assert got.shape == want.shape
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    off = np.abs(got[fine] - want[fine]) - np.broadcast_to(bar, want.shape)[fine]
    assert (off <= 0).all(), float(off.max())


def check(x, given, K, scale, io, entropy=True, pad=0, rows=None):
    """Forward against the reference; x fp64 numpy of values that io holds (as many rows as
    wanted, again and again)."""
    R, V = rows or len(x), x.shape[1]
    some, x = len(x), np.resize(x, (R, V))
    given = None if given is None else np.resize(given, (R, given.shape[1]))
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    wide = torch.full((R, V + pad), 50.0, dtype=dt)
    wide[:, :V] = torch.from_numpy(x).to(dt)
    logits = wide.to(DEV)[:, :V]
    G = 0 if given is None else given.shape[1]
    tok = None if given is None else torch.from_numpy(given).to(torch.int32).to(DEV)
    op = runner.TokenLogprobs(R, V, G, K, io, scale, entropy, device=DEV)
    logp, lse, ent, top, top_logp = op.forward(logits, tok)
    want = ref.logprobs(f64(logits[:some]), None if given is None else given[:some], K, scale)
    want = [w if w is None else np.resize(w, (R, *w.shape[1:])) for w in want]
    finite = np.where(np.isfinite(want[1]), want[1], 0)
    if G:
        same_or_near(logp, want[0], 7.5e-6 + 2.0 ** -23 * np.abs(want[0]))
    same_or_near(lse, want[1], 7.5e-6 + 2.0 ** -22 * np.abs(finite))
    if entropy:
        same_or_near(ent, want[2], 1.5e-5 * (2 + 2 * np.abs(np.nan_to_num(want[2]))
                                             + np.log(V)))
    if K:
        assert np.array_equal(top.cpu().numpy(), want[3])
        same_or_near(top_logp, want[4], 7.5e-6 + 2.0 ** -23 * np.abs(want[4]))
    return logits, tok, op


def draw(R, V, seed=0, size=3.0):
    return size * np.random.default_rng(seed + V).normal(size=(R, V))


def tokens(R, V, G, seed=0):
    """Some given twice, some padding, some past the vocabulary."""
    r = np.random.default_rng(seed + V + G)
    t = r.integers(0, V, (R, G))
    t[r.random((R, G)) < 0.1] = -1
    if G > 3:
        t[:, 1] = t[:, 0]
    return t


SIZES = [(1, 1, 1, 1), (3, 2, 2, 2), (5, 7, 1, 7), (4, 64, 4, 64), (9, 100, 0, 20), (2, 513, 5, 64),
         (3, 2047, 1, 5), (3, 2048, 1, 64), (3, 2049, 64, 64), (2, 4097, 1, 1), (7, 8192, 0, 0),
         (2, 8193, 1, 33), (3, 20001, 256, 20), (1, 70000, 1, 64), (2, 131072, 3, 8)]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("R,V,G,K", SIZES)
def test_sizes(R, V, G, K, io):
    check(draw(R, V), tokens(R, V, G) if G else None, K, 0.8, io, entropy=V % 2 == 0, pad=V % 5)


def test_many_rows():
    """More rows than any cut into parts."""
    check(draw(700, 300), tokens(700, 300, 2), 10, 1.0, "bf16")
    check(draw(530, 9000), tokens(530, 9000, 1), 3, 1.0, "f32")


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 1000, 9000, 30000])
def test_masks(io, V):
    """-inf and the type's lowest value as masks; rows that they leave nothing, one, fewer than K;
    NaN and +inf; signed zeros."""
    x = draw(12, V)
    r = np.random.default_rng(1)
    low = float(torch.finfo(torch.bfloat16).min)
    x[0] = -np.inf
    x[1], x[1, V // 2] = -np.inf, 3.0
    x[2, r.random(V) < 0.9] = -np.inf
    x[3, r.random(V) < 0.9] = low
    x[4] = low
    x[5], x[5, [3, V - 1]] = -np.inf, [-2.0, 4.0]
    x[6, 5] = np.nan
    x[7], x[7, [1, V - 2]] = np.nan, [-np.inf, 0.5]
    x[8, 9] = np.inf
    x[9] = np.nan
    x[10] = np.where(r.random(V) < 0.5, -0.0, 0.0)
    x[11], x[11, V - 3:] = -np.inf, np.nan
    given = np.tile(np.array([[0, V // 2, V, -1, V - 1]]), (12, 1))
    for K in (1, 6, 33):
        check(x, given, K, 1.0, io)
    check(x, given, 20, 0.5, io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_equal_logits(io):
    """All equal, two values, rising, falling, the best ones side by side: ties go to the lower
    token whatever part, chunk or lane they are in."""
    for V in (300, 2048, 9000, 50000):
        r = np.random.default_rng(V)
        x = np.zeros((8, V))
        x[1] = (r.random(V) < 0.5) * 1.0
        x[2] = np.arange(V) // 256 * 2.0 ** -4
        x[3] = -(np.arange(V) // 256) * 2.0 ** -4
        x[4, V // 3:V // 3 + 100] = 1.0
        x[5] = r.integers(0, 3, V)
        x[6, ::64] = 2.0
        x[7, -70:] = 5.0
        for K in (1, 17, 64):
            check(x, None, K, 1.0, io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("R,V,K", [
    (40, 512, 64), (40, 513, 48), (40, 600, 49), (40, 1024, 20), (40, 1025, 48), (40, 2048, 48),
    (40, 2048, 49), (40, 2049, 0), (40, 3001, 1), (40, 4095, 64), (40, 4096, 20), (40, 4097, 64),
    (2047, 4097, 32), (2048, 4097, 32), (2048, 4097, 33), (2048, 4097, 0), (2050, 9000, 1),
    (2048, 16384, 20), (2048, 16385, 20)])
def test_rows_at_the_bounds_of_the_choices(R, V, K, io):
    some = min(R, 40)
    check(draw(some, V), tokens(some, V, 2), K, 1.0, io, pad=V % 3, rows=R)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("R,V,K", [(24, 900, 20), (24, 1500, 64), (24, 3000, 20), (24, 4096, 64),
                                   (2048, 5000, 1), (2048, 5000, 32), (2048, 13000, 20)])
def test_hard_rows(R, V, K, io):
    """Rows of equal values, ties, rising and falling ones, masks, NaN and +inf, side by side."""
    r = np.random.default_rng(V)
    x = np.zeros((12, V))
    x[1] = (r.random(V) < 0.5) * 1.0
    x[2] = np.arange(V) // 64 * 2.0 ** -4
    x[3] = -(np.arange(V) // 64) * 2.0 ** -4
    x[4, V // 3:V // 3 + 100] = 1.0
    x[5] = r.integers(0, 3, V)
    x[6] = -np.inf
    x[7], x[7, [V // 2, V - 1]] = -np.inf, 3.0
    x[8, r.random(V) < 0.9] = -np.inf
    x[9, 5] = np.nan
    x[10], x[10, V - 2] = draw(1, V)[0], np.inf
    x[11], x[11, V - 3:] = -np.inf, np.nan
    check(x, tokens(12, V, 1), K, 1.0, io, rows=R)


def test_large_logits():
    """Logits far from 0: log probabilities come from differences."""
    x = draw(4, 5000).astype(np.float32).astype(np.float64)
    x = (x + 4096.0).astype(np.float32).astype(np.float64)
    x[1] = 1e30 * np.sign(x[1] - 4096.0)
    check(x, tokens(4, 5000, 3), 5, 1.0, "f32")


def grad_check(x, given, scale, io, lse_only=False, ent=False, pad=0, seed=0):
    R, V = x.shape
    r = np.random.default_rng(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    wide = torch.zeros((R, V + pad), dtype=dt)
    wide[:, :V] = torch.from_numpy(x).to(dt)
    logits = wide.to(DEV)[:, :V]
    x = f64(logits)
    G = 0 if given is None else given.shape[1]

    def vector(*shape):
        return r.normal(size=shape).astype(np.float32)

    dlogp = vector(R, G) if G else None
    dlse = vector(R) if lse_only or not G or ent else None
    dent = vector(R) if ent else None
    _, lse, entropy, _, _ = ref.logprobs(x, None, 0, scale)
    dev = [None if t is None else torch.from_numpy(np.asarray(t, np.float32)).to(DEV)
           for t in (lse, dlogp, dlse, entropy, dent)]
    tok = None if given is None else torch.from_numpy(given).to(torch.int32).to(DEV)
    op = runner.TokenLogprobs(R, V, G, 0, io, scale, backward=True, device=DEV)
    got = op.backward(logits, tok, *dev)
    want, size = ref.logprobs_backward(x, given, dlogp, dlse, dent, scale)
    same_or_near(got, want, 2e-5 * size + (2.0 ** -8 * np.abs(want) if io == "bf16" else 0) + 1e-37)
    return op, logits, tok, dev, got


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("R,V,G,ent", [(1, 1, 1, False), (3, 2, 2, True), (5, 7, 0, False),
                                       (2, 513, 5, True), (4, 4096, 1, False), (3, 4097, 1, True),
                                       (2, 9001, 256, True), (600, 100, 1, False),
                                       (1, 70001, 64, False)])
def test_gradient(R, V, G, ent, io):
    grad_check(draw(R, V), tokens(R, V, G) if G else None, 0.8, io, ent=ent, pad=V % 3)


def test_gradient_of_masked_rows():
    x = draw(6, 3000)
    r = np.random.default_rng(4)
    x[0] = -np.inf
    x[1, r.random(3000) < 0.9] = -np.inf
    x[2], x[2, 77] = -np.inf, 1.0
    x[3, 5:] = -3e38
    given = np.tile(np.array([[1, 77, -1]]), (6, 1))
    given[5, 0] = 3000  # past the vocabulary: the row is NaN
    for io in ("bf16", "f32"):
        for ent in (False, True):
            grad_check(x, given, 1.0, io, ent=ent)


def test_gradient_in_place():
    op, logits, tok, dev, got = grad_check(draw(9, 5001), tokens(9, 5001, 4), 1.0, "bf16", ent=True)
    want, dense = got.clone(), logits.contiguous().clone()
    assert op.backward(dense, tok, *dev, out=dense) is dense
    assert torch.equal(dense, want)


def test_gradient_against_differences():
    """Differences of the kernel's own outputs (fp32, step 2^-6)."""
    R, V, G, h = 5, 200, 3, 2.0 ** -6
    g = torch.Generator().manual_seed(3)
    x, d = (torch.randn((R, V), generator=g).to(DEV) for _ in range(2))
    tok = torch.randint(0, V, (R, G), generator=g).to(torch.int32).to(DEV)
    dl, ds, dh = (torch.randn(s, generator=g).to(DEV) for s in ((R, G), (R,), (R,)))
    op = runner.TokenLogprobs(R, V, G, 0, "f32", entropy=True, device=DEV)
    _, lse, ent, _, _ = (None if t is None else t.clone() for t in op.forward(x, tok))
    grad = runner.TokenLogprobs(R, V, G, 0, "f32", backward=True, device=DEV).backward(
        x, tok, lse, dl, ds, ent, dh)
    vals = []
    for s in (h, -h):
        logp, l, e, _, _ = op.forward(x + s * d, tok)
        vals.append(float((logp.double() * dl).sum() + (l.double() * ds).sum() +
                          (e.double() * dh).sum()))
    assert abs((vals[0] - vals[1]) / (2 * h) - float((grad.double() * d).sum())) <= \
        2e-3 * float(grad.norm()) * float(d.norm())


def test_outputs_that_are_not_wanted_and_no_rows():
    x = torch.randn((3, 50), device=DEV)
    cfg = ab.make_logprob_config(3, 50, 0, 0, "f32")
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    ab.onela_token_logprobs(cfg, x, None, None, None, None, None, None, ws, 256)
    cfg = ab.make_logprob_config(0, 50, 2, 3, "f32")
    ab.onela_token_logprobs(cfg, None, None, None, None, None, None, None, ws, 256)
    ab.onela_token_logprobs_backward(cfg, None, None, None, None, None, None, None, None)
    torch.cuda.synchronize()


def test_more_than_32_bits_of_offset():
    R, V = 66000, 32768  # 2.16e9 elements, 4.3 GB
    x = torch.zeros((R, V), dtype=torch.bfloat16, device=DEV)
    x[-3:] = (3 * torch.randn((3, V), device=DEV)).bfloat16()
    tok = torch.full((R, 1), 7, dtype=torch.int32, device=DEV)
    op = runner.TokenLogprobs(R, V, 1, 4, "bf16", entropy=True, device=DEV)
    out = [t.clone() for t in op.forward(x, tok)]
    want = ref.logprobs(f64(x[-3:]), np.full((3, 1), 7), 4, 1.0)
    same_or_near(out[0][-3:], want[0], 7.5e-6 + 2.0 ** -23 * np.abs(want[0]))
    assert np.array_equal(out[3][-3:].cpu().numpy(), want[3])
    assert bool((out[3][:-3] == torch.arange(4, device=DEV)).all())
    d = torch.ones((R, 1), device=DEV)
    got = runner.TokenLogprobs(R, V, 1, 0, "bf16", backward=True, device=DEV).backward(
        x, tok, out[1], d)
    want, size = ref.logprobs_backward(f64(x[-3:]), np.full((3, 1), 7), np.ones((3, 1)), None, None,
                                       1.0)
    same_or_near(got[-3:], want, 2e-5 * size + 2.0 ** -8 * np.abs(want))
    assert bool((got[:-3, 8:] == got[0, 8]).all())


@pytest.mark.parametrize("R,V,K", [(2, 40000, 20), (600, 5000, 8)])
def test_graph_stream_and_same_bits(R, V, K):
    """Two objects captured into two graphs and replayed in turn, and again on another stream."""
    io, given = "bf16", tokens(R, V, 3)
    x = torch.from_numpy(draw(R, V)).bfloat16().to(DEV)
    tok = torch.from_numpy(given).to(torch.int32).to(DEV)
    ops = [runner.TokenLogprobs(R, V, 3, K, io, entropy=True, device=DEV) for _ in range(2)]
    back = runner.TokenLogprobs(R, V, 3, K, io, backward=True, device=DEV)
    dl = torch.randn((R, 3), device=DEV)

    def both(op):
        out = op.forward(x, tok)
        return [*out, back.backward(x, tok, out[1], dl, None, out[2], out[2])]

    want = [t.clone() for t in both(ops[0])]
    torch.cuda.synchronize()
    graphs, got = [], []
    for op in ops:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(both(op))
    for _ in range(3):
        for one in got:
            for t in one:
                t.fill_(-5)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for one in got:
            assert all(torch.equal(a, b) for a, b in zip(want, one))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = both(ops[1])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, again))


def test_beam_scores_less_lse_select_from_logits():
    """The selection over logits with beam_scores - lse gives what it gives over log
    probabilities: same parents and tokens where scores differ by more than roundings."""
    W, V = 64, 2048
    x = torch.from_numpy(draw(W, V)).float().to(DEV)
    x[:, 100:1500] = float("-inf")
    beam = torch.randn((1, W), device=DEV)
    _, lse, _, _, _ = runner.TokenLogprobs(W, V, 0, 0, "f32", device=DEV).forward(x)
    parents, toks, scores = (t.clone() for t in runner.BeamSelector(1, W, V, W, device=DEV)(
        x[None], beam - lse))
    want = (f64(beam)[0][:, None] + ref_logp(f64(x))).reshape(-1)
    order = np.argsort(-want, kind="stable")[:W + 1]
    got = parents[0].cpu().numpy().astype(np.int64) * V + toks[0].cpu().numpy()
    assert np.abs(f64(scores)[0] - want[got]).max() <= 2e-5
    gap = want[order][:-1] - want[order][1:]
    assert len(set(got) ^ set(order[:W])) == 0 or gap[-1] < 2e-5


def ref_logp(x):
    m = x.max(1, keepdims=True)
    return x - m - np.log(np.exp(x - m).sum(1, keepdims=True))


def far_rows(V, io):
    """Rows whose lse is far from 0: a large offset, finite masks' values throughout (and in all
    columns but one), large values of either sign, and ordinary and masked rows beside them."""
    x = draw(12, V)
    low = float(torch.finfo(torch.bfloat16).min)
    x[0] += 4096.0
    x[1] -= 4096.0
    x[2] = -1e9
    x[3] = -1e9 + x[3]
    x[4] = low
    x[5], x[5, V // 2] = low, 2.0
    x[6] = 1e30 * np.sign(x[6])
    x[7] = -low
    x[8] += 100.0
    x[9] = -np.inf
    x[10], x[10, [1, V - 2]] = -np.inf, -4e9
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    return f64(torch.from_numpy(x).to(dt))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("V,G,ent,place", [(70, 2, False, False), (1000, 5, True, True),
                                           (4096, 1, False, False), (9001, 0, True, True),
                                           (9001, 256, True, False), (50001, 1, False, True)])
@pytest.mark.parametrize("scale", [1.0, 0.7, 1.5])
def test_gradient_of_rows_far_from_zero(scale, V, G, ent, place, io):
    """p comes from differences to the row's largest logit wherever lse alone has lost ln s: its
    error is the sum's 7.5e-6, half a step of an lse up to 128 (4e-6) and the exponential's
    argument, 2^-23 |ln p| (|ln p| < 40: 5e-6), of every term.  In place too."""
    x = far_rows(V, io)
    R, given = len(x), tokens(len(x), V, G) if G else None
    if G:
        given[given >= V] = -1
        given[2], given[4], given[7] = -1, -1, -1  # padding alone: 0 without the others
    r = np.random.default_rng(V)
    dlogp = r.normal(size=(R, G)).astype(np.float32) if G else None
    dlse, dent = ((r.normal(size=R).astype(np.float32) for _ in range(2)) if ent or not G
                  else (None, None))
    dent = dent if ent else None
    with np.errstate(over="ignore"):
        _, lse, entropy, _, _ = ref.logprobs(x, None, 0, scale)
        dev = [None if t is None else torch.from_numpy(np.asarray(t, np.float32)).to(DEV)
               for t in (lse, dlogp, dlse, entropy, dent)]
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    logits = torch.from_numpy(x).to(dt).to(DEV)
    tok = None if given is None else torch.from_numpy(given).to(torch.int32).to(DEV)
    op = runner.TokenLogprobs(R, V, G, 0, io, scale, backward=True, device=DEV)
    got = op.backward(logits, tok, *dev, out=logits if place else None)
    want, size = ref.logprobs_backward(x, given, dlogp, dlse, dent, scale)
    same_or_near(got, want, 2e-5 * size + (2.0 ** -8 * np.abs(want) if io == "bf16" else 0) + 1e-37)
    if not ent and G:
        assert float(got[[2, 4, 7]].float().abs().max()) == 0.0


@pytest.mark.parametrize("scale", [0.7, 1.5])
def test_gradient_from_the_forward_calls_own_sums(scale):
    """What the forward call leaves is what the gradient takes, far rows among it: each row's
    gradient of the sum of all log probabilities adds up to 0 (V terms of 1 and of V p each, with
    their 2e-5 and the roundings of V sums)."""
    V = 5000
    x = torch.from_numpy(far_rows(V, "f32")).float().to(DEV)
    R = x.shape[0]
    tok = torch.randint(0, V, (R, 3), generator=torch.Generator().manual_seed(1)).int().to(DEV)
    tok[10] = 1  # (its mask leaves this token and one other)
    _, lse, *_ = runner.TokenLogprobs(R, V, 3, 0, "f32", scale, device=DEV).forward(x, tok)
    one = torch.ones((R, 3), device=DEV)
    got = runner.TokenLogprobs(R, V, 3, 0, "f32", scale, backward=True, device=DEV).backward(
        x, tok, lse, one)
    assert bool(torch.isfinite(got).all())
    assert float(got.double().sum(1).abs().max()) <= scale * 6 * 2e-5
    assert float(got[9].abs().max()) == 0.0


def test_selection_from_logits_with_dead_beams():
    """Beams whose mask leaves nothing have candidates of -inf, as with log probabilities, in this step
    and the next one; the selections are the same (all scores differ by more than roundings, candidates of
    -inf go by their places)."""
    W, V = 8, 40
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn((2, W, V), generator=g, device=DEV)
    x[0, :] = float("-inf")
    x[0, 2, [3, 30]], x[0, 5, 7] = torch.tensor([0.5, 2.0], device=DEV), -1.0
    x[1, 0] = float("-inf")
    x[1, 3:, 5:] = float("-inf")
    logp = torch.log_softmax(x.double(), -1).float()
    logp[torch.isneginf(x)] = float("-inf")
    direct, select = (runner.BeamSelector(1, W, V, W, device=DEV) for _ in range(2))
    want = got = torch.tensor([[-1.0, -2.0, -3.5, -0.5, -4.0, -2.5, float("-inf"), 0.0]], device=DEV)
    for t in range(2):
        _, lse, *_ = runner.TokenLogprobs(W, V, 0, 0, "f32", device=DEV).forward(x[t])
        a = [v.clone() for v in direct(logp[t][None], want)]
        b = [v.clone() for v in select(x[t][None], runner.scores_for_logits(got, lse[None]))]
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        want, got = a[2], b[2]
        assert torch.equal(torch.isneginf(want), torch.isneginf(got))
        assert not bool(got.isnan().any())
        live = torch.isfinite(want)
        assert int(live.sum()) == (3, W)[t]
        assert float((want - got)[live].abs().max()) <= 2e-5
