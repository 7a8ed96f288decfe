"""Short causal convolution, its gradient and its step, through the C ABI, against 64-bit
references.

Bars, relative to the sum of the sizes of a result's terms.  y: 5 products and sums (2^-24 each),
the exponential's argument (|pre| 2^-24 of it, |pre| < 12 here) and three roundings more: 2e-6.
dx, state gradients: the slope takes the same errors once more, then 4 products: 4e-6.  Weight
gradients: sums along a run (48 tokens here at most), over a workgroup's runs (256 at most,
in a row) and over the workgroups (16 apart, then 16) make at most 340 roundings: 2.5e-5.  bf16
results: one rounding, 2^-8 of the value, on top.  States are copies."""
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


def near(got, want, size, bar, io="f32"):
    got = f64(got)
    assert got.shape == want.shape and np.isfinite(got).all()
    bar = bar * size + (2.0 ** -8 * np.abs(want) if io == "bf16" else 0)
    assert (np.abs(got - want) <= bar + 1e-37).all(), float((np.abs(got - want) - bar).max())


class Case:
    def __init__(self, lengths, C, taps, io, bias=True, state=True, wide=0, seed=0, tail=0):
        g = torch.Generator().manual_seed(seed + C)
        dt = torch.bfloat16 if io == "bf16" else torch.float32
        self.lengths, self.C, self.taps, self.io, self.dt = lengths, C, taps, io, dt
        self.N, self.n = len(lengths), sum(lengths)

        def draw(*shape, dtype=dt):
            return torch.randn(shape, generator=g).to(dtype).to(DEV)

        rows = draw(self.n + tail, C + wide)
        self.x = rows[:, wide // 2:wide // 2 + C] if wide else rows
        self.w = draw(C, taps, dtype=torch.float32) * 0.7
        self.bias = draw(C, dtype=torch.float32) * 0.3 if bias else None
        self.state = draw(self.N, taps - 1, C) if state else None
        self.off = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32,
                                device=DEV)
        self.dy, self.dlast = draw(self.n + tail, C), draw(self.N, taps - 1, C)

    def numbers(self):
        bias = np.zeros(self.C) if self.bias is None else f64(self.bias)
        return self.lengths, f64(self.x)[:self.n], f64(self.w), bias, f64(self.state)


CASES = [
    ([1], 8, 2, "f32", True, False, 0, True),
    ([1], 2048, 4, "bf16", False, True, 64, True),
    ([3, 1, 2], 24, 4, "f32", True, True, 8, True),
    ([0, 5, 1, 0, 130, 2, 0], 80, 4, "bf16", True, True, 16, True),
    ([0, 5, 1, 0, 130, 2, 0], 80, 3, "f32", False, False, 0, False),
    ([200], 512, 4, "bf16", False, False, 0, True),
    ([70, 70, 70], 520, 3, "bf16", True, True, 0, False),
    ([333, 4, 12], 264, 2, "f32", True, True, 40, True),
    ([1] * 70 + [9, 0, 30], 16, 4, "f32", True, True, 0, True),
    ([500, 41], 1032, 4, "bf16", True, True, 16, True),
]


@pytest.mark.parametrize("lengths,C,taps,io,bias,state,wide,silu", CASES)
def test_conv_and_gradient(lengths, C, taps, io, bias, state, wide, silu):
    c = Case(lengths, C, taps, io, bias, state, wide)
    act = "silu" if silu else None
    op = runner.ShortConv(c.N, c.n, C, taps, io, act, device=DEV)
    y, last = op.forward(c.x, c.w, c.bias, c.off, c.state)
    want, wlast, size = ref.conv(*c.numbers(), silu)
    near(y, want, size, 2e-6, io)
    assert np.array_equal(f64(last), wlast)
    back = runner.ShortConv(c.N, c.n, C, taps, io, act, backward=True, device=DEV)
    got = back.backward(c.x, c.w, c.dy, c.bias, c.off, c.state, c.dlast)
    grads, sizes = ref.conv_backward(*c.numbers(), silu, f64(c.dy), f64(c.dlast))
    near(got[0], grads[0], sizes[0], 4e-6, io)
    near(got[1], grads[1], sizes[1], 2.5e-5)
    if bias:
        near(got[2], grads[2], sizes[2], 2.5e-5)
    else:
        assert got[2] is None
    if state:
        near(got[3], grads[3], sizes[3], 4e-6, io)
    else:
        assert got[3] is None


def test_equal_lengths_without_offsets():
    c = Case([37] * 5, 96, 4, "f32")
    op = runner.ShortConv(5, 185, 96, 4, "f32", device=DEV)
    a = [t.clone() for t in op.forward(c.x, c.w, c.bias, c.off, c.state)]
    b = op.forward(c.x, c.w, c.bias, None, c.state)
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    back = runner.ShortConv(5, 185, 96, 4, "f32", backward=True, device=DEV)
    a = [t.clone() for t in back.backward(c.x, c.w, c.dy, c.bias, c.off, c.state, c.dlast)]
    b = back.backward(c.x, c.w, c.dy, c.bias, None, c.state, c.dlast)
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_gradient_against_differences():
    """Differences of the kernel's own outputs (fp32, step 2^-7): the curvature of silu adds some
    step^2, roundings 2e-7 / step of the sum over the outputs."""
    c = Case([0, 6, 19], 16, 4, "f32", seed=5)
    op = runner.ShortConv(3, 25, 16, 4, "f32", device=DEV)
    back = runner.ShortConv(3, 25, 16, 4, "f32", backward=True, device=DEV)
    grads = back.backward(c.x, c.w, c.dy, c.bias, c.off, c.state, c.dlast)
    h, g = 2.0 ** -7, torch.Generator().manual_seed(9)
    for i, grad in enumerate(grads):
        args = [c.x, c.w, c.bias, c.state]
        d = torch.randn(args[i].shape, generator=g).to(DEV)
        vals = []
        for s in (h, -h):
            moved = list(args)
            moved[i] = (args[i] + s * d).contiguous()
            y, last = op.forward(moved[0], moved[1], moved[2], c.off, moved[3])
            vals.append(float((y.double() * c.dy).sum() + (last.double() * c.dlast).sum()))
        want = float((grad.double() * d).sum())
        assert abs((vals[0] - vals[1]) / (2 * h) - want) <= \
            1e-3 * float(grad.norm()) * float(d.norm())


def test_rows_behind_the_last_sequence_are_left():
    c = Case([5, 40], 64, 4, "bf16", tail=30)
    op = runner.ShortConv(2, 75, 64, 4, "bf16", device=DEV)
    c.x[45:] = float("nan")
    op.y.fill_(7.0)
    y, last = op.forward(c.x, c.w, c.bias, c.off, c.state)
    want, wlast, size = ref.conv(*c.numbers(), True)
    near(y[:45], want, size, 2e-6, "bf16")
    assert bool((y[45:] == 7.0).all()) and np.array_equal(f64(last), wlast)
    back = runner.ShortConv(2, 75, 64, 4, "bf16", backward=True, device=DEV)
    back.dx.fill_(7.0)
    c.dy[45:] = float("nan")
    got = back.backward(c.x, c.w, c.dy, c.bias, c.off, c.state)
    grads, sizes = ref.conv_backward(*c.numbers(), True, f64(c.dy), None)
    near(got[0][:45], grads[0], sizes[0], 4e-6, "bf16")
    assert bool((got[0][45:] == 7.0).all())
    near(got[1], grads[1], sizes[1], 2.5e-5)


def test_sequences_of_nothing():
    """No tokens at all: the states pass through, the weights' gradients are 0."""
    c = Case([0, 0, 0], 40, 4, "bf16")
    op = runner.ShortConv(3, 0, 40, 4, "bf16", device=DEV)
    _, last = op.forward(c.x, c.w, c.bias, c.off, c.state)
    assert torch.equal(last, c.state)
    back = runner.ShortConv(3, 0, 40, 4, "bf16", backward=True, device=DEV)
    _, dw, db, ds = back.backward(c.x, c.w, c.dy, c.bias, c.off, c.state, c.dlast)
    assert torch.equal(ds, c.dlast) and float(dw.abs().max()) == float(db.abs().max()) == 0.0
    _, _, _, ds = back.backward(c.x, c.w, c.dy, c.bias, None, c.state)
    assert float(ds.abs().max()) == 0.0


def test_last_state_in_the_place_of_the_first():
    """Sequences longer than a run, so that other workgroups read the first state."""
    c = Case([1, 0, 300, 2], 48, 4, "f32")
    op = runner.ShortConv(4, 303, 48, 4, "f32", device=DEV)
    y, last = (t.clone() for t in op.forward(c.x, c.w, c.bias, c.off, c.state))
    state = c.state.clone()
    ab.onela_short_conv(op.cfg, c.off, c.x, c.w, c.bias, state, op.y, state)
    assert torch.equal(op.y, y) and torch.equal(state, last)


def test_offsets_that_are_wrong_stay_inside():
    """Offsets out of range or order give wrong sequences and no access outside (the tensors
    stand in the middle of larger ones that keep their values)."""
    T, C = 64, 32
    for off in ([0, 500, 20, 64], [-9, 30, 10, 900], [70, 80, 90, 64], [64, 0, 64, 0]):
        whole = torch.full((3 * T, C), 5.0, device=DEV)
        x = torch.randn((T, C), device=DEV)
        state, last = torch.randn((3, 3, C), device=DEV), torch.full((9, 3, C), 5.0, device=DEV)
        w = torch.randn((C, 4), device=DEV)
        cfg = ab.make_conv_config(3, T, C, 4, "f32")
        o = torch.tensor(off, dtype=torch.int32, device=DEV)
        ab.onela_short_conv(cfg, o, x, w, None, state, whole[T:2 * T], last[3:6])
        nbytes = ab.onela_short_conv_workspace_bytes(cfg)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
        dx, ds = torch.full((3 * T, C), 5.0, device=DEV), torch.full((9, 3, C), 5.0, device=DEV)
        dw = torch.empty((C, 4), device=DEV)
        ab.onela_short_conv_backward(cfg, o, x, w, None, state, x, last[3:6], dx[T:2 * T], dw, None,
                                     ds[3:6], ws, nbytes)
        torch.cuda.synchronize()
        for t, n in ((whole, T), (last, 3), (dx, T), (ds, 3)):
            assert bool((t[:n] == 5.0).all()) and bool((t[2 * n:] == 5.0).all())


@pytest.mark.parametrize("io,C,taps,T,silu", [("f32", 8, 2, 1, True), ("bf16", 520, 4, 1, True),
                                              ("bf16", 2048, 4, 2, False), ("f32", 96, 3, 5, True)])
def test_step_goes_on_from_a_prompt(io, C, taps, T, silu):
    """A prompt's last tokens in steps give the prompt's own bits, in place and from pool to
    pool; slots outside the pool give zeros and store nothing."""
    N, act = 5, "silu" if silu else None
    c = Case([11] * N, C, taps, io, wide=16)
    whole, last = runner.ShortConv(N, 11 * N, C, taps, io, act, device=DEV).forward(
        c.x, c.w, c.bias, None, c.state)
    whole = whole.unflatten(0, (N, 11))
    x = c.x.unflatten(0, (N, 11))
    first = x[:, :11 - T].flatten(0, 1).contiguous()
    _, mid = runner.ShortConv(N, N * (11 - T), C, taps, io, act, device=DEV).forward(
        first, c.w, c.bias, None, c.state)
    new = x[:, 11 - T:].flatten(0, 1)
    pool = torch.full((9, taps - 1, C), 3.0, dtype=c.dt, device=DEV)
    slots = torch.tensor([7, 2, -1, 0, 9], dtype=torch.int32, device=DEV)
    for n in (0, 1, 3):
        pool[int(slots[n])] = mid[n]
    out = torch.full((6, taps - 1, C), 4.0, dtype=c.dt, device=DEV)
    step = runner.ShortConvStep(N, N * T, C, taps, io, 9, act, device=DEV)
    for target in (out, None):
        where = torch.tensor([5, 1, 2, -3, 0], dtype=torch.int32, device=DEV)
        before = pool.clone()
        y = step.step(pool, slots, new, c.w, c.bias, pool_out=target,
                      slots_out=None if target is None else where).unflatten(0, (N, T))
        for n in range(N):
            if n in (0, 1, 3):
                assert torch.equal(y[n], whole[n, 11 - T:])
            else:
                assert float(y[n].float().abs().max()) == 0.0
        if target is not None:
            assert torch.equal(pool, before)
            assert torch.equal(out[5], last[0]) and torch.equal(out[1], last[1])
            assert bool((out[[0, 2, 3, 4]] == 4.0).all())
        else:
            for n in (0, 1, 3):
                assert torch.equal(pool[int(slots[n])], last[n])
            assert bool((pool[[1, 3, 4, 5, 6, 8]] == 3.0).all())


def test_beams_go_on_from_their_parents():
    """Several sequences from one state; ragged steps, one without a token (its state is its
    parent's)."""
    c = Case([2, 0, 1, 3], 64, 4, "f32")
    pool = torch.randn((3, 3, 64), device=DEV)
    parents = torch.tensor([1, 1, 1, 0], dtype=torch.int32, device=DEV)
    out = torch.zeros((4, 3, 64), device=DEV)
    step = runner.ShortConvStep(4, 6, 64, 4, "f32", 3, device=DEV)
    y = step.step(pool, parents, c.x, c.w, c.bias, c.off, pool_out=out)
    want, wlast, size = ref.conv(c.lengths, f64(c.x), f64(c.w), f64(c.bias),
                                 f64(pool)[parents.cpu().numpy()], True)
    near(y, want, size, 2e-6)
    assert np.array_equal(f64(out), wlast)


def test_not_finite_stays_near():
    """NaN and infinities of an input reach the taps tokens from it on, in its channel."""
    c = Case([20, 20], 16, 4, "f32", state=False)
    c.x[6, 3], c.x[17, 5] = float("nan"), float("inf")
    op = runner.ShortConv(2, 40, 16, 4, "f32", None, device=DEV)
    y, _ = op.forward(c.x, c.w, c.bias, c.off)
    bad = ~torch.isfinite(y).cpu()
    want = torch.zeros_like(bad)
    want[6:10, 3] = True
    want[17:20, 5] = True
    assert torch.equal(bad, want)


def test_more_than_32_bits_of_offset():
    T, C = 350000, 6144  # 2.15e9 elements, 4.3 GB
    x = torch.zeros((T, C), dtype=torch.bfloat16, device=DEV)
    x[-6:] = torch.randn((6, C), device=DEV).bfloat16()
    w = torch.randn((C, 4), device=DEV)
    op = runner.ShortConv(1, T, C, 4, "bf16", device=DEV)
    op.y.fill_(float("nan"))
    y, last = op.forward(x, w)
    want, _, size = ref.conv([6], f64(x[-6:]), f64(w), np.zeros(C), None, True)
    near(y[-6:], want, size, 2e-6, "bf16")
    assert torch.equal(last[0], x[-3:]) and not bool(y[:, ::997].isnan().any())
    del op, y
    back = runner.ShortConv(1, T, C, 4, "bf16", backward=True, device=DEV)
    back.dx.fill_(float("nan"))
    dx, dw, _, _ = back.backward(x, w, x)
    grads, sizes = ref.conv_backward([6], f64(x[-6:]), f64(w), np.zeros(C), None, True,
                                     f64(x[-6:]), None)
    near(dx[-6:], grads[0], sizes[0], 4e-6, "bf16")
    near(dw, grads[1], sizes[1], 2.5e-5)
    assert not bool(dx[:, ::997].isnan().any())


def test_graph_stream_and_same_bits():
    """Replays of a captured call, beside eager calls on another stream, give the same bits."""
    c = Case([100, 0, 57], 264, 4, "bf16")
    op = runner.ShortConv(3, 157, 264, 4, "bf16", device=DEV)
    back = runner.ShortConv(3, 157, 264, 4, "bf16", backward=True, device=DEV)
    other = runner.ShortConv(3, 157, 264, 4, "bf16", backward=True, device=DEV)

    def both(b):
        return [*op.forward(c.x, c.w, c.bias, c.off, c.state),
                *b.backward(c.x, c.w, c.dy, c.bias, c.off, c.state, c.dlast)]

    want = [t.clone() for t in both(back)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(back)
    side = torch.cuda.Stream()
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            again = other.backward(c.x, c.w, c.dy, c.bias, c.off, c.state, c.dlast)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        assert all(torch.equal(a, b) for a, b in zip(want[2:], again))


@pytest.mark.parametrize("C,taps", [(1 << 26, 4), (54 << 20, 4), (1 << 24, 2)])
def test_weight_gradients_of_the_most_channels(C, taps):
    """The second launch alone writes them where there are no tokens: all of them, in more turns
    than a grid has workgroups (a thread for each of their 16ths would pass 2^32)."""
    cfg = ab.make_conv_config(1, 0, C, taps, "bf16")
    n = ab.onela_short_conv_workspace_bytes(cfg)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    w = torch.zeros((C, taps), device=DEV)
    dw, db = torch.full((C, taps), 7.0, device=DEV), torch.full((C,), 7.0, device=DEV)
    ab.onela_short_conv_backward(cfg, None, None, w, None, None, None, None, None, dw, db, None, ws,
                                 n)
    assert float(dw.abs().max()) == float(db.abs().max()) == 0.0


def test_step_over_its_inputs():
    """y in the place of x: the same bits, several tokens per sequence, slots outside among them."""
    c = Case([3] * 4, 72, 4, "bf16")
    pool = torch.randn((5, 3, 72), device=DEV).bfloat16()
    slots = torch.tensor([4, -1, 0, 2], dtype=torch.int32, device=DEV)
    step = runner.ShortConvStep(4, 12, 72, 4, "bf16", 5, device=DEV)
    first, x = pool.clone(), c.x.clone()
    y = step.step(pool, slots, c.x, c.w, c.bias)
    ab.onela_short_conv_step(step.cfg, None, x, c.w, c.bias, first, 5, slots, None, 0, None, x)
    assert torch.equal(x, y) and torch.equal(first, pool)


@pytest.mark.parametrize("lengths,tail,C,io", [
    ([5, 40], 30, 64, "bf16"), ([5, 0, 40, 0], 1, 2048, "f32"), ([300], 700, 520, "bf16"),
    ([0, 0], 77, 96, "f32"), ([33, 31], 0, 256, "bf16"), ([2000, 1, 48], 5000, 8, "f32")])
def test_rows_behind_the_last_sequence_are_cleared(lengths, tail, C, io):
    """With clear_rest they are 0 and all others have the bits that they have without; so without
    offsets, where no row is behind."""
    c = Case(lengths, C, 4, io, tail=tail)
    rows = c.n + tail
    for off in (c.off, None):
        N = c.N if off is not None else 1
        state, dlast = (None, None) if off is None else (c.state, c.dlast)
        for backward in (False, True):
            got = []
            for clear in (False, True):
                op = runner.ShortConv(N, rows, C, 4, io, backward=backward, device=DEV,
                                      clear_rest=clear)
                (op.dx if backward else op.y).fill_(7.0)
                got.append(op.backward(c.x, c.w, c.dy, c.bias, off, state, dlast) if backward else
                           op.forward(c.x, c.w, c.bias, off, state))
            end = c.n if off is not None else rows
            assert bool((got[0][0][end:] == 7.0).all())
            assert not bool(got[1][0][end:].any())
            assert torch.equal(got[0][0][:end], got[1][0][:end])
            for a, b in zip(got[0][1:], got[1][1:]):
                assert a is b is None or torch.equal(a, b)


def test_clearing_by_offsets_that_are_wrong_stays_inside():
    T, C = 64, 32
    x, w = torch.randn((T, C), device=DEV), torch.randn((C, 4), device=DEV)
    for off in ([0, 500, 20, 64], [-9, 30, 10, 900], [70, 80, 90, 64], [64, 0, 64, 0], [0, 5, 9, -7]):
        cfg = ab.make_conv_config(3, T, C, 4, "f32", clear_rest=True)
        o = torch.tensor(off, dtype=torch.int32, device=DEV)
        y, dx = (torch.full((3 * T, C), 5.0, device=DEV) for _ in range(2))
        ab.onela_short_conv(cfg, o, x, w, None, None, y[T:2 * T], None)
        ab.onela_short_conv_backward(cfg, o, x, w, None, None, x, None, dx[T:2 * T])
        for t in (y, dx):
            assert bool((t[:T] == 5.0).all()) and bool((t[2 * T:] == 5.0).all())
