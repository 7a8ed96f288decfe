"""Norms before and after a block with its gate and residual scale, and their gradients, through
the C ABI, against 64-bit references.

Bars, relative to the sizes of a result's terms (a row's largest, since every element takes its
row's means): h: the mean of squares (some 20 roundings in a row of sums, half of that in the
root), the gate's exponential (|g| 2^-24, |g| < 6 here) and six products: 3e-6.  y: the second mean
takes those of h once more: 6e-6.  dx, dres, dgate: two more means: 1.2e-5.  Weight gradients: sums
along a workgroup's rows (6 here), its lane groups (64 at most) and the workgroups (16 and 64)
add 150 roundings at most: 2.1e-5.  bf16 results: one rounding, 2^-8 of the value, on top."""
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


def near(got, want, size, bar, dtype=None):
    got = f64(got)
    assert got.shape == want.shape and np.isfinite(got).all()
    big = size.max(-1, keepdims=True) if size.ndim > 1 else size
    bar = bar * big + (2.0 ** -8 * np.abs(want) if dtype is torch.bfloat16 else 0)
    assert (np.abs(got - want) <= bar + 1e-37).all(), float((np.abs(got - want) - bar).max())


class Case:
    def __init__(self, T, H, D, io, rio, after, before, act, res, cs, weights=True, wide=False):
        g = torch.Generator().manual_seed(T * 7 + D)
        types = {"bf16": torch.bfloat16, "f32": torch.float32}
        dt, rt = types[io], types[rio]
        self.io, self.rio, self.dt, self.rt = io, rio, dt, rt
        self.T, self.H, self.D = T, H, D

        def draw(dtype, more=0):
            x = torch.randn((T, H * D + more), generator=g).to(dtype).to(DEV)
            return x[:, more:].unflatten(1, (H, D))

        def vector(on):
            return (1 + 0.3 * torch.randn(D, generator=g)).to(DEV) if on else None

        self.x = draw(dt, 24 if wide else 0)
        self.gate = draw(dt, 8 if wide else 0) if act else None
        self.res = draw(rt) * 2 if res else None
        self.wa, self.wb, self.cs = vector(after and weights), vector(before and weights), vector(cs)
        self.dy = draw(dt) if before or not res else None
        self.dh = draw(rt) if res else None
        self.args = dict(after=after, before=before, act=act, scale=0.6, eps=1e-5)
        self.make = dict(num_heads=H, io=io, residual_io=rio, norm_after=after, norm_before=before,
                         gate=act, residual_scale=0.6, eps=1e-5, device=DEV)

    def tensors(self):
        return self.x, self.res, self.gate, self.wa, self.wb, self.cs

    def forward(self):
        return runner.BlockNorm(self.T, self.D, **self.make).forward(*self.tensors())

    def backward(self, op=None):
        op = op or runner.BlockNorm(self.T, self.D, backward=True, **self.make)
        return op.backward(self.x, self.dy, *self.tensors()[1:], self.dh)


#  T, H, D, io, residual, after, before, gate, res, channel scale, weights, wide
CASES = [
    (1, 1, 8, "f32", "f32", True, True, "silu", True, True, True, False),
    (3, 2, 24, "f32", "f32", True, False, "sigmoid", False, False, True, True),
    (33, 16, 128, "bf16", "bf16", True, False, "silu", False, False, True, True),
    (7, 3, 64, "bf16", "f32", False, True, None, True, False, True, False),
    (5, 1, 136, "bf16", "f32", True, True, "silu", True, True, True, True),
    (9, 1, 512, "f32", "bf16", True, True, "sigmoid", True, False, False, False),
    (4, 1, 520, "f32", "f32", False, True, "silu", True, True, True, True),
    (6, 2, 1024, "bf16", "bf16", False, True, None, True, False, True, True),
    (11, 1, 2048, "bf16", "f32", True, True, "silu", True, True, True, False),
    (2, 1, 2056, "f32", "bf16", True, True, None, True, True, True, False),
    (3, 1, 4096, "bf16", "bf16", True, True, "sigmoid", True, True, True, True),
    (2, 1, 8192, "f32", "f32", True, True, "silu", True, True, True, False),
    (3, 1, 4104, "bf16", "f32", True, True, "silu", True, True, True, True),
    (1500, 1, 8192, "bf16", "bf16", False, True, None, True, False, True, False),
    (10, 1, 256, "bf16", "f32", False, False, None, True, True, True, False),  # residual alone
    (10, 2, 40, "f32", "f32", False, False, "silu", False, True, True, False),  # a gate alone
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_norm_and_gradient(case):
    c = Case(*case)
    y, h = c.forward()
    want = ref.block_norm(*map(f64, c.tensors()), **c.args)
    if y is not None:
        near(y, want[0], want[2], 6e-6, c.dt)
    if c.res is not None:
        near(h, want[1], want[3], 3e-6, c.rt)
    assert (y is None) == (c.res is not None and not c.args["before"])
    assert (h is None) == (c.res is None)
    got = c.backward()
    grads, sizes = ref.block_norm_backward(*map(f64, c.tensors()), f64(c.dy), f64(c.dh), **c.args)
    for i, (g, w, s) in enumerate(zip(got, grads, sizes)):
        if c.tensors()[i] is None:
            assert g is None
        else:
            near(g, w, s, 1.2e-5 if i < 3 else 2.1e-5, (c.dt, c.rt, c.dt, None, None, None)[i])


def test_gradient_against_differences():
    """Differences of the kernel's own outputs (fp32, step 2^-7): third derivatives add some
    step^2, roundings 1e-6 / step of the sum."""
    c = Case(4, 2, 32, "f32", "f32", True, True, "silu", True, True)
    op = runner.BlockNorm(4, 32, **c.make)
    g = torch.Generator().manual_seed(2)
    for i, grad in enumerate(c.backward()):
        args, h = list(c.tensors()), 2.0 ** -7
        d = torch.randn(args[i].shape, generator=g).to(DEV)
        vals = []
        for s in (h, -h):
            moved = list(args)
            moved[i] = args[i] + s * d
            y, r = op.forward(*moved)
            vals.append(float((y.double() * c.dy).sum() + (r.double() * c.dh).sum()))
        assert abs((vals[0] - vals[1]) / (2 * h) - float((grad.double() * d).sum())) <= \
            2e-3 * float(grad.norm()) * float(d.norm())


def test_outputs_that_are_not_wanted():
    """y or the residual alone, one weight gradient alone, one incoming gradient alone: the same
    bits, and nothing else is written."""
    c = Case(20, 1, 512, "bf16", "f32", True, True, "silu", True, True)
    y, h = c.forward()
    op = runner.BlockNorm(20, 512, **c.make)
    for wy, wh in ((True, False), (False, True)):
        y2, h2 = torch.full_like(y, 9.0), torch.full_like(h, 9.0)
        ab.onela_block_norm(op.cfg, c.x, c.gate, c.res, c.wa, c.wb, c.cs, y2 if wy else None,
                            h2 if wh else None)
        assert torch.equal(y2, y) if wy else bool((y2 == 9.0).all())
        assert torch.equal(h2, h) if wh else bool((h2 == 9.0).all())
    back = runner.BlockNorm(20, 512, backward=True, **c.make)
    want = [t.clone() for t in c.backward(back)]
    back.dw.fill_(9.0)
    dx = torch.empty_like(c.x)
    ab.onela_block_norm_backward(back.cfg, c.x, c.gate, c.res, c.wa, c.wb, c.cs, c.dy, c.dh, dx,
                                 dbefore_weight=back.dw[1], workspace=back.workspace,
                                 workspace_bytes=back.ws_bytes)
    assert torch.equal(dx, want[0]) and torch.equal(back.dw[1], want[4])
    assert bool((back.dw[[0, 2]] == 9.0).all())
    zero = torch.zeros_like(c.dy)
    a = [t.clone() for t in back.backward(c.x, zero, *c.tensors()[1:], c.dh)]
    b = back.backward(c.x, None, *c.tensors()[1:], c.dh)
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_residual_in_place():
    c = Case(700, 1, 264, "bf16", "f32", False, True, None, True, False)
    y, h = c.forward()
    op = runner.BlockNorm(700, 264, **c.make)
    res, y2 = c.res.clone(), torch.empty_like(y)
    ab.onela_block_norm(op.cfg, c.x, None, res, None, c.wb, None, y2, res)
    assert torch.equal(res, h) and torch.equal(y2, y)
    want = [None if t is None else t.clone() for t in c.backward()]
    back = runner.BlockNorm(700, 264, backward=True, **c.make)
    d = c.dh.clone()
    ab.onela_block_norm_backward(back.cfg, c.x, None, c.res, None, c.wb, None, c.dy, d, y2, None, d)
    assert torch.equal(y2, want[0]) and torch.equal(d, want[1])


def test_rows_of_zeros_and_not_finite():
    """Zeros give zeros (eps); NaN and infinities stay in their row."""
    c = Case(6, 2, 128, "f32", "f32", True, True, "silu", True, False)
    c.x[1], c.res[1] = 0.0, 0.0
    c.x[2, 1, 5], c.gate[4, 0, 7] = float("nan"), float("inf")
    for t in c.forward():
        assert float(t[1].abs().max()) == 0.0
        bad = (~torch.isfinite(t)).any(-1).cpu()
        want = torch.zeros_like(bad)
        want[2, 1] = want[4, 0] = True
        assert torch.equal(bad, want)


def test_no_rows():
    cfg = ab.make_block_norm_config(0, 1, 64, "bf16", "f32", True, True, "silu")
    ab.onela_block_norm(cfg, None, None, None, None, None, None, None, None)
    n = ab.onela_block_norm_workspace_bytes(cfg)
    ws, dw = torch.empty(n, dtype=torch.uint8, device=DEV), torch.full((64,), 3.0, device=DEV)
    ab.onela_block_norm_backward(cfg, None, None, None, None, None, None, None, None, None,
                                 dafter_weight=dw, workspace=ws, workspace_bytes=n)
    assert float(dw.abs().max()) == 0.0


@pytest.mark.parametrize("T,H,D", [(5000, 4, 64), (3000, 1, 2048)])
def test_many_rows_same_bits_graph_and_stream(T, H, D):
    """More rows than there are workgroups: against the reference by rows of their own, the same
    bits again, replayed and on another stream."""
    c = Case(T, H, D, "bf16", "f32", True, True, "silu", True, True, wide=True)
    op, back = (runner.BlockNorm(T, D, backward=b, **c.make) for b in (False, True))

    def both():
        return [*op.forward(*c.tensors()), *c.backward(back)]

    want = [t.clone() for t in both()]
    at = [0, 1, T // 2, T - 2, T - 1]
    some = [None if t is None else f64(t[at] if t.ndim == 3 else t) for t in c.tensors()]
    y, h, ys, hs = ref.block_norm(*some, **c.args)
    near(want[0][at], y, ys, 6e-6, c.dt)
    near(want[1][at], h, hs, 3e-6)
    grads, sizes = ref.block_norm_backward(*some, f64(c.dy[at]), f64(c.dh[at]), **c.args)
    for i in range(3):
        near(want[2 + i][at], grads[i], sizes[i], 1.2e-5, (c.dt, c.rt, c.dt)[i])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_weight_gradients_of_many_rows():
    """Sums over 4000 x 4 rows (bar: 16 rows along a lane group, 64 groups, 16 + 64 of the second
    sum: 250 roundings and the terms' own, 3e-5)."""
    c = Case(4000, 4, 32, "f32", "f32", True, True, "silu", True, True)
    got = c.backward()
    grads, sizes = ref.block_norm_backward(*map(f64, c.tensors()), f64(c.dy), f64(c.dh), **c.args)
    for i in range(3, 6):
        near(got[i], grads[i], sizes[i], 3e-5)


def test_more_than_32_bits_of_offset():
    T, D = 270000, 8192  # 2.2e9 elements, 4.4 GB
    x = torch.zeros((T, 1, D), dtype=torch.bfloat16, device=DEV)
    x[-3:] = torch.randn((3, 1, D), device=DEV).bfloat16()
    op = runner.BlockNorm(T, D, norm_after=True, norm_before=False, eps=1e-6, device=DEV)
    y, _ = op.forward(x)
    want = ref.block_norm(f64(x[-3:]), *[None] * 5, after=True, before=False, act=None, scale=1.0,
                          eps=1e-6)
    near(y[-3:], want[0], want[2], 6e-6, torch.bfloat16)
    assert float(y[:-3].abs().max()) == 0.0


@pytest.mark.parametrize("act", ["silu", "sigmoid"])
@pytest.mark.parametrize("D", [128, 2048, 8192])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_gradients_of_large_gates(io, D, act):
    """The activation's slope stays right to 2^-22 of 1 wherever the gate stands: s and g (1 - s) have
    half a step of s each, |g| 2^-24 where s is not 1 (|g| < 17): 1e-6, beside the 1.2e-5 of dgate."""
    c = Case(5, 1, D, io, "f32", True, False, act, False, False)
    at = torch.tensor([40.3, -40.3, 1000.7, -1000.7, 2.0 ** 24 + 2, 2.0 ** 25, 2.0 ** 25 + 4, 3e9,
                       1e30, -1e30, 17.2, -17.2, 88.9, -88.9, 0.0])
    c.gate[1, 0, :15] = at.to(c.dt).to(DEV)
    c.gate[2, 0, -15:] = at.to(c.dt).to(DEV)
    got = c.backward()
    grads, sizes = ref.block_norm_backward(*map(f64, c.tensors()), f64(c.dy), None, **c.args)
    near(got[2], grads[2], sizes[2], 1.2e-5, c.dt)


@pytest.mark.parametrize("T,H,D", [(900, 3, 40), (700, 1, 512), (600, 1, 2048), (300, 1, 8192)])
def test_outputs_in_the_place_of_inputs(T, H, D):
    """Every output in the place of each dense input of its type, in turn: the same bits."""
    c = Case(T, H, D, "bf16", "bf16", True, True, "silu", True, True)
    forward, back = (runner.BlockNorm(T, D, backward=b, **c.make) for b in (False, True))
    want = [t.clone() for t in (*c.forward(), *c.backward()[:3])]
    for i, j in ((0, 1), (1, 2), (2, 0)):
        x, gate, res = ins = [c.x.clone(), c.gate.clone(), c.res.clone()]
        ab.onela_block_norm(forward.cfg, x, gate, res, c.wa, c.wb, c.cs, ins[i], ins[j])
        assert torch.equal(ins[i], want[0]) and torch.equal(ins[j], want[1])
    for i, j, k in ((0, 1, 2), (3, 4, 0), (2, 0, 3), (4, 3, 1)):  # dx, d_residual, dgate
        x, gate, res, dy, dh = ins = [t.clone() for t in (c.x, c.gate, c.res, c.dy, c.dh)]
        ab.onela_block_norm_backward(back.cfg, x, gate, res, c.wa, c.wb, c.cs, dy, dh, ins[i],
                                     ins[k], ins[j])
        assert torch.equal(ins[i], want[2]) and torch.equal(ins[j], want[3])
        assert torch.equal(ins[k], want[4])
