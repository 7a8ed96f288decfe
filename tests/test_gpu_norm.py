"""Norm and rotation of queries and keys and their gradients, through the C ABI, against 64-bit
references.

Bars: fp32 results 2e-6 of the row's largest value (sums of up to 512 squares, a root, a
division and a rotation: some 2^-24 each); weight gradients are fp32 sums over all rows in a
fixed order, 4e-6 of the largest.  bf16 results: one rounding, 2^-8 of the value, on top."""
import numpy as np
import pytest

from paper_2609_12399_amd import onela as ab
from paper_2609_12399_amd import runner
from tests import delta_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def near(got, want, io, sums=None):
    got = f64(got)
    assert np.isfinite(got).all()
    big = np.abs(want).max(-1, keepdims=True) if sums is None else np.abs(want).max()
    bar = (2e-6 if sums is None else 4e-6) * big + (2.0 ** -8 * np.abs(want) if io == "bf16" and
                                                   sums is None else 0)
    assert (np.abs(got - want) <= bar + 1e-30).all(), float((np.abs(got - want) - bar).max())


def table(rows, rot):
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return torch.tensor(np.concatenate([np.cos(a), np.sin(a)], 1), dtype=torch.float32, device=DEV)


def case(T, HQ, HK, D, io, weights, rot, seed=0, wide=False):
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    H = HQ + HK + (1 if wide else 0)
    x = torch.randn((T, H, D), generator=g).to(dt).to(DEV)
    q, k = x[:, :HQ], x[:, HQ:HQ + HK]
    if not wide:
        q, k = q.contiguous(), k.contiguous()
    w = [1 + 0.2 * torch.randn(D, generator=g).to(DEV) if weights else None for _ in range(2)]
    cs = table(50, rot) if rot else None
    pos = torch.randint(0, 50, (T,), generator=g).to(torch.int32).to(DEV) if rot else None
    d = [torch.randn((T, h, D), generator=g).to(dt).to(DEV) for h in (HQ, HK)]
    return q, k, w, pos, cs, d


@pytest.mark.parametrize("T,HQ,HK,D,io,norm,weights,rot,rotation,wide", [
    (1, 1, 1, 8, "f32", "rms", True, 0, "halves", False),
    (5, 3, 1, 16, "bf16", "l2", False, 16, "halves", True),
    (7, 2, 2, 32, "f32", "l2", False, 16, "pairs", False),
    (33, 4, 2, 64, "bf16", "rms", True, 64, "halves", True),
    (3, 8, 1, 96, "f32", "rms", True, 32, "halves", True),
    (17, 2, 1, 80, "bf16", "rms", True, 80, "pairs", False),
    (129, 16, 16, 128, "bf16", "l2", False, 0, "halves", True),
    (40, 16, 4, 128, "bf16", "rms", True, 128, "halves", False),
    (9, 8, 2, 256, "bf16", "rms", True, 64, "halves", True),
    (9, 8, 2, 256, "f32", "rms", True, 256, "pairs", True),
    (6, 3, 3, 512, "bf16", "rms", True, 512, "halves", False),
    (6, 1, 2, 408, "f32", "l2", True, 400, "halves", False),
])
def test_norm_and_gradient(T, HQ, HK, D, io, norm, weights, rot, rotation, wide):
    q, k, w, pos, cs, d = case(T, HQ, HK, D, io, weights, rot, seed=D, wide=wide)
    rms, pairs, eps = norm == "rms", rotation == "pairs", 1e-5
    args = dict(norm=norm, rotary_dim=rot, rotation=rotation, eps=eps, device=DEV)
    out = runner.QkNormRope(T, HQ, HK, D, io, **args).forward(q, k, *w, pos, cs)
    grad = runner.QkNormRope(T, HQ, HK, D, io, backward=True, **args).backward(q, k, *d, *w, pos,
                                                                              cs)
    at = None if cs is None else f64(cs)[pos.cpu().numpy()]
    for x, y, wt, dz, dx, dw in zip((q, k), out, w, d, grad[:2], grad[2:]):
        near(y, ref.norm(f64(x), f64(wt), rms, eps, rot, at, pairs), io)
        gx, gw = ref.norm_backward(f64(x), f64(wt), f64(dz), rms, eps, rot, at, pairs)
        near(dx, gx, io)
        if weights:
            near(dw, gw, io, sums=True)
        else:
            assert dw is None


def test_default_positions_and_rows_of_zeros():
    """No positions: token t is at position t.  A row of zeros gives zeros (eps)."""
    T, D = 12, 64
    q, k, w, _, cs, _ = case(T, 2, 1, D, "f32", True, 32)
    q[3] = 0
    out = runner.QkNormRope(T, 2, 1, D, "f32", norm="rms", rotary_dim=32, eps=1e-6,
                            device=DEV).forward(q, k, *w, None, cs)
    near(out[0], ref.norm(f64(q), f64(w[0]), True, 1e-6, 32, f64(cs)[:T]), "f32")
    assert float(out[0][3].abs().max()) == 0.0


def test_positions_outside_the_table_are_nan():
    T, D = 6, 64
    q, k, w, pos, cs, d = case(T, 2, 1, D, "bf16", True, 64)
    pos[1], pos[4] = -1, 50
    out = runner.QkNormRope(T, 2, 1, D, "bf16", norm="rms", rotary_dim=64, device=DEV).forward(
        q, k, *w, pos, cs)
    for x in out:
        bad = torch.isnan(x).all(-1).all(-1).cpu().tolist()
        assert bad == [False, True, False, False, True, False]
        assert torch.isfinite(x[[0, 2, 3, 5]].float()).all()


def test_queries_alone_and_no_tokens():
    q, _, w, pos, cs, d = case(10, 4, 1, 64, "f32", True, 64)
    op = runner.QkNormRope(10, 4, 0, 64, "f32", norm="rms", rotary_dim=64, device=DEV)
    y, _ = op.forward(q, None, w[0], None, pos, cs)
    near(y, ref.norm(f64(q), f64(w[0]), True, 1e-6, 64, f64(cs)[pos.cpu().numpy()]), "f32")
    cfg = ab.make_norm_config(0, 4, 2, 64, "f32", "rms")
    ab.onela_qk_norm_rope(cfg, None, None, w[0], w[1], None, None, None, None)
    nbytes = ab.onela_qk_norm_rope_workspace_bytes(cfg)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    dw = torch.full((2, 64), float("nan"), device=DEV)
    ab.onela_qk_norm_rope_backward(cfg, None, None, w[0], w[1], None, None, None, None, None, None,
                                   dw[0], dw[1], ws, nbytes)
    assert float(dw.abs().max()) == 0.0  # sums over no rows


def test_one_weight_gradient_alone():
    q, k, w, pos, cs, d = case(30, 4, 2, 128, "bf16", True, 0)
    both = runner.QkNormRope(30, 4, 2, 128, "bf16", norm="rms", backward=True, device=DEV)
    a = [x.clone() for x in both.backward(q, k, *d, *w)]
    one = runner.QkNormRope(30, 4, 2, 128, "bf16", norm="rms", backward=True, device=DEV)
    one.dw.fill_(7.0)
    ab.onela_qk_norm_rope_backward(one.cfg, q, k, *w, None, None, *d, one.q, one.k, None,
                                   one.dw[1], one.workspace, one.ws_bytes)
    assert torch.equal(one.dw[1], a[3]) and float((one.dw[0] - 7.0).abs().max()) == 0.0
    assert torch.equal(one.q, a[0]) and torch.equal(one.k, a[1])


def test_many_rows_same_bits_again_and_graph():
    """More rows than the backward pass has workgroups; the sums are in a fixed order."""
    T, HQ, HK, D = 3000, 8, 8, 64
    q, k, w, pos, cs, d = case(T, HQ, HK, D, "bf16", True, 64, wide=True)
    op = runner.QkNormRope(T, HQ, HK, D, "bf16", norm="rms", rotary_dim=64, backward=True,
                           device=DEV)
    a = [x.clone() for x in op.backward(q, k, *d, *w, pos, cs)]
    at = f64(cs)[pos.cpu().numpy()]
    for x, wt, dz, dx, dw in zip((q, k), w, d, a[:2], a[2:]):
        gx, gw = ref.norm_backward(f64(x), f64(wt), f64(dz), True, 1e-6, 64, at)
        near(dx, gx, "bf16")
        near(dw, gw, "bf16", sums=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = op.backward(q, k, *d, *w, pos, cs)
    for _ in range(3):
        for x in got:
            x.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(a, got):
            assert torch.equal(x, y)


def test_more_rows_than_one_launch_takes():
    """Rows past the 2^32 threads that one grid may hold (here 2^26 rows of 64 lanes): every row
    is written, none twice."""
    T, D = (1 << 26) + 100, 264
    q = torch.ones((T, 1, D), dtype=torch.bfloat16, device=DEV)
    q[-200:] = torch.randn((200, 1, D), device=DEV).bfloat16()
    q[:5] = q[-5:]
    op = runner.QkNormRope(T, 1, 0, D, "bf16", norm="rms", eps=0.0, device=DEV)
    op.q.fill_(float("nan"))
    out, _ = op.forward(q, None)
    for part in (slice(0, 5), slice(T - 200, T)):
        near(out[part], ref.norm(f64(q[part]), None, True, 0.0), "bf16")
    middle = out[5:-200].view(torch.int16)
    assert int(middle.min()) == int(middle.max()) == 0x3f80  # 1 in bf16
