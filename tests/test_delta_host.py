"""What the delta-rule and norm entry points refuse on the host, and their workspace sizes; no
GPU and no HIP call is needed (every argument here is rejected before one)."""
import ctypes

import pytest

from paper_2609_12399_amd import onela as ab

A = 1 << 20  # an address that is aligned and never used


@pytest.fixture(scope="module")
def lib():
    return ab.load_library()


def delta(**kw):
    base = dict(num_seqs=2, total_tokens=128, num_qk_heads=2, num_v_heads=4, d_k=128, d_v=128,
                io_dtype="bf16")
    base.update(kw)
    return ab.make_delta_config(**base)


def norm(**kw):
    base = dict(num_tokens=4, num_q_heads=2, num_k_heads=1, head_dim=64, io_dtype="bf16")
    base.update(kw)
    return ab.make_norm_config(**base)


BAD_DELTA = [dict(num_seqs=0), dict(num_qk_heads=0), dict(num_v_heads=0), dict(num_v_heads=3),
             dict(d_k=96, d_v=96), dict(d_k=128, d_v=64), dict(d_k=512, d_v=512),
             dict(d_k=256, d_v=256, io_dtype="f32"), dict(io_dtype=5), dict(total_tokens=-1),
             dict(total_tokens=1 << 31), dict(q_stride=128), dict(q_stride=2 * 128 + 4),
             dict(k_stride=-256), dict(v_stride=511), dict(v_stride=1 << 23),
             dict(total_tokens=2147483646, num_qk_heads=64, num_v_heads=64)]


def forward(lib, cfg, off=None, q=A, k=A, v=A, la=A, beta=A, s0=None, o=A, last=A, ws=A,
            nbytes=1 << 40):
    return lib.onela_delta_rule_forward(ctypes.byref(cfg), off, q, k, v, la, beta, s0, o, last, ws,
                                        nbytes, None)


def backward(lib, cfg, off=None, q=A, k=A, v=A, la=A, beta=A, s0=None, do=A, ds=None, dq=A, dk=A,
             dv=A, dla=A, db=A, ds0=None, ws=A, nbytes=1 << 40):
    return lib.onela_delta_rule_backward(ctypes.byref(cfg), off, q, k, v, la, beta, s0, do, ds, dq,
                                         dk, dv, dla, db, ds0, ws, nbytes, None)


def step(lib, cfg, off=None, q=A, k=A, v=A, la=A, beta=A, state=A, num=2, slots=None, o=A):
    return lib.onela_delta_rule_step(ctypes.byref(cfg), off, q, k, v, la, beta, state, num, slots,
                                     o, None)


@pytest.mark.parametrize("bad", BAD_DELTA, ids=str)
def test_delta_shapes_refused(lib, bad):
    cfg = delta(**bad)
    assert forward(lib, cfg) == ab.ONELA_EINVAL
    assert backward(lib, cfg) == ab.ONELA_EINVAL
    assert step(lib, cfg) == ab.ONELA_EINVAL
    assert ab.onela_delta_rule_workspace_bytes(cfg) == 0


def test_lengths_that_do_not_divide_need_offsets(lib):
    cfg = delta(total_tokens=127)
    assert forward(lib, cfg) == ab.ONELA_EINVAL
    assert forward(lib, cfg, off=A, nbytes=0) == ab.ONELA_ECAPACITY
    assert ab.onela_delta_rule_workspace_bytes(cfg) > 0


@pytest.mark.parametrize("call", [forward, backward])
def test_delta_arguments_refused(lib, call):
    cfg = delta()
    need = ab.onela_delta_rule_workspace_bytes(cfg, call is backward)
    assert call(lib, cfg, nbytes=0) == ab.ONELA_ECAPACITY
    assert call(lib, cfg, off=A, nbytes=need - 1) == ab.ONELA_ECAPACITY
    names = ["q", "k", "v", "la", "beta", "ws"]
    names += ["o"] if call is forward else ["do", "dq", "dk", "dv", "dla", "db"]
    for name in names:
        assert call(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
        odd = A + (2 if name in ("la", "beta", "dla", "db") else 128 if name == "ws" else 8)
        assert call(lib, cfg, **{name: odd}) == ab.ONELA_EINVAL, name
    for name in ("s0", "off") + (("last",) if call is forward else ("ds", "ds0")):
        assert call(lib, cfg, **{name: A + 2}) == ab.ONELA_EINVAL, name


def test_step_arguments_refused(lib):
    cfg = delta()
    for name in ("q", "k", "v", "la", "beta", "state", "o"):
        assert step(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
        assert step(lib, cfg, **{name: A + 2}) == ab.ONELA_EINVAL, name
    assert step(lib, cfg, slots=A + 2) == ab.ONELA_EINVAL
    assert step(lib, cfg, num=0) == ab.ONELA_EINVAL
    assert step(lib, cfg, num=1) == ab.ONELA_ECAPACITY
    assert lib.onela_delta_rule_step(None, None, A, A, A, A, A, A, 2, None, A, None) == \
        ab.ONELA_EINVAL


def test_delta_workspace_bytes(lib):
    """Never less for more tokens or sequences, at least a chunk's factors (a triangular
    64 x 64 matrix in two 16-bit parts, twice) per value head and chunk, more for the backward
    pass, and multiples of 256."""
    last = 0
    for seqs, tokens in ((1, 0), (1, 63), (1, 64), (2, 64), (2, 6400), (5, 6400), (5, 64000)):
        cfg = delta(num_seqs=seqs, total_tokens=tokens)
        n, back = (ab.onela_delta_rule_workspace_bytes(cfg, b) for b in (False, True))
        assert n % 256 == 0 and back % 256 == 0 and back > n >= last
        assert n >= (tokens // 64 + seqs) * 4 * 2 * 12288
        last = n


BAD_NORM = [dict(num_tokens=-1), dict(num_tokens=1 << 31), dict(num_q_heads=0),
            dict(num_k_heads=-1), dict(head_dim=4), dict(head_dim=60), dict(head_dim=520),
            dict(rotary_dim=8, table_rows=4), dict(rotary_dim=80, table_rows=4),
            dict(rotary_dim=-16, table_rows=4), dict(rotary_dim=32), dict(io_dtype=3),
            dict(norm=2), dict(rotation=-1), dict(eps=-1.0), dict(eps=float("nan")),
            dict(q_stride=64), dict(k_stride=68), dict(num_q_heads=1 << 30),
            dict(num_tokens=2147483647, num_q_heads=64)]


def rope(lib, cfg, q=A, k=A, wq=None, wk=None, pos=None, cs=None, qo=A, ko=A):
    return lib.onela_qk_norm_rope(ctypes.byref(cfg), q, k, wq, wk, pos, cs, qo, ko, None)


def rope_back(lib, cfg, q=A, k=A, wq=None, wk=None, pos=None, cs=None, dqo=A, dko=A, dq=A, dk=A,
              dwq=None, dwk=None, ws=None, nbytes=0):
    return lib.onela_qk_norm_rope_backward(ctypes.byref(cfg), q, k, wq, wk, pos, cs, dqo, dko, dq,
                                           dk, dwq, dwk, ws, nbytes, None)


@pytest.mark.parametrize("bad", BAD_NORM, ids=str)
def test_norm_shapes_refused(lib, bad):
    cfg = norm(**bad)
    assert rope(lib, cfg, cs=A) == ab.ONELA_EINVAL
    assert rope_back(lib, cfg, cs=A) == ab.ONELA_EINVAL
    assert ab.onela_qk_norm_rope_workspace_bytes(cfg) == 0


def test_norm_arguments_refused(lib):
    cfg = norm()
    for name in ("q", "k", "qo", "ko"):
        assert rope(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
        assert rope(lib, cfg, **{name: A + 8}) == ab.ONELA_EINVAL, name
    for name in ("wq", "wk", "pos", "cs"):
        assert rope(lib, cfg, **{name: A + 2}) == ab.ONELA_EINVAL, name
    for name in ("q", "k", "dqo", "dko", "dq", "dk"):
        assert rope_back(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
        assert rope_back(lib, cfg, **{name: A + 8}) == ab.ONELA_EINVAL, name
    assert rope(lib, norm(rotary_dim=32, table_rows=9)) == ab.ONELA_EINVAL  # no table
    need = ab.onela_qk_norm_rope_workspace_bytes(cfg)
    assert rope_back(lib, cfg, dwq=A) == ab.ONELA_EINVAL
    assert rope_back(lib, cfg, dwk=A, ws=A + 64, nbytes=need) == ab.ONELA_EINVAL
    assert rope_back(lib, cfg, dwq=A, ws=A, nbytes=need - 1) == ab.ONELA_ECAPACITY
    assert rope_back(lib, cfg, dwq=A + 2, ws=A, nbytes=need) == ab.ONELA_EINVAL


def test_binding_refuses_tensors_that_are_not_there():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)  # a CPU tensor
    with pytest.raises(ValueError):
        ab.onela_qk_norm_rope(norm(), x, x, None, None, None, None, x, x, 0)
    with pytest.raises(ValueError):
        ab.onela_qk_norm_rope(norm(q_stride=256), x, x, None, None, None, None, x, x, 0)
    with pytest.raises(ValueError):
        ab.onela_delta_rule_forward(delta(), None, None, A, A, A, A, None, A, A, A, 0, 0)


# Grids of 2^32 threads and more, which the runtime would start with fewer and without an error:
# many chunks of small heads (256 threads a chunk and head), many short sequences of wide ones
# (1024 threads a sequence and head of 512), gradients (512 a chunk and query/key head of 128).
@pytest.mark.parametrize("big", [
    dict(num_seqs=1, total_tokens=(1 << 18) * 64, num_qk_heads=64, num_v_heads=64, d_k=32, d_v=32),
    dict(num_seqs=1 << 16, total_tokens=1 << 16, num_qk_heads=1, num_v_heads=64, d_k=128, d_v=512),
    dict(num_seqs=1 << 17, total_tokens=1 << 17, num_qk_heads=64, num_v_heads=64),
], ids=str)
def test_more_threads_than_a_grid_holds(lib, big):
    cfg = delta(**big)
    assert backward(lib, cfg, off=A) == ab.ONELA_EINVAL
    assert ab.onela_delta_rule_workspace_bytes(cfg, True) == 0
    if cfg.num_seqs == 1 << 17:
        assert ab.onela_delta_rule_workspace_bytes(cfg, False) > 0
    else:
        assert forward(lib, cfg, off=A) == ab.ONELA_EINVAL
        assert ab.onela_delta_rule_workspace_bytes(cfg, False) == 0


def test_step_with_more_threads_than_a_grid_holds(lib):
    cfg = delta(num_seqs=1 << 18, total_tokens=1 << 18, num_qk_heads=1, num_v_heads=32)
    assert step(lib, cfg, num=1 << 18) == ab.ONELA_EINVAL


def test_clear_rest_refused(lib):
    for bad in (2, -1):
        cfg = delta()
        cfg.clear_rest = bad
        assert forward(lib, cfg) == backward(lib, cfg) == step(lib, cfg) == ab.ONELA_EINVAL
        assert ab.onela_delta_rule_workspace_bytes(cfg, False) == 0
    assert step(lib, delta(clear_rest=True)) == ab.ONELA_EINVAL
    assert ab.onela_delta_rule_workspace_bytes(delta(clear_rest=True), True) > 0
