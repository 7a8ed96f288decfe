"""What the short convolution, the norms around a block and the log probabilities refuse before any
device work: configurations, pointers, overlapping tensors (C ABI), and tensors that are not
the object's (runner).  No GPU is needed."""
import ctypes

import pytest

from paper_2609_12399_amd import onela as ab
from paper_2609_12399_amd import runner

A, B, C, D, E, F = (0x10000000 * i for i in range(1, 7))  # aligned addresses far apart; never read


@pytest.fixture(scope="module")
def lib():
    return ab.load_library()



# ---- short causal convolution -----------------------------------------------------------------

def conv_cfg(**kw):
    base = dict(num_seqs=2, total_tokens=10, channels=64, taps=4, io_dtype=ab.ONELA_BF16)
    return ab.make_conv_config(**{**base, **kw})


def conv(lib, cfg, off=None, x=A, w=B, bias=None, s=None, y=C, last=None):
    return lib.onela_short_conv(ctypes.byref(cfg), off, x, w, bias, s, y, last, None)


def conv_back(lib, cfg, off=None, x=A, w=B, bias=None, s=None, dy=C, dlast=None, dx=D, dw=None,
              db=None, ds=None, ws=None, n=0):
    return lib.onela_short_conv_backward(ctypes.byref(cfg), off, x, w, bias, s, dy, dlast, dx, dw,
                                         db, ds, ws, n, None)


def conv_step(lib, cfg, off=None, x=A, w=B, bias=None, s=C, num=2, slots=None, out=None, num_out=0,
              slots_out=None, y=D):
    return lib.onela_short_conv_step(ctypes.byref(cfg), off, x, w, bias, s, num, slots, out,
                                     num_out, slots_out, y, None)


@pytest.mark.parametrize("bad", [
    dict(num_seqs=0), dict(total_tokens=-1), dict(total_tokens=1 << 31), dict(channels=4),
    dict(channels=60), dict(channels=0), dict(taps=1), dict(taps=5), dict(io_dtype=2),
    dict(activation=2), dict(activation=-1), dict(x_stride=56), dict(x_stride=68),
    dict(x_stride=1 << 41), dict(num_seqs=1 << 30, channels=1 << 20),
    dict(channels=(1 << 26) + 8),
    dict(total_tokens=(1 << 31) - 1, num_seqs=1, channels=1 << 20)], ids=str)
def test_conv_shapes_refused(lib, bad):
    cfg = conv_cfg(**bad)
    for call in (conv, conv_back, conv_step):
        assert call(lib, cfg, off=E) == ab.ONELA_EINVAL
    assert ab.onela_short_conv_workspace_bytes(cfg) == 0
    assert conv(lib, conv_cfg(num_seqs=3)) == ab.ONELA_EINVAL  # no offsets: equal lengths


def test_conv_arguments_refused(lib):
    cfg = conv_cfg()
    for name in ("x", "w", "y"):
        assert conv(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
    for name, off in (("x", 8), ("y", 8), ("s", 8), ("last", 4), ("w", 2), ("bias", 2), ("off", 2)):
        assert conv(lib, cfg, **{name: E + off}) == ab.ONELA_EINVAL, name
    # 10 tokens of 64 bf16 channels are 1280 bytes, the states 2 x 3 rows of 128
    assert conv(lib, cfg, y=A) == conv(lib, cfg, y=A + 1264) == ab.ONELA_EINVAL
    assert conv(lib, conv_cfg(x_stride=128), y=A + 9 * 256 + 112) == ab.ONELA_EINVAL
    assert conv(lib, cfg, s=E, last=E + 128) == ab.ONELA_EINVAL
    for name in ("x", "w", "dy", "dx"):
        assert conv_back(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
    for name, off in (("dy", 8), ("dx", 8), ("s", 8), ("dlast", 8), ("ds", 8), ("dw", 2), ("db", 2)):
        assert conv_back(lib, cfg, **{name: E + off}, ws=F, n=1 << 20) == ab.ONELA_EINVAL, name
    assert conv_back(lib, cfg, dx=C) == conv_back(lib, cfg, dx=A + 16) == ab.ONELA_EINVAL
    assert conv_back(lib, cfg, s=E, dlast=F, ds=F) == ab.ONELA_EINVAL
    assert conv_back(lib, cfg, s=E, ds=E + 256) == ab.ONELA_EINVAL
    need = ab.onela_short_conv_workspace_bytes(cfg)
    assert need % 256 == 0 and need >= 5 * 64 * 4
    assert conv_back(lib, cfg, dw=E) == ab.ONELA_EINVAL
    assert conv_back(lib, cfg, db=E, ws=F + 128, n=need) == ab.ONELA_EINVAL
    assert conv_back(lib, cfg, dw=E, ws=F, n=need - 1) == ab.ONELA_ECAPACITY


def test_conv_step_arguments_refused(lib):
    cfg = conv_cfg(total_tokens=2)
    for name in ("x", "w", "s", "y"):
        assert conv_step(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
    for name, off in (("x", 8), ("s", 8), ("y", 8), ("slots", 2)):
        assert conv_step(lib, cfg, **{name: E + off}) == ab.ONELA_EINVAL, name
    assert conv_step(lib, cfg, num=0, slots=E) == ab.ONELA_EINVAL
    assert conv_step(lib, cfg, num=1) == ab.ONELA_ECAPACITY
    assert conv_step(lib, cfg, slots_out=E) == ab.ONELA_EINVAL  # in place there is one slot
    assert conv_step(lib, cfg, out=E) == ab.ONELA_EINVAL
    assert conv_step(lib, cfg, out=E, num_out=1) == ab.ONELA_ECAPACITY
    assert conv_step(lib, cfg, out=E + 8, num_out=2) == ab.ONELA_EINVAL
    # the pools: 2 x 3 rows of 128 bytes each
    for out in (C, C + 640, C - 752):
        assert conv_step(lib, cfg, out=out, num_out=2) == ab.ONELA_EINVAL


# ---- norms around a block -----------------------------------------------------------------------

def norm_cfg(**kw):
    base = dict(num_tokens=4, num_heads=2, width=64, io_dtype=ab.ONELA_BF16,
                residual_dtype=ab.ONELA_F32, norm_after=True, norm_before=True, gate="silu")
    return ab.make_block_norm_config(**{**base, **kw})


def norm(lib, cfg, x=A, gate=B, res=C, wa=None, wb=None, cs=None, y=D, h=E):
    return lib.onela_block_norm(ctypes.byref(cfg), x, gate, res, wa, wb, cs, y, h, None)


def norm_back(lib, cfg, x=A, gate=B, res=C, wa=None, wb=None, cs=None, dy=D, dh=E, dx=F, dg=None,
              dr=None, dwa=None, dwb=None, dcs=None, ws=None, n=0):
    return lib.onela_block_norm_backward(ctypes.byref(cfg), x, gate, res, wa, wb, cs, dy, dh, dx,
                                         dg, dr, dwa, dwb, dcs, ws, n, None)


@pytest.mark.parametrize("bad", [
    dict(num_tokens=-1), dict(num_tokens=1 << 31), dict(num_heads=0), dict(width=0), dict(width=4),
    dict(width=60), dict(width=8200), dict(io_dtype=2), dict(residual_dtype=-1),
    dict(norm_after=2), dict(norm_before=-1), dict(gate=3), dict(gate=-1), dict(x_stride=120),
    dict(x_stride=132), dict(gate_stride=127), dict(gate_stride=1 << 41), dict(eps=-1e-6),
    dict(eps=float("nan")), dict(residual_scale=float("inf")), dict(residual_scale=float("nan")),
    dict(num_tokens=(1 << 31) - 1, num_heads=(1 << 31) - 1)], ids=str)
def test_norm_shapes_refused(lib, bad):
    cfg = norm_cfg(**bad)
    assert norm(lib, cfg) == norm_back(lib, cfg) == ab.ONELA_EINVAL
    assert ab.onela_block_norm_workspace_bytes(cfg) == 0


def test_norm_arguments_refused(lib):
    cfg = norm_cfg()
    assert norm(lib, cfg, x=None) == norm(lib, cfg, gate=None) == ab.ONELA_EINVAL
    assert norm(lib, norm_cfg(gate=None)) == ab.ONELA_EINVAL  # a gate that no one asked for
    assert norm(lib, cfg, y=None, h=None) == ab.ONELA_EINVAL
    assert norm(lib, norm_cfg(norm_after=False), wa=F) == ab.ONELA_EINVAL
    assert norm(lib, norm_cfg(norm_before=False), wb=F) == ab.ONELA_EINVAL
    for name, off in (("x", 8), ("gate", 8), ("res", 8), ("wa", 2), ("wb", 2), ("cs", 2), ("y", 8),
                      ("h", 8)):
        assert norm(lib, cfg, **{name: F + off}) == ab.ONELA_EINVAL, name
    assert norm_back(lib, cfg, dx=None) == norm_back(lib, cfg, dy=None, dh=None) == ab.ONELA_EINVAL
    for name, off in (("dy", 8), ("dh", 8), ("dx", 8), ("dg", 8), ("dr", 8), ("dwa", 2),
                      ("dwb", 2), ("dcs", 2)):
        assert norm_back(lib, cfg, **{name: F + off}, ws=F, n=1 << 30) == ab.ONELA_EINVAL, name
    bare = norm_cfg(gate=None, norm_after=False)
    assert norm_back(lib, bare, gate=None, dg=F) == ab.ONELA_EINVAL
    assert norm_back(lib, bare, gate=None, dwa=F, ws=F, n=1 << 30) == ab.ONELA_EINVAL
    need = ab.onela_block_norm_workspace_bytes(cfg)
    assert need >= 3 * 64 * 4
    for name in ("dwa", "dwb", "dcs"):
        assert norm_back(lib, cfg, **{name: A}) == ab.ONELA_EINVAL
        assert norm_back(lib, cfg, **{name: A}, ws=F + 64, n=need) == ab.ONELA_EINVAL
        assert norm_back(lib, cfg, **{name: A}, ws=F, n=need - 1) == ab.ONELA_ECAPACITY


# ---- log probabilities ----------------------------------------------------------------------------

def logp_cfg(**kw):
    base = dict(num_rows=4, vocab=100, num_given=2, num_top=3, io_dtype=ab.ONELA_BF16)
    return ab.make_logprob_config(**{**base, **kw})


def logp(lib, cfg, x=A, given=B, lp=C, lse=D, ent=None, top=E, topl=F, ws=A, n=1 << 30):
    return lib.onela_token_logprobs(ctypes.byref(cfg), x, given, lp, lse, ent, top, topl, ws, n,
                                    None)


def logp_back(lib, cfg, x=A, given=B, lse=C, ent=None, dl=D, dlse=None, dent=None, dx=E):
    return lib.onela_token_logprobs_backward(ctypes.byref(cfg), x, given, lse, ent, dl, dlse, dent,
                                             dx, None)


@pytest.mark.parametrize("bad", [
    dict(num_rows=-1), dict(num_rows=1 << 31), dict(vocab=0), dict(vocab=1 << 28),
    dict(num_given=-1), dict(num_given=257), dict(num_top=-1), dict(num_top=65),
    dict(vocab=5, num_top=6), dict(io_dtype=-1), dict(logits_stride=99), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=2e30),
    dict(logits_stride=1 << 41), dict(num_rows=1 << 24), dict(num_rows=1 << 20, vocab=1 << 17)],
    ids=str)
def test_logprob_shapes_refused(lib, bad):
    cfg = logp_cfg(**bad)
    assert logp(lib, cfg) == logp_back(lib, cfg) == ab.ONELA_EINVAL
    assert ab.onela_token_logprobs_workspace_bytes(cfg) == 0


def test_logprob_arguments_refused(lib):
    cfg = logp_cfg()
    for name in ("x", "given", "lp", "top", "topl", "ws"):
        assert logp(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
    for name, off in (("x", 1), ("given", 2), ("lp", 2), ("lse", 2), ("ent", 2), ("top", 2),
                      ("topl", 2), ("ws", 128)):
        assert logp(lib, cfg, **{name: F + off}) == ab.ONELA_EINVAL, name
    assert logp(lib, logp_cfg(io_dtype=ab.ONELA_F32), x=A + 2) == ab.ONELA_EINVAL
    need = ab.onela_token_logprobs_workspace_bytes(cfg)
    assert need >= 256 and logp(lib, cfg, n=need - 1) == ab.ONELA_ECAPACITY
    for name in ("x", "given", "lse", "dl", "dx"):
        assert logp_back(lib, cfg, **{name: None}) == ab.ONELA_EINVAL, name
    for name, off in (("x", 1), ("given", 2), ("lse", 2), ("ent", 2), ("dl", 2), ("dlse", 2),
                      ("dent", 2), ("dx", 1)):
        assert logp_back(lib, cfg, **{name: F + off}) == ab.ONELA_EINVAL, name
    assert logp_back(lib, cfg, dent=F) == ab.ONELA_EINVAL  # without the entropy
    # 4 rows of 100 bf16: over the logits only where those are dense
    assert logp_back(lib, cfg, dx=A + 798) == logp_back(lib, cfg, dx=A - 2) == ab.ONELA_EINVAL
    assert logp_back(lib, logp_cfg(logits_stride=104), dx=A) == ab.ONELA_EINVAL


def test_workspace_of_parts(lib):
    """Few long rows are worked on in parts; the workspace holds every part's sums and best."""
    for rows, vocab, top in ((1, 131072, 64), (3, 131072, 0), (200, 50001, 8)):
        n = ab.onela_token_logprobs_workspace_bytes(logp_cfg(num_rows=rows, vocab=vocab,
                                                             num_top=top))
        assert n % 256 == 0 and n >= rows * (16 + 8 * top)


# ---- the runner's objects ---------------------------------------------------------------------------

torch = pytest.importorskip("torch")
BF, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


@pytest.fixture
def entries(monkeypatch):
    """The entry points, called with anything, write down that they were."""
    calls = []
    for name in ("onela_short_conv", "onela_short_conv_backward", "onela_short_conv_step",
                 "onela_block_norm", "onela_block_norm_backward", "onela_token_logprobs",
                 "onela_token_logprobs_backward"):
        monkeypatch.setattr(ab, name, lambda *a, name=name, **k: calls.append(name))
    return calls


def refuses(call, good, bad):
    for name, shape, dtype in bad:
        with pytest.raises(ValueError, match=name):
            call(**{**good, name: torch.zeros(shape, dtype=dtype)})


def test_conv_objects_refuse(entries):
    rows = torch.zeros(10, 64, dtype=BF)
    good = dict(x=rows, weight=torch.zeros(64, 4), bias=torch.zeros(64),
                seq_offsets=torch.zeros(3, dtype=I32), initial_state=torch.zeros(2, 3, 64, dtype=BF))
    bad = [("x", (10, 64), F32), ("x", (9, 64), BF), ("x", (640,), BF), ("weight", (64, 4), BF),
           ("weight", (4, 64), F32), ("bias", (64,), BF), ("bias", (4,), F32),
           ("seq_offsets", (3,), I64), ("seq_offsets", (2,), I32),
           ("initial_state", (2, 3, 64), F32), ("initial_state", (2, 4, 64), BF)]
    op, back = (runner.ShortConv(2, 10, 64, 4, "bf16", backward=b, device="cpu")
                for b in (False, True))
    refuses(op.forward, good, bad)
    refuses(back.backward, dict(good, d_y=rows), bad + [("d_y", (10, 64), F32),
                                                       ("d_final_state", (2, 3, 64), F32)])
    step = runner.ShortConvStep(10, 10, 64, 4, "bf16", 12, device="cpu")
    pool = torch.zeros(12, 3, 64, dtype=BF)
    some = dict(good, pool=pool, slots=torch.zeros(10, dtype=I32), seq_offsets=None)
    del some["initial_state"]
    refuses(step.step, some, [*bad[:7], ("slots", (10,), I64), ("slots", (9,), I32),
                              ("pool", (12, 3, 64), F32), ("pool", (11, 3, 64), BF),
                              ("pool_out", (12, 2, 64), BF), ("slots_out", (10,), I64)])
    with pytest.raises(ValueError, match="backward"):
        back.forward(**good)
    with pytest.raises(ValueError, match="forward"):
        op.backward(**good, d_y=rows)
    assert entries == []
    op.forward(**good)
    back.backward(**good, d_y=rows)
    step.step(**{**some, "pool": torch.zeros(15, 3, 64, dtype=BF)}, pool_out=pool)
    assert len(entries) == 3


def test_norm_objects_refuse(entries):
    x = torch.zeros(4, 2, 64, dtype=BF)
    good = dict(x=x, residual=torch.zeros(4, 2, 64), gate=x, after_weight=torch.zeros(64),
                before_weight=torch.zeros(64), channel_scale=torch.zeros(64))
    bad = [("x", (4, 2, 64), F32), ("x", (4, 128), BF), ("gate", (4, 2, 64), F32),
           ("gate", (4, 1, 64), BF), ("residual", (4, 2, 64), BF), ("residual", (8, 64), F32),
           ("after_weight", (64,), BF), ("before_weight", (2, 64), F32),
           ("channel_scale", (128,), F32)]
    op, back = (runner.BlockNorm(4, 64, 2, "bf16", "f32", True, True, "silu", backward=b,
                                 device="cpu") for b in (False, True))
    refuses(op.forward, good, bad)
    refuses(back.backward, dict(good, d_y=x), bad + [("d_y", (4, 2, 64), F32),
                                                    ("d_residual_out", (4, 2, 64), BF)])
    with pytest.raises(ValueError, match="gate"):
        op.forward(**{**good, "gate": None})
    with pytest.raises(ValueError, match="gate"):
        runner.BlockNorm(4, 64, 2, "bf16", "f32", True, device="cpu").forward(**good)
    assert entries == []
    op.forward(**good)
    back.backward(**good, d_y=x)
    assert len(entries) == 2


def test_logprob_objects_refuse(entries):
    x, given = torch.zeros(4, 100, dtype=BF), torch.zeros(4, 2, dtype=I32)
    op, back = (runner.TokenLogprobs(4, 100, 2, 3, "bf16", entropy=True, backward=b, device="cpu")
                for b in (False, True))
    bad = [("logits", (4, 100), F32), ("logits", (4, 99), BF), ("given", (4, 2), I64),
           ("given", (4,), I32)]
    refuses(op.forward, dict(logits=x, given=given), bad)
    good = dict(logits=x, given=given, lse=torch.zeros(4), d_logp=torch.zeros(4, 2))
    refuses(back.backward, good, bad + [("lse", (4, 1), F32), ("d_logp", (4, 2), BF),
                                        ("d_lse", (3,), F32), ("entropy", (4,), BF),
                                        ("d_entropy", (5,), F32), ("out", (4, 100), F32)])
    with pytest.raises(ValueError, match="given"):
        op.forward(x)
    with pytest.raises(ValueError, match="given"):
        runner.TokenLogprobs(4, 100, 0, 3, "bf16", device="cpu").forward(x, given[:, :0])
    assert entries == []
    op.forward(x, given)
    back.backward(**good)
    assert len(entries) == 2


@pytest.mark.parametrize("make", [
    lambda: runner.ShortConv(1, 4, 12, 4, device="cpu"),
    lambda: runner.BlockNorm(4, 8200, device="cpu"),
    lambda: runner.TokenLogprobs(4, 10, num_top=11, device="cpu")])
def test_objects_of_refused_sizes(make):
    with pytest.raises(ab.OnelaError):
        make()


class OnGpu:
    """What the checks look at of a tensor on GPU `at`."""
    is_cuda = True

    def __init__(self, like, at):
        self.dtype, self.shape, self.device = like.dtype, like.shape, f"cuda:{at}"
        self.get_device, self.is_contiguous = (lambda: at), (lambda: True)


def test_tensors_on_other_devices_are_refused(entries, monkeypatch):
    x, w, dy = torch.zeros(4, 64, dtype=BF), torch.zeros(64), torch.zeros(4, 64, dtype=BF)
    ids, rows = torch.zeros(4, dtype=I32), torch.zeros(4, 1, dtype=I32)
    heads, lse, pool = x[:, None], torch.zeros(4), torch.zeros(5, 3, 64, dtype=BF)
    conv = dict(x=x, weight=torch.zeros(64, 4), bias=w, seq_offsets=ids[:2],
                initial_state=pool[:1])
    norm = dict(x=heads, residual=heads, gate=heads, after_weight=w, before_weight=w,
                channel_scale=w)
    step = dict(x=x, weight=conv["weight"], pool=pool, slots=ids)
    convs, norms, probs = ([make(b) for b in (False, True)] for make in (
        lambda b: runner.ShortConv(1, 4, 64, 4, "bf16", backward=b, device="cpu"),
        lambda b: runner.BlockNorm(4, 64, 1, "bf16", norm_after=True, gate="silu", backward=b,
                                   device="cpu"),
        lambda b: runner.TokenLogprobs(4, 64, 1, 0, "bf16", backward=b, device="cpu")))
    steps = runner.ShortConvStep(4, 4, 64, 4, "bf16", 5, device="cpu")
    calls = [(convs[0], "forward", conv), (convs[1], "backward", dict(conv, d_y=dy)),
             (convs[1], "backward", dict(conv, d_y=dy, d_final_state=pool[:1])),
             (norms[0], "forward", norm), (norms[1], "backward", dict(norm, d_y=heads)),
             (norms[1], "backward", dict(norm, d_y=heads, d_residual_out=heads)),
             (probs[0], "forward", dict(logits=x, given=rows)),
             (probs[1], "backward", dict(logits=x, given=rows, lse=lse,
                                         d_logp=torch.zeros(4, 1), d_lse=lse, out=x)),
             (steps, "step", step), (steps, "step", dict(step, pool_out=pool, slots_out=ids))]
    for op in (*convs, *norms, *probs, steps):
        op.on = 0
    for current in (0, 1):
        monkeypatch.setattr(ab, "current_device", lambda: current)
        for op, name, args in calls:
            here = {k: OnGpu(v, 0) for k, v in args.items()}
            for k, v in args.items():
                with pytest.raises(ValueError, match="current device"):
                    getattr(op, name)(**{**here, k: OnGpu(v, 1)})
            if current == 1:  # (the object and its tensors on another device than the current one)
                with pytest.raises(ValueError, match="current device"):
                    getattr(op, name)(**here)
    assert entries == []


# ---- the functions and layers on them -----------------------------------------------------------------

mixer = pytest.importorskip("paper_2609_12399_amd.mixer")


def test_second_derivatives_are_refused(entries):
    x, w = torch.randn(6, 16, requires_grad=True), torch.randn(16, 4, requires_grad=True)
    outs = [mixer.ShortConvFunction.apply(x, w, None, None, None, 2, "silu")[0],
            mixer.BlockNormFunction.apply(x[:, None], x[:, None], None, None, None, None, True, True,
                                          None, 1.0, 1e-6)[0],
            mixer.TokenLogprobsFunction.apply(x, None, 0, 1.0, True)[2]]
    for y in outs:
        dx, = torch.autograd.grad(y.sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once"):
            (dx.square().sum() + x.sum()).backward()


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_layer_with_convolution_and_gates_under_autocast(entries, monkeypatch, io):
    """The operators take what the autocast products give; states and gates go with them."""
    for name in ("onela_delta_rule_forward", "onela_delta_rule_step", "onela_qk_norm_rope"):
        monkeypatch.setattr(ab, name, lambda *a, name=name, **k: entries.append(name))
    layer = mixer.DeltaMixer(16, 1, 2, 32, 32, io, device="cpu", conv_taps=3, gated=True)
    x = torch.randn(6, 16).to(layer.w_qkv.dtype)
    off = torch.tensor([0, 2, 6], dtype=I32)
    with torch.autocast("cpu", dtype=BF):
        y, (state, conv) = layer.prompt(x, off)
        assert conv.shape == (2, 2, layer.qkv_width) and conv.dtype is BF
        layer.prompt(x, off, None, (state, conv))
        layer.step(x[:2], (state, conv), torch.zeros(2, dtype=I32))
        beams = mixer.BeamStates(conv)
        layer.beam_step_inputs(x.unflatten(0, (2, 3)), None, None, beams)
        assert beams.conv.shape == (6, 2, layer.qkv_width)
        layer.beam_step_inputs(x.unflatten(0, (2, 3)), torch.zeros(2, 3, dtype=I32), None, beams)
        layer.beam_outputs(torch.zeros(2, 3, 2, 32), beams)
    prompt = ["onela_short_conv", "onela_qk_norm_rope", "onela_delta_rule_forward",
              "onela_block_norm"]
    step = ["onela_short_conv_step", "onela_qk_norm_rope"]
    assert entries == [*prompt, *prompt, *step, "onela_delta_rule_step", "onela_block_norm", *step,
                       *step, "onela_block_norm"]


def test_recommender_on_the_entry_points(entries, monkeypatch):
    """One training step calls, per layer, the convolution, the norm, the delta rule and two
    block norms, and the log probabilities once, each with its gradient."""
    recommender = pytest.importorskip("paper_2609_12399_amd.recommender")
    for name in ("onela_delta_rule_forward", "onela_delta_rule_backward", "onela_qk_norm_rope",
                 "onela_qk_norm_rope_backward"):
        monkeypatch.setattr(ab, name, lambda *a, name=name, **k: entries.append(name))
    model = recommender.Recommender(20, 16, 2, 1, 2, 32, "f32", device="cpu")
    off = torch.tensor([0, 2, 6], dtype=I32)
    model.loss(torch.arange(6), torch.arange(6).int(), off).backward()
    assert all(w.grad is not None and w.grad.shape == w.shape for w in model.weights())
    for name, n in (("onela_short_conv", 2), ("onela_short_conv_backward", 2),
                    ("onela_block_norm", 5), ("onela_block_norm_backward", 5),
                    ("onela_token_logprobs", 1), ("onela_token_logprobs_backward", 1),
                    ("onela_delta_rule_backward", 2)):
        assert entries.count(name) == n, name


@pytest.mark.parametrize("bounds,steps", [([0, 3, 3], 2), ([0, 0, 3], 2), ([0, 2, 3], 0)])
def test_search_refuses_empty_prompts(bounds, steps):
    recommender = pytest.importorskip("paper_2609_12399_amd.recommender")
    model = recommender.Recommender(20, 16, 2, 1, 2, 32, "f32", device="cpu")
    with pytest.raises(ValueError, match="one token"):
        model.search(torch.zeros(3, dtype=I64), torch.tensor(bounds, dtype=I32), 4, steps)


def test_norm_overlaps_refused(lib):
    """4 tokens of 2 x 64 bf16 are 1024 bytes, the residual in fp32 2048, a weight's vector 256."""
    cfg, wide = norm_cfg(), norm_cfg(x_stride=256, gate_stride=256)
    for out in ("y", "h"):
        for at in (A + 16, A - 16, B + 1008, C + 2032, C - 16):
            assert norm(lib, cfg, **{out: at}) == ab.ONELA_EINVAL, (out, at)
        # between the rows of a wider x or gate, and in their place
        for at in (A + 256, B + 3 * 512, A, B):
            assert norm(lib, wide, **{out: at}) == ab.ONELA_EINVAL, (out, at)
    assert norm(lib, cfg, h=A) == norm(lib, cfg, y=C) == ab.ONELA_EINVAL  # of another type
    assert norm(lib, cfg, y=D, h=D) == norm(lib, cfg, y=D, h=D + 1008) == ab.ONELA_EINVAL
    for name in ("wa", "wb", "cs"):
        assert norm(lib, cfg, **{name: D + 512}) == norm(lib, cfg, **{name: E - 240}) == ab.ONELA_EINVAL
    need = ab.onela_block_norm_workspace_bytes(cfg)
    far = 0x70000000
    for out in ("dx", "dg", "dr"):
        for at in (A + 16, B - 16, C + 2032, D + 1008, E - 16):
            assert norm_back(lib, cfg, **{out: at}) == ab.ONELA_EINVAL, (out, at)
        for at in (A + 256, B + 3 * 512):
            assert norm_back(lib, wide, **{out: at}) == ab.ONELA_EINVAL, (out, at)
    assert norm_back(lib, cfg, dr=D) == norm_back(lib, cfg, dx=E) == ab.ONELA_EINVAL
    assert norm_back(lib, cfg, dg=F) == norm_back(lib, cfg, dg=F + 1008) == ab.ONELA_EINVAL
    assert norm_back(lib, cfg, dr=F - 2032) == ab.ONELA_EINVAL
    for name in ("dwa", "dwb", "dcs"):
        for at in (A, D + 512, F + 1020):
            assert norm_back(lib, cfg, **{name: at}, ws=far, n=need) == ab.ONELA_EINVAL, (name, at)
    for ws in (A, F, F - need + 256):
        assert norm_back(lib, cfg, dwa=far, ws=ws, n=need) == ab.ONELA_EINVAL, ws
    assert norm_back(lib, cfg, dwa=far, dwb=far + 128, ws=far + 4096, n=need) == ab.ONELA_EINVAL
    assert norm_back(lib, cfg, dwa=far + 8192, ws=far, n=need) == ab.ONELA_EINVAL


def test_conv_overlaps_refused(lib):
    """10 tokens of 64 bf16 channels are 1280 bytes, the states 768, the weights 1024, offsets 12."""
    cfg, far = conv_cfg(), 0x70000000
    for at in (A, A + 1264, A - 752, B + 1008, C + 16, C - 752):
        assert conv(lib, cfg, last=at) == ab.ONELA_EINVAL, at
    for at in (B, B - 1264, E, E - 512, F, F + 752):
        assert conv(lib, cfg, off=E, s=F, y=at) == ab.ONELA_EINVAL, at
    assert conv(lib, cfg, bias=C + 128) == conv(lib, cfg, s=C, last=C) == ab.ONELA_EINVAL
    assert conv(lib, cfg, off=E, last=E) == conv(lib, cfg, s=E, last=E + 752) == ab.ONELA_EINVAL
    need = ab.onela_short_conv_workspace_bytes(cfg)
    grads = dict(s=E, dlast=F, dw=far, db=far + 4096, ds=far + 8192, ws=far + 65536, n=need)
    for name in ("dx", "ds", "dw", "db"):
        for at in (A, A + 1264, C + 16, E, F + 752):
            assert conv_back(lib, cfg, **{**grads, name: at}) == ab.ONELA_EINVAL, (name, at)
    for name in ("dx", "ds"):
        assert conv_back(lib, cfg, **{**grads, name: B}) == ab.ONELA_EINVAL, name
        assert conv_back(lib, cfg, bias=far + 512, **{**grads, "dw": None, name: far + 256}) == \
            ab.ONELA_EINVAL
    assert conv_back(lib, cfg, **{**grads, "dw": B + 512}) == ab.ONELA_EINVAL
    assert conv_back(lib, cfg, **{**grads, "db": far + 1020}) == ab.ONELA_EINVAL
    for ws in (A, B, D, far + 8192 - 256):
        assert conv_back(lib, cfg, **{**grads, "ws": ws}) == ab.ONELA_EINVAL, ws
    assert conv_back(lib, cfg, off=far, **grads) == ab.ONELA_EINVAL
    cfg = conv_cfg(total_tokens=2)  # 256 bytes, pools of two slots 768
    for y in (A + 16, A - 240, B, B + 1008, C, C + 752, E, F):
        assert conv_step(lib, cfg, slots=E, out=F, num_out=2, y=y) == ab.ONELA_EINVAL, y
    assert conv_step(lib, conv_cfg(total_tokens=2, x_stride=128), y=A) == ab.ONELA_EINVAL
    for at in (A, A - 752, B + 16, E):
        assert conv_step(lib, cfg, slots=E, s=at) == ab.ONELA_EINVAL, at
        assert conv_step(lib, cfg, slots=E, out=at, num_out=2) == ab.ONELA_EINVAL, at
    assert conv_step(lib, cfg, out=F, num_out=2, slots_out=F + 16) == ab.ONELA_EINVAL
    assert conv_step(lib, cfg, y=B, bias=B + 240, w=E) == ab.ONELA_EINVAL


def test_logprob_overlaps_refused(lib):
    """4 rows: logits 800 bytes, 2 given tokens 32, the 3 best 48, a number for each row 16."""
    cfg, far = logp_cfg(), 0x70000000
    base = dict(x=A, given=B, lp=C, lse=D, ent=far, top=E, topl=F, ws=far + 4096)
    sizes = dict(lp=32, lse=16, ent=16, top=48, topl=48)
    for name, n in sizes.items():
        for at in (A + 796, A - n + 4, B + 28, B - n + 4):
            assert logp(lib, cfg, **{**base, name: at}) == ab.ONELA_EINVAL, (name, at)
        for other, m in sizes.items():
            if other != name:
                at = base[other]
                assert logp(lib, cfg, **{**base, name: at + m - 4}) == ab.ONELA_EINVAL, (name, other)
    parts = logp_cfg(num_rows=1, vocab=131072, num_top=0, num_given=0)
    need = ab.onela_token_logprobs_workspace_bytes(parts)
    for ws in (A, A + 262144 - 256, D):
        assert logp(lib, parts, ws=ws, n=need) == ab.ONELA_EINVAL, ws
    for name, n in (("given", 32), ("lse", 16), ("ent", 16), ("dl", 32), ("dlse", 16), ("dent", 16)):
        for at in (E, E + 796, E - n + 4):
            assert logp_back(lib, cfg, **{**dict(ent=F, dlse=far, dent=far + 256), name: at}) == \
                ab.ONELA_EINVAL, (name, at)


def test_scores_for_logits():
    inf = float("inf")
    lse = torch.tensor([2.0, -inf, -inf, 1.0, float("nan")])
    score = torch.tensor([1.0, -3.0, -inf, -inf, 0.0])
    logits = torch.tensor([[1.5, -inf], [-inf, -inf], [-inf, -inf], [0.0, -inf], [0.0, 0.0]])
    got = runner.scores_for_logits(score, lse)[:, None] + logits
    assert torch.equal(got[:4], torch.tensor([[0.5, -inf]] + [[-inf, -inf]] * 3))
    assert bool(got[4].isnan().all())
    assert runner.scores_for_logits(None, lse[:1]).tolist() == [-2.0]


def test_conv_clear_rest_refused(lib):
    for bad in (2, -1):
        cfg = conv_cfg()
        cfg.clear_rest = bad
        for call in (conv, conv_back, conv_step):
            assert call(lib, cfg, off=E) == ab.ONELA_EINVAL
        assert ab.onela_short_conv_workspace_bytes(cfg) == 0
    assert conv_step(lib, conv_cfg(total_tokens=2, clear_rest=True)) == ab.ONELA_EINVAL
    assert ab.onela_short_conv_workspace_bytes(conv_cfg(clear_rest=True)) > 0
