"""The delta rule over whole sequences, its gradient and its recurrent step, through the C
ABI, against the 64-bit recurrence.

Metrics, per value (or query/key) head: the largest error over the largest reference value.
Bars, from the arithmetic:
  fp32 results (states, gradients by beta and log(alpha), all of fp32 tensors): every
  product of operands is exact to 2^-24 of its largest factor and sums run in fp32, so that
  a chunk contributes some tens of 2^-24 and later chunks shrink what earlier ones
  left: 4e-6 (64 x 2^-24).  The gradient by log(alpha) sums up to 64 tokens' terms that cancel:
  four times that.
  bf16 results: one rounding, 2^-8 of the value itself, plus two-part operands, 2^-17 of
  each of up to 8 comparable terms: 2^-8 |value| + 6.1e-5 of the largest."""
import numpy as np
import pytest

from paper_2609_12399_amd import onela as ab
from paper_2609_12399_amd import runner
from tests import delta_reference as ref
from tests.gpu_common import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"
F32, SUMS = 4e-6, 1.6e-5


def draw(lengths, HK, HV, dk, dv, io, seed=0, alpha_mu=-3.0):
    """q, k, v, log_alpha, beta on the device (bits that both sides read)."""
    g = torch.Generator().manual_seed(seed)
    n, dt = sum(lengths), torch.bfloat16 if io == "bf16" else torch.float32

    def unit(h):
        x = torch.randn((n, h, dk), generator=g)
        return (x / x.norm(dim=-1, keepdim=True)).to(dt)

    x = [unit(HK), unit(HK), torch.randn((n, HV, dv), generator=g).to(dt),
         -torch.nn.functional.softplus(torch.randn((n, HV), generator=g) + alpha_mu),
         torch.sigmoid(torch.randn((n, HV), generator=g))]
    return [t.to(DEV) for t in x], g


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def offsets(lengths):
    return torch.tensor(ref.bounds(lengths), dtype=torch.int32, device=DEV)


def head_err(got, want, axis):
    """Largest error over the largest value, per head."""
    got, want = np.moveaxis(f64(got), axis, 0), np.moveaxis(want, axis, 0)
    if not want.size:
        return 0.0
    got, want = got.reshape(got.shape[0], -1), want.reshape(want.shape[0], -1)
    assert np.isfinite(got).all()
    return float((np.abs(got - want).max(1) / np.maximum(np.abs(want).max(1), 1e-30)).max())


def check(name, got, want, axis, io="f32", bar=F32):
    if io == "bf16":
        g, w = np.moveaxis(f64(got), axis, 0), np.moveaxis(want, axis, 0)
        if not w.size:
            return
        big = np.abs(w).reshape(w.shape[0], -1).max(1).reshape(-1, *[1] * (w.ndim - 1))
        over = np.abs(g - w) - 2.0 ** -8 * np.abs(w) - 6.1e-5 * big
        assert np.isfinite(g).all() and over.max() <= 0, (name, float(over.max()))
        return
    err = head_err(got, want, axis)
    log(f"[delta] {name} {err:.2e}")
    assert err <= bar, (name, err)


def op_of(lengths, HK, HV, dk, dv, io, scale, backward=False):
    return runner.DeltaRule(len(lengths), sum(lengths), HK, HV, dk, dv, io, scale, backward, DEV)


def run_both(lengths, HK, HV, dk, dv, io, seed=0, state=True, scale=None, equal=False,
             tweak=None, alpha_mu=-3.0):
    x, g = draw(lengths, HK, HV, dk, dv, io, seed, alpha_mu)
    if tweak:
        tweak(x)
    N, n = len(lengths), sum(lengths)
    scale = dk ** -0.5 if scale is None else scale
    s0 = torch.randn((N, HV, dv, dk), generator=g).to(DEV) if state else None
    ds = torch.randn((N, HV, dv, dk), generator=g).to(DEV) if state else None
    do = torch.randn((n, HV, dv), generator=g).to(x[2].dtype).to(DEV)
    off = None if equal else offsets(lengths)
    host = [f64(t) for t in x]
    o, last, _ = ref.forward(lengths, *host, scale, f64(s0))
    want = ref.backward(lengths, *host, scale, f64(s0), f64(do), f64(ds))
    fo, fs = op_of(lengths, HK, HV, dk, dv, io, scale).forward(*x, off, s0)
    got = op_of(lengths, HK, HV, dk, dv, io, scale, True).backward(*x, do, off, s0, ds)
    torch.cuda.synchronize()
    check("o", fo, o, 1, io)
    check("final state", fs, last, 1)
    for name, a, w in zip(("dq", "dk", "dv"), got[:3], want[:3]):
        check(name, a, w, 1, io)
    check("dlog_alpha", got[3], want[3], 1, bar=SUMS)
    check("dbeta", got[4], want[4], 1)
    if state:
        check("d initial state", got[5], want[5], 1)
    else:
        assert got[5] is None


@pytest.mark.parametrize("lengths", [[1], [2], [63], [64], [65], [200], [0, 5, 0, 130, 1, 64, 0],
                                     [127, 129]])
def test_lengths(lengths):
    run_both(lengths, 2, 4, 64, 64, "bf16", seed=sum(lengths))


@pytest.mark.parametrize("HK,HV,dk,dv,io", [
    (1, 1, 32, 32, "f32"), (2, 2, 32, 32, "bf16"), (2, 2, 64, 64, "f32"), (1, 3, 64, 64, "bf16"),
    (2, 4, 128, 128, "f32"), (2, 4, 128, 128, "bf16"), (1, 2, 128, 256, "bf16"),
    (1, 1, 128, 512, "bf16"), (2, 2, 256, 256, "bf16"), (1, 2, 256, 512, "bf16")])
def test_geometries(HK, HV, dk, dv, io):
    run_both([70, 3, 131], HK, HV, dk, dv, io, seed=dk + dv)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_equal_lengths_without_offsets_and_states(io):
    run_both([90, 90, 90], 2, 2, 64, 64, io, state=False, equal=True, scale=1.0)


def test_many_sequences():
    """More sequences than a wave has lanes: the slot's sequence is found in blocks."""
    r = np.random.default_rng(3)
    run_both([int(x) for x in r.integers(0, 9, 150)], 1, 2, 32, 32, "f32")


def test_long_memory():
    """Decays near 1 over many chunks."""
    run_both([700], 1, 2, 64, 64, "f32", alpha_mu=-7.0)


def test_vanishing_decays():
    """alpha = 0 (log -inf), e^-200 and e^-40 among ordinary ones: no 0 / 0, the decays
    after them keep their precision, and the gradient by such a log_alpha is 0."""
    def tweak(x):
        x[3][[0, 5, 70, 71, 127]] = float("-inf")
        x[3][[10, 80]] = -200.0
        x[3][[20, 100]] = -40.0
        x[3][30] = -3e5
    run_both([130, 20], 1, 2, 64, 64, "f32", tweak=tweak)
    run_both([130, 20], 1, 2, 64, 64, "bf16", tweak=tweak)


def test_gates_at_their_ends():
    """beta = 0 (nothing is written; its gradient is not), beta = 1 and alpha = 1."""
    def tweak(x):
        x[4][::3] = 0.0
        x[4][1::3] = 1.0
        x[3][::2] = 0.0
    run_both([100], 2, 2, 32, 32, "f32", tweak=tweak)


def test_repeated_keys():
    """The same key at every token: the chunk's triangular system is as full as it gets."""
    def tweak(x):
        x[1][:] = x[1][:1]
    run_both([100], 2, 2, 64, 64, "bf16", tweak=tweak)


def test_views_into_wider_rows():
    """q, k and v as slices of one projection's output."""
    n, HK, HV, d = 150, 2, 4, 64
    x, g = draw([n], HK, HV, d, d, "bf16")
    wide = torch.full((n, 2 * HK * d + HV * d + 8), float("nan"), dtype=torch.bfloat16, device=DEV)
    q, k = wide[:, :HK * d].view(n, HK, d), wide[:, HK * d:2 * HK * d].view(n, HK, d)
    v = wide[:, 2 * HK * d:2 * HK * d + HV * d].view(n, HV, d)
    q.copy_(x[0]), k.copy_(x[1]), v.copy_(x[2])
    do = torch.randn((n, HV, d), generator=g).bfloat16().to(DEV)
    for back in (False, True):
        a, b = (op_of([n], HK, HV, d, d, "bf16", 1.0, back) for _ in range(2))
        if back:
            ra, rb = a.backward(*x, do), b.backward(q, k, v, *x[3:], do)
        else:
            ra, rb = a.forward(*x), b.forward(q, k, v, *x[3:])
        for s, t in zip(ra, rb):
            assert (s is None and t is None) or torch.equal(s, t)


def test_state_in_place_and_split_sequence():
    """A sequence cut at any token, the state handed on in place, gives the whole's
    outputs to the bars' sum."""
    n, HK, HV, d = 200, 1, 2, 128
    x, g = draw([n], HK, HV, d, d, "f32")
    s0 = torch.randn((1, HV, d, d), generator=g).to(DEV)
    o, last = op_of([n], HK, HV, d, d, "f32", 1.0).forward(*x, None, s0)
    for cut in (1, 64, 131):
        state, outs = s0.clone(), []
        for a, b in ((0, cut), (cut, n)):
            op = op_of([b - a], HK, HV, d, d, "f32", 1.0)
            op.final_state = state
            outs.append(op.forward(*[t[a:b] for t in x], None, state)[0])
        check("o", torch.cat(outs), f64(o), 1, bar=2 * F32)
        check("state", state, f64(last), 1, bar=2 * F32)


def test_no_final_state_wanted_and_no_tokens():
    x, g = draw([0, 0], 1, 2, 64, 64, "bf16")
    s0 = torch.randn((2, 2, 64, 64), generator=g).to(DEV)
    for off in (None, offsets([0, 0])):
        cfg = ab.make_delta_config(2, 0, 1, 2, 64, 64, "bf16")
        last = torch.full_like(s0, float("nan"))
        nbytes = ab.onela_delta_rule_workspace_bytes(cfg)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
        ab.onela_delta_rule_forward(cfg, off, *x, s0, None, last, ws, nbytes)
        assert torch.equal(last, s0)
        ds = torch.full_like(s0, float("nan"))
        nbytes = ab.onela_delta_rule_workspace_bytes(cfg, True)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
        ab.onela_delta_rule_backward(cfg, off, *x, s0, None, s0, None, None, None, None, None, ds,
                                     ws, nbytes)
        assert torch.equal(ds, s0)
    x, _ = draw([70], 1, 2, 64, 64, "bf16")
    cfg = ab.make_delta_config(1, 70, 1, 2, 64, 64, "bf16")
    nbytes = ab.onela_delta_rule_workspace_bytes(cfg)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    o = torch.empty_like(x[2])
    ab.onela_delta_rule_forward(cfg, None, *x, None, o, None, ws, nbytes)
    assert torch.equal(o, op_of([70], 1, 2, 64, 64, "bf16", 1.0).forward(*x)[0])


def test_offsets_that_leave_tokens_out():
    """Offsets that do not rise, or leave the tokens, are cut to them: the call ends, and
    sequences that are in order are right."""
    x, _ = draw([300], 1, 2, 32, 32, "f32")
    for bad in ([0, 200, 100, 300], [0, 64, 5000, 2000000000], [-7, 64, 64, 64]):
        op = runner.DeltaRule(3, 300, 1, 2, 32, 32, "f32", 1.0, device=DEV)
        off = torch.tensor(bad, dtype=torch.int32, device=DEV)
        o, _ = op.forward(*x, off)
        torch.cuda.synchronize()
        first = min(max(bad[1], 0), 300)
        if bad == [0, 200, 100, 300]:
            continue  # the first two share tokens and slots
        want, _, _ = ref.forward([first], *[f64(t)[:first] for t in x], 1.0)
        check("o", o[:first], want, 1)


def test_nan_stays_in_its_sequence():
    x, _ = draw([70, 70], 1, 2, 64, 64, "bf16")
    clean, _ = op_of([70, 70], 1, 2, 64, 64, "bf16", 1.0).forward(*x)
    x[2][10] = float("nan")
    o, s = op_of([70, 70], 1, 2, 64, 64, "bf16", 1.0).forward(*x)
    assert torch.isnan(o[10]).all() and torch.isnan(s[0]).any()
    assert torch.equal(o[70:], clean[70:]) and not torch.isnan(s[1]).any()


def test_same_bits_again_and_on_another_stream():
    lengths = [130, 64, 7]
    x, g = draw(lengths, 2, 4, 128, 128, "bf16")
    do = torch.randn_like(x[2])
    off = offsets(lengths)
    fwd, bwd = op_of(lengths, 2, 4, 128, 128, "bf16", 1.0), op_of(lengths, 2, 4, 128, 128, "bf16",
                                                                  1.0, True)
    a = [t.clone() for t in (*fwd.forward(*x, off), *bwd.backward(*x, do, off)[:5])]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for op in (fwd, bwd):
        op.stream = side
        op.workspace.fill_(255)  # what is left in it means nothing
    torch.cuda.synchronize()
    b = (*fwd.forward(*x, off), *bwd.backward(*x, do, off)[:5])
    side.synchronize()
    for s, t in zip(a, b):
        assert torch.equal(s, t)


def test_graph_replays():
    lengths = [130, 7]
    x, g = draw(lengths, 1, 2, 128, 128, "bf16")
    do, off = torch.randn_like(x[2]), offsets(lengths)
    fwd, bwd = op_of(lengths, 1, 2, 128, 128, "bf16", 1.0), op_of(lengths, 1, 2, 128, 128, "bf16",
                                                                  1.0, True)
    want = [t.clone() for t in (*fwd.forward(*x, off), *bwd.backward(*x, do, off)[:5])]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = (*fwd.forward(*x, off), *bwd.backward(*x, do, off)[:5])
    for _ in range(4):
        for t in got:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for s, t in zip(got, want):
            assert torch.equal(s, t)


# ---- recurrent step ------------------------------------------------------------------

def run_step(lengths, HK, HV, dk, dv, io, slots, num_slots, equal=False, tweak=None, seed=0):
    x, g = draw(lengths, HK, HV, dk, dv, io, seed)
    if tweak:
        tweak(x)
    pool = torch.randn((num_slots, HV, dv, dk), generator=g).to(DEV)
    before = f64(pool)
    slot = None if slots is None else torch.tensor(slots, dtype=torch.int32, device=DEV)
    ids = list(range(len(lengths))) if slots is None else slots
    scale = dk ** -0.5
    op = runner.DeltaRuleStep(len(lengths), sum(lengths), HK, HV, dk, dv, io, num_slots, scale,
                              DEV)
    op.o.fill_(float("nan"))
    o = op.step(pool, slot, *x, None if equal else offsets(lengths))
    torch.cuda.synchronize()
    live = [i for i in ids if 0 <= i < num_slots]
    s0 = np.stack([before[i] if 0 <= i < num_slots else np.zeros_like(before[0]) for i in ids])
    want, last, _ = ref.forward(lengths, *[f64(t) for t in x], scale, s0)
    b = ref.bounds(lengths)
    for n, i in enumerate(ids):
        if i in live:
            before[i] = last[n]
        else:
            want[b[n]:b[n + 1]] = 0.0
    check("step o", o, want, 1, io)
    check("pool", pool, before, 1)


@pytest.mark.parametrize("HK,HV,dk,dv,io", [
    (1, 1, 32, 32, "f32"), (2, 2, 32, 32, "bf16"), (1, 3, 64, 64, "f32"), (2, 2, 64, 64, "bf16"),
    (2, 4, 128, 128, "f32"), (2, 4, 128, 128, "bf16"), (1, 2, 128, 256, "bf16"),
    (1, 1, 128, 512, "bf16"), (2, 2, 256, 256, "bf16"), (1, 2, 256, 512, "bf16")])
def test_step_geometries(HK, HV, dk, dv, io):
    run_step([1, 1, 1], HK, HV, dk, dv, io, [4, 0, 2], 5, equal=True)


def test_step_several_tokens_and_slots_left_out():
    """Sequences of 0 to 5 tokens; slots outside the pool leave it alone and give zeros."""
    run_step([1, 3, 0, 5, 2, 1], 1, 2, 128, 128, "bf16", [3, -1, 2, 0, 9, 1], 6)
    run_step([2, 2, 2], 2, 2, 64, 64, "f32", None, 3, equal=True)


def test_step_zero_decay():
    def tweak(x):
        x[3][1] = float("-inf")
    run_step([1, 1], 1, 2, 64, 64, "bf16", None, 2, equal=True, tweak=tweak)


def test_step_continues_the_chunked_form():
    n, HK, HV, d = 140, 2, 4, 128
    x, _ = draw([n], HK, HV, d, d, "bf16")
    o, last = op_of([n], HK, HV, d, d, "bf16", 1.0).forward(*x)
    m = n - 5
    _, pool = op_of([m], HK, HV, d, d, "bf16", 1.0).forward(*[t[:m] for t in x])
    step = runner.DeltaRuleStep(1, 1, HK, HV, d, d, "bf16", 1, 1.0, DEV)
    outs = [step.step(pool, None, *[t[i:i + 1] for t in x]).clone() for i in range(m, n)]
    check("state", pool, f64(last), 1, bar=2 * F32)
    check("o", torch.cat(outs), f64(o[m:]), 1, bar=2.0 ** -7)


@pytest.mark.slow
def test_offsets_beyond_32_bits():
    """More than 2^31 elements (and 2^32 bytes) before the last tokens of v and o."""
    HK, HV, d = 16, 64, 128
    N, L = 9, 30000
    n = N * L  # 270000 x 64 x 128 = 2.2e9 elements
    g = torch.Generator(device=DEV).manual_seed(0)
    k = torch.randn((n, HK, d), generator=g, device=DEV, dtype=torch.bfloat16)
    k.div_(k.norm(dim=-1, keepdim=True))
    v = torch.randn((n, HV, d), generator=g, device=DEV, dtype=torch.bfloat16)
    la = -torch.rand((n, HV), generator=g, device=DEV)
    beta = torch.rand((n, HV), generator=g, device=DEV)
    op = runner.DeltaRule(N, n, HK, HV, d, d, "bf16", 1.0, device=DEV)
    o, last = op.forward(k, k, v, la, beta)
    tail = slice(n - 300, n)  # decays of e^-0.5 a token leave nothing of what is before
    want, state, _ = ref.forward([300], *[f64(t[tail])[:, s] for t, s in (
        (k, [15]), (k, [15]), (v, [60, 63]), (la, [60, 63]), (beta, [60, 63]))], 1.0)
    check("o", o[tail][200:, [60, 63]], want[200:], 1, "bf16")
    check("state", last[N - 1:, [60, 63]], state, 1)


# ---- the chain in segments --------------------------------------------------------------
# Long sequences of few heads are cut into segments that run at once (the number is the
# library's choice by the device's compute units); a chained segment adds one product with its
# transition matrix (2^-24 of its largest terms), within the bars above.

@pytest.mark.parametrize("lengths,HK,HV,dk,dv,io,equal", [
    ([64 * 21 + 5], 1, 2, 64, 64, "bf16", False), ([64 * 16], 1, 1, 128, 128, "bf16", True),
    ([64 * 9 + 1, 3, 64 * 14], 1, 2, 128, 128, "bf16", False),
    ([64 * 12] * 3, 1, 1, 32, 32, "f32", True), ([64 * 13 - 1, 0, 64 * 5], 1, 3, 64, 64, "f32", False),
    ([64 * 10 + 30], 1, 1, 256, 256, "bf16", False), ([64 * 9], 1, 1, 128, 256, "bf16", True),
    ([64 * 11 + 17], 1, 1, 128, 128, "f32", False)])
def test_segments(lengths, HK, HV, dk, dv, io, equal):
    run_both(lengths, HK, HV, dk, dv, io, seed=7, equal=equal, alpha_mu=-5.0)


@pytest.mark.parametrize("size", [1e-6, 1e6])
def test_magnitudes(size):
    """Values and states scaled by a power of ten: results scale with them (parts of fp32
    operands carry scales of their own; nothing overflows or vanishes)."""
    def tweak(x):
        x[2].mul_(size)
    x, g = draw([140], 1, 2, 64, 64, "f32", 5)
    tweak(x)
    s0 = size * torch.randn((1, 2, 64, 64), generator=g).to(DEV)
    do = torch.randn((140, 2, 64), generator=g).to(DEV) / size
    ds = torch.randn((1, 2, 64, 64), generator=g).to(DEV) / size
    host = [f64(t) for t in x]
    o, last, _ = ref.forward([140], *host, 1.0, f64(s0))
    fo, fs = op_of([140], 1, 2, 64, 64, "f32", 1.0).forward(*x, None, s0)
    check("o", fo, o, 1)
    check("final state", fs, last, 1)
    want = ref.backward([140], *host, 1.0, f64(s0), f64(do), f64(ds))
    got = op_of([140], 1, 2, 64, 64, "f32", 1.0, True).backward(*x, do, None, s0, ds)
    for name, a, w, bar in zip(("dq", "dk", "dv", "dla", "db", "ds"), got, want,
                               (F32, F32, F32, SUMS, F32, F32)):
        check(name, a, w, 1, bar=bar)


def test_keys_and_queries_of_any_size():
    """Unnormalised keys (small ones beside large ones, whole tokens of zeros) and queries."""
    def tweak(x):
        x[1].mul_(0.02 + torch.arange(x[1].shape[0], device=DEV)[:, None, None] % 7 * 0.2)
        x[1][5] = 0
        x[0].mul_(300.0)
    run_both([130], 1, 2, 64, 64, "f32", tweak=tweak)
    run_both([130], 1, 2, 64, 64, "bf16", tweak=tweak)


@pytest.mark.parametrize("lengths,HK,HV,d,io", [
    ([64 * 32], 4, 4, 64, "bf16"), ([64 * 20 + 3], 1, 2, 64, "f32"),
    ([64 * 24 - 7, 0, 40, 64 * 11], 1, 2, 128, "bf16"), ([64 * 16], 1, 1, 256, "bf16")])
def test_states_in_place_in_segments(lengths, HK, HV, d, io):
    """final_state may be initial_state and d_initial_state d_final_state where the chain is cut
    into segments: bit for bit the results of the calls with tensors of their own."""
    x, g = draw(lengths, HK, HV, d, d, io, seed=11)
    shape = (len(lengths), HV, d, d)
    s0, ds = (torch.randn(shape, generator=g).to(DEV) for _ in range(2))
    do, off = torch.randn(x[2].shape, generator=g).to(x[2]), offsets(lengths)
    want = op_of(lengths, HK, HV, d, d, io, 1.0).forward(*x, off, s0)
    op = op_of(lengths, HK, HV, d, d, io, 1.0)
    op.final_state = s0.clone()
    for a, b in zip(op.forward(*x, off, op.final_state), want):
        assert torch.equal(a, b)
    want = op_of(lengths, HK, HV, d, d, io, 1.0, True).backward(*x, do, off, s0, ds)
    op = op_of(lengths, HK, HV, d, d, io, 1.0, True)
    op.d_initial_state = ds.clone()
    for a, b in zip(op.backward(*x, do, off, s0, op.d_initial_state), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("chunks,tail", [(3, 1), (3, 64), (20, 1), (20, 128)])
@pytest.mark.parametrize("size", [1.0, 1e-6, 1e-8])
def test_gradients_before_tokens_without_one(chunks, tail, size):
    """d_o is zero over a sequence's last chunks (tokens without a label) and there is no
    d_final_state: nothing of the empty adjoint's scale reaches the chunks before.  In one
    segment and in several, decays near 1."""
    n = 64 * chunks + tail
    x, g = draw([n], 1, 2, 64, 64, "f32", 21, alpha_mu=-7.0)
    do = size * torch.randn((n, 2, 64), generator=g)
    do[64 * chunks - (64 if tail == 128 else 0):] = 0
    do = do.to(DEV)
    want = ref.backward([n], *[f64(t) for t in x], 1.0, None, f64(do), None)
    got = op_of([n], 1, 2, 64, 64, "f32", 1.0, True).backward(*x, do, offsets([n]))
    for name, a, w, bar in zip(("dq", "dk", "dv", "dla", "db"), got, want,
                               (F32, F32, F32, SUMS, F32)):
        check(name, a, w, 1, bar=bar)


@pytest.mark.parametrize("chunks", [3, 20])
@pytest.mark.parametrize("size", [1.0, 1e-6, 1e-8])
def test_values_after_tokens_without_any(chunks, size):
    """Values that are zero over the first chunks, from a zero state, and small after."""
    n = 64 * chunks + 5
    x, g = draw([n], 1, 2, 64, 64, "f32", 22, alpha_mu=-7.0)
    x[2].mul_(size)
    x[2][:64 * (chunks - 1)] = 0
    do = torch.randn((n, 2, 64), generator=g).to(DEV)
    host = [f64(t) for t in x]
    o, last, _ = ref.forward([n], *host, 1.0)
    fo, fs = op_of([n], 1, 2, 64, 64, "f32", 1.0).forward(*x, offsets([n]))
    check("o", fo, o, 1)
    check("final state", fs, last, 1)
    want = ref.backward([n], *host, 1.0, None, f64(do), None)
    got = op_of([n], 1, 2, 64, 64, "f32", 1.0, True).backward(*x, do, offsets([n]))
    for name, a, w, bar in zip(("dq", "dk", "dv", "dla", "db"), got, want,
                               (F32, F32, F32, SUMS, F32)):
        check(name, a, w, 1, bar=bar)


def different_sizes(lengths, HK, HV, d, io):
    """Value channels from 1 to 1e-5 beside one another, output gradients the other way round:
    (o, final state), the gradients, and the 64-bit references of both."""
    x, g = draw(lengths, HK, HV, d, d, io, 23, alpha_mu=-5.0)
    size = (10.0 ** -(torch.arange(d) % 6).double()).float().to(DEV)
    n, N = sum(lengths), len(lengths)
    s0, ds = (torch.randn((N, HV, d, d), generator=g).to(DEV) for _ in range(2))
    do = torch.randn((n, HV, d), generator=g).to(DEV)
    x[2], s0 = (x[2].float() * size).to(x[2].dtype), s0 * size[:, None]
    do, ds = (do / size).to(x[2].dtype), ds / size[:, None]
    host = [f64(t) for t in x]
    off = offsets(lengths)
    got = (op_of(lengths, HK, HV, d, d, io, 1.0).forward(*x, off, s0),
           op_of(lengths, HK, HV, d, d, io, 1.0, True).backward(*x, do, off, s0, ds))
    return got, (ref.forward(lengths, *host, 1.0, f64(s0))[:2],
                 ref.backward(lengths, *host, 1.0, f64(s0), f64(do), f64(ds)))


SIZES = [([200], 1, 2, 64, "f32"), ([64 * 18], 1, 2, 64, "f32"), ([150, 70], 1, 2, 128, "bf16")]


@pytest.mark.parametrize("lengths,HK,HV,d,io", SIZES)
def test_channels_of_different_sizes(lengths, HK, HV, d, io):
    """Every row of the state is a recurrence of its own, so the bars hold for each size of channel
    by itself."""
    (got, grads), (want, wgrads) = different_sizes(lengths, HK, HV, d, io)
    for c in range(6):
        check(f"o {c}", got[0][..., c::6], want[0][..., c::6], 1, io)
        check(f"state {c}", got[1][:, :, c::6], want[1][:, :, c::6], 1)
        check(f"dv {c}", grads[2][..., c::6], wgrads[2][..., c::6], 1, io)
        check(f"d initial state {c}", grads[5][:, :, c::6], wgrads[5][:, :, c::6], 1)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("d,io", [(64, "f32"), (128, "bf16")])
def test_channels_that_are_not_finite(bad, d, io):
    """A channel of the values, a row of the state to start from, of d_o or of d_final_state that
    is not finite: the other channels keep their bits."""
    lengths = [150]
    x, g = draw(lengths, 1, 2, d, d, io, 24)
    x[2].mul_(50.0)
    s0, ds = (10 * torch.randn((1, 2, d, d), generator=g).to(DEV) for _ in range(2))
    do = torch.randn(x[2].shape, generator=g).to(x[2])
    off = offsets(lengths)

    def run(v, s0, do, ds):
        o, last = op_of(lengths, 1, 2, d, d, io, 1.0).forward(*x[:2], v, *x[3:], off, s0)
        b = op_of(lengths, 1, 2, d, d, io, 1.0, True).backward(*x[:2], v, *x[3:], do, off, s0, ds)
        return o, last, b[2], b[5]

    clean = run(x[2], s0, do, ds)
    one, other = 6, d - 1  # and their neighbours 7 and d - 2
    keep = [c for c in range(d) if c not in (one, other)]
    v, s, w, e = (t.clone() for t in (x[2], s0, do, ds))
    v[:, :, one], s[:, :, other], w[:, :, one], e[:, :, other] = bad, bad, bad, bad
    v[70:, :, other], w[:70, :, other] = bad, bad
    o, last, dv, d0 = run(v, s, w, e)
    for a, b in ((o, clean[0]), (dv, clean[2])):
        assert torch.equal(a[..., keep], b[..., keep])
        assert not torch.isfinite(a[..., [one, other]]).any()
    for a, b in ((last, clean[1]), (d0, clean[3])):
        assert torch.equal(a[:, :, keep], b[:, :, keep])
        assert not torch.isfinite(a[:, :, [one, other]]).any()


@pytest.mark.parametrize("lengths,HK,HV,d,io", SIZES)
def test_gradients_over_channels_of_different_sizes(lengths, HK, HV, d, io):
    """The gradients by q, k and the gates are sums over channels, here of one size."""
    (_, got), (_, want) = different_sizes(lengths, HK, HV, d, io)
    check("dq", got[0], want[0], 1, io)
    check("dk", got[1], want[1], 1, io)
    check("dlog_alpha", got[3], want[3], 1, bar=SUMS)
    check("dbeta", got[4], want[4], 1)


def test_long_sequences_that_forget_nothing():
    """alpha = 1 throughout, as many heads as compute units, so that the chain is not cut: the
    recurrence in 32 bits stays near 3e-7 of the state at any length, and so has the chain."""
    n, HV, d, heads = 32768, 256, 64, [0, 255]
    g = torch.Generator(device=DEV).manual_seed(25)
    k = torch.randn((n, 1, d), generator=g, device=DEV)
    k.div_(k.norm(dim=-1, keepdim=True))
    v = torch.randn((n, HV, d), generator=g, device=DEV)
    beta = torch.rand((n, HV), generator=g, device=DEV)
    la = torch.zeros_like(beta)
    o, last = op_of([n], 1, HV, d, d, "f32", 1.0).forward(k, k, v, la, beta)
    want, state, _ = ref.forward([n], f64(k), f64(k), *[f64(t[:, heads]) for t in (v, la, beta)],
                                 1.0)
    check("o", o[:, heads], want, 1)
    check("state", last[:, heads], state, 1)
    m = 8192
    do = torch.randn((m, HV, d), generator=g, device=DEV)
    x = [t[:m] for t in (k, k, v, la, beta)]
    got = op_of([m], 1, HV, d, d, "f32", 1.0, True).backward(*x, do)
    want = ref.backward([m], f64(x[0]), f64(x[1]), *[f64(t[:, heads]) for t in x[2:]], 1.0, None,
                        f64(do[:, heads]), None)
    check("dv", got[2][:, heads], want[2], 1)
    check("dlog_alpha", got[3][:, heads], want[3], 1, bar=SUMS)
    check("dbeta", got[4][:, heads], want[4], 1)


@pytest.mark.parametrize("chunks", [2, 9])
@pytest.mark.parametrize("big,small", [(1e25, 1e-10), (1e-25, 1e10), (1e30, 1e-30)])
def test_states_forgotten_for_values_of_another_size(big, small, chunks):
    """alpha = 0 at the first token after a state of a size far from the values': the rows' scale
    changes by more than a float holds, and nothing overflows or stays scaled for the old state."""
    n = 64 * chunks
    x, g = draw([n], 1, 2, 64, 64, "f32", 26, alpha_mu=-5.0)
    x[2].mul_(small)
    x[3][64] = float("-inf")
    x[2][:64] = 0
    x[4][:64] = 0
    s0 = big * torch.randn((1, 2, 64, 64), generator=g).to(DEV)
    host = [f64(t) for t in x]
    o, last, _ = ref.forward([n], *host, 1.0, f64(s0))
    fo, fs = op_of([n], 1, 2, 64, 64, "f32", 1.0).forward(*x, None, s0)
    check("o before", fo[:64], o[:64], 1)
    check("o after", fo[64:], o[64:], 1)
    check("final state", fs, last, 1)


@pytest.mark.parametrize("lengths,HK,HV,dk,dv,io", [
    ([2] * 9, 8, 16, 128, 256, "bf16"), ([1620, 727, 632, 99, 1979], 16, 16, 64, 64, "f32"),
    ([343, 2605, 662, 883], 8, 16, 128, 256, "bf16"), ([300] * 24, 8, 16, 128, 128, "bf16"),
    ([200] * 16, 4, 8, 256, 512, "bf16")])
def test_same_bits_of_many_workgroups(lengths, HK, HV, dk, dv, io):
    """Enough workgroups that they share compute units and memory: every call gives the same bits,
    and single heads the reference's values."""
    x, g = draw(lengths, HK, HV, dk, dv, io, seed=27)
    s0 = torch.randn((len(lengths), HV, dv, dk), generator=g).to(DEV)
    do, off = torch.randn(x[2].shape, generator=g).to(x[2]), offsets(lengths)
    ops = [op_of(lengths, HK, HV, dk, dv, io, 1.0, b) for b in (False, True)]

    def call():
        return [t.clone() for t in (*ops[0].forward(*x, off, s0), *ops[1].backward(*x, do, off, s0))]

    first = call()
    for _ in range(5):
        for a, b in zip(first, call()):
            assert torch.equal(a, b)
    G, n = HV // HK, min(sum(lengths), 400)
    part, rows = [], 0
    for m in lengths:
        if rows + m <= n or not part:
            part.append(m)
            rows += m
    hv = slice(HV - G, HV)  # the last query/key head and its value heads, the first sequences
    if rows > 700:
        return
    host = [f64(t[:rows])[:, s] for t, s in zip(x, (slice(HK - 1, HK),) * 2 + (hv,) * 3)]
    want = ref.backward(part, *host, 1.0, f64(s0[:len(part), hv]), f64(do[:rows, hv]), None)
    got = first[2:]
    check("dq", got[0][:rows, HK - 1:], want[0], 1, io)
    check("dk", got[1][:rows, HK - 1:], want[1], 1, io)
    check("dlog_alpha", got[3][:rows, hv], want[3], 1, bar=SUMS)
    check("dbeta", got[4][:rows, hv], want[4], 1)


@pytest.mark.parametrize("lengths,tail,HK,HV,d,io", [
    ([5, 40], 30, 1, 2, 64, "bf16"), ([64, 0, 64], 64, 2, 2, 32, "f32"), ([300], 700, 2, 6, 128, "bf16"),
    ([0, 0], 77, 1, 1, 32, "f32"), ([63], 1, 1, 3, 256, "bf16"), ([33, 31], 0, 1, 2, 64, "f32"),
    ([1, 2000, 48], 3000, 1, 2, 128, "f32")])
def test_rows_behind_the_last_sequence(lengths, tail, HK, HV, d, io):
    """They are not read and left as they were, or with clear_rest 0; all others have the same bits."""
    x, g = draw([*lengths, tail], HK, HV, d, d, io)
    n, N = sum(lengths), len(lengths)
    do = torch.randn((n + tail, HV, d), generator=g).to(x[2].dtype).to(DEV)
    for t in (*x, do):
        t[n:] = float("nan")
    s0, ds = (torch.randn((N, HV, d, d), generator=g).to(DEV) for _ in range(2))
    off = offsets(lengths)
    for backward, names in ((False, ["o"]), (True, ["dq", "dk", "dv", "dlog_alpha", "dbeta"])):
        got = []
        for clear in (False, True):
            op = runner.DeltaRule(N, n + tail, HK, HV, d, d, io, 0.5, backward, DEV, clear_rest=clear)
            for name in names:
                getattr(op, name).fill_(7.0)
            got.append(op.backward(*x, do, off, s0, ds) if backward else op.forward(*x, off, s0))
        for a, b in zip(got[0][:len(names)], got[1]):
            assert bool((a[n:] == 7.0).all()) and not bool(b[n:].any())
            assert torch.equal(a[:n], b[:n]) and bool(torch.isfinite(b).all())
        assert torch.equal(got[0][len(names)], got[1][len(names)])


def test_clearing_by_offsets_that_are_wrong_stays_inside():
    x, _ = draw([100], 1, 2, 32, 32, "f32")
    for bad in ([0, 500, 20, 64], [-9, 30, 10, 900], [70, 80, 90, 64], [64, 0, 64, 0], [0, 5, 9, -7]):
        op, back = (runner.DeltaRule(3, 100, 1, 2, 32, 32, "f32", 1.0, b, DEV, clear_rest=True)
                    for b in (False, True))
        whole = {}
        for one, names in ((op, ["o"]), (back, ["dq", "dk", "dv", "dlog_alpha", "dbeta"])):
            for name in names:
                t = getattr(one, name)
                whole[name] = torch.full((3 * 128, *t.shape[1:]), 5.0, device=DEV)
                setattr(one, name, whole[name][128:228])
        off = torch.tensor(bad, dtype=torch.int32, device=DEV)
        op.forward(*x, off)
        back.backward(*x, x[2], off)
        torch.cuda.synchronize()
        for name, t in whole.items():
            assert bool((t[:128] == 5.0).all()) and bool((t[228:] == 5.0).all()), (bad, name)
