"""The mixing layer (paper_2609_12399_amd/mixer.py): gradients of the whole layer against
differences of a 64-bit copy, training, and its three ways of serving against each other."""
import numpy as np
import pytest

from paper_2609_12399_amd import runner
from paper_2609_12399_amd.workload import WorkloadSpec
from tests import delta_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
mixer = pytest.importorskip("paper_2609_12399_amd.mixer")
DEV = "cuda:0"


def f64(t):
    return t.detach().cpu().double().numpy()


def layer64(layer, weights, x, lengths, pos):
    """The layer's outputs in 64 bits from the formulas."""
    wqkv, wg, wo = weights
    n, qk = x.shape[0], layer.HK * layer.dk
    rows = x @ wqkv
    at = None if layer.cos_sin is None else f64(layer.cos_sin)[pos]
    q, k = (ref.norm(rows[:, a:a + qk].reshape(n, layer.HK, layer.dk), None, False, 1e-6,
                     layer.rotary_dim, at) for a in (0, qk))
    v = rows[:, 2 * qk:].reshape(n, layer.HV, layer.dv)
    g = x @ wg
    la = -np.logaddexp(0.0, g[:, :layer.HV] - 3.0)
    b = 1.0 / (1.0 + np.exp(-g[:, layer.HV:]))
    o, _, _ = ref.forward(lengths, q, k, v, la, b, 1.0)
    return o.reshape(n, -1) @ wo


def make(io, rotary=16):
    layer = mixer.DeltaMixer(48, 2, 4, 32, 32, io, rotary_dim=rotary, max_positions=200,
                             device=DEV)
    lengths = [70, 5]
    off = torch.tensor([0, 70, 75], dtype=torch.int32, device=DEV)
    pos = torch.cat([torch.arange(n) for n in lengths]).to(torch.int32).to(DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((75, 48), generator=g, device=DEV).to(layer.w_qkv.dtype)
    return layer, lengths, off, pos, x, g


def test_layer_gradients_match_differences():
    """fp32 layer: directional derivatives along random directions of each weight and of the
    input, against central differences of the 64-bit copy.  Bar 1e-4 of the gradient's norm
    times the direction's (fp32 library products of some 100 terms on both sides of the
    operators, differences good to 1e-9)."""
    layer, lengths, off, pos, x, g = make("f32")
    x.requires_grad_()
    c = torch.randn((75, 48), generator=g, device=DEV)
    y, _ = layer(x, off, pos)
    want = layer64(layer, [f64(w) for w in layer.weights()], f64(x), lengths, f64(pos).astype(int))
    assert np.abs(f64(y) - want).max() <= 2e-5 * np.abs(want).max()
    (y * c).sum().backward()
    r = np.random.default_rng(0)
    tensors = [*layer.weights(), x]
    for i, t in enumerate(tensors):
        d = r.normal(size=tuple(t.shape))
        h, vals = 1e-5, []
        for s in (h, -h):
            args = [f64(u) for u in tensors]
            args[i] = args[i] + s * d
            vals.append((f64(c) * layer64(layer, args[:3], args[3], lengths,
                                          f64(pos).astype(int))).sum())
        grad = f64(t.grad)
        assert abs((vals[0] - vals[1]) / (2 * h) - (grad * d).sum()) <= \
            1e-4 * np.linalg.norm(grad) * np.linalg.norm(d)


def test_training_lowers_the_loss():
    layer, _, off, pos, x, _ = make("bf16")
    losses = mixer.train(layer, x, torch.roll(x, 1, 0).float(), off, pos, steps=20)
    assert np.isfinite(losses).all() and losses[-1] < 0.9 * losses[0]


def test_prompt_step_and_beams_agree():
    """The last tokens of a prompt one by one on a pool, and as beams of a search, give the
    prompt's own outputs (two bf16 roundings each)."""
    layer, lengths, off, pos, x, _ = make("bf16")
    y, _ = layer.prompt(x, off, pos)
    m = 66  # the first sequence up to here, then its tokens one by one
    cut = torch.tensor([0, m], dtype=torch.int32, device=DEV)
    _, state = layer.prompt(x[:m], cut, pos[:m])
    pool = torch.zeros((3, *state.shape[1:]), device=DEV)
    pool[2] = state[0]
    slots = torch.tensor([2], dtype=torch.int32, device=DEV)
    spec = WorkloadSpec("mixer", 1, layer.HK, layer.HV, layer.dk, layer.dv, 0, (3,) * 4, "bf16",
                        "uniform")
    dec = runner.Decoder(spec, state, DEV)
    big = float(y[:70].float().abs().max())
    for t in range(4):
        one = layer.step(x[m + t:m + t + 1], pool, slots, pos[m + t:m + t + 1])
        bx = x[m + t].expand(1, 3, -1).contiguous()
        par = None if t == 0 else torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV)
        o = torch.empty((1, 3, layer.HV, layer.dv), device=DEV)
        dec.step(t, layer.beam_step_inputs(bx, par, pos[m + t].repeat(3)), o, fused=bool(t % 2))
        beams = layer.beam_outputs(o)
        for got in (one[0], *beams[0]):
            assert float((got.float() - y[m + t].float()).abs().max()) <= 2.0 ** -6 * big
    assert float(pool[:2].abs().max()) == 0.0
    dec.close()


def test_example_runs(capsys):
    mixer.main()
    out = capsys.readouterr().out
    assert "training: loss" in out and "beams:" in out


def test_prompt_goes_on_from_states():
    """A prompt cut in two, the second part from the first one's states, gives the whole's outputs
    and states (two bf16 roundings each: products over other numbers of tokens may round the
    projections the other way)."""
    layer, lengths, off, pos, x, _ = make("bf16")
    y, state = layer.prompt(x, off, pos)
    a, b = 41, 3  # of each sequence's tokens, the first part
    first = torch.cat([torch.arange(a), 70 + torch.arange(b)]).to(DEV)
    rest = torch.cat([torch.arange(a, 70), 70 + torch.arange(b, 5)]).to(DEV)
    at = [torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([0, a, a + b], [0, 70 - a, 75 - a - b])]
    _, mid = layer.prompt(x[first], at[0], pos[first])
    z, end = layer.prompt(x[rest], at[1], pos[rest], initial_state=mid)
    assert float((z.float() - y[rest].float()).abs().max()) <= 2.0 ** -6 * float(y.float().abs().max())
    assert float((end - state).abs().max()) <= 2.0 ** -6 * float(state.abs().max())
