"""What the runner's objects and the example layer's autograd functions refuse before anything is
enqueued: tensors of another type or shape than the object's, which the kernels would read past
their ends or as other numbers; derivatives of derivatives.  No GPU is needed: the library's entry
points are replaced by ones that accept everything."""
import pytest

from paper_2609_12399_amd import onela as ab
from paper_2609_12399_amd import runner

torch = pytest.importorskip("torch")
mixer = pytest.importorskip("paper_2609_12399_amd.mixer")

N, T, HK, HV, DK, DV = 2, 6, 1, 2, 32, 32
BF, F32, F64, I32, I64 = (torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64)


@pytest.fixture(autouse=True)
def entries(monkeypatch):
    """The entry points, called with anything, write down that they were."""
    calls = []
    for name in ("onela_delta_rule_forward", "onela_delta_rule_backward", "onela_delta_rule_step",
                 "onela_qk_norm_rope", "onela_qk_norm_rope_backward"):
        monkeypatch.setattr(ab, name, lambda *a, name=name, **k: calls.append(name))
    return calls


def delta_args(dt=BF):
    return dict(q=torch.zeros(T, HK, DK, dtype=dt), k=torch.zeros(T, HK, DK, dtype=dt),
                v=torch.zeros(T, HV, DV, dtype=dt), log_alpha=torch.zeros(T, HV),
                beta=torch.zeros(T, HV))


STATE = (N, HV, DV, DK)
BAD_DELTA = [("q", (T, HK, DK), F32), ("k", (T, HK, DK), torch.float16), ("v", (T, HV, DV), F32),
             ("q", (T - 1, HK, DK), BF), ("k", (T, HK + 1, DK), BF), ("v", (T, HV, DV + 8), BF),
             ("v", (T, HV * DV), BF), ("log_alpha", (T, HV), BF), ("beta", (T, HV), BF),
             ("beta", (T, HV), F64), ("log_alpha", (T - 1, HV), F32), ("beta", (T, HV, 1), F32),
             ("seq_offsets", (N + 1,), I64), ("seq_offsets", (N,), I32),
             ("initial_state", STATE, BF), ("initial_state", (N - 1, *STATE[1:]), F32)]


@pytest.mark.parametrize("name,shape,dtype", BAD_DELTA, ids=str)
def test_delta_rule_refuses(entries, name, shape, dtype):
    bad = torch.zeros(shape, dtype=dtype)
    do = torch.zeros(T, HV, DV, dtype=BF)
    op = runner.DeltaRule(N, T, HK, HV, DK, DV, "bf16", device="cpu")
    back = runner.DeltaRule(N, T, HK, HV, DK, DV, "bf16", backward=True, device="cpu")
    with pytest.raises(ValueError, match=name):
        op.forward(**{**delta_args(), name: bad})
    with pytest.raises(ValueError, match=name):
        back.backward(**{**delta_args(), name: bad}, d_o=do)
    assert entries == []
    op.forward(**delta_args())
    back.backward(**delta_args(), d_o=do)
    assert len(entries) == 2


@pytest.mark.parametrize("name,shape,dtype", [
    ("d_o", (T, HV, DV), F32), ("d_o", (T, HV, DV - 8), BF), ("d_final_state", STATE, BF),
    ("d_final_state", (N, HV, DK), F32)], ids=str)
def test_delta_rule_backward_refuses(entries, name, shape, dtype):
    op = runner.DeltaRule(N, T, HK, HV, DK, DV, "bf16", backward=True, device="cpu")
    with pytest.raises(ValueError, match=name):
        op.backward(**{**delta_args(), "d_o": torch.zeros(T, HV, DV, dtype=BF),
                       name: torch.zeros(shape, dtype=dtype)})
    assert entries == []


@pytest.mark.parametrize("name,shape,dtype", [
    *[b for b in BAD_DELTA if b[0] != "initial_state"], ("pool", (4, *STATE[1:]), F32),
    ("pool", (5, *STATE[1:]), BF), ("slots", (N,), I64), ("slots", (N + 1,), I32)], ids=str)
def test_delta_step_refuses(entries, name, shape, dtype):
    op = runner.DeltaRuleStep(N, T, HK, HV, DK, DV, "bf16", 5, device="cpu")
    good = dict(delta_args(), pool=torch.zeros(5, *STATE[1:]), slots=torch.zeros(N, dtype=I32))
    with pytest.raises(ValueError, match=name):
        op.step(**{**good, name: torch.zeros(shape, dtype=dtype)})
    assert entries == []
    op.step(**good)
    op.step(**{**good, "pool": torch.zeros(7, *STATE[1:])})  # more slots than are told of
    assert len(entries) == 2


def norm_args():
    return dict(q=torch.zeros(T, 3, 32, dtype=BF), k=torch.zeros(T, 1, 32, dtype=BF),
                q_weight=torch.zeros(32), k_weight=torch.zeros(32),
                positions=torch.zeros(T, dtype=I32), cos_sin=torch.zeros(9, 16))


@pytest.mark.parametrize("name,shape,dtype", [
    ("q", (T, 3, 32), F32), ("q", (T, 2, 32), BF), ("k", (T, 1, 40), BF), ("k", (T, 1, 32), F32),
    ("q_weight", (32,), F64), ("k_weight", (32,), BF), ("q_weight", (31,), F32),
    ("positions", (T,), I64), ("positions", (T - 1,), I32), ("cos_sin", (9, 32), F32),
    ("cos_sin", (9, 16), F64), ("cos_sin", (9 * 16,), F32)], ids=str)
def test_norm_refuses(entries, name, shape, dtype):
    bad = {**norm_args(), name: torch.zeros(shape, dtype=dtype)}
    d = dict(d_q_out=torch.zeros(T, 3, 32, dtype=BF), d_k_out=torch.zeros(T, 1, 32, dtype=BF))
    op, back = (runner.QkNormRope(T, 3, 1, 32, "bf16", rotary_dim=16, backward=b, device="cpu")
                for b in (False, True))
    with pytest.raises(ValueError, match=name):
        op.forward(**bad)
    with pytest.raises(ValueError, match=name):
        back.backward(**bad, **d)
    for one in d:
        with pytest.raises(ValueError, match=one):
            back.backward(**norm_args(), **{**d, one: d[one].float()})
    assert entries == []
    op.forward(**norm_args())
    back.backward(**norm_args(), **d)
    assert len(entries) == 2
    alone = runner.QkNormRope(T, 3, 0, 32, "bf16", device="cpu")  # queries alone
    alone.forward(norm_args()["q"], None)
    with pytest.raises(ValueError, match="k"):
        alone.forward(norm_args()["q"], norm_args()["k"])


def test_second_derivatives_are_refused():
    """The functions' backward passes are not differentiable themselves: a penalty on their
    gradients raises, and does not count as a constant."""
    q, k = (torch.randn(T, HK, DK, requires_grad=True) for _ in range(2))
    v, la, b = (torch.randn(*s, requires_grad=True) for s in ((T, HV, DV), (T, HV), (T, HV)))
    for y in (mixer.DeltaRuleFunction.apply(q, k, v, la, b, None, None, 2, 1.0)[0],
              mixer.QkNormRopeFunction.apply(q, k, None, None, None, None, "l2", 0, 1e-6)[0]):
        dq, = torch.autograd.grad(y.sum(), q, create_graph=True)
        with pytest.raises(RuntimeError, match="once"):
            (dq.square().sum() + q.sum()).backward()


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_layer_under_autocast(entries, io):
    """torch.autocast changes the types of the layer's products: the gates stay in 32 bits, and the
    operators take queries, keys and values as they come."""
    layer = mixer.DeltaMixer(16, HK, HV, DK, DV, io, rotary_dim=16, max_positions=9, device="cpu")
    x = torch.randn(T, 16).to(layer.w_qkv.dtype)
    off, pos = torch.tensor([0, 2, T], dtype=I32), torch.arange(T, dtype=I32)
    with torch.autocast("cpu", dtype=BF):
        _, _, _, la, b = layer._inputs(x, pos)
        assert la.dtype is F32 and b.dtype is F32
        gates = x.float().double() @ layer.w_gates.double()
        assert (b - torch.sigmoid(gates[:, HV:])).abs().max() < 1e-5
        y, state = layer(x, off, pos)
        layer.step(x[:2], torch.zeros(3, *STATE[1:]), torch.zeros(2, dtype=I32), pos[:2])
        beams = layer.beam_step_inputs(x[None], positions=pos)
        assert {t.dtype for t in (beams.q, beams.k, beams.v)} == {layer.w_qkv.dtype}
        assert beams.alpha.dtype is F32 and beams.beta.dtype is F32
    assert entries == ["onela_qk_norm_rope", "onela_qk_norm_rope", "onela_delta_rule_forward",
                       "onela_qk_norm_rope", "onela_delta_rule_step", "onela_qk_norm_rope"]


def test_layer_positions(monkeypatch):
    """Without positions a packed sequence's tokens count from its own start; single tokens and
    beams of a layer that rotates cannot be placed and are refused."""
    seen = []
    monkeypatch.setattr(ab, "onela_qk_norm_rope", lambda cfg, q, k, wq, wk, positions, *a, **kw:
                        seen.append(positions))
    layer = mixer.DeltaMixer(16, HK, HV, DK, DV, "f32", rotary_dim=16, max_positions=9,
                             device="cpu")
    x = torch.randn(T, 16)
    for off, want in (([0, 2, T], [0, 1, 0, 1, 2, 3]), ([0, 0, 2, 2, T], [0, 1, 0, 1, 2, 3]),
                      ([0, T], [0, 1, 2, 3, 4, 5])):
        layer.prompt(x, torch.tensor(off, dtype=I32))
        assert seen.pop().tolist() == want and not seen
    pos = torch.tensor([4, 5, 3, 3, 2, 1], dtype=I32)
    layer.prompt(x, torch.tensor([0, T], dtype=I32), pos)
    assert seen.pop() is pos
    with pytest.raises(ValueError, match="positions"):
        layer.step(x, torch.zeros(T, *STATE[1:]), None)
    with pytest.raises(ValueError, match="positions"):
        layer.beam_step_inputs(x[None])
    plain = mixer.DeltaMixer(16, HK, HV, DK, DV, "f32", device="cpu")
    plain.step(x, torch.zeros(T, *STATE[1:]), None)
    plain.prompt(x, torch.tensor([0, T], dtype=I32))
    assert seen == [None, None]


def test_layer_positions_behind_the_last_sequence(monkeypatch):
    """A padded batch's rest is at position 0, however long it is."""
    seen = []
    monkeypatch.setattr(ab, "onela_qk_norm_rope", lambda cfg, q, k, wq, wk, positions, *a, **kw:
                        seen.append(positions))
    layer = mixer.DeltaMixer(16, HK, HV, DK, DV, "f32", rotary_dim=16, max_positions=9,
                             device="cpu")
    x = torch.randn(30, 16)
    for off, want in (([0, 2, 5], [0, 1, 0, 1, 2]), ([0, 0, 0], []), ([0, 9, 9], list(range(9)))):
        layer.prompt(x, torch.tensor(off, dtype=I32))
        got = seen.pop()
        assert got.tolist() == want + [0] * (30 - len(want)) and got.dtype is I32
