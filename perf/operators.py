"""Performance cases of the gated delta rule over whole sequences (outputs, state and
gradients), of its recurrent step on a pool of states, and of the norm and rotation of
queries and keys.

Each case is one call that a model around this framework's decode makes: a layer's prompt
pass, the backward pass of a training step, one token of a serving batch, the norm of the
queries and keys that those calls take.  Geometries are those of
``paper_2609_12399_amd.workload`` (heads of 32 to 256, 1 to 16 requests, prompts of up to
8192 tokens, 16 heads of 128 as the paper's model has); ragged lengths are drawn from the
case's own sizes.  Inputs follow the distributions given there: q, k normalised N(0, 1),
v ~ N(0, 1), beta = sigmoid(N(0, 1)), alpha = exp(-softplus(N(-3, 1))), handed over as
log(alpha).

The plain forms are the chunkwise equations in products of 32 bits, 64 tokens per chunk,
with the only loop where a chunk needs the state of the one before; ``exact`` walks the
recurrence token by token in 64 bits.
"""
import random

import torch

own = False

DEV = "cuda:0"
C = 64  # tokens per chunk of the plain form


# ---- cases -------------------------------------------------------------------------

def _delta(name, kind, N, T, HK, HV, dk, dv, io="bf16", ragged=False, state=False):
    """N sequences of T tokens, or with ``ragged`` of lengths from 0 to about 2 T."""
    c = {"kind": kind, "N": N, "T": T, "HK": HK, "HV": HV, "dk": dk, "dv": dv, "io": io,
         "ragged": ragged, "state": state}
    return c if name is None else dict(c, name=name)


def _step(name, N, slots, T, HK, HV, dk, dv, io="bf16"):
    c = {"kind": "step", "N": N, "slots": slots, "T": T, "HK": HK, "HV": HV, "dk": dk,
         "dv": dv, "io": io}
    return c if name is None else dict(c, name=name)


def _norm(name, kind, T, HQ, HK, D, rot, rms, io="bf16"):
    c = {"kind": kind, "T": T, "HQ": HQ, "HK": HK, "D": D, "rot": rot, "rms": rms, "io": io}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the smallest layer (2 heads of 32, one chunk, fp32): what a call costs
        _delta("forward_tiny_f32", "forward", 1, 64, 2, 2, 32, 32, io="f32"),
        # one user's prompt through a layer, few heads for the card
        _delta("forward_t4096", "forward", 1, 4096, 16, 16, 128, 128),
        # a packed batch of prompts of any length, grouped heads, continued from states
        _delta("forward_ragged16", "forward", 16, 1000, 16, 32, 128, 128, ragged=True,
               state=True),
        # heads of 256
        _delta("forward_k256", "forward", 4, 2048, 8, 8, 256, 256),
        # gradients of a small fp32 layer, lengths that fill no chunk
        _delta("backward_f32_d64", "backward", 2, 500, 4, 4, 64, 64, io="f32", state=True),
        # gradients of one long sequence
        _delta("backward_t4096", "backward", 1, 4096, 16, 16, 128, 128),
        # gradients of a packed training batch, grouped heads: the largest
        _delta("backward_ragged8", "backward", 8, 2048, 16, 32, 128, 128, ragged=True),
        # one token for one user: latency
        _step("step_1", 1, 1, 1, 16, 16, 128, 128),
        # one token for a serving batch on a pool of states
        _step("step_256", 256, 320, 1, 16, 32, 128, 128),
        # queries and keys of a few tokens of an attention layer, a quarter of the head rotated
        _norm("norm_t8", "norm", 8, 8, 2, 256, 64, True),
        # queries and keys of a batch of prompts of a delta-rule layer: L2, no rotation
        _norm("norm_t16384", "norm", 16384, 16, 16, 128, 0, False),
        # gradients of norm and rotation in a training step
        _norm("norm_backward_t8191", "norm_backward", 8191, 16, 16, 128, 128, True),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(lo * (hi / lo) ** rng.random() + 0.5)))


_GEOMETRIES = [(16, 16, 128, 128), (16, 32, 128, 128), (8, 8, 128, 128), (16, 16, 64, 64),
               (4, 4, 32, 32), (2, 6, 64, 64), (8, 8, 256, 256), (4, 8, 256, 512),
               (8, 16, 128, 256)]
# Drawn calls compute at most what the largest listed one of their kind does.
_MOST = {"forward": 16 * 1000 * 32 * 128 * 128, "backward": 8 * 2048 * 32 * 128 * 128,
         "step": 256 * 32 * 128 * 128}


def draw(rng):
    while True:
        kind = rng.choice(["forward", "forward", "backward", "backward", "step", "norm",
                           "norm_backward"])
        if kind in ("norm", "norm_backward"):
            D = rng.choice([32, 64, 96, 128, 256])
            HQ = rng.choice([1, 3, 8, 16, 32])
            c = _norm(None, kind, _log_int(rng, 1, 16384), HQ, rng.choice([1, 2, HQ]), D,
                      rng.choice([0, 32, D]), rng.random() < 0.6,
                      "f32" if rng.random() < 0.25 else "bf16")
            if c["T"] * (c["HQ"] + c["HK"]) * D <= 16384 * 32 * 128:
                return c
            continue
        HK, HV, dk, dv = rng.choice(_GEOMETRIES)
        io = "f32" if dk == dv and dk <= 128 and rng.random() < 0.25 else "bf16"
        if kind == "step":
            N = _log_int(rng, 1, 256)
            c = _step(None, N, N + rng.randrange(0, 64), rng.choice([1, 1, 1, 2, 4]), HK, HV,
                      dk, dv, io)
            if N * c["T"] * HV * dk * dv <= _MOST[kind]:
                return c
            continue
        N = _log_int(rng, 1, 16)
        c = _delta(None, kind, N, _log_int(rng, 1 if N > 1 else 40, 8192), HK, HV, dk, dv, io,
                   N > 1 and rng.random() < 0.6, rng.random() < 0.5)
        n = sum(_lengths(c))
        if 1 <= n <= _MOST[kind] / (HV * dk * dv) and max(_lengths(c)) <= 8192:
            return c


def _lengths(c):
    if not c["ragged"]:
        return [c["T"]] * c["N"]
    r = random.Random(c["N"] * 100003 + c["T"])
    return [r.randrange(0, 2 * c["T"] + 1) for _ in range(c["N"])]


# ---- inputs --------------------------------------------------------------------------

def _unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def _io(c):
    return torch.bfloat16 if c["io"] == "bf16" else torch.float32


class _Draws:
    """Draws on the GPU from one seeded generator."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=torch.float32)

    def state(self, n, c):
        """States with the content of long prompts: decayed outer products of the last 32
        tokens, the memory that the gates leave."""
        S = torch.zeros((n, c["HV"], c["dv"], c["dk"]), device=DEV)
        for _ in range(32):
            k = _unit(self.normal(n, c["HV"], 1, c["dk"]))
            S.mul_(0.94).add_(0.5 * self.normal(n, c["HV"], c["dv"], 1) * k)
        return S

    def tokens(self, c, n):
        """q, k, v, log(alpha), beta of n tokens."""
        q = _unit(self.normal(n, c["HK"], c["dk"])).to(_io(c))
        k = _unit(self.normal(n, c["HK"], c["dk"])).to(_io(c))
        v = self.normal(n, c["HV"], c["dv"]).to(_io(c))
        la = -torch.nn.functional.softplus(self.normal(n, c["HV"]) - 3.0)
        return q, k, v, la, torch.sigmoid(self.normal(n, c["HV"]))


def prepare(case, seed):
    c, d, x = dict(case), _Draws(seed), {}
    x["case"], x["op"] = c, None
    if c["kind"] in ("forward", "backward"):
        x["lengths"] = _lengths(c)
        n = sum(x["lengths"])
        x["tokens"] = d.tokens(c, n)
        x["s0"] = d.state(c["N"], c) if c["state"] else None
        x["offsets"] = None
        if c["ragged"]:
            off = torch.tensor([0] + x["lengths"], device=DEV)
            x["offsets"] = torch.cumsum(off, 0).to(torch.int32)
        x["scale"] = c["dk"] ** -0.5
        if c["kind"] == "backward":
            x["do"] = d.normal(n, c["HV"], c["dv"]).to(_io(c))
            x["ds"] = d.normal(c["N"], c["HV"], c["dv"], c["dk"]) if c["state"] else None
    elif c["kind"] == "step":
        x["tokens"] = d.tokens(c, c["N"] * c["T"])
        x["pool"] = d.state(c["slots"], c)
        x["slots"] = torch.randperm(c["slots"], generator=d.g,
                                    device=DEV)[:c["N"]].to(torch.int32)
        x["scale"] = c["dk"] ** -0.5
    else:
        # queries and keys stand side by side in a projection's output
        H = c["HQ"] + c["HK"]
        qk = d.normal(c["T"], H, c["D"]).to(_io(c))
        x["q"], x["k"] = qk[:, :c["HQ"]], qk[:, c["HQ"]:]
        x["wq"] = x["wk"] = x["positions"] = x["cos_sin"] = None
        if c["rms"]:
            x["wq"] = 1.0 + 0.1 * d.normal(c["D"])
            x["wk"] = 1.0 + 0.1 * d.normal(c["D"])
        if c["rot"]:
            most = 16384
            f = 10000.0 ** (-torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64)
                            / c["rot"])
            a = torch.arange(most, device=DEV, dtype=torch.float64)[:, None] * f
            x["cos_sin"] = torch.cat([a.cos(), a.sin()], 1).float()
            x["positions"] = torch.randint(0, most, (c["T"],), generator=d.g,
                                           device=DEV).to(torch.int32)
        x["eps"] = 1e-6
        if c["kind"] == "norm_backward":
            x["dqo"] = d.normal(c["T"], c["HQ"], c["D"]).to(_io(c))
            x["dko"] = d.normal(c["T"], c["HK"], c["D"]).to(_io(c))
    return x


# ---- one pass ------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(x):
    from paper_2609_12399_amd import runner
    c, op = x["case"], x["op"]
    if op is None:  # the object that a program keeps: its workspace and output tensors
        if c["kind"] in ("forward", "backward"):
            op = runner.DeltaRule(c["N"], x["tokens"][0].shape[0], c["HK"], c["HV"], c["dk"],
                                  c["dv"], c["io"], scale=x["scale"],
                                  backward=c["kind"] == "backward", device=DEV)
        elif c["kind"] == "step":
            op = runner.DeltaRuleStep(c["N"], c["N"] * c["T"], c["HK"], c["HV"], c["dk"],
                                      c["dv"], c["io"], c["slots"], scale=x["scale"],
                                      device=DEV)
        else:
            op = runner.QkNormRope(c["T"], c["HQ"], c["HK"], c["D"], c["io"],
                                   norm="rms" if c["rms"] else "l2", rotary_dim=c["rot"],
                                   eps=x["eps"], backward=c["kind"] == "norm_backward",
                                   device=DEV)
        x["op"] = op
    if c["kind"] == "forward":
        return op.forward(*x["tokens"], seq_offsets=x["offsets"], initial_state=x["s0"])
    if c["kind"] == "backward":
        return op.backward(*x["tokens"], x["do"], seq_offsets=x["offsets"],
                           initial_state=x["s0"], d_final_state=x["ds"])
    if c["kind"] == "step":
        return op.step(x["pool"], x["slots"], *x["tokens"]), x["pool"]
    if c["kind"] == "norm":
        return op.forward(x["q"], x["k"], x["wq"], x["wk"], x["positions"], x["cos_sin"])
    return op.backward(x["q"], x["k"], x["dqo"], x["dko"], x["wq"], x["wk"], x["positions"],
                       x["cos_sin"])


def _run_plain(x):
    return {"forward": _plain_forward, "backward": _plain_backward, "step": _plain_step,
            "norm": _plain_norm, "norm_backward": _plain_norm_backward}[x["case"]["kind"]](x)


# ---- plain forms ---------------------------------------------------------------------

def _chunks(x, rows):
    """rows [n][H][...] of the packed tokens as [N][H][chunks][C][...] in 32 bits, zero past a
    sequence's end (log(alpha) = 0, beta = 0, k = v = 0 leave the state as it is)."""
    c, most = x["case"], max(1, -(-max(x["lengths"]) // C)) * C
    t = torch.arange(most, device=DEV)
    if x["offsets"] is None:
        begin = torch.arange(c["N"], device=DEV)[:, None] * c["T"]
        end = begin + c["T"]
    else:
        begin, end = x["offsets"][:-1, None], x["offsets"][1:, None]
    at = begin + t
    inside = at < end
    at = torch.where(inside, at, rows.shape[0])
    rows = torch.cat([rows.float(), torch.zeros_like(rows[:1], dtype=torch.float32)])
    y = rows[at].movedim(2, 1)
    return y.reshape(c["N"], rows.shape[1], most // C, C, *rows.shape[2:])


def _packed(x, y):
    """The inverse of _chunks: [N][H][chunks][C][...] -> [n][H][...]."""
    y = y.flatten(2, 3).movedim(1, 2)
    if x["offsets"] is None:
        return y[:, :x["case"]["T"]].flatten(0, 1)
    length = (x["offsets"][1:] - x["offsets"][:-1])[:, None]
    return y[torch.arange(y.shape[1], device=DEV) < length]


def _factors(x):
    c, G = x["case"], x["case"]["HV"] // x["case"]["HK"]
    q, k, v, la, b = (_chunks(x, t) for t in x["tokens"])
    q, k = q.repeat_interleave(G, 1), k.repeat_interleave(G, 1)
    g = la.cumsum(-1)
    low = torch.ones(C, C, device=DEV).tril()
    # exp of the decays between two tokens, above the diagonal nothing
    gam2 = torch.exp((g[..., :, None] - g[..., None, :]) * low) * low
    kk = gam2 * (k @ k.transpose(-1, -2)) * low.tril(-1)
    qk = gam2 * (q @ k.transpose(-1, -2)) * x["scale"]
    A = kk * b[..., None, :]
    eye = torch.eye(C, device=DEV)
    # (I + A)^-1 of a strictly lower A: (I - A) (I + A^2) (I + A^4) ... (I + A^32)
    A2 = A @ A
    A4 = A2 @ A2
    A8 = A4 @ A4
    A16 = A8 @ A8
    T = (eye - A) @ (eye + A2) @ ((eye + A4) @ (eye + A8)) @ ((eye + A16) @ (eye + A16 @ A16))
    gam, sig = torch.exp(g)[..., None], torch.exp(g[..., -1:] - g)[..., None]
    return q, k, v, b[..., None], gam, sig, gam2, kk, qk, T


def _states(x, k, v, b, gam, sig, T):
    """The state before every chunk, e of every chunk and the last state."""
    c = x["case"]
    S = torch.zeros(c["N"], c["HV"], c["dv"], c["dk"], device=DEV) if x["s0"] is None else x["s0"]
    before, es = [], []
    gk, sk = gam * k, b * sig * k
    for i in range(k.shape[2]):
        e = T[:, :, i] @ (v[:, :, i] - gk[:, :, i] @ S.transpose(-1, -2))
        before.append(S)
        es.append(e)
        S = gam[:, :, i, -1:] * S + e.transpose(-1, -2) @ sk[:, :, i]
    return torch.stack(before, 2), torch.stack(es, 2), S


def _plain_forward(x):
    q, k, v, b, gam, sig, gam2, kk, qk, T = _factors(x)
    S, e, last = _states(x, k, v, b, gam, sig, T)
    o = x["scale"] * ((gam * q) @ S.transpose(-1, -2)) + qk @ (b * e)
    return _packed(x, o).to(_io(x["case"])), last


def _plain_backward(x):
    c, io, scale = x["case"], _io(x["case"]), x["scale"]
    q, k, v, b, gam, sig, gam2, kk, qk, T = _factors(x)
    S, e, last = _states(x, k, v, b, gam, sig, T)
    do = _chunks(x, x["do"])
    intra = qk.transpose(-1, -2) @ do
    dS = torch.zeros_like(last) if x["ds"] is None else x["ds"]
    after, dvs = [], []
    sk, gk, gdo = sig * k, gam * k, scale * gam * do
    for i in range(k.shape[2] - 1, -1, -1):
        dD = intra[:, :, i] + sk[:, :, i] @ dS.transpose(-1, -2)
        dv = T[:, :, i].transpose(-1, -2) @ (b[:, :, i] * dD)
        after.append(dS)
        dvs.append(dv)
        dS = (gam[:, :, i, -1:] * dS + gdo[:, :, i].transpose(-1, -2) @ q[:, :, i]
              - dv.transpose(-1, -2) @ gk[:, :, i])
    after, dv = torch.stack(after[::-1], 2), torch.stack(dvs[::-1], 2)
    doe = do @ e.transpose(-1, -2)
    dve = (dv @ e.transpose(-1, -2)).tril(-1)
    bt = b.transpose(-1, -2)
    L, M = scale * gam2 * bt * doe, -gam2 * bt * dve
    qS, kS, kD = scale * gam * (do @ S), gam * (dv @ S), b * sig * (e @ after)
    dq = qS + L @ k
    dk = L.transpose(-1, -2) @ q + (M + M.transpose(-1, -2)) @ k + kD - kS
    db = (qk * doe).sum(-2) - (kk * dve).sum(-2) + (sig * k * (e @ after)).sum(-1)
    # the decay of token t weighs every pair (i, j) with i >= t > j
    Z = L * (q @ k.transpose(-1, -2)) + M * (k @ k.transpose(-1, -2))
    kd = (kD * k).sum(-1)
    own_t = (qS * q).sum(-1) - (kS * k).sum(-1) + Z.sum(-1) - Z.sum(-2) - kd
    whole = gam[..., -1, 0] * (S * after).sum((-1, -2)) + kd.sum(-1)
    dg = own_t.flip(-1).cumsum(-1).flip(-1) + whole[..., None]
    G = c["HV"] // c["HK"]
    dq, dk = (t.unflatten(1, (c["HK"], G)).sum(2) for t in (dq, dk))
    out = [_packed(x, t) for t in (dq, dk, dv, dg, db)]
    return (*(t.to(io) for t in out[:3]), *out[3:], dS if c["state"] else None)


def _plain_step(x):
    c, G, N, T = x["case"], x["case"]["HV"] // x["case"]["HK"], x["case"]["N"], x["case"]["T"]
    q, k, v, la, b = (t.float().unflatten(0, (N, T)) for t in x["tokens"])
    q, k = q.repeat_interleave(G, 2), k.repeat_interleave(G, 2)
    S, out = x["pool"][x["slots"].long()], []
    for t in range(T):
        S = torch.exp(la[:, t])[..., None, None] * S
        d = b[:, t, :, None] * (v[:, t] - (S * k[:, t, :, None]).sum(-1))
        S = S + d[..., None] * k[:, t, :, None]
        out.append(x["scale"] * (S * q[:, t, :, None]).sum(-1))
    x["pool"][x["slots"].long()] = S
    return torch.stack(out, 1).flatten(0, 1).to(_io(c)), x["pool"]


def _norm_of(x, t, w):
    c, t = x["case"], t.float()
    n = c["D"] if c["rms"] else 1
    r = torch.rsqrt((t * t).sum(-1, keepdim=True) / n + x["eps"])
    return t, r, n, torch.ones(c["D"], device=DEV) if w is None else w


def _turn(x, y, sign):
    """Rotates the first rot columns: pairs (i, i + rot / 2)."""
    rot = x["case"]["rot"]
    if not rot:
        return y
    cs = x["cos_sin"][x["positions"].long()][:, None]
    co, si = cs[..., :rot // 2], sign * cs[..., rot // 2:]
    a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    return torch.cat([a * co - b * si, b * co + a * si, y[..., rot:]], -1)


def _plain_norm(x):
    out = []
    for t, w in ((x["q"], x["wq"]), (x["k"], x["wk"])):
        t, r, n, w = _norm_of(x, t, w)
        out.append(_turn(x, t * r * w, 1.0).to(_io(x["case"])))
    return tuple(out)


def _plain_norm_backward(x):
    grads, weights = [], []
    for t, w, dz in ((x["q"], x["wq"], x["dqo"]), (x["k"], x["wk"], x["dko"])):
        given = w is not None
        t, r, n, w = _norm_of(x, t, w)
        dy = _turn(x, dz.float(), -1.0)
        weights.append((dy * t * r).sum((0, 1)) if given else None)
        dx = r * (w * dy - t * r * r * (w * dy * t).sum(-1, keepdim=True) / n)
        grads.append(dx.to(_io(x["case"])))
    return (*grads, *weights)


# ---- what a pass cannot do without ---------------------------------------------------

def work(case):
    c, e = case, 2 if case["io"] == "bf16" else 4
    if c["kind"] in ("norm", "norm_backward"):
        n = c["T"] * (c["HQ"] + c["HK"]) * c["D"]
        extra = 4 * c["T"] * (c["rot"] + 1) if c["rot"] else 0
        return {"bytes": n * e * (2 if c["kind"] == "norm" else 3) + extra,
                "flops": n * (6 if c["kind"] == "norm" else 14)}
    state = 4 * c["HV"] * c["dv"] * c["dk"]
    n = c["N"] * c["T"] if c["kind"] == "step" else sum(_lengths(c))
    unit = n * c["HV"] * c["dv"] * c["dk"]
    qk, v, gates = e * c["HK"] * c["dk"], e * c["HV"] * c["dv"], 4 * c["HV"]
    if c["kind"] == "step":
        return {"bytes": n * (2 * qk + 2 * v + 2 * gates) + 2 * c["N"] * state,
                "flops": 6 * unit}
    states = c["N"] * state * (2 if c["state"] else 1)
    if c["kind"] == "forward":
        # S k, the rank-one update and S q of every token
        return {"bytes": n * (2 * qk + 2 * v + 2 * gates) + states, "flops": 6 * unit}
    # the states again, their adjoints' two products with q, k, the output's gradient, and
    # the five products of gradients with a state
    return {"bytes": n * (4 * qk + 3 * v + 4 * gates) + (3 * c["N"] * state if c["state"] else 0),
            "flops": 18 * unit}


# ---- the same in 64 bits -------------------------------------------------------------

def _dense(x, t):
    """[n][...] of the packed tokens as [N][longest][...], zero past a sequence's end."""
    n, at = x["lengths"], 0
    y = torch.zeros(len(n), max(max(n), 1), *t.shape[1:], dtype=torch.float64, device=DEV)
    for i, m in enumerate(n):
        y[i, :m] = t[at:at + m].double()
        at += m
    return y


def _undense(x, y):
    return torch.cat([y[i, :m] for i, m in enumerate(x["lengths"])])


def exact(case, seed):
    x = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "norm_backward"):
        return _exact_norm(x, kind)
    G = case["HV"] // case["HK"]
    if kind == "step":
        x["lengths"] = [case["T"]] * case["N"]
        S = x["pool"].double()[x["slots"].long()]
    else:
        S = torch.zeros(case["N"], case["HV"], case["dv"], case["dk"], dtype=torch.float64,
                        device=DEV) if x["s0"] is None else x["s0"].double()
    q, k, v, la, b = (_dense(x, t) for t in x["tokens"])
    q, k = q.repeat_interleave(G, 2), k.repeat_interleave(G, 2)
    a, n = torch.exp(la), q.shape[1]
    o, keep = torch.zeros_like(v), kind == "backward"
    # alpha_t S_{t-1} and the error v_t - alpha_t S_{t-1} k_t of every token
    old = torch.zeros(n if keep else 0, *S.shape, dtype=torch.float64, device=DEV)
    err = torch.zeros_like(v)
    for t in range(n):
        S = a[:, t, :, None, None] * S
        err[:, t] = v[:, t] - (S @ k[:, t, :, :, None])[..., 0]
        if keep:
            old[t] = S
        S = S + (b[:, t, :, None] * err[:, t])[..., None] * k[:, t, :, None]
        o[:, t] = x["scale"] * (S @ q[:, t, :, :, None])[..., 0]
    if kind == "forward":
        return _undense(x, o), S
    if kind == "step":
        pool = x["pool"].double()
        pool[x["slots"].long()] = S
        return _undense(x, o), pool
    do = _dense(x, x["do"])
    dS = torch.zeros_like(S) if x["ds"] is None else x["ds"].double()
    dq, dk, dv, dg, db = (torch.zeros_like(t) for t in (q, k, v, la, b))
    for t in range(n - 1, -1, -1):
        kt, d = k[:, t, :, None], x["scale"] * do[:, t]
        new = old[t] + (b[:, t, :, None] * err[:, t])[..., None] * kt
        dq[:, t] = (d[..., None, :] @ new)[..., 0, :]
        dS = dS + d[..., None] * q[:, t, :, None]
        u = (dS @ kt.transpose(-1, -2))[..., 0]  # adjoint of beta_t err_t
        db[:, t] = (u * err[:, t]).sum(-1)
        dv[:, t] = b[:, t, :, None] * u
        w = dv[:, t][..., None, :]
        dk[:, t] = ((b[:, t, :, None] * err[:, t])[..., None, :] @ dS - w @ old[t])[..., 0, :]
        dS = dS - dv[:, t][..., None] * kt
        dg[:, t] = (dS * old[t]).sum((-1, -2))
        dS = a[:, t, :, None, None] * dS
    dq, dk = (t.unflatten(2, (case["HK"], G)).sum(3) for t in (dq, dk))
    return (*(_undense(x, t) for t in (dq, dk, dv, dg, db)), dS if case["state"] else None)


def _exact_norm(x, kind):
    c, rot, grads, weights = x["case"], x["case"]["rot"], [], []
    for t, w, dz in ((x["q"], x["wq"], x.get("dqo")), (x["k"], x["wk"], x.get("dko"))):
        t = t.double()
        size = torch.sqrt((t ** 2).mean(-1) + x["eps"]) if c["rms"] else \
            torch.sqrt((t ** 2).sum(-1) + x["eps"])
        unit = t / size[..., None]
        gain = torch.ones(c["D"], dtype=torch.float64, device=DEV) if w is None else w.double()
        turn = torch.ones(c["T"], 1, max(rot // 2, 1), dtype=torch.complex128, device=DEV)
        if rot:
            cs = x["cos_sin"].double()[x["positions"].long()]
            turn = torch.complex(cs[:, :rot // 2], cs[:, rot // 2:])[:, None]

        def rotated(y, by):
            if not rot:
                return y
            z = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * by
            return torch.cat([z.real, z.imag, y[..., rot:]], -1)

        if kind == "norm":
            grads.append(rotated(unit * gain, turn))
            continue
        dy = rotated(dz.double(), turn.conj())
        weights.append(None if w is None else (dy * unit).sum((0, 1)))
        dn = dy * gain
        along = (dn * unit).mean(-1) if c["rms"] else (dn * unit).sum(-1)
        grads.append((dn - unit * along[..., None]) / size[..., None])
    return (*grads, *weights)
