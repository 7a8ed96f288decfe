"""Performance cases of what stands before and after the delta rule in a model: the short
causal convolution of a layer's projections (over packed sequences, its gradient, its step
on a pool of states), the norms before and after a block with its gate and residual scale,
and the log probabilities that a model's logits give to tokens, with their gradients.

Each case is one call that a model around this framework's decode makes: a layer's prompt
pass, the backward pass of a training step, one step of a beam search whose beams go on from
their parents' states, the logits of a beam search before the selection.  Geometries are those of
``paper_2609_12399_amd.workload``: 16 heads of 128 (rows of 2048 columns, 6144 channels of
queries, keys and values side by side), 512 beams, a codebook of 8192 tokens; the wider
vocabularies are generic.  Activations are N(0, 1), a training step's logits N(0, 2^2) with one
token that the model is surer of, gates N(0, 1).

The plain forms are the formulas in elementary products and sums of 32 bits; ``exact`` takes the
definitions in 64 bits and, for gradients, lets torch differentiate them.
"""
import random

import torch

own = False

DEV = "cuda:0"


# ---- cases -------------------------------------------------------------------------

def _named(name, c):
    return c if name is None else dict(c, name=name)


def _logits(name, kind, R, V, G, K, io="bf16", entropy=True, masked=False, pad=0, scale=1.0):
    """R rows of V logits (the rows V + pad apart), G given tokens, K alternatives per row.
    ``masked``: most logits are -inf, in one row all."""
    return _named(name, {"kind": kind, "R": R, "V": V, "G": G, "K": K, "io": io,
                         "entropy": entropy, "masked": masked, "pad": pad, "scale": scale})


def _norm(name, kind, T, H, D, after, before, gate, residual, channel, io="bf16"):
    """T tokens of H rows of D columns; norm after the block, norm before the next, gate
    ("", "silu", "sigmoid"), residual ("", "bf16", "f32"), a scale for each channel."""
    return _named(name, {"kind": kind, "T": T, "H": H, "D": D, "after": after, "before": before,
                         "gate": gate, "residual": residual, "channel": channel, "io": io})


def _conv(name, kind, N, T, C, taps, io="bf16", silu=True, bias=False, ragged=False,
          state=False):
    """N sequences of T tokens, or with ``ragged`` of lengths from 0 to about 2 T."""
    return _named(name, {"kind": kind, "N": N, "T": T, "C": C, "taps": taps, "io": io,
                         "silu": silu, "bias": bias, "ragged": ragged, "state": state})


def _step(name, N, T, C, taps, beams, io="bf16", silu=True, bias=False):
    """N sequences of T tokens on a pool of states, or with ``beams`` from the states of parents
    in one pool to another pool."""
    return _named(name, {"kind": "conv_step", "N": N, "T": T, "C": C, "taps": taps,
                         "beams": beams, "io": io, "silu": silu, "bias": bias})


def listed():
    return [
        # the next token of one user: its log probability and the alternatives beside it
        _logits("logprobs_1", "logprobs", 1, 8192, 1, 8),
        # 512 beams before the selection, tokens that may not follow masked: latency and HBM
        _logits("logprobs_beams512", "logprobs", 512, 8192, 0, 0, io="f32", entropy=False,
                masked=True),
        # a batch of texts scored with a wide, odd vocabulary and 20 alternatives: the largest read
        _logits("logprobs_4096", "logprobs", 4096, 50001, 1, 20),
        # gradient of a training step's loss, one target per token: the largest
        _logits("logprobs_backward_8192", "logprobs_backward", 8192, 32768, 1, 0,
                entropy=False),
        # gradient of a distillation from a teacher's 64 best tokens, with entropy
        _logits("logprobs_backward_300", "logprobs_backward", 300, 50001, 64, 0, io="f32"),
        # one token between two blocks: latency
        _norm("norm_1", "norm", 1, 1, 2048, False, True, "", "bf16", False),
        # a batch of prompts between two blocks, residual stream in 32 bits
        _norm("norm_16384", "norm", 16384, 1, 2048, True, True, "", "f32", True),
        # the outputs of the delta rule's heads, normed and gated before the output projection
        _norm("norm_heads_16384", "norm", 16384, 16, 128, True, False, "silu", "", False),
        # gradients of everything between two blocks in a training step
        _norm("norm_backward_8191", "norm_backward", 8191, 1, 2048, True, True, "silu", "bf16",
              True),
        # queries, keys and values of ragged prompts that go on from states
        _conv("conv_ragged16", "conv", 16, 1000, 6144, 4, ragged=True, state=True),
        # gradients of a packed training batch
        _conv("conv_backward_8", "conv_backward", 8, 1024, 6144, 4, bias=True),
        # one step of 512 beams, each from its parent's state
        _step("conv_step_beams512", 512, 1, 6144, 4, True),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(lo * (hi / lo) ** rng.random() + 0.5)))


def draw(rng):
    while True:
        kind = rng.choice(["logprobs", "logprobs", "logprobs_backward", "norm", "norm_backward",
                           "conv", "conv_backward", "conv_step"])
        io = "f32" if rng.random() < 0.25 else "bf16"
        wide = 2 if io == "f32" else 1
        if kind in ("logprobs", "logprobs_backward"):
            R, V = _log_int(rng, 1, 8192), _log_int(rng, 2, 131072)
            if rng.random() < 0.4:
                V = max(8, V // 8 * 8)
            G = rng.choice([0, 1, 1, 1, 4, _log_int(rng, 1, 64)])
            K = rng.choice([0, 1, 5, 20, _log_int(rng, 1, 64)]) if kind == "logprobs" else 0
            most = 4096 * 50001 if kind == "logprobs" else 8192 * 32768
            c = _logits(None, kind, R, V, G, min(K, V), io, rng.random() < 0.5,
                        kind == "logprobs" and rng.random() < 0.25, rng.choice([0, 0, 8, 3]),
                        rng.choice([1.0, 1.0, 0.7, 1.5]))
            if R * V * wide <= most:
                return c
        elif kind in ("norm", "norm_backward"):
            after, before = rng.random() < 0.6, rng.random() < 0.7
            gate = rng.choice(["", "silu", "sigmoid"])
            residual = rng.choice(["", "bf16", "f32"])
            T = _log_int(rng, 1, 16384)
            H = rng.choice([1, 1, 3, 8, 16])
            D = rng.choice([32, 64, 80, 128, 256, 8 * _log_int(rng, 2, 512)])
            most = 16384 * 2048 if kind == "norm" else 8191 * 2048
            c = _norm(None, kind, T, H, D, after, before, gate, residual,
                      rng.random() < 0.4, io)
            if (after or before or gate or residual) and T * H * D * wide <= most:
                return c
        elif kind == "conv_step":
            beams = rng.random() < 0.5
            c = _step(None, _log_int(rng, 1, 512), rng.choice([1, 1, 1, 2, 5]),
                      8 * _log_int(rng, 1, 1024), rng.choice([2, 3, 4, 4]), beams, io,
                      rng.random() < 0.8, rng.random() < 0.3)
            if c["N"] * (c["T"] + 4) * c["C"] * wide <= 512 * 5 * 6144:
                return c
        else:
            N = _log_int(rng, 1, 16)
            c = _conv(None, kind, N, _log_int(rng, 1, 8192), 8 * _log_int(rng, 1, 1024),
                      rng.choice([2, 3, 4, 4]), io, rng.random() < 0.8, rng.random() < 0.3,
                      N > 1 and rng.random() < 0.6, rng.random() < 0.5)
            most = sum(_lengths({"N": 16, "T": 1000, "ragged": True})) * 6144
            if kind == "conv_backward":
                most = 8192 * 6144
            n = sum(_lengths(c))
            if 1 <= n and (n + 3 * N) * c["C"] * wide <= most:
                return c


def _lengths(c):
    if not c["ragged"]:
        return [c["T"]] * c["N"]
    r = random.Random(c["N"] * 100003 + c["T"])
    return [r.randrange(0, 2 * c["T"] + 1) for _ in range(c["N"])]


# ---- inputs --------------------------------------------------------------------------

def _dtype(io):
    return torch.bfloat16 if io == "bf16" else torch.float32


class _Draws:
    """Draws on the GPU from one seeded generator."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=torch.float32)

    def index(self, most, *shape):
        return torch.randint(0, most, shape, generator=self.g, device=DEV)


def prepare(case, seed):
    c, d = dict(case), _Draws(seed)
    x = {"case": c, "op": None}
    if c["kind"].startswith("logprobs"):
        _prepare_logits(c, d, x)
    elif c["kind"].startswith("norm"):
        _prepare_norm(c, d, x)
    else:
        _prepare_conv(c, d, x)
    return x


def _prepare_logits(c, d, x):
    R, V, G = c["R"], c["V"], c["G"]
    z = torch.empty((R, V + c["pad"]), dtype=_dtype(c["io"]), device=DEV)
    for i in range(0, R, 1024):  # (a part at a time: the draws are in 32 bits)
        part = 2.0 * d.normal(min(1024, R - i), V + c["pad"])
        part.scatter_add_(1, d.index(V, part.shape[0], 1), torch.full_like(part[:, :1], 9.0))
        if c["masked"]:
            part[torch.rand(part.shape, generator=d.g, device=DEV) < 0.7] = float("-inf")
            if i == 0 and R > 1:
                part[0] = float("-inf")
        z[i:i + 1024] = part
    x["logits"] = z[:, :V]
    x["given"] = None
    if G:
        given = d.index(V, R, G).to(torch.int32)
        given[torch.rand(given.shape, generator=d.g, device=DEV) < 0.06] = -1  # padding
        x["given"] = given
    if c["kind"] == "logprobs_backward":
        # what the forward call left
        x["lse"], x["entropy"] = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
        for i in range(0, R, 1024):
            logp = c["scale"] * x["logits"][i:i + 1024].double()
            lse = torch.logsumexp(logp, 1)
            logp -= lse[:, None]
            x["lse"][i:i + 1024] = lse
            x["entropy"][i:i + 1024] = -(logp.exp() * logp).sum(1)
        x["dlogp"] = -torch.rand((R, G), generator=d.g, device=DEV) / R if G else None
        x["dlse"] = 1e-4 * d.normal(R) if not G or c["entropy"] else None
        x["dentropy"] = 1e-2 * d.normal(R) / R if c["entropy"] else None


def _prepare_norm(c, d, x):
    T, H, D = c["T"], c["H"], c["D"]
    dt = _dtype(c["io"])
    x["eps"], x["scale"] = 1e-6, 0.5
    x["x"] = d.normal(T, H, D).to(dt)
    # the gate stands in a projection's output, beside other columns
    x["gate"] = d.normal(T, H * D + 64).to(dt)[:, 64:].unflatten(1, (H, D)) if c["gate"] else None
    x["residual"] = (2.0 * d.normal(T, H, D)).to(_dtype(c["residual"])) if c["residual"] else None
    x["wa"] = 1.0 + 0.1 * d.normal(D) if c["after"] else None
    x["wb"] = 1.0 + 0.1 * d.normal(D) if c["before"] else None
    x["cs"] = 1.0 + 0.3 * d.normal(D) if c["channel"] else None
    if c["kind"] == "norm_backward":
        x["dy"] = d.normal(T, H, D).to(dt) if c["before"] or not c["residual"] else None
        x["dres"] = d.normal(T, H, D).to(_dtype(c["residual"])) if c["residual"] else None


def _prepare_conv(c, d, x):
    C, S = c["C"], c["taps"] - 1
    dt = _dtype(c["io"])
    x["w"] = d.normal(C, c["taps"]) * c["taps"] ** -0.5
    x["bias"] = 0.1 * d.normal(C) if c["bias"] else None
    if c["kind"] == "conv_step":
        N = c["N"]
        rows = d.normal(N * c["T"], C + 64).to(dt)
        x["x"] = rows[:, :C]
        slots = N + 7
        x["pool"] = d.normal(slots, S, C).to(dt)
        if c["beams"]:
            x["slots"] = d.index(max(1, N // 2), N).to(torch.int32)  # parents, some of several
            x["pool_out"] = torch.zeros((N, S, C), dtype=dt, device=DEV)
        else:
            x["slots"] = torch.randperm(slots, generator=d.g, device=DEV)[:N].to(torch.int32)
            x["pool_out"] = None
        return
    x["lengths"] = _lengths(c)
    n = sum(x["lengths"])
    # the convolution's channels stand beside a gate in a projection's output
    x["x"] = d.normal(n, C + 64).to(dt)[:, :C]
    x["offsets"] = None
    if c["ragged"]:
        off = torch.tensor([0] + x["lengths"], device=DEV)
        x["offsets"] = torch.cumsum(off, 0).to(torch.int32)
    x["state"] = d.normal(c["N"], S, C).to(dt) if c["state"] else None
    if c["kind"] == "conv_backward":
        x["dy"] = d.normal(n, C).to(dt)
        x["dstate"] = d.normal(c["N"], S, C).to(dt) if c["state"] else None


# ---- one pass ------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _make_own(x):
    """The object that a program keeps: its workspace and output tensors."""
    from paper_2609_12399_amd import runner
    c = x["case"]
    if c["kind"].startswith("logprobs"):
        return runner.TokenLogprobs(c["R"], c["V"], num_given=c["G"], num_top=c["K"], io=c["io"],
                                    scale=c["scale"], entropy=c["entropy"],
                                    backward=c["kind"] == "logprobs_backward", device=DEV)
    if c["kind"].startswith("norm"):
        return runner.BlockNorm(c["T"], c["D"], num_heads=c["H"], io=c["io"],
                                residual_io=c["residual"] or None, norm_after=c["after"],
                                norm_before=c["before"], gate=c["gate"] or None,
                                residual_scale=x["scale"], eps=x["eps"],
                                backward=c["kind"] == "norm_backward", device=DEV)
    act = "silu" if c["silu"] else None
    if c["kind"] == "conv_step":
        return runner.ShortConvStep(c["N"], c["N"] * c["T"], c["C"], c["taps"], c["io"],
                                    x["pool"].shape[0], activation=act, device=DEV)
    return runner.ShortConv(c["N"], x["x"].shape[0], c["C"], c["taps"], c["io"], activation=act,
                            backward=c["kind"] == "conv_backward", device=DEV)


def _run_own(x):
    c, op = x["case"], x["op"]
    if op is None:
        op = x["op"] = _make_own(x)
    if c["kind"] == "logprobs":
        return op.forward(x["logits"], x["given"])
    if c["kind"] == "logprobs_backward":
        return op.backward(x["logits"], x["given"], x["lse"], x["dlogp"], x["dlse"], x["entropy"],
                           x["dentropy"])
    if c["kind"] == "norm":
        return op.forward(x["x"], x["residual"], x["gate"], x["wa"], x["wb"], x["cs"])
    if c["kind"] == "norm_backward":
        return op.backward(x["x"], x["dy"], x["residual"], x["gate"], x["wa"], x["wb"], x["cs"],
                           x["dres"])
    if c["kind"] == "conv":
        return op.forward(x["x"], x["w"], x["bias"], x["offsets"], x["state"])
    if c["kind"] == "conv_backward":
        return op.backward(x["x"], x["w"], x["dy"], x["bias"], x["offsets"], x["state"],
                           x["dstate"])
    y = op.step(x["pool"], x["slots"], x["x"], x["w"], x["bias"], pool_out=x["pool_out"])
    return y, x["pool"] if x["pool_out"] is None else x["pool_out"]


def _run_plain(x):
    return {"logprobs": _plain_logprobs, "logprobs_backward": _plain_logprobs_backward,
            "norm": _plain_norm, "norm_backward": _plain_norm_backward, "conv": _plain_conv,
            "conv_backward": _plain_conv_backward, "conv_step": _plain_step}[x["case"]["kind"]](x)


# ---- plain forms ---------------------------------------------------------------------
# Outputs that a call does not make are None.

def _plain_logprobs(x):
    c, V = x["case"], x["case"]["V"]
    z = x["logits"].float()
    m = z.amax(1, keepdim=True)
    gone = torch.isinf(m) & (m < 0)  # a row whose mask leaves nothing
    d = (z - torch.where(gone, 0.0, m)) * c["scale"]
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    logs = torch.log(s)
    lse = torch.where(gone, m, m * c["scale"] + logs)
    entropy = logp = tokens = top = None
    if c["entropy"]:
        h = logs - (e * torch.where(e > 0, d, 0.0)).sum(1, keepdim=True) / s
        entropy = torch.where(gone, 0.0, h)[:, 0]
    if c["G"]:
        given = x["given"].long()
        logp = d.gather(1, given.clamp(0, V - 1)) - logs
        logp = torch.where(gone, m, logp)
        logp = torch.where(given < 0, 0.0, torch.where(given >= V, float("nan"), logp))
    if c["K"]:
        # ties go to the lowest index: one whole number of the value's order and the index
        bits = (z + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
        index = torch.arange(V - 1, -1, -1, device=DEV)
        key = torch.topk(order * 2 ** 32 + index, c["K"], 1).values
        at = V - 1 - key % 2 ** 32
        tokens = at.to(torch.int32)
        top = torch.where(gone, m, d.gather(1, at) - logs)
    return logp, lse[:, 0], entropy, tokens, top


def _plain_logprobs_backward(x):
    c, V = x["case"], x["case"]["V"]
    logp = x["logits"].float() * c["scale"] - x["lse"][:, None]
    a = torch.zeros_like(x["lse"]) if x["dlse"] is None else x["dlse"]
    if c["G"]:
        keep = x["given"] >= 0
        dl = torch.where(keep, x["dlogp"], 0.0)
        a = a - dl.sum(1)
    a = a[:, None]
    if c["entropy"]:
        a = a - x["dentropy"][:, None] * (logp + x["entropy"][:, None])
    dz = torch.exp(logp) * a
    if c["G"]:
        dz.scatter_add_(1, x["given"].clamp(0, V - 1).long(), dl)
    return (c["scale"] * dz).to(_dtype(c["io"]))


def _act(kind, g):
    """The gate's activation and its derivative."""
    s = 1.0 / (1.0 + torch.exp(-g))
    return (g * s, s * (1.0 + g * (1.0 - s))) if kind == "silu" else (s, s * (1.0 - s))


def _rms(x, t):
    return torch.rsqrt((t * t).mean(-1, keepdim=True) + x["eps"])


def _norm_parts(x):
    """x normed, the block's output u, its factor s, the sum h."""
    c, t = x["case"], x["x"].float()
    n = t * _rms(x, t) if c["after"] else t
    u = n * x["wa"] if c["after"] else n
    if c["gate"]:
        u = u * _act(c["gate"], x["gate"].float())[0]
    s = x["scale"] * (torch.ones(c["D"], device=DEV) if x["cs"] is None else x["cs"])
    h = s * u if x["residual"] is None else x["residual"].float() + s * u
    return n, u, s, h


def _plain_norm(x):
    c = x["case"]
    n, u, s, h = _norm_parts(x)
    y = h * _rms(x, h) * x["wb"] if c["before"] else h
    return (y.to(_dtype(c["io"])) if c["before"] or not c["residual"] else None,
            h.to(_dtype(c["residual"])) if c["residual"] else None)


def _back(x, t, d):
    """The gradient by t of t * _rms(t) from that of the result."""
    r = _rms(x, t)
    return r * (d - t * (r * r * (t * d).mean(-1, keepdim=True)))


def _plain_norm_backward(x):
    c, dt = x["case"], _dtype(x["case"]["io"])
    n, u, s, h = _norm_parts(x)
    dh = 0.0 if x["dres"] is None else x["dres"].float()
    dwa = dwb = dcs = dgate = dres = None
    if x["dy"] is not None:
        dy = x["dy"].float()
        if c["before"]:
            dwb = (dy * h * _rms(x, h)).sum((0, 1))
            dh = dh + _back(x, h, dy * x["wb"])
        else:
            dh = dh + dy
    if c["residual"]:
        dres = dh.to(_dtype(c["residual"]))
    if c["channel"]:
        dcs = x["scale"] * (dh * u).sum((0, 1))
    du = dh * s
    if c["gate"]:
        a, da = _act(c["gate"], x["gate"].float())
        dgate = (du * da * (n * x["wa"] if c["after"] else n)).to(dt)
        du = du * a
    if c["after"]:
        dwa = (du * n).sum((0, 1))
        du = _back(x, x["x"].float(), du * x["wa"])
    return du.to(dt), dres, dgate, dwa, dwb, dcs


def _places(x):
    """Where the inputs of every token stand in the rows of x followed by those of the states
    (or by one row of zeros): [taps][tokens]; the same for the last states."""
    c, n, S = x["case"], x["x"].shape[0], x["case"]["taps"] - 1
    t = torch.arange(n, device=DEV)
    if x["offsets"] is None:
        begin = torch.arange(c["N"] + 1, device=DEV) * c["T"]
    else:
        begin = x["offsets"].long()
    seq = torch.searchsorted(begin, t, right=True) - 1

    def place(seq, p):  # of input p (below 0: before the sequence)
        old = n + seq * S + S + p if c["state"] else torch.full_like(p, n)
        return torch.where(p >= 0, begin[seq] + p, old)

    tap = torch.arange(-S, 1, device=DEV)[:, None]
    ends = place(torch.arange(c["N"], device=DEV)[:, None],
                 (begin[1:] - begin[:-1])[:, None] + tap[:-1, 0])
    return place(seq[None], (t - begin[seq])[None] + tap), ends


def _rows(x):
    """The rows that _places speaks of, in 32 bits."""
    old = (x["state"].flatten(0, 1).float() if x["case"]["state"] else
           torch.zeros((1, x["case"]["C"]), device=DEV))
    return torch.cat([x["x"].float(), old])


def _pre(x, rows, at):
    """The sums before the activation, tap by tap."""
    y = sum(x["w"][:, j] * rows[at[j]] for j in range(x["case"]["taps"]))
    return y if x["bias"] is None else y + x["bias"]


def _plain_conv(x):
    c, dt = x["case"], _dtype(x["case"]["io"])
    (at, ends), rows = _places(x), _rows(x)
    y = _pre(x, rows, at)
    return (_act("silu", y)[0] if c["silu"] else y).to(dt), rows[ends].to(dt)


def _plain_conv_backward(x):
    c, dt, n = x["case"], _dtype(x["case"]["io"]), x["x"].shape[0]
    (at, ends), rows = _places(x), _rows(x)
    g = x["dy"].float()
    if c["silu"]:
        g = g * _act("silu", _pre(x, rows, at))[1]
    dw = torch.stack([(g * rows[at[j]]).sum(0) for j in range(c["taps"])], 1)
    db = None if x["bias"] is None else g.sum(0)
    # (of one tap no two tokens read the same row, but for the row of zeros)
    drows = torch.zeros_like(rows)
    drows = sum((drows.clone().index_add_(0, at[j], x["w"][:, j] * g) for j in range(c["taps"])),
                drows)
    if x["dstate"] is not None:
        drows.index_add_(0, ends.flatten(), x["dstate"].flatten(0, 1).float())
    dstate = drows[n:].unflatten(0, (c["N"], c["taps"] - 1)).to(dt) if c["state"] else None
    return drows[:n].to(dt), dw, db, dstate


def _plain_step(x):
    c, dt = x["case"], _dtype(x["case"]["io"])
    new = x["x"].float().unflatten(0, (c["N"], c["T"]))
    rows = torch.cat([x["pool"][x["slots"].long()].float(), new], 1)
    y = sum(x["w"][:, j] * rows[:, j:j + c["T"]] for j in range(c["taps"]))
    if x["bias"] is not None:
        y = y + x["bias"]
    y = (_act("silu", y)[0] if c["silu"] else y).flatten(0, 1).to(dt)
    last = rows[:, c["T"]:].to(dt)
    if x["pool_out"] is None:
        x["pool"][x["slots"].long()] = last
        return y, x["pool"]
    x["pool_out"].copy_(last)
    return y, x["pool_out"]


# ---- work ----------------------------------------------------------------------------

def work(case):
    c = case
    size = 2 if c["io"] == "bf16" else 4
    if c["kind"].startswith("logprobs"):
        n, rows = c["R"] * c["V"], c["R"] * 4
        given = 2 * rows * c["G"]  # the tokens and their log probabilities (or gradients)
        if c["kind"] == "logprobs":
            return {"bytes": n * size + given + rows * (1 + c["entropy"] + 2 * c["K"]),
                    "flops": n * (4 + 2 * c["entropy"])}
        more = 1 + 2 * c["entropy"] + (not c["G"] or c["entropy"])
        return {"bytes": 2 * n * size + given + rows * more, "flops": n * (4 + 3 * c["entropy"])}
    if c["kind"].startswith("norm"):
        n, res = c["T"] * c["H"] * c["D"], {"": 0, "bf16": 2, "f32": 4}[c["residual"]]
        gate, y = bool(c["gate"]) * size, (c["before"] or not c["residual"]) * size
        vectors = 4 * c["D"] * (c["after"] + c["before"] + c["channel"])
        if c["kind"] == "norm":
            return {"bytes": n * (size + gate + 2 * res + y) + vectors,
                    "flops": n * (4 * c["after"] + 4 * c["before"] + 6 * bool(gate) + 2)}
        # x, gate, residual and the outputs' gradients read, three gradients written
        return {"bytes": n * (2 * size + 2 * gate + 3 * res + y) + 2 * vectors,
                "flops": n * (12 * c["after"] + 12 * c["before"] + 12 * bool(gate) + 4)}
    rows = c["N"] * c["T"] if c["kind"] == "conv_step" else sum(_lengths(c))
    n, states = rows * c["C"], c["N"] * (c["taps"] - 1) * c["C"] * size
    vectors = 4 * c["C"] * (c["taps"] + c["bias"])
    if c["kind"] == "conv_step":
        # (a parent's state is read once, however many go on from it)
        read = 0.5 * states if c["beams"] else states
        return {"bytes": 2 * n * size + read + states + vectors,
                "flops": n * (2 * c["taps"] + 6 * c["silu"])}
    if c["kind"] == "conv":
        return {"bytes": 2 * n * size + states * (1 + c["state"]) + vectors,
                "flops": n * (2 * c["taps"] + 6 * c["silu"])}
    return {"bytes": 3 * n * size + 3 * states * c["state"] + 2 * vectors,
            "flops": n * (6 * c["taps"] + 12 * c["silu"])}


# ---- the definitions in 64 bits ----------------------------------------------------------

def exact(case, seed):
    x = prepare(case, seed)
    with torch.enable_grad():
        if case["kind"].startswith("logprobs"):
            return _exact_logits(x)
        if case["kind"].startswith("norm"):
            return _exact_norm(x)
        return _exact_step(x) if case["kind"] == "conv_step" else _exact_conv(x)


def _exact_logits(x):
    """In parts of some rows."""
    c, parts = x["case"], []
    rows = max(1, 2 ** 26 // c["V"])
    for i in range(0, c["R"], rows):
        z = x["logits"][i:i + rows].double()
        given = None if x["given"] is None else x["given"][i:i + rows].long()
        gone = torch.isneginf(z).all(1)
        if c["kind"] == "logprobs":
            logp = torch.log_softmax(torch.where(gone[:, None], 0.0, z) * c["scale"], 1)
            logp[gone] = float("-inf")
            lse = torch.logsumexp(z * c["scale"], 1)
            p = torch.exp(logp)
            picked = entropy = tokens = top = None
            if c["entropy"]:
                entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
            if c["G"]:
                picked = logp.gather(1, given.clamp(min=0)) .masked_fill(given < 0, 0.0)
            if c["K"]:
                tokens = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :c["K"]]
                top, tokens = logp.gather(1, tokens), tokens.to(torch.int32)
            parts.append((picked, lse, entropy, tokens, top))
            continue
        z.requires_grad_()
        logp = torch.log_softmax(z * c["scale"], 1)
        total = 0.0
        if c["G"]:
            picked = logp.gather(1, given.clamp(min=0)).masked_fill(given < 0, 0.0)
            total = total + (picked * x["dlogp"][i:i + rows].double()).sum()
        if x["dlse"] is not None:
            lse = torch.logsumexp(z * c["scale"], 1)
            total = total + (lse * x["dlse"][i:i + rows].double()).sum()
        if c["entropy"]:
            h = -(torch.exp(logp) * logp).sum(1)
            total = total + (h * x["dentropy"][i:i + rows].double()).sum()
        parts.append(torch.autograd.grad(total, z)[0])
    if c["kind"] == "logprobs_backward":
        return torch.cat(parts)
    return tuple(None if p[0] is None else torch.cat(p) for p in zip(*parts))


def _exact_norm(x):
    c = x["case"]

    def leaf(t):
        return None if t is None else t.double().requires_grad_()

    t, res, gate, wa, wb, cs = (leaf(x[k]) for k in ("x", "residual", "gate", "wa", "wb", "cs"))

    def normed(v, w):
        return w * v / torch.sqrt(v.square().sum(-1, keepdim=True) / c["D"] + x["eps"])

    u = normed(t, wa) if c["after"] else t
    if c["gate"]:
        u = u * (torch.nn.functional.silu(gate) if c["gate"] == "silu" else torch.sigmoid(gate))
    u = u * x["scale"]
    if c["channel"]:
        u = u * cs
    h = u + res if c["residual"] else u
    y = normed(h, wb) if c["before"] else h
    y = y if c["before"] or not c["residual"] else None
    h = h if c["residual"] else None
    if c["kind"] == "norm":
        return tuple(None if v is None else v.detach() for v in (y, h))
    total = 0.0
    if y is not None:
        total = total + (y * x["dy"].double()).sum()
    if h is not None:
        total = total + (h * x["dres"].double()).sum()
    wanted = [v for v in (t, res, gate, wa, wb, cs) if v is not None]
    grads = iter(torch.autograd.grad(total, wanted))
    return tuple(None if v is None else next(grads) for v in (t, res, gate, wa, wb, cs))


def _exact_conv(x):
    c, S = x["case"], x["case"]["taps"] - 1
    backward = c["kind"] == "conv_backward"
    t = x["x"].double().requires_grad_(backward)
    w = x["w"].double().requires_grad_(backward)
    bias = None if x["bias"] is None else x["bias"].double().requires_grad_(backward)
    if x["state"] is None:
        state = torch.zeros((c["N"], S, c["C"]), dtype=torch.float64, device=DEV)
    else:
        state = x["state"].double().requires_grad_(backward)
    ys, lasts, start = [], [], 0
    for i, n in enumerate(x["lengths"]):
        rows = torch.cat([state[i], t[start:start + n]])
        y = (rows.unfold(0, S + 1, 1) * w).sum(-1) if n else rows[:0]
        if bias is not None:
            y = y + bias
        ys.append(torch.nn.functional.silu(y) if c["silu"] else y)
        lasts.append(rows[n:])
        start += n
    y, last = torch.cat(ys), torch.stack(lasts)
    if not backward:
        return y, last
    total = (y * x["dy"].double()).sum()
    if x["dstate"] is not None:
        total = total + (last * x["dstate"].double()).sum()
    wanted = [v for v in (t, w, bias, state if c["state"] else None) if v is not None]
    grads = iter(torch.autograd.grad(total, wanted))
    return tuple(None if v is None else next(grads)
                 for v in (t, w, bias, state if c["state"] else None))


def _exact_step(x):
    c, S = x["case"], x["case"]["taps"] - 1
    slots = x["slots"].long()
    rows = torch.cat([x["pool"].double()[slots], x["x"].double().unflatten(0, (c["N"], c["T"]))],
                     1)
    y = (rows.unfold(1, S + 1, 1) * x["w"].double()).sum(-1)
    if x["bias"] is not None:
        y = y + x["bias"].double()
    y = torch.nn.functional.silu(y) if c["silu"] else y
    pool = x["pool"].double() if x["pool_out"] is None else x["pool_out"].double()
    pool[slots if x["pool_out"] is None else slice(None)] = rows[:, c["T"]:]
    return y.flatten(0, 1), pool
