"""A Gated DeltaNet mixing layer on the library's operators: what stands around the
large-beam decode in a model.

One layer projects its input to queries, keys, values and two gates per value head, may pass
them through a short causal convolution (``onela_short_conv*``), norms and turns the queries and
keys (``onela_qk_norm_rope``), mixes the tokens by the delta rule (``onela_delta_rule_*``), may norm
the heads' outputs and gate them (``onela_block_norm``) and projects back.  The same weights serve

* a training step: :meth:`DeltaMixer.__call__` is differentiable (the operators' own
  backward passes);
* a prompt: :meth:`DeltaMixer.prompt` gives the outputs and the states after it;
* single tokens: :meth:`DeltaMixer.step` moves the states of a pool on in place;
* a beam search from a prompt's state: :meth:`DeltaMixer.beam_step_inputs` gives what
  one step of :class:`runner.Decoder` takes.

Rows behind the last sequence of a padded batch are 0 in the functions' outputs and gradients
(the calls' ``clear_rest``), since products and sums over tokens follow.

The operators' functions may be captured into a graph, forward and backward together.  As with
anything in torch, no outputs of an eager pass on the same leaves may be alive then: their nodes
belong to the stream of that pass, and a capture that meets them ends in an error or the process.

A layer with a convolution has two states, (the delta rule's, the convolution's), wherever one
without has the first alone.  :mod:`recommender` puts such layers into a model.

    python -m paper_2609_12399_amd.mixer        # trains a small layer, then serves with it
"""
from __future__ import annotations

import torch

from . import runner


def _io(x) -> str:
    return {torch.bfloat16: "bf16", torch.float32: "f32"}[x.dtype]


class _Once(torch.autograd.Function):
    """A gradient that cannot be differentiated itself."""

    @staticmethod
    def forward(ctx, g):
        return g.view_as(g)

    @staticmethod
    def backward(ctx, d):
        raise RuntimeError("the gradients of the library's operators are differentiable once")


def _once(grads):
    """The results of a backward pass: where it runs to be differentiated (create_graph), ones that
    refuse it.  (torch's own mark for this lets them pass as constants when the gradients that
    come in are some.)"""
    if not torch.is_grad_enabled():
        return grads
    return tuple(None if g is None else _Once.apply(g.detach().requires_grad_()) for g in grads)


class QkNormRopeFunction(torch.autograd.Function):
    """q, k [tokens][heads][D], weights fp32 [D] or None -> both normed and turned."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, cos_sin, norm, rotary_dim, eps):
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, cos_sin)
        ctx.args = dict(norm=norm, rotary_dim=rotary_dim, eps=eps, device=q.device)
        op = runner.QkNormRope(q.shape[0], q.shape[1], k.shape[1], q.shape[2], _io(q), **ctx.args)
        return op.forward(q, k, q_weight, k_weight, positions, cos_sin)

    @staticmethod
    def backward(ctx, d_q, d_k):
        q, k, q_weight, k_weight, positions, cos_sin = ctx.saved_tensors
        op = runner.QkNormRope(q.shape[0], q.shape[1], k.shape[1], q.shape[2], _io(q),
                               backward=True, **ctx.args)
        grads = op.backward(q, k, d_q.contiguous(), d_k.contiguous(), q_weight, k_weight,
                            positions, cos_sin)
        return (*_once(grads), None, None, None, None, None)


class DeltaRuleFunction(torch.autograd.Function):
    """(o, final state) of packed sequences; seq_offsets int32 [num_seqs + 1] or None."""

    @staticmethod
    def forward(ctx, q, k, v, log_alpha, beta, seq_offsets, initial_state, num_seqs, scale):
        ctx.save_for_backward(q, k, v, log_alpha, beta, seq_offsets, initial_state)
        ctx.sizes = (num_seqs, q.shape[0], q.shape[1], v.shape[1], q.shape[2], v.shape[2], _io(q))
        ctx.scale = scale
        op = runner.DeltaRule(*ctx.sizes, scale=scale, device=q.device, clear_rest=True)
        return op.forward(q, k, v, log_alpha, beta, seq_offsets, initial_state)

    @staticmethod
    def backward(ctx, d_o, d_state):
        q, k, v, log_alpha, beta, seq_offsets, initial_state = ctx.saved_tensors
        op = runner.DeltaRule(*ctx.sizes, scale=ctx.scale, backward=True, device=q.device,
                              clear_rest=True)
        dq, dk, dv, dla, db, ds = _once(op.backward(
            q, k, v, log_alpha, beta, d_o.contiguous(), seq_offsets, initial_state,
            d_state.contiguous()))
        return dq, dk, dv, dla, db, None, ds, None, None


class ShortConvFunction(torch.autograd.Function):
    """x [tokens][channels], weight fp32 [channels][taps] -> (y, last states); seq_offsets int32
    [num_seqs + 1] or None, initial_state [num_seqs][taps - 1][channels] or None."""

    @staticmethod
    def forward(ctx, x, weight, bias, seq_offsets, initial_state, num_seqs, activation):
        ctx.save_for_backward(x, weight, bias, seq_offsets, initial_state)
        ctx.sizes = (num_seqs, *x.shape, weight.shape[1], _io(x), activation)
        op = runner.ShortConv(*ctx.sizes, device=x.device, clear_rest=True)
        return op.forward(x, weight, bias, seq_offsets, initial_state)

    @staticmethod
    def backward(ctx, d_y, d_state):
        x, weight, bias, seq_offsets, initial_state = ctx.saved_tensors
        op = runner.ShortConv(*ctx.sizes, backward=True, device=x.device, clear_rest=True)
        dx, dw, db, ds = _once(op.backward(x, weight, d_y.contiguous(), bias, seq_offsets,
                                           initial_state, d_state.contiguous()))
        return dx, dw, db, None, ds, None, None


class BlockNormFunction(torch.autograd.Function):
    """(y, h) of runner.BlockNorm: x and gate [tokens][heads][width], residual of either type;
    what is None is left out (y with a residual and without norm_before, h without a residual)."""

    @staticmethod
    def forward(ctx, x, residual, gate, after_weight, before_weight, channel_scale, norm_after,
                norm_before, activation, residual_scale, eps):
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x, residual, gate, after_weight, before_weight, channel_scale)
        T, H, D = x.shape
        ctx.sizes = (T, D, H, _io(x), None if residual is None else _io(residual), norm_after,
                     norm_before, activation, residual_scale, eps)
        op = runner.BlockNorm(*ctx.sizes, device=x.device)
        return op.forward(x, residual, gate, after_weight, before_weight, channel_scale)

    @staticmethod
    def backward(ctx, d_y, d_h):
        x, residual, gate, wa, wb, cs = ctx.saved_tensors
        if d_y is None and d_h is None:
            return (None,) * 11
        d_y, d_h = (None if d is None else d.contiguous() for d in (d_y, d_h))
        op = runner.BlockNorm(*ctx.sizes, backward=True, device=x.device)
        grads = op.backward(x, d_y, residual, gate, wa, wb, cs, d_h)
        return (*_once(grads), None, None, None, None, None)


class TokenLogprobsFunction(torch.autograd.Function):
    """(logp of the given tokens, lse, entropy, best tokens, their logp) of runner.TokenLogprobs;
    the best ones are not differentiated (given again, they are)."""

    @staticmethod
    def forward(ctx, logits, given, num_top, scale, entropy):
        ctx.set_materialize_grads(False)
        num_given = 0 if given is None else given.shape[1]
        ctx.sizes = (*logits.shape, num_given, 0, _io(logits), scale)
        op = runner.TokenLogprobs(*logits.shape, num_given, num_top, _io(logits), scale, entropy,
                                  device=logits.device)
        out = op.forward(logits, given)
        ctx.save_for_backward(logits, given, out[1], out[2])
        ctx.mark_non_differentiable(*(t for t in out[3:] if t is not None))
        return out

    @staticmethod
    def backward(ctx, d_logp, d_lse, d_entropy, *_):
        logits, given, lse, entropy = ctx.saved_tensors
        if d_logp is None and d_lse is None and d_entropy is None:
            return (None,) * 5
        if d_logp is None and given is not None:
            d_logp = torch.zeros(given.shape, device=logits.device)
        d_logp, d_lse, d_entropy = (None if d is None else d.contiguous()
                                    for d in (d_logp, d_lse, d_entropy))
        op = runner.TokenLogprobs(*ctx.sizes, backward=True, device=logits.device)
        return (*_once((op.backward(logits, given, lse, d_logp, d_lse, entropy, d_entropy),)),
                None, None, None, None)


class BeamStates:
    """What one layer keeps of a search's beams beside the decoder: the convolution's states, one
    for each beam of the last step (at first one for each request, of its prompt), and the
    present step's output gates."""

    def __init__(self, conv=None):
        self.conv, self.gate = conv, None


class DeltaMixer:
    """One layer's weights and its four uses.  ``rotary_dim`` columns of each query and key
    turn with the token's position (0: none, as the delta rule has it by itself); with
    ``conv_taps`` queries, keys and values pass a causal convolution of that length and silu;
    ``gated`` norms every value head's output and multiplies it by the silu of a projection."""

    def __init__(self, width: int, num_qk_heads: int, num_v_heads: int, d_k: int, d_v: int,
                 io: str = "bf16", rotary_dim: int = 0, max_positions: int = 0, seed: int = 0,
                 device="cuda:0", conv_taps: int = 0, gated: bool = False):
        g = torch.Generator(device=device).manual_seed(seed)
        dt = {"bf16": torch.bfloat16, "f32": torch.float32}[io]
        self.HK, self.HV, self.dk, self.dv = num_qk_heads, num_v_heads, d_k, d_v
        self.io, self.rotary_dim, self.device = io, rotary_dim, device
        self.qkv_width = 2 * num_qk_heads * d_k + num_v_heads * d_v

        def weight(n, m, dtype):
            w = torch.randn((n, m), generator=g, device=device) * n ** -0.5
            return w.to(dtype).requires_grad_()

        self.conv_taps, self.gated = conv_taps, gated
        # (the output gate's columns stand behind those of queries, keys and values)
        self.w_qkv = weight(width, self.qkv_width + (num_v_heads * d_v if gated else 0), dt)
        self.w_gates = weight(width, 2 * num_v_heads, torch.float32)
        self.w_out = weight(num_v_heads * d_v, width, dt)
        self.w_conv = self.w_norm = None
        if conv_taps:
            self.w_conv = weight(conv_taps, self.qkv_width, torch.float32).detach().T.contiguous()
            self.w_conv.requires_grad_()
        if gated:
            self.w_norm = torch.ones(d_v, device=device, requires_grad=True)
        self.cos_sin = None
        if rotary_dim:
            f = 10000.0 ** (-torch.arange(0, rotary_dim, 2, device=device) / rotary_dim)
            a = torch.arange(max_positions, device=device)[:, None] * f
            self.cos_sin = torch.cat([a.cos(), a.sin()], 1)

    def weights(self):
        return [w for w in (self.w_qkv, self.w_gates, self.w_out, self.w_conv, self.w_norm)
                if w is not None]

    def _project(self, x):
        """Rows of queries, keys and values side by side, and the output gates or None (views)."""
        rows = x @ self.w_qkv
        if not self.gated:
            return rows, None
        return rows[:, :self.qkv_width], rows[:, self.qkv_width:].unflatten(1, (self.HV, self.dv))

    def _read_out(self, o, gate):
        """The delta rule's outputs [tokens][heads][d_v] through the gate, projected back."""
        if self.gated:
            o, _ = BlockNormFunction.apply(o, None, gate, self.w_norm, None, None, True, False,
                                           "silu", 1.0, 1e-6)
        return o.flatten(1) @ self.w_out

    def _inputs(self, x, positions, rows=None):
        """q, k (normed, turned), v (a view of the projection), log(alpha), beta of tokens x, whose
        projected (and convolved) rows are given where they are not x @ w_qkv."""
        if self.rotary_dim and positions is None:
            raise ValueError("a layer that rotates needs the tokens' positions")
        qk = self.HK * self.dk
        if rows is None:
            rows, _ = self._project(x)
        q = rows[:, :qk].unflatten(1, (self.HK, self.dk))
        k = rows[:, qk:2 * qk].unflatten(1, (self.HK, self.dk))
        v = rows[:, 2 * qk:].unflatten(1, (self.HV, self.dv))
        q, k = QkNormRopeFunction.apply(q, k, None, None, positions, self.cos_sin, "l2",
                                        self.rotary_dim, 1e-6)
        with torch.autocast(x.device.type, enabled=False):  # (the gates are fp32 throughout)
            gates = x.float() @ self.w_gates
            log_alpha = -torch.nn.functional.softplus(gates[:, :self.HV] - 3.0)
            return q, k, v, log_alpha, torch.sigmoid(gates[:, self.HV:])

    def __call__(self, x, seq_offsets, positions=None, initial_state=None):
        """Outputs [tokens][width] and states of packed sequences; differentiable.  Without
        positions every sequence's tokens count from 0 (rows behind the last sequence have 0: a
        position outside the table has NaN for its gradients, which would reach the weights; given
        ones have to be inside in these rows too)."""
        if self.rotary_dim and positions is None:
            t = torch.arange(x.shape[0], dtype=torch.int32, device=x.device)
            positions = t - seq_offsets[torch.searchsorted(seq_offsets, t, right=True) - 1]
            positions = positions * (t < seq_offsets[-1])
        N = seq_offsets.numel() - 1
        rows, gate = self._project(x)
        if self.conv_taps:
            initial_state, conv = (None, None) if initial_state is None else initial_state
            rows, conv = ShortConvFunction.apply(rows, self.w_conv, None, seq_offsets, conv, N,
                                                 "silu")
        q, k, v, la, b = self._inputs(x, positions, rows)
        o, state = DeltaRuleFunction.apply(q, k, v, la.contiguous(), b.contiguous(), seq_offsets,
                                           initial_state, N, 1.0)
        return self._read_out(o, gate), (state, conv) if self.conv_taps else state

    @torch.no_grad()
    def prompt(self, x, seq_offsets, positions=None, initial_state=None):
        """As the call, without gradients; from initial_state (another prompt's states) or zeros."""
        return self(x, seq_offsets, positions, initial_state)

    @torch.no_grad()
    def step(self, x, pool, slots, positions=None):
        """One token for each row of x on the states slots of the pool, in place."""
        n = x.shape[0]
        rows, gate = self._project(x)
        if self.conv_taps:
            pool, conv = pool
            rows = runner.ShortConvStep(n, n, self.qkv_width, self.conv_taps, _io(rows),
                                        conv.shape[0], device=self.device).step(
                                            conv, slots, rows, self.w_conv)
        q, k, v, la, b = self._inputs(x, positions, rows)
        op = runner.DeltaRuleStep(n, n, self.HK, self.HV, self.dk, self.dv, _io(q), pool.shape[0],
                                  device=self.device)
        o = op.step(pool, slots, q, k, v, la.contiguous(), b.contiguous())
        return self._read_out(o, gate)

    @torch.no_grad()
    def beam_step_inputs(self, x, parents=None, positions=None,
                         beams: BeamStates | None = None) -> runner.DeviceStep:
        """x [requests][beams][width] -> the step that runner.Decoder takes; its output o
        goes through :meth:`beam_outputs`.  A layer with a convolution or output gates takes the
        search's ``beams``, which move on."""
        R, W = x.shape[:2]
        x = x.flatten(0, 1)
        rows, gate = self._project(x)
        if (self.conv_taps or self.gated) and beams is None:
            raise ValueError("a layer with a convolution or gates needs the beams' states")
        if self.conv_taps:
            old = beams.conv
            each = old.shape[0] // R  # states of a request
            slots = torch.arange(R, dtype=torch.int32, device=x.device)[:, None] * each
            slots = (slots + (0 if parents is None else parents)).expand(R, W)
            beams.conv = old.new_empty((R * W, *old.shape[1:]))
            rows = runner.ShortConvStep(R * W, R * W, self.qkv_width, self.conv_taps, _io(rows),
                                        old.shape[0], device=self.device).step(
                                            old, slots.flatten().contiguous(), rows, self.w_conv,
                                            pool_out=beams.conv)
        if self.gated:
            beams.gate = gate
        q, k, v, la, b = self._inputs(x, positions, rows)
        q, k, v = (t.to(self.w_qkv.dtype).contiguous().unflatten(0, (R, W)) for t in (q, k, v))
        alpha = torch.exp(la).contiguous().unflatten(0, (R, W))
        return runner.DeviceStep(q, k, v, alpha, b.contiguous().unflatten(0, (R, W)), parents, W)

    @torch.no_grad()
    def beam_outputs(self, o, beams: BeamStates | None = None):
        if not self.gated:
            return o.flatten(2).to(self.w_out.dtype) @ self.w_out
        return self._read_out(o.flatten(0, 1).to(beams.gate.dtype), beams.gate).unflatten(
            0, o.shape[:2])


def train(layer: DeltaMixer, x, target, seq_offsets, positions=None, steps: int = 30,
          lr: float = 3e-3):
    """Adam on the squared error of the layer's outputs; the losses."""
    masters = [w.detach().float().requires_grad_() for w in layer.weights()]
    opt, losses = torch.optim.Adam(masters, lr=lr), []
    for _ in range(steps):
        y, _ = layer(x, seq_offsets, positions)
        loss = torch.nn.functional.mse_loss(y.float(), target)
        for w in layer.weights():
            w.grad = None
        loss.backward()
        for m, w in zip(masters, layer.weights()):
            m.grad = w.grad.float()
        opt.step()
        with torch.no_grad():
            for m, w in zip(masters, layer.weights()):
                w.copy_(m)
        losses.append(float(loss.detach()))
    return losses


def main():
    device, width, HK, HV, d = "cuda:0", 256, 2, 4, 64
    layer = DeltaMixer(width, HK, HV, d, d, rotary_dim=16, max_positions=512, device=device)
    lengths = [300, 17, 130]
    off = torch.tensor([0, 300, 317, 447], dtype=torch.int32, device=device)
    pos = torch.cat([torch.arange(n) for n in lengths]).to(torch.int32).to(device)
    g = torch.Generator(device=device).manual_seed(1)
    x = torch.randn((447, width), generator=g, device=device).bfloat16()
    losses = train(layer, x, torch.roll(x, 1, 0).float(), off, pos)
    print(f"training: loss {losses[0]:.4f} -> {losses[-1]:.4f}")

    y, state = layer.prompt(x, off, pos)
    pool, slots = state.clone(), torch.arange(3, dtype=torch.int32, device=device)
    for t in range(3):
        tok = torch.randn((3, width), generator=g, device=device).bfloat16()
        y = layer.step(tok, pool, slots, torch.tensor(lengths, device=device).int() + t)
    print(f"serving: 3 tokens on 3 states, output norm {float(y.float().norm()):.3f}")

    from .workload import WorkloadSpec
    W = 8
    spec = WorkloadSpec("mixer", 3, HK, HV, d, d, 0, (W,), "bf16", "uniform")
    dec = runner.Decoder(spec, state, device)
    bx = torch.randn((3, W, width), generator=g, device=device).bfloat16()
    bpos = torch.tensor(lengths, device=device).int().repeat_interleave(W)
    o = torch.empty((3, W, HV, d), device=device)
    dec.step(0, layer.beam_step_inputs(bx, positions=bpos), o, fused=True)
    print(f"beams: {W} per request, output norm {float(layer.beam_outputs(o).float().norm()):.3f}")
    dec.close()


if __name__ == "__main__":
    main()
