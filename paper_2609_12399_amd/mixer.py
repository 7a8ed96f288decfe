"""A Gated DeltaNet mixing layer on the library's operators: what stands around the
large-beam decode in a model.

One layer projects its input to queries, keys, values and two gates per value head, norms and
turns the queries and keys (``onela_qk_norm_rope``), mixes the tokens by the delta rule
(``onela_delta_rule_*``) and projects back.  The same weights serve

* a training step: :meth:`DeltaMixer.__call__` is differentiable (the operators' own
  backward passes);
* a prompt: :meth:`DeltaMixer.prompt` gives the outputs and the states after it;
* single tokens: :meth:`DeltaMixer.step` moves the states of a pool on in place;
* a beam search from a prompt's state: :meth:`DeltaMixer.beam_step_inputs` gives what
  one step of :class:`runner.Decoder` takes.

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
        raise RuntimeError("the gradients of the delta rule and of the norm are differentiable once")


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
        op = runner.DeltaRule(*ctx.sizes, scale=scale, device=q.device)
        return op.forward(q, k, v, log_alpha, beta, seq_offsets, initial_state)

    @staticmethod
    def backward(ctx, d_o, d_state):
        q, k, v, log_alpha, beta, seq_offsets, initial_state = ctx.saved_tensors
        op = runner.DeltaRule(*ctx.sizes, scale=ctx.scale, backward=True, device=q.device)
        dq, dk, dv, dla, db, ds = _once(op.backward(
            q, k, v, log_alpha, beta, d_o.contiguous(), seq_offsets, initial_state,
            d_state.contiguous()))
        return dq, dk, dv, dla, db, None, ds, None, None


class DeltaMixer:
    """One layer's weights and its four uses.  ``rotary_dim`` columns of each query and key
    turn with the token's position (0: none, as the delta rule has it by itself)."""

    def __init__(self, width: int, num_qk_heads: int, num_v_heads: int, d_k: int, d_v: int,
                 io: str = "bf16", rotary_dim: int = 0, max_positions: int = 0, seed: int = 0,
                 device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        dt = {"bf16": torch.bfloat16, "f32": torch.float32}[io]
        self.HK, self.HV, self.dk, self.dv = num_qk_heads, num_v_heads, d_k, d_v
        self.io, self.rotary_dim, self.device = io, rotary_dim, device
        self.qkv_width = 2 * num_qk_heads * d_k + num_v_heads * d_v

        def weight(n, m, dtype):
            w = torch.randn((n, m), generator=g, device=device) * n ** -0.5
            return w.to(dtype).requires_grad_()

        self.w_qkv = weight(width, self.qkv_width, dt)
        self.w_gates = weight(width, 2 * num_v_heads, torch.float32)
        self.w_out = weight(num_v_heads * d_v, width, dt)
        self.cos_sin = None
        if rotary_dim:
            f = 10000.0 ** (-torch.arange(0, rotary_dim, 2, device=device) / rotary_dim)
            a = torch.arange(max_positions, device=device)[:, None] * f
            self.cos_sin = torch.cat([a.cos(), a.sin()], 1)

    def weights(self):
        return [self.w_qkv, self.w_gates, self.w_out]

    def _inputs(self, x, positions):
        """q, k (normed, turned), v (a view of the projection), log(alpha), beta of tokens x."""
        if self.rotary_dim and positions is None:
            raise ValueError("a layer that rotates needs the tokens' positions")
        n, qk = x.shape[0], self.HK * self.dk
        rows = x @ self.w_qkv
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
        positions every sequence's tokens count from 0."""
        if self.rotary_dim and positions is None:
            t = torch.arange(x.shape[0], dtype=torch.int32, device=x.device)
            positions = t - seq_offsets[torch.searchsorted(seq_offsets, t, right=True) - 1]
        q, k, v, la, b = self._inputs(x, positions)
        o, state = DeltaRuleFunction.apply(q, k, v, la.contiguous(), b.contiguous(), seq_offsets,
                                           initial_state, seq_offsets.numel() - 1, 1.0)
        return o.flatten(1) @ self.w_out, state

    @torch.no_grad()
    def prompt(self, x, seq_offsets, positions=None, initial_state=None):
        """As the call, without gradients; from initial_state (another prompt's states) or zeros."""
        return self(x, seq_offsets, positions, initial_state)

    @torch.no_grad()
    def step(self, x, pool, slots, positions=None):
        """One token for each row of x on the states slots of the pool, in place."""
        q, k, v, la, b = self._inputs(x, positions)
        op = runner.DeltaRuleStep(x.shape[0], x.shape[0], self.HK, self.HV, self.dk, self.dv,
                                  _io(q), pool.shape[0], device=self.device)
        o = op.step(pool, slots, q, k, v, la.contiguous(), b.contiguous())
        return o.flatten(1) @ self.w_out

    @torch.no_grad()
    def beam_step_inputs(self, x, parents=None, positions=None) -> runner.DeviceStep:
        """x [requests][beams][width] -> the step that runner.Decoder takes; its output o
        goes through :meth:`beam_outputs`."""
        R, W = x.shape[:2]
        q, k, v, la, b = self._inputs(x.flatten(0, 1), positions)
        q, k, v = (t.to(self.w_qkv.dtype).contiguous().unflatten(0, (R, W)) for t in (q, k, v))
        alpha = torch.exp(la).contiguous().unflatten(0, (R, W))
        return runner.DeviceStep(q, k, v, alpha, b.contiguous().unflatten(0, (R, W)), parents, W)

    @torch.no_grad()
    def beam_outputs(self, o):
        return o.flatten(2).to(self.w_out.dtype) @ self.w_out


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
