"""Host-side driver of the decode path on one GPU.

Moves a :mod:`workload` to device memory (PyTorch is used only for
allocation and streams) and drives the C ABI in protocol order: for each
decode step t, ``onela_resolve_ancestry`` -> ``onela_append_records`` ->
``onela_decode_step``.  No arithmetic of the method happens here.
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

from . import onela as ab
from .workload import Tensor, Workload, WorkloadSpec


def _torch():
    import torch
    return torch


def device_tensor(x, device):
    """Copy a workload Tensor / numpy array to the device, keeping its bits."""
    torch = _torch()
    if isinstance(x, Tensor):
        arr = x.dev
        t = torch.from_numpy(np.ascontiguousarray(arr))
        if x.dtype == "bf16":
            t = t.view(torch.bfloat16)
        return t.to(device)
    return torch.from_numpy(np.ascontiguousarray(x)).to(device)


@dataclass
class DeviceStep:
    q: object
    k: object
    v: object
    alpha: object
    beta: object
    parents: object  # None at step 0
    width: int


@dataclass
class DeviceWorkload:
    spec: WorkloadSpec
    steps: list
    prompt: tuple | None  # (k, v, alpha, beta) or None


def to_device(wl: Workload, device="cuda:0", with_prompt: bool = True) -> DeviceWorkload:
    steps = []
    for t, st in enumerate(wl.steps):
        steps.append(DeviceStep(
            device_tensor(st.q, device), device_tensor(st.k, device),
            device_tensor(st.v, device), device_tensor(st.alpha, device),
            device_tensor(st.beta, device),
            None if st.parents is None else device_tensor(st.parents.astype(np.int32), device),
            int(wl.spec.widths[t])))
    prompt = None
    if with_prompt and wl.prompt_k is not None:
        prompt = tuple(device_tensor(x, device) for x in
                       (wl.prompt_k, wl.prompt_v, wl.prompt_alpha, wl.prompt_beta))
    return DeviceWorkload(wl.spec, steps, prompt)


def config_for(spec: WorkloadSpec, max_beams: int | None = None,
               max_steps: int | None = None, records: str = "inputs",
               storage: str = "copy") -> ab.onela_config_t:
    return ab.make_config(spec.R, spec.HK, spec.HV, spec.dk, spec.dv,
                          max_beams or spec.W, max_steps or spec.T, spec.io_dtype, records,
                          storage)


def prefill_state(spec: WorkloadSpec, prompt, device="cuda:0", stream=None):
    """S_ctx [R][HV][dv][dk] fp32 from the prompt, on the GPU."""
    torch = _torch()
    cfg = config_for(spec)
    s0 = torch.empty((spec.R, spec.HV, spec.dv, spec.dk), dtype=torch.float32, device=device)
    k, v, a, b = prompt
    ab.onela_prefill_state(cfg, spec.P, k, v, a, b, s0, stream)
    return s0


class Decoder:
    """One decode context (workspace + onela_ctx_t) bound to a stream."""

    def __init__(self, spec: WorkloadSpec, s0, device="cuda:0", stream=None,
                 max_beams: int | None = None, max_steps: int | None = None,
                 records: str = "inputs", storage: str = "copy"):
        """storage="borrow": the steps' k/v/alpha/beta tensors are the record
        slabs and must outlive the beam search (run() keeps them referenced)."""
        torch = _torch()
        self.spec = spec
        self.cfg = config_for(spec, max_beams, max_steps, records, storage)
        self._borrowed = []
        self.ws_bytes = ab.onela_workspace_bytes(self.cfg)
        if self.ws_bytes == 0:
            raise ab.OnelaError(ab.ONELA_EINVAL, "onela_workspace_bytes")
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.stream = stream
        self.s0 = s0  # borrowed by the context until close()
        self.ctx = ab.onela_init(self.cfg, s0, self.workspace, self.ws_bytes, stream)

    def step(self, t: int, st: DeviceStep, o, gather_out=None, fused: bool = False):
        if self.cfg.record_storage == ab.ONELA_RECORDS_BORROW:
            self._borrowed.append(st)
        if fused:
            ab.onela_decode_step_fused(self.ctx, t, st.width, st.parents, st.k, st.v, st.alpha,
                                       st.beta, st.q, o, gather_out)
            return
        ab.onela_resolve_ancestry(self.ctx, t, st.width, st.parents, gather_out)
        ab.onela_append_records(self.ctx, t, st.k, st.v, st.alpha, st.beta)
        ab.onela_decode_step(self.ctx, t, st.q, o)

    def alloc_outputs(self, dw: DeviceWorkload):
        torch = _torch()
        s = self.spec
        return [torch.empty((s.R, st.width, s.HV, s.dv), dtype=torch.float32,
                            device=self.workspace.device) for st in dw.steps]

    def run(self, dw: DeviceWorkload, outs=None, gathers=None, fused=False):
        """Run every step; ``fused`` is a bool or a per-step list of bools."""
        if outs is None:
            outs = self.alloc_outputs(dw)
        for t, st in enumerate(dw.steps):
            f = fused[t] if isinstance(fused, (list, tuple)) else fused
            self.step(t, st, outs[t], None if gathers is None else gathers[t], f)
        return outs

    def reset(self):
        ab.onela_reset(self.ctx)
        self._borrowed = []

    def status(self) -> int:
        return ab.onela_get_device_status(self.ctx)

    def close(self):
        if self.ctx:
            ab.onela_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class FullStateBaseline:
    """The per-beam materialised-state GPU baseline (one call per step)."""

    def __init__(self, spec: WorkloadSpec, s0, device="cuda:0", stream=None):
        torch = _torch()
        self.spec = spec
        self.cfg = config_for(spec)
        self.s0 = s0
        self.ws_bytes = ab.onela_fullstate_workspace_bytes(self.cfg)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.status_word = torch.zeros(4, dtype=torch.int32, device=device)
        self.stream = stream

    def run(self, dw: DeviceWorkload, outs=None):
        torch = _torch()
        s = self.spec
        if outs is None:
            outs = [torch.empty((s.R, st.width, s.HV, s.dv), dtype=torch.float32,
                                device=self.workspace.device) for st in dw.steps]
        prev = 0
        for t, st in enumerate(dw.steps):
            ab.onela_fullstate_step(self.cfg, t, st.width, prev, st.parents, self.s0, st.q,
                                    st.k, st.v, st.alpha, st.beta, outs[t], self.workspace,
                                    self.ws_bytes, self.status_word, self.stream)
            prev = st.width
        return outs


class BeamSelector:
    """Global top-W beam selection (onela_select_beams) for fixed
    (R, W_prev, V, W): owns the workspace and the three output tensors."""

    def __init__(self, R: int, prev_width: int, vocab: int, width: int, device="cuda:0",
                 stream=None):
        torch = _torch()
        self.R, self.prev_width, self.vocab, self.width = R, prev_width, vocab, width
        self.ws_bytes = ab.onela_select_workspace_bytes(R, prev_width, vocab, width)
        # zero-filled once: the selection keeps its cross-workgroup state
        # here (a call counter, bound words, tagged summaries) and leaves it
        # ready for the next call
        self.workspace = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=device)
        self.parents = torch.empty((R, width), dtype=torch.int32, device=device)
        self.tokens = torch.empty((R, width), dtype=torch.int32, device=device)
        self.scores = torch.empty((R, width), dtype=torch.float32, device=device)
        self.stream = stream

    def __call__(self, logp, beam_scores=None):
        ab.onela_select_beams(self.R, self.prev_width, self.vocab, self.width, logp,
                              beam_scores, self.parents, self.tokens, self.scores,
                              self.workspace, self.ws_bytes, self.stream)
        return self.parents, self.tokens, self.scores


def _io_tensor_dtype(io: str):
    torch = _torch()
    return {"bf16": torch.bfloat16, "f32": torch.float32}[io]


def _expect(*tensors):
    """ValueError unless each (tensor, name, shape, dtype) has this shape and type: the kernels read
    by the object's sizes.  (None and plain addresses are the binding's to judge.)"""
    for x, name, shape, dtype in tensors:
        if x is not None and not isinstance(x, int) and (x.dtype is not dtype or x.shape != shape):
            raise ValueError(f"{name} must be {dtype} {list(shape)}, not {x.dtype} {list(x.shape)}")


def _set_strides(cfg, q, k, v):
    """Elements between the tokens of [tokens][heads][width] views (0: dense)."""
    strides = [0 if x.is_contiguous() else x.stride(0) for x in (q, k, v)]
    cfg.q_stride, cfg.k_stride, cfg.v_stride = strides


class DeltaRule:
    """The gated delta rule over whole sequences (onela_delta_rule_forward and, with
    ``backward``, onela_delta_rule_backward) for fixed sizes: owns the workspace and
    the output tensors, which every call writes again.

    Sequences are packed: ``seq_offsets`` [N + 1] gives their bounds in the
    ``total_tokens`` tokens, None N equal lengths.  q, k and v may be views into
    wider rows (a projection's output)."""

    def __init__(self, num_seqs: int, total_tokens: int, num_qk_heads: int, num_v_heads: int,
                 d_k: int, d_v: int, io: str = "bf16", scale: float = 1.0,
                 backward: bool = False, device="cuda:0", stream=None):
        torch = _torch()
        self.cfg = ab.make_delta_config(num_seqs, total_tokens, num_qk_heads, num_v_heads, d_k,
                                        d_v, io, scale)
        self.ws_bytes = ab.onela_delta_rule_workspace_bytes(self.cfg, backward)
        if self.ws_bytes == 0:
            raise ab.OnelaError(ab.ONELA_EINVAL, "onela_delta_rule_workspace_bytes")
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.stream = stream
        self.is_backward = backward

        def tensor(heads, width, dtype):
            shape = (total_tokens, heads) + ((width,) if width else ())
            return torch.empty(shape, dtype=dtype, device=device)

        dt, f32 = _io_tensor_dtype(io), torch.float32
        state = (num_seqs, num_v_heads, d_v, d_k)
        self.dtypes = dt, f32, torch.int32
        self.shapes = ((total_tokens, num_qk_heads, d_k), (total_tokens, num_v_heads, d_v),
                       (total_tokens, num_v_heads), (num_seqs + 1,), state)
        if backward:
            self.dq, self.dk = tensor(num_qk_heads, d_k, dt), tensor(num_qk_heads, d_k, dt)
            self.dv = tensor(num_v_heads, d_v, dt)
            self.dlog_alpha, self.dbeta = tensor(num_v_heads, 0, f32), tensor(num_v_heads, 0, f32)
            self.d_initial_state = torch.empty(state, dtype=f32, device=device)
        else:
            self.o = tensor(num_v_heads, d_v, dt)
            self.final_state = torch.empty(state, dtype=f32, device=device)

    def _set(self, q, k, v, log_alpha, beta, seq_offsets, initial_state):
        dt, f32, i32 = self.dtypes
        qk, values, gates, bounds, state = self.shapes
        _expect((q, "q", qk, dt), (k, "k", qk, dt), (v, "v", values, dt),
                (log_alpha, "log_alpha", gates, f32), (beta, "beta", gates, f32),
                (seq_offsets, "seq_offsets", bounds, i32),
                (initial_state, "initial_state", state, f32))
        _set_strides(self.cfg, q, k, v)

    def forward(self, q, k, v, log_alpha, beta, seq_offsets=None, initial_state=None):
        """(o, final_state)"""
        if self.is_backward:
            raise ValueError("this object holds the backward call's tensors")
        self._set(q, k, v, log_alpha, beta, seq_offsets, initial_state)
        ab.onela_delta_rule_forward(self.cfg, seq_offsets, q, k, v, log_alpha, beta,
                                    initial_state, self.o, self.final_state, self.workspace,
                                    self.ws_bytes, self.stream)
        return self.o, self.final_state

    def backward(self, q, k, v, log_alpha, beta, d_o, seq_offsets=None, initial_state=None,
                 d_final_state=None):
        """(dq, dk, dv, dlog_alpha, dbeta, d_initial_state or None without one)"""
        if not self.is_backward:
            raise ValueError("this object holds the forward call's tensors")
        self._set(q, k, v, log_alpha, beta, seq_offsets, initial_state)
        _expect((d_o, "d_o", self.shapes[1], self.dtypes[0]),
                (d_final_state, "d_final_state", self.shapes[4], self.dtypes[1]))
        ds = None if initial_state is None else self.d_initial_state
        ab.onela_delta_rule_backward(self.cfg, seq_offsets, q, k, v, log_alpha, beta,
                                     initial_state, d_o, d_final_state, self.dq, self.dk,
                                     self.dv, self.dlog_alpha, self.dbeta, ds, self.workspace,
                                     self.ws_bytes, self.stream)
        return self.dq, self.dk, self.dv, self.dlog_alpha, self.dbeta, ds


class DeltaRuleStep:
    """The recurrent form on a pool of ``num_slots`` states (onela_delta_rule_step) for
    fixed sizes: owns the output tensor."""

    def __init__(self, num_seqs: int, total_tokens: int, num_qk_heads: int, num_v_heads: int,
                 d_k: int, d_v: int, io: str, num_slots: int, scale: float = 1.0,
                 device="cuda:0", stream=None):
        torch = _torch()
        self.cfg = ab.make_delta_config(num_seqs, total_tokens, num_qk_heads, num_v_heads, d_k,
                                        d_v, io, scale)
        self.num_slots, self.stream = num_slots, stream
        self.dense = True  # the configuration's strides are those of dense tensors
        self.pool = num_slots, num_v_heads, d_v, d_k
        dt = _io_tensor_dtype(io)
        self.dtypes = dt, torch.float32, torch.int32
        self.shapes = ((total_tokens, num_qk_heads, d_k), (total_tokens, num_v_heads, d_v),
                       (total_tokens, num_v_heads), (num_seqs + 1,), (num_seqs,))
        self.o = torch.empty((total_tokens, num_v_heads, d_v), dtype=dt, device=device)

    def step(self, pool, slots, q, k, v, log_alpha, beta, seq_offsets=None):
        """o; the pool's states move on in place."""
        dt, f32, i32 = self.dtypes
        qk, values, gates, bounds, seqs = self.shapes
        try:  # (in one expression: these checks are a seventh of a single token's call)
            fits = (q.dtype is dt and q.shape == qk and k.dtype is dt and k.shape == qk and
                    v.dtype is dt and v.shape == values and log_alpha.dtype is f32 and
                    log_alpha.shape == gates and beta.dtype is f32 and beta.shape == gates and
                    pool.dtype is f32 and pool.shape == self.pool and
                    (slots is None or slots.dtype is i32 and slots.shape == seqs) and
                    (seq_offsets is None or seq_offsets.dtype is i32 and
                     seq_offsets.shape == bounds))
        except AttributeError:
            fits = False
        if not fits:
            _expect((q, "q", qk, dt), (k, "k", qk, dt), (v, "v", values, dt),
                    (log_alpha, "log_alpha", gates, f32), (beta, "beta", gates, f32),
                    (seq_offsets, "seq_offsets", bounds, i32), (slots, "slots", seqs, i32))
            if not isinstance(pool, int) and pool is not None:  # (more slots do no harm)
                _expect((pool, "pool", (max(self.num_slots, *pool.shape[:1]), *self.pool[1:]), f32))
        dense = q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
        if not (dense and self.dense):
            _set_strides(self.cfg, q, k, v)
            self.dense = dense
        ab.onela_delta_rule_step(self.cfg, seq_offsets, q, k, v, log_alpha, beta, pool,
                                 self.num_slots, slots, self.o, self.stream)
        return self.o


class QkNormRope:
    """Norm and rotation of queries and keys (onela_qk_norm_rope and, with ``backward``,
    onela_qk_norm_rope_backward) for fixed sizes: owns the output tensors and the
    workspace.  q and k may be views into wider rows."""

    def __init__(self, num_tokens: int, num_q_heads: int, num_k_heads: int, head_dim: int,
                 io: str = "bf16", norm: str = "l2", rotary_dim: int = 0,
                 rotation: str = "halves", eps: float = 1e-6, backward: bool = False,
                 device="cuda:0", stream=None):
        torch = _torch()
        self.cfg = ab.make_norm_config(num_tokens, num_q_heads, num_k_heads, head_dim, io, norm,
                                       rotary_dim, max(1, rotary_dim), rotation, eps)
        self.ws_bytes = ab.onela_qk_norm_rope_workspace_bytes(self.cfg)
        if self.ws_bytes == 0:
            raise ab.OnelaError(ab.ONELA_EINVAL, "onela_qk_norm_rope_workspace_bytes")
        self.stream = stream
        self.is_backward = backward
        self.dtypes = _io_tensor_dtype(io), torch.float32, torch.int32
        self.rotary_dim = rotary_dim
        self.shapes = ((num_tokens, num_q_heads, head_dim), (num_tokens, num_k_heads, head_dim),
                       (head_dim,), (num_tokens,))

        def like(heads):
            return torch.empty((num_tokens, heads, head_dim), dtype=_io_tensor_dtype(io),
                               device=device)

        self.q, self.k = like(num_q_heads), like(num_k_heads)
        if backward:
            self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
            self.dw = torch.empty((2, head_dim), dtype=torch.float32, device=device)

    def _set(self, q, k, q_weight, k_weight, positions, cos_sin):
        dt, f32, i32 = self.dtypes
        queries, keys, width, tokens = self.shapes
        try:  # (in one expression, as the step's)
            fits = (q.dtype is dt and q.shape == queries and
                    (k is None or k.dtype is dt and k.shape == keys) and
                    (q_weight is None or q_weight.dtype is f32 and q_weight.shape == width) and
                    (k_weight is None or k_weight.dtype is f32 and k_weight.shape == width) and
                    (positions is None or positions.dtype is i32 and positions.shape == tokens))
        except AttributeError:
            fits = False
        if not fits:
            _expect((q, "q", queries, dt), (k, "k", keys, dt), (q_weight, "q_weight", width, f32),
                    (k_weight, "k_weight", width, f32), (positions, "positions", tokens, i32))
        self.cfg.q_stride = 0 if q.is_contiguous() else q.stride(0)
        self.cfg.k_stride = 0 if k is None or k.is_contiguous() else k.stride(0)
        if cos_sin is not None:
            table = cos_sin.shape
            if self.rotary_dim and (cos_sin.dtype is not f32 or table[1:] != (self.rotary_dim,)):
                raise ValueError(f"cos_sin must be {f32} [rows, {self.rotary_dim}], not "
                                 f"{cos_sin.dtype} {list(table)}")
            self.cfg.table_rows = table[0]

    def forward(self, q, k, q_weight=None, k_weight=None, positions=None, cos_sin=None):
        """(q, k) normed and turned"""
        if self.is_backward:
            raise ValueError("this object holds the backward call's tensors")
        self._set(q, k, q_weight, k_weight, positions, cos_sin)
        ab.onela_qk_norm_rope(self.cfg, q, k, q_weight, k_weight, positions, cos_sin, self.q,
                              self.k, self.stream)
        return self.q, self.k

    def backward(self, q, k, d_q_out, d_k_out, q_weight=None, k_weight=None, positions=None,
                 cos_sin=None):
        """(dq, dk, dq_weight, dk_weight; None for a weight that is not given)"""
        if not self.is_backward:
            raise ValueError("this object holds the forward call's tensors")
        self._set(q, k, q_weight, k_weight, positions, cos_sin)
        _expect((d_q_out, "d_q_out", self.shapes[0], self.dtypes[0]),
                (d_k_out, "d_k_out", self.shapes[1], self.dtypes[0]))
        dwq = None if q_weight is None else self.dw[0]
        dwk = None if k_weight is None else self.dw[1]
        ab.onela_qk_norm_rope_backward(self.cfg, q, k, q_weight, k_weight, positions, cos_sin,
                                       d_q_out, d_k_out, self.q, self.k, dwq, dwk,
                                       self.workspace, self.ws_bytes, self.stream)
        return self.q, self.k, dwq, dwk
