// Host side of libonela: argument validation, workspace carving, per-step
// protocol bookkeeping and kernel launches.  Every check that can fail runs
// before anything is enqueued, so a rejected call leaves no device work and
// no change in the context.
#include <atomic>
#include <cstdint>
#include <cstdlib>
#include <new>

#include "../../include/onela.h"
#include "delta_params.h"
#include "internal.h"

using onela::aligned16;
using onela::aligned4;
using onela::Arena;
using onela::Layout;
using onela::Protocol;
using onela::Shape;
using onela::shape_of;

struct onela_ctx_s {
  Shape shape;
  Arena arena;
  hipStream_t stream;
  Protocol pr;  // steps resolved / appended, widths, status-word state
};

namespace {

bool launch_ok(hipError_t e) { return e == hipSuccess; }

// Registers the caller's buffers as step t's record slab (borrowed records).
void borrow_step(onela_ctx_s* c, int t, const void* k, const void* v, const float* alpha,
                 const float* beta) {
  c->arena.bk[t] = k;
  c->arena.bv[t] = v;
  c->arena.balpha[t] = alpha;
  c->arena.bbeta[t] = beta;
  c->arena.bw[t] = c->pr.widths[t];
}

}  // namespace


extern "C" {

const char* onela_status_str(onela_status_t st) {
  switch (st) {
    case ONELA_OK: return "ok";
    case ONELA_EINVAL: return "invalid argument";
    case ONELA_ESTEP: return "call out of step order";
    case ONELA_EPARENT: return "parent index out of range (device)";
    case ONELA_ECAPACITY: return "capacity exceeded";
    case ONELA_EHIP: return "HIP runtime error";
    case ONELA_ENOMEM: return "host allocation failed";
  }
  return "unknown status";
}

onela_status_t onela_check_config(const onela_config_t* cfg) {
  Shape s;
  return shape_of(cfg, &s);
}

size_t onela_workspace_bytes(const onela_config_t* cfg) {
  Shape s;
  if (shape_of(cfg, &s) != ONELA_OK) return 0;
  return onela::layout_of(s).total;
}

namespace {
// Compute units of the current device, queried once per device (a host-side
// attribute query; nothing is enqueued).  0 if it cannot be read.
int device_compute_units() {
  static std::atomic<int> cache[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 0;
  int v = cache[dev].load(std::memory_order_relaxed);
  if (v <= 0) {
    if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess)
      return 0;
    cache[dev].store(v, std::memory_order_relaxed);
  }
  return v > 0 ? v : 0;
}
}  // namespace

onela_status_t onela_init(const onela_config_t* cfg, const float* s0,
                          void* workspace, size_t workspace_bytes, void* stream,
                          onela_ctx_t* out) {
  Shape s;
  onela_status_t rc = shape_of(cfg, &s);
  if (rc != ONELA_OK) return rc;
  if (!s0 || !workspace || !out || !aligned16(s0)) return ONELA_EINVAL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return ONELA_EINVAL;
  const Layout l = onela::layout_of(s);
  if (workspace_bytes < l.total) return ONELA_ECAPACITY;
  s.cus = device_compute_units();

  onela_ctx_s* c = new (std::nothrow) onela_ctx_s();
  if (!c) return ONELA_ENOMEM;
  c->shape = s;
  c->stream = static_cast<hipStream_t>(stream);
  c->pr = Protocol{};
  char* p = static_cast<char*>(workspace);
  c->arena.status = reinterpret_cast<int*>(p);
  p += l.status;
  c->arena.anc[0] = reinterpret_cast<int*>(p);
  p += l.anc;
  c->arena.anc[1] = reinterpret_cast<int*>(p);
  p += l.anc;
  c->arena.s0 = s0;
  c->arena.s_frag = reinterpret_cast<uint16_t*>(p);
  p += l.s_frag;
  c->arena.k = s.borrow ? nullptr : p;
  p += l.k;
  c->arena.v = s.borrow ? nullptr : p;
  p += l.v;
  c->arena.ab = s.borrow ? nullptr : reinterpret_cast<float2*>(p);
  p += l.ab;
  c->arena.d = s.delta ? p : nullptr;
  p += l.d;
  c->arena.dsc = s.delta ? reinterpret_cast<unsigned*>(p) : nullptr;

  *out = c;
  return ONELA_OK;
}

onela_status_t onela_reset(onela_ctx_t c) {
  if (!c) return ONELA_EINVAL;
  c->pr.resolved = -1;
  c->pr.appended = -1;
  c->pr.search_zeroed = false;
  return ONELA_OK;
}

onela_status_t onela_resolve_ancestry(onela_ctx_t c, int32_t step, int32_t width,
                                      const int32_t* parents, int32_t* gather_out) {
  if (!c) return ONELA_EINVAL;
  const Shape& s = c->shape;
  Protocol& pr = c->pr;
  const onela_status_t rc = onela::check_resolve(s, pr, step, width, parents, gather_out);
  if (rc != ONELA_OK) return rc;
  if (step > 0) {
    // The step-0 decode launch zeroes the status word of a new search.  When
    // the caller resolves step 1 without having decoded step 0, zero it here
    // first, so that what the resolve kernel flags is not mixed with a word
    // that was never cleared (or still holds an earlier search's error).
    if (!pr.search_zeroed) {
      if (!launch_ok(onela::launch_clear_status(c->arena.status, c->stream))) return ONELA_EHIP;
      pr.search_zeroed = true;
      pr.status_live = true;
    }
    hipError_t e = onela::launch_resolve(s, step, width, pr.widths[step - 1], parents,
                                         c->arena.anc[(step - 1) & 1],
                                         c->arena.anc[step & 1], gather_out,
                                         c->arena.status, c->stream);
    if (!launch_ok(e)) return ONELA_EHIP;
  }
  pr.widths[step] = width;
  pr.resolved = step;
  return ONELA_OK;
}

onela_status_t onela_append_records(onela_ctx_t c, int32_t step, const void* k,
                                    const void* v, const float* alpha,
                                    const float* beta) {
  if (!c) return ONELA_EINVAL;
  const onela_status_t rc = onela::check_append(c->pr, step, k, v, alpha, beta);
  if (rc != ONELA_OK) return rc;
  if (c->shape.borrow) {
    borrow_step(c, step, k, v, alpha, beta);
  } else {
    hipError_t e = onela::launch_append(c->shape, step, c->pr.widths[step], k, v, alpha,
                                        beta, c->arena, c->stream);
    if (!launch_ok(e)) return ONELA_EHIP;
  }
  c->pr.appended = step;
  return ONELA_OK;
}

onela_status_t onela_decode_step(onela_ctx_t c, int32_t step, const void* q, float* o) {
  if (!c) return ONELA_EINVAL;
  const onela_status_t rc = onela::check_decode(c->pr, step, q, o);
  if (rc != ONELA_OK) return rc;
  const int width = c->pr.widths[step];
  hipError_t e = c->shape.delta
                     ? onela::launch_replay_decode(c->shape, step, width, q, o, c->arena,
                                                   c->stream)
                     : onela::launch_decode(c->shape, step, width, q, o, c->arena, c->stream);
  if (!launch_ok(e)) return ONELA_EHIP;
  if (step == 0) c->pr.status_live = c->pr.search_zeroed = true;
  return ONELA_OK;
}

onela_status_t onela_decode_step_fused(onela_ctx_t c, int32_t step, int32_t width,
                                       const int32_t* parents, const void* k, const void* v,
                                       const float* alpha, const float* beta, const void* q,
                                       float* o, int32_t* gather_out) {
  if (!c) return ONELA_EINVAL;
  const Shape& s = c->shape;
  Protocol& pr = c->pr;
  const onela_status_t rc =
      onela::check_fused(s, pr, step, width, parents, k, v, alpha, beta, q, o, gather_out);
  if (rc != ONELA_OK) return rc;
  const int prev = step > 0 ? pr.widths[step - 1] : 0;
  hipError_t e = s.delta ? onela::launch_replay_fused(s, step, width, prev, parents, k, v, alpha,
                                                      beta, q, o, gather_out, c->arena, c->stream)
                         : onela::launch_fused_step(s, step, width, prev, parents, k, v, alpha,
                                                    beta, q, o, gather_out, c->arena, c->stream);
  if (!launch_ok(e)) return ONELA_EHIP;
  pr.widths[step] = width;
  if (s.borrow) borrow_step(c, step, k, v, alpha, beta);
  pr.resolved = step;
  pr.appended = step;
  if (step == 0) pr.status_live = pr.search_zeroed = true;
  return ONELA_OK;
}

onela_status_t onela_get_device_status(onela_ctx_t c) {
  if (!c) return ONELA_EINVAL;
  if (hipStreamSynchronize(c->stream) != hipSuccess) return ONELA_EHIP;
  if (!c->pr.status_live) return ONELA_OK;  // no step has run: nothing was flagged
  int word = 0;
  if (hipMemcpy(&word, c->arena.status, sizeof(int), hipMemcpyDeviceToHost) != hipSuccess)
    return ONELA_EHIP;
  if (word == 0) return ONELA_OK;
  if (!launch_ok(onela::launch_clear_status(c->arena.status, c->stream)) ||
      hipStreamSynchronize(c->stream) != hipSuccess)
    return ONELA_EHIP;
  return ONELA_EPARENT;
}

void onela_destroy(onela_ctx_t c) { delete c; }

onela_status_t onela_prefill_state(const onela_config_t* cfg, int32_t prompt_len,
                                   const void* k, const void* v, const float* alpha,
                                   const float* beta, float* s0_out, void* stream) {
  Shape s;
  onela_status_t rc = shape_of(cfg, &s);
  if (rc != ONELA_OK) return rc;
  if (prompt_len < 0 || !s0_out || !aligned16(s0_out)) return ONELA_EINVAL;
  if (prompt_len > 0 && (!k || !v || !alpha || !beta || !aligned16(k) || !aligned16(v) ||
                         !aligned4(alpha) || !aligned4(beta)))
    return ONELA_EINVAL;
  hipError_t e = onela::launch_prefill(s, prompt_len, k, v, alpha, beta, s0_out,
                                       static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

size_t onela_prefill_workspace_bytes(const onela_config_t* cfg, int32_t prompt_len) {
  Shape s;
  if (shape_of(cfg, &s) != ONELA_OK || prompt_len < 0) return 0;
  return onela::prefill_chunked_workspace_bytes(s, prompt_len);
}

onela_status_t onela_prefill_state_chunked(const onela_config_t* cfg, int32_t prompt_len,
                                           const void* k, const void* v, const float* alpha,
                                           const float* beta, float* s0_out, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  Shape s;
  const onela_status_t rc = shape_of(cfg, &s);
  if (rc != ONELA_OK) return rc;
  if (prompt_len < 0 || !s0_out || !aligned16(s0_out)) return ONELA_EINVAL;
  if (prompt_len > 0 && (!k || !v || !alpha || !beta || !aligned16(k) || !aligned16(v) ||
                         !aligned4(alpha) || !aligned4(beta)))
    return ONELA_EINVAL;
  const size_t need = onela::prefill_chunked_workspace_bytes(s, prompt_len);
  if (need > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
    return ONELA_EINVAL;
  if (workspace_bytes < need) return ONELA_ECAPACITY;
  s.cus = device_compute_units();
  const hipError_t e =
      onela::launch_prefill_chunked(s, prompt_len, k, v, alpha, beta, s0_out, workspace,
                                    static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

size_t onela_fullstate_workspace_bytes(const onela_config_t* cfg) {
  Shape s;
  if (shape_of(cfg, &s) != ONELA_OK) return 0;
  return 2 * sizeof(float) * size_t(s.R) * s.wmax * s.HV * size_t(s.dv) * s.dk;
}

onela_status_t onela_fullstate_step(const onela_config_t* cfg, int32_t step,
                                    int32_t width, int32_t prev_width,
                                    const int32_t* parents, const float* s0,
                                    const void* q, const void* k, const void* v,
                                    const float* alpha, const float* beta, float* o,
                                    void* workspace, size_t workspace_bytes,
                                    int32_t* status_word, void* stream) {
  Shape s;
  onela_status_t rc = shape_of(cfg, &s);
  if (rc != ONELA_OK) return rc;
  if (step < 0 || width < 1 || width > s.wmax) return ONELA_ECAPACITY;
  if (step > 0 && (prev_width < 1 || prev_width > s.wmax)) return ONELA_ECAPACITY;
  if (step == 0 && parents) return ONELA_EINVAL;
  if (step > 0 && (!parents || !aligned4(parents))) return ONELA_EINVAL;
  if (!s0 || !q || !k || !v || !alpha || !beta || !o || !workspace) return ONELA_EINVAL;
  if (!aligned16(s0) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) ||
      !aligned4(alpha) || !aligned4(beta) || !aligned16(workspace))
    return ONELA_EINVAL;
  if (status_word && !aligned4(status_word)) return ONELA_EINVAL;
  const size_t half = sizeof(float) * size_t(s.R) * s.wmax * s.HV * size_t(s.dv) * s.dk;
  if (workspace_bytes < 2 * half) return ONELA_ECAPACITY;
  float* base = static_cast<float*>(workspace);
  float* buf[2] = {base, base + half / sizeof(float)};
  hipError_t e = onela::launch_fullstate(s, step, width, prev_width, parents, s0, q, k, v,
                                         alpha, beta, o, buf[(step + 1) & 1], buf[step & 1],
                                         status_word, static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

uint64_t onela_capacity_bytes(int32_t R, int32_t HV, int32_t dk, int32_t dv, int32_t beams,
                              int32_t steps, int32_t state_bytes, int32_t record_bytes) {
  if (R < 0 || HV < 0 || dk < 0 || dv < 0 || beams < 0 || steps < 0 || state_bytes < 0 ||
      record_bytes < 0)
    return 0;
  const uint64_t ctx = uint64_t(R) * HV * uint64_t(dv) * dk * state_bytes;
  const uint64_t rec = uint64_t(steps) * R * uint64_t(beams) * HV * record_bytes;
  return ctx + rec;
}

uint64_t onela_fullstate_capacity_bytes(int32_t R, int32_t HV, int32_t dk, int32_t dv,
                                        int32_t beams, int32_t state_bytes) {
  if (R < 0 || HV < 0 || dk < 0 || dv < 0 || beams < 0 || state_bytes < 0) return 0;
  return uint64_t(R) * beams * HV * uint64_t(dv) * dk * state_bytes;
}

onela_status_t onela_select_workspace_bytes(int32_t num_requests, int32_t prev_width,
                                            int32_t vocab, int32_t width, size_t* bytes) {
  if (!bytes) return ONELA_EINVAL;
  *bytes = 0;
  onela::SelectPlan plan;
  const onela_status_t rc = onela::check_select(num_requests, prev_width, vocab, width, &plan);
  if (rc != ONELA_OK) return rc;
  *bytes = plan.total;
  return ONELA_OK;
}

onela_status_t onela_select_beams(int32_t num_requests, int32_t prev_width, int32_t vocab,
                                  int32_t width, const float* logp, const float* beam_scores,
                                  int32_t* parents_out, int32_t* tokens_out, float* scores_out,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const onela_status_t st =
      onela_select_workspace_bytes(num_requests, prev_width, vocab, width, &need);
  if (st != ONELA_OK) return st;
  if (!logp || !parents_out || !tokens_out || !scores_out || !aligned4(logp) ||
      !aligned4(parents_out) || !aligned4(tokens_out) || !aligned4(scores_out))
    return ONELA_EINVAL;
  if (beam_scores && !aligned4(beam_scores)) return ONELA_EINVAL;
  if (need > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
    return ONELA_EINVAL;
  if (workspace_bytes < need) return ONELA_ECAPACITY;
  onela::SelectPlan plan;
  onela::select_plan(num_requests, unsigned(prev_width) * unsigned(vocab), unsigned(width),
                     &plan);
  const hipError_t e = onela::launch_select(plan, num_requests, prev_width, vocab, width, logp,
                                            beam_scores, parents_out, tokens_out, scores_out,
                                            workspace, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ONELA_OK : ONELA_EHIP;
}

onela_status_t onela_select_beams_noalloc(int32_t num_requests, int32_t prev_width,
                                          int32_t vocab, int32_t width, const float* logp,
                                          const float* beam_scores, int32_t* parents_out,
                                          int32_t* tokens_out, float* scores_out,
                                          void* stream) {
  size_t need = 0;
  const onela_status_t st =
      onela_select_workspace_bytes(num_requests, prev_width, vocab, width, &need);
  if (st != ONELA_OK) return st;
  if (need > onela::kSelectScratchBytes) return ONELA_ECAPACITY;
  if (!logp || !parents_out || !tokens_out || !scores_out || !aligned4(logp) ||
      !aligned4(parents_out) || !aligned4(tokens_out) || !aligned4(scores_out))
    return ONELA_EINVAL;
  if (beam_scores && !aligned4(beam_scores)) return ONELA_EINVAL;
  void* ws = nullptr;
  if (onela::select_scratch(&ws) != hipSuccess) return ONELA_EHIP;
  onela::SelectPlan plan;
  onela::select_plan(num_requests, unsigned(prev_width) * unsigned(vocab), unsigned(width),
                     &plan);
  const hipError_t e = onela::launch_select(plan, num_requests, prev_width, vocab, width, logp,
                                            beam_scores, parents_out, tokens_out, scores_out,
                                            ws, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ONELA_OK : ONELA_EHIP;
}

// ---- delta rule over sequences ----------------------------------------------------

namespace {
// What the three entry points share: ONELA_EINVAL unless the tensors of the
// sequences are there and aligned.
onela_status_t delta_inputs(const onela_delta_config_t* cfg, const int32_t* offsets,
                            const void* q, const void* k, const void* v, const float* la,
                            const float* beta, onela::DeltaShape* s, onela::DeltaParams* p) {
  const onela_status_t rc = onela::delta_shape_of(cfg, offsets != nullptr, s);
  if (rc != ONELA_OK) return rc;
  if (offsets && !aligned4(offsets)) return ONELA_EINVAL;
  if (s->total > 0 && (!q || !k || !v || !la || !beta)) return ONELA_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned4(la) || !aligned4(beta))
    return ONELA_EINVAL;
  *p = onela::DeltaParams{};
  p->q = q;
  p->k = k;
  p->v = v;
  p->la = la;
  p->beta = beta;
  p->offsets = offsets;
  p->total = s->total;
  p->qs = s->qs;
  p->ks = s->ks;
  p->vs = s->vs;
  p->scale = s->scale;
  p->N = s->N;
  p->HK = s->HK;
  p->HV = s->HV;
  p->DV = s->dv;
  p->L = s->L;
  p->nch_l = onela::delta_chunks(s->L);
  p->slots = s->slots;
  p->clear = cfg->clear_rest && offsets;  // (without offsets there is no rest)
  return ONELA_OK;
}

onela_status_t delta_workspace(const onela::DeltaShape& s, bool backward, const void* workspace,
                               size_t bytes) {
  if (!onela::delta_grids_fit(s, backward)) return ONELA_EINVAL;
  const size_t need = onela::delta_workspace_bytes(s, backward);
  if (need > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
    return ONELA_EINVAL;
  return bytes < need ? ONELA_ECAPACITY : ONELA_OK;
}
}  // namespace

size_t onela_delta_rule_workspace_bytes(const onela_delta_config_t* cfg, int32_t backward) {
  // (any lengths: as many chunk slots as ragged sequences can need, or more)
  onela::DeltaShape s;
  if (onela::delta_shape_of(cfg, true, &s) != ONELA_OK) return 0;
  if (!onela::delta_grids_fit(s, backward != 0)) return 0;
  return onela::delta_workspace_bytes(s, backward != 0);
}

onela_status_t onela_delta_rule_forward(const onela_delta_config_t* cfg,
                                        const int32_t* seq_offsets, const void* q,
                                        const void* k, const void* v, const float* log_alpha,
                                        const float* beta, const float* initial_state, void* o,
                                        float* final_state, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  onela::DeltaShape s;
  onela::DeltaParams p;
  onela_status_t rc = delta_inputs(cfg, seq_offsets, q, k, v, log_alpha, beta, &s, &p);
  if (rc != ONELA_OK) return rc;
  if ((s.total > 0 && !o) || !aligned16(o) || !aligned16(initial_state) || !aligned16(final_state))
    return ONELA_EINVAL;
  rc = delta_workspace(s, false, workspace, workspace_bytes);
  if (rc != ONELA_OK) return rc;
  s.cus = device_compute_units();
  p.s_in = initial_state;
  p.s_out = final_state;
  p.o = o;
  const hipError_t e =
      onela::launch_delta_rule(s, p, false, workspace, static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

onela_status_t onela_delta_rule_backward(
    const onela_delta_config_t* cfg, const int32_t* seq_offsets, const void* q, const void* k,
    const void* v, const float* log_alpha, const float* beta, const float* initial_state,
    const void* d_o, const float* d_final_state, void* dq, void* dk, void* dv,
    float* dlog_alpha, float* dbeta, float* d_initial_state, void* workspace,
    size_t workspace_bytes, void* stream) {
  onela::DeltaShape s;
  onela::DeltaParams p;
  onela_status_t rc = delta_inputs(cfg, seq_offsets, q, k, v, log_alpha, beta, &s, &p);
  if (rc != ONELA_OK) return rc;
  if (s.total > 0 && (!d_o || !dq || !dk || !dv || !dlog_alpha || !dbeta)) return ONELA_EINVAL;
  if (!aligned16(d_o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) ||
      !aligned4(dlog_alpha) || !aligned4(dbeta) || !aligned16(initial_state) ||
      !aligned16(d_final_state) || !aligned16(d_initial_state))
    return ONELA_EINVAL;
  rc = delta_workspace(s, true, workspace, workspace_bytes);
  if (rc != ONELA_OK) return rc;
  s.cus = device_compute_units();
  p.s_in = initial_state;
  p.ds_in = d_final_state;
  p.ds_out = d_initial_state;
  p.d_o = d_o;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  p.dla = dlog_alpha;
  p.db = dbeta;
  const hipError_t e =
      onela::launch_delta_rule(s, p, true, workspace, static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

onela_status_t onela_delta_rule_step(const onela_delta_config_t* cfg,
                                     const int32_t* seq_offsets, const void* q, const void* k,
                                     const void* v, const float* log_alpha, const float* beta,
                                     float* state, int32_t num_slots, const int32_t* slots,
                                     void* o, void* stream) {
  onela::DeltaShape s;
  onela::DeltaParams p;
  const onela_status_t rc = delta_inputs(cfg, seq_offsets, q, k, v, log_alpha, beta, &s, &p);
  if (rc != ONELA_OK) return rc;
  if (cfg->clear_rest || !onela::delta_step_grid_fits(s)) return ONELA_EINVAL;
  if (num_slots < 1 || !state || !aligned16(state) || !aligned4(slots)) return ONELA_EINVAL;
  if ((s.total > 0 && !o) || !aligned16(o)) return ONELA_EINVAL;
  if (!slots && num_slots < s.N) return ONELA_ECAPACITY;
  if (s.total == 0) return ONELA_OK;
  p.pool = state;
  p.num_slots = num_slots;
  p.slot = slots;
  p.o = o;
  const hipError_t e = onela::launch_delta_step(s, p, static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

// ---- norm and rotation of queries and keys --------------------------------------

namespace {
onela_status_t norm_inputs(const onela_norm_config_t* c, const void* q, const void* k,
                           const float* wq, const float* wk, const int32_t* positions,
                           const float* cos_sin, onela::NormParams* p) {
  const onela_status_t rc = onela::check_norm(c);
  if (rc != ONELA_OK) return rc;
  if (c->num_tokens > 0 && (!q || (c->num_k_heads > 0 && !k) || (c->rotary_dim > 0 && !cos_sin)))
    return ONELA_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned4(wq) || !aligned4(wk) || !aligned4(positions) ||
      !aligned4(cos_sin))
    return ONELA_EINVAL;
  *p = onela::NormParams{};
  p->q = q;
  p->k = k;
  p->wq = wq;
  p->wk = wk;
  p->positions = positions;
  p->cos_sin = cos_sin;
  p->HQ = c->num_q_heads;
  p->HK = c->num_k_heads;
  p->D = c->head_dim;
  p->rot = c->rotary_dim;
  p->table = c->table_rows;
  p->pairs = c->rotation == ONELA_ROTATE_PAIRS;
  p->rows = long(c->num_tokens) * (p->HQ + p->HK);
  p->qs = c->q_stride ? long(c->q_stride) : long(p->HQ) * p->D;
  p->ks = c->k_stride ? long(c->k_stride) : long(p->HK) * p->D;
  p->eps = c->eps;
  p->inv_n = c->norm == ONELA_NORM_RMS ? 1.f / float(p->D) : 1.f;
  return ONELA_OK;
}
}  // namespace

onela_status_t onela_qk_norm_rope(const onela_norm_config_t* cfg, const void* q, const void* k,
                                  const float* q_weight, const float* k_weight,
                                  const int32_t* positions, const float* cos_sin, void* q_out,
                                  void* k_out, void* stream) {
  onela::NormParams p;
  const onela_status_t rc = norm_inputs(cfg, q, k, q_weight, k_weight, positions, cos_sin, &p);
  if (rc != ONELA_OK) return rc;
  if ((p.rows > 0 && (!q_out || (p.HK > 0 && !k_out))) || !aligned16(q_out) || !aligned16(k_out))
    return ONELA_EINVAL;
  p.qo = q_out;
  p.ko = k_out;
  const hipError_t e = onela::launch_norm_rope(p, cfg->io_dtype == ONELA_BF16, false,
                                               static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

size_t onela_qk_norm_rope_workspace_bytes(const onela_norm_config_t* cfg) {
  return onela::check_norm(cfg) == ONELA_OK ? onela::norm_workspace_bytes(cfg) : 0;
}

onela_status_t onela_qk_norm_rope_backward(const onela_norm_config_t* cfg, const void* q,
                                           const void* k, const float* q_weight,
                                           const float* k_weight, const int32_t* positions,
                                           const float* cos_sin, const void* d_q_out,
                                           const void* d_k_out, void* dq, void* dk,
                                           float* dq_weight, float* dk_weight, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  onela::NormParams p;
  const onela_status_t rc = norm_inputs(cfg, q, k, q_weight, k_weight, positions, cos_sin, &p);
  if (rc != ONELA_OK) return rc;
  if (p.rows > 0 && (!d_q_out || !dq || (p.HK > 0 && (!d_k_out || !dk)))) return ONELA_EINVAL;
  if (!aligned16(d_q_out) || !aligned16(d_k_out) || !aligned16(dq) || !aligned16(dk) ||
      !aligned4(dq_weight) || !aligned4(dk_weight))
    return ONELA_EINVAL;
  if (dq_weight || dk_weight) {
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return ONELA_EINVAL;
    if (workspace_bytes < onela::norm_workspace_bytes(cfg)) return ONELA_ECAPACITY;
    p.partial = static_cast<float*>(workspace);
  }
  p.dqo = d_q_out;
  p.dko = d_k_out;
  p.dq = dq;
  p.dk = dk;
  p.dwq = dq_weight;
  p.dwk = dk_weight;
  const hipError_t e = onela::launch_norm_rope(p, cfg->io_dtype == ONELA_BF16, true,
                                               static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}


// ---- short causal convolution ----------------------------------------------------------

namespace {
bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }
size_t io_bytes(int32_t dtype) { return dtype == ONELA_BF16 ? 2 : 4; }
// Bytes from the first to the last element of n tokens of `own` elements, `stride` apart.
size_t span(int64_t n, int64_t stride, int64_t own, int32_t dtype) {
  return n > 0 ? size_t((n - 1) * stride + own) * io_bytes(dtype) : 0;
}

onela_status_t conv_inputs(const onela_conv_config_t* c, const int32_t* offsets, const void* x,
                           const float* weight, const float* bias, onela::ConvParams* p) {
  const onela_status_t rc = onela::check_conv(c, offsets != nullptr);
  if (rc != ONELA_OK) return rc;
  if (!weight || (c->total_tokens > 0 && !x)) return ONELA_EINVAL;
  if (!aligned16(x) || !aligned4(weight) || !aligned4(bias) || !aligned4(offsets))
    return ONELA_EINVAL;
  *p = onela::ConvParams{};
  p->x = x;
  p->w = weight;
  p->bias = bias;
  p->offsets = offsets;
  p->total = long(c->total_tokens);
  p->xs = c->x_stride ? long(c->x_stride) : long(c->channels);
  p->N = c->num_seqs;
  p->C = c->channels;
  p->L = offsets ? 0 : int(c->total_tokens / c->num_seqs);
  p->silu = c->activation == ONELA_ACT_SILU;
  p->clear = c->clear_rest && offsets;  // (without offsets there is no rest)
  return ONELA_OK;
}
size_t conv_x_bytes(const onela_conv_config_t* c) {
  return span(c->total_tokens, c->x_stride ? c->x_stride : c->channels, c->channels, c->io_dtype);
}
size_t conv_rows_bytes(const onela_conv_config_t* c, int64_t rows) {
  return size_t(rows) * size_t(c->channels) * io_bytes(c->io_dtype);
}
struct ConvVectors {
  onela::Bytes weight, bias, offsets;
};
ConvVectors conv_vectors(const onela_conv_config_t* c, const float* weight, const float* bias,
                         const int32_t* offsets) {
  const size_t channels = size_t(c->channels) * sizeof(float);
  return {{weight, channels * size_t(c->taps)},
          {bias, channels},
          {offsets, (size_t(c->num_seqs) + 1) * sizeof(int32_t)}};
}
}  // namespace

onela_status_t onela_short_conv(const onela_conv_config_t* cfg, const int32_t* seq_offsets,
                                const void* x, const float* weight, const float* bias,
                                const void* initial_state, void* y, void* final_state,
                                void* stream) {
  onela::ConvParams p;
  const onela_status_t rc = conv_inputs(cfg, seq_offsets, x, weight, bias, &p);
  if (rc != ONELA_OK) return rc;
  if ((p.total > 0 && !y) || !aligned16(y) || !aligned16(initial_state) || !aligned16(final_state))
    return ONELA_EINVAL;
  const size_t states = conv_rows_bytes(cfg, int64_t(p.N) * (cfg->taps - 1));
  const onela::Bytes out = {y, conv_rows_bytes(cfg, p.total)}, last = {final_state, states};
  const onela::Bytes first = {initial_state, states};
  const ConvVectors v = conv_vectors(cfg, weight, bias, seq_offsets);
  if (onela::clash({out, last}, {{x, conv_x_bytes(cfg)}, v.weight, v.bias, v.offsets}, false) ||
      onela::clash({out}, {first}, false) || onela::clash({last}, {first}, true))
    return ONELA_EINVAL;
  p.s_in = initial_state;
  p.s_out = final_state;
  p.y = y;
  const hipError_t e = onela::launch_conv(p, onela::conv_plan(cfg, false), cfg->taps,
                                          cfg->io_dtype == ONELA_BF16,
                                          static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

size_t onela_short_conv_workspace_bytes(const onela_conv_config_t* cfg) {
  return onela::check_conv(cfg, true) == ONELA_OK ? onela::conv_workspace_bytes(cfg) : 0;
}

onela_status_t onela_short_conv_backward(const onela_conv_config_t* cfg,
                                         const int32_t* seq_offsets, const void* x,
                                         const float* weight, const float* bias,
                                         const void* initial_state, const void* d_y,
                                         const void* d_final_state, void* dx, float* dweight,
                                         float* dbias, void* d_initial_state, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  onela::ConvParams p;
  const onela_status_t rc = conv_inputs(cfg, seq_offsets, x, weight, bias, &p);
  if (rc != ONELA_OK) return rc;
  if (p.total > 0 && (!d_y || !dx)) return ONELA_EINVAL;
  if (!aligned16(d_y) || !aligned16(dx) || !aligned16(initial_state) ||
      !aligned16(d_final_state) || !aligned16(d_initial_state) || !aligned4(dweight) ||
      !aligned4(dbias))
    return ONELA_EINVAL;
  const size_t states = conv_rows_bytes(cfg, int64_t(p.N) * (cfg->taps - 1));
  const size_t rows = conv_rows_bytes(cfg, p.total);
  if (dweight || dbias) {
    if (!workspace || !aligned256(workspace)) return ONELA_EINVAL;
    if (workspace_bytes < onela::conv_workspace_bytes(cfg)) return ONELA_ECAPACITY;
    p.partial = static_cast<float*>(workspace);
  }
  // (a run reads rows of its neighbours)
  const ConvVectors v = conv_vectors(cfg, weight, bias, seq_offsets);
  const onela::Bytes grad = {dx, rows}, dfirst = {d_initial_state, states};
  const onela::Bytes dw = {dweight, v.weight.n}, db = {dbias, size_t(p.C) * sizeof(float)};
  const onela::Bytes work = {p.partial, onela::conv_workspace_bytes(cfg)};
  if (onela::clash({grad, dfirst, dw, db, work},
                   {{x, conv_x_bytes(cfg)}, {initial_state, states}, {d_y, rows},
                    {d_final_state, states}, v.offsets}, false) ||
      onela::clash({grad, dfirst, work}, {v.weight, v.bias}, false) ||
      onela::clash({dw, db}, {v.weight, v.bias}, true))
    return ONELA_EINVAL;
  p.s_in = initial_state;
  p.dy = d_y;
  p.ds_in = d_final_state;
  p.dx = dx;
  p.ds_out = d_initial_state;
  p.dw = dweight;
  p.db = dbias;
  const hipError_t e = onela::launch_conv_backward(p, onela::conv_plan(cfg, true), cfg->taps,
                                                   cfg->io_dtype == ONELA_BF16,
                                                   static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

onela_status_t onela_short_conv_step(const onela_conv_config_t* cfg, const int32_t* seq_offsets,
                                     const void* x, const float* weight, const float* bias,
                                     void* state, int32_t num_slots, const int32_t* slots,
                                     void* state_out, int32_t num_slots_out,
                                     const int32_t* slots_out, void* y, void* stream) {
  onela::ConvParams p;
  const onela_status_t rc = conv_inputs(cfg, seq_offsets, x, weight, bias, &p);
  if (rc != ONELA_OK) return rc;
  if (cfg->clear_rest || (p.total > 0 && !y) || !aligned16(y)) return ONELA_EINVAL;
  if (!state || num_slots < 1 || !aligned16(state) || !aligned4(slots)) return ONELA_EINVAL;
  if (state_out ? num_slots_out < 1 : slots_out != nullptr) return ONELA_EINVAL;
  if (!aligned16(state_out) || !aligned4(slots_out)) return ONELA_EINVAL;
  if (!slots && num_slots < p.N) return ONELA_ECAPACITY;
  if (state_out && !slots_out && num_slots_out < p.N) return ONELA_ECAPACITY;
  const int64_t rows = cfg->taps - 1;
  const ConvVectors v = conv_vectors(cfg, weight, bias, seq_offsets);
  const onela::Bytes out = {y, conv_rows_bytes(cfg, p.total)}, in = {x, conv_x_bytes(cfg)};
  const onela::Bytes pool = {state, conv_rows_bytes(cfg, num_slots * rows)};
  const onela::Bytes pool_out = {state_out, conv_rows_bytes(cfg, num_slots_out * rows)};
  const onela::Bytes list = {slots, size_t(p.N) * sizeof(int32_t)};
  const onela::Bytes list_out = {slots_out, size_t(p.N) * sizeof(int32_t)};
  // (a thread reads the input of a token and channel before it writes the output)
  if (onela::clash({out}, {in}, true) || onela::clash({state_out ? pool_out : pool}, {in}, false) ||
      onela::clash({out, state_out ? pool_out : pool},
                   {v.weight, v.bias, v.offsets, list, list_out}, false) ||
      (state_out && onela::clash({out, pool_out}, {pool}, false)))
    return ONELA_EINVAL;
  p.s_in = state;
  p.s_out = state_out;
  p.slot = slots;
  p.slot_out = slots_out;
  p.slots = num_slots;
  p.slots_out = num_slots_out;
  p.y = y;
  const hipError_t e = onela::launch_conv_step(p, cfg->taps, cfg->io_dtype == ONELA_BF16,
                                               static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

// ---- norms around a block -----------------------------------------------------------

namespace {
onela_status_t block_norm_inputs(const onela_block_norm_config_t* c, const void* x,
                                 const void* gate, const void* residual, const float* wa,
                                 const float* wb, const float* cs, onela::BlockNormParams* p) {
  const onela_status_t rc = onela::check_block_norm(c);
  if (rc != ONELA_OK) return rc;
  const bool gated = c->gate_act != ONELA_ACT_NONE;
  if (c->num_tokens > 0 && (!x || gated != (gate != nullptr))) return ONELA_EINVAL;
  if ((wa && !c->norm_after) || (wb && !c->norm_before)) return ONELA_EINVAL;
  if (!aligned16(x) || !aligned16(gate) || !aligned16(residual) || !aligned4(wa) ||
      !aligned4(wb) || !aligned4(cs))
    return ONELA_EINVAL;
  const long own = long(c->num_heads) * c->width;
  *p = onela::BlockNormParams{};
  p->x = x;
  p->gate = gate;
  p->res = residual;
  p->wa = wa;
  p->wb = wb;
  p->cs = cs;
  p->rows = long(c->num_tokens) * c->num_heads;
  p->xs = c->x_stride ? long(c->x_stride) : own;
  p->gs = c->gate_stride ? long(c->gate_stride) : own;
  p->scale = c->residual_scale;
  p->eps = c->eps;
  p->H = c->num_heads;
  p->D = c->width;
  p->after = c->norm_after != 0;
  p->before = c->norm_before != 0;
  p->silu = c->gate_act == ONELA_ACT_SILU;
  return ONELA_OK;
}
size_t block_norm_bytes(const onela_block_norm_config_t* c, int64_t stride, int32_t dtype) {
  const int64_t own = int64_t(c->num_heads) * c->width;
  return span(c->num_tokens, stride ? stride : own, own, dtype);
}
size_t width_bytes(const onela_block_norm_config_t* c) { return size_t(c->width) * 4; }
}  // namespace

onela_status_t onela_block_norm(const onela_block_norm_config_t* cfg, const void* x,
                                const void* gate, const void* residual,
                                const float* after_weight, const float* before_weight,
                                const float* channel_scale, void* y, void* residual_out,
                                void* stream) {
  onela::BlockNormParams p;
  const onela_status_t rc =
      block_norm_inputs(cfg, x, gate, residual, after_weight, before_weight, channel_scale, &p);
  if (rc != ONELA_OK) return rc;
  if ((p.rows > 0 && !y && !residual_out) || !aligned16(y) || !aligned16(residual_out))
    return ONELA_EINVAL;
  const size_t rows = block_norm_bytes(cfg, 0, cfg->io_dtype), vector = width_bytes(cfg);
  const size_t res = block_norm_bytes(cfg, 0, cfg->residual_dtype);
  if (onela::clash({{y, rows}, {residual_out, res}},
                   {{x, block_norm_bytes(cfg, cfg->x_stride, cfg->io_dtype)},
                    {gate, block_norm_bytes(cfg, cfg->gate_stride, cfg->io_dtype)},
                    {residual, res},
                    {after_weight, vector},
                    {before_weight, vector},
                    {channel_scale, vector}},
                   true))
    return ONELA_EINVAL;
  p.y = y;
  p.h = residual_out;
  const hipError_t e = onela::launch_block_norm(
      p, cfg->io_dtype == ONELA_BF16, cfg->residual_dtype == ONELA_BF16, device_compute_units(),
      static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

size_t onela_block_norm_workspace_bytes(const onela_block_norm_config_t* cfg) {
  return onela::check_block_norm(cfg) == ONELA_OK ? onela::block_norm_workspace_bytes(cfg) : 0;
}

onela_status_t onela_block_norm_backward(
    const onela_block_norm_config_t* cfg, const void* x, const void* gate, const void* residual,
    const float* after_weight, const float* before_weight, const float* channel_scale,
    const void* d_y, const void* d_residual_out, void* dx, void* dgate, void* d_residual,
    float* dafter_weight, float* dbefore_weight, float* dchannel_scale, void* workspace,
    size_t workspace_bytes, void* stream) {
  onela::BlockNormParams p;
  const onela_status_t rc =
      block_norm_inputs(cfg, x, gate, residual, after_weight, before_weight, channel_scale, &p);
  if (rc != ONELA_OK) return rc;
  if (p.rows > 0 && (!dx || (!d_y && !d_residual_out))) return ONELA_EINVAL;
  if (dgate && cfg->gate_act == ONELA_ACT_NONE) return ONELA_EINVAL;
  if ((dafter_weight && !cfg->norm_after) || (dbefore_weight && !cfg->norm_before))
    return ONELA_EINVAL;
  if (!aligned16(d_y) || !aligned16(d_residual_out) || !aligned16(dx) || !aligned16(dgate) ||
      !aligned16(d_residual) || !aligned4(dafter_weight) || !aligned4(dbefore_weight) ||
      !aligned4(dchannel_scale))
    return ONELA_EINVAL;
  if (dafter_weight || dbefore_weight || dchannel_scale) {
    if (!workspace || !aligned256(workspace)) return ONELA_EINVAL;
    if (workspace_bytes < onela::block_norm_workspace_bytes(cfg)) return ONELA_ECAPACITY;
    p.partial = static_cast<float*>(workspace);
  }
  const size_t rows = block_norm_bytes(cfg, 0, cfg->io_dtype), vector = width_bytes(cfg);
  const size_t res = block_norm_bytes(cfg, 0, cfg->residual_dtype);
  if (onela::clash({{dx, rows},
                    {dgate, rows},
                    {d_residual, res},
                    {dafter_weight, vector},
                    {dbefore_weight, vector},
                    {dchannel_scale, vector},
                    {p.partial, onela::block_norm_workspace_bytes(cfg)}},
                   {{x, block_norm_bytes(cfg, cfg->x_stride, cfg->io_dtype)},
                    {gate, block_norm_bytes(cfg, cfg->gate_stride, cfg->io_dtype)},
                    {residual, res},
                    {d_y, rows},
                    {d_residual_out, res},
                    {after_weight, vector},
                    {before_weight, vector},
                    {channel_scale, vector}},
                   true))
    return ONELA_EINVAL;
  p.dy = d_y;
  p.dh = d_residual_out;
  p.dx = dx;
  p.dgate = dgate;
  p.dres = d_residual;
  p.dwa = dafter_weight;
  p.dwb = dbefore_weight;
  p.dcs = dchannel_scale;
  const hipError_t e = onela::launch_block_norm_backward(
      p, cfg->io_dtype == ONELA_BF16, cfg->residual_dtype == ONELA_BF16, device_compute_units(),
      static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

// ---- log probabilities of tokens --------------------------------------------------------

namespace {
bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

onela_status_t logprob_inputs(const onela_logprob_config_t* c, const void* logits,
                              const int32_t* given, onela::LogprobParams* p) {
  const onela_status_t rc = onela::check_logprob(c);
  if (rc != ONELA_OK) return rc;
  if (c->num_rows > 0 && (!logits || (c->num_given > 0 && !given))) return ONELA_EINVAL;
  if (!aligned_to(logits, io_bytes(c->io_dtype)) || !aligned4(given)) return ONELA_EINVAL;
  *p = onela::LogprobParams{};
  p->x = logits;
  p->given = given;
  p->R = long(c->num_rows);
  p->xs = c->logits_stride ? long(c->logits_stride) : long(c->vocab);
  p->scale = c->scale;
  p->V = c->vocab;
  p->G = c->num_given;
  return ONELA_OK;
}
}  // namespace

size_t onela_token_logprobs_workspace_bytes(const onela_logprob_config_t* cfg) {
  return onela::check_logprob(cfg) == ONELA_OK ? onela::logprob_workspace_bytes(cfg) : 0;
}

onela_status_t onela_token_logprobs(const onela_logprob_config_t* cfg, const void* logits,
                                    const int32_t* given, float* logp_out, float* lse_out,
                                    float* entropy_out, int32_t* top_tokens_out,
                                    float* top_logp_out, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  onela::LogprobParams p;
  const onela_status_t rc = logprob_inputs(cfg, logits, given, &p);
  if (rc != ONELA_OK) return rc;
  if (p.R > 0 && ((p.G > 0 && !logp_out) ||
                  (cfg->num_top > 0 && (!top_tokens_out || !top_logp_out))))
    return ONELA_EINVAL;
  if (!aligned4(logp_out) || !aligned4(lse_out) || !aligned4(entropy_out) ||
      !aligned4(top_tokens_out) || !aligned4(top_logp_out))
    return ONELA_EINVAL;
  if (!workspace || !aligned256(workspace)) return ONELA_EINVAL;
  if (workspace_bytes < onela::logprob_workspace_bytes(cfg)) return ONELA_ECAPACITY;
  const onela::LogprobPlan plan = onela::logprob_plan(cfg);
  const size_t row = size_t(p.R) * 4, tokens = row * size_t(p.G), best = row * size_t(cfg->num_top);
  if (onela::clash({{logp_out, tokens},
                    {lse_out, row},
                    {entropy_out, row},
                    {top_tokens_out, best},
                    {top_logp_out, best},
                    {workspace, plan.parts > 1 ? onela::logprob_workspace_bytes(cfg) : 0}},
                   {{logits, span(p.R, p.xs, p.V, cfg->io_dtype)}, {given, tokens}}, false))
    return ONELA_EINVAL;
  p.logp = logp_out;
  p.lse = lse_out;
  p.entropy = entropy_out;
  p.K = cfg->num_top;
  p.top = top_tokens_out;
  p.top_logp = top_logp_out;
  p.parts = static_cast<float*>(workspace);
  const hipError_t e =
      onela::launch_logprobs(p, plan, cfg->io_dtype == ONELA_BF16,
                             static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

onela_status_t onela_token_logprobs_backward(const onela_logprob_config_t* cfg,
                                             const void* logits, const int32_t* given,
                                             const float* lse, const float* entropy,
                                             const float* d_logp, const float* d_lse,
                                             const float* d_entropy, void* d_logits,
                                             void* stream) {
  onela::LogprobParams p;
  const onela_status_t rc = logprob_inputs(cfg, logits, given, &p);
  if (rc != ONELA_OK) return rc;
  if (p.R > 0 && (!lse || !d_logits || (p.G > 0 && !d_logp) || (d_entropy && !entropy)))
    return ONELA_EINVAL;
  if (!aligned4(lse) || !aligned4(entropy) || !aligned4(d_logp) || !aligned4(d_lse) ||
      !aligned4(d_entropy) || !aligned_to(d_logits, io_bytes(cfg->io_dtype)))
    return ONELA_EINVAL;
  // (in place: where every row is written over itself)
  const size_t row = size_t(p.R) * 4, tokens = row * size_t(p.G);
  const onela::Bytes out = {d_logits, span(p.R, p.V, p.V, cfg->io_dtype)};
  if (onela::clash({out}, {{logits, span(p.R, p.xs, p.V, cfg->io_dtype)}}, true) ||
      onela::clash({out},
                   {{given, tokens}, {lse, row}, {entropy, row}, {d_logp, tokens}, {d_lse, row},
                    {d_entropy, row}}, false))
    return ONELA_EINVAL;
  p.lse_in = lse;
  p.entropy_in = entropy;
  p.dlogp = d_logp;
  p.dlse = d_lse;
  p.dentropy = d_entropy;
  p.dx = d_logits;
  const hipError_t e = onela::launch_logprobs_backward(p, cfg->io_dtype == ONELA_BF16,
                                                       static_cast<hipStream_t>(stream));
  return launch_ok(e) ? ONELA_OK : ONELA_EHIP;
}

}  // extern "C"
