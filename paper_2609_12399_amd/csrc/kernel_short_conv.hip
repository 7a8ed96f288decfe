// Short causal convolution of every channel over packed sequences, its gradient, and its step on
// pools of states.
//
//   pre_t = b + sum_j w_j x_{t-K+1+j},  y_t = pre_t or silu(pre_t),  0 <= j < K (taps);
//   g_t = dy_t act'(pre_t),  dx_t = sum_j w_j g_{t+K-1-j},  dw_j = sum_t g_t x_{t-K+1+j},
// the inputs before a sequence being its state.  dx of those is the state's gradient, and the
// gradient of the last state is added to the dx of the inputs that it holds.
//
// A thread takes 4 channels and walks a run of tokens with the last K inputs in registers, so that
// x is read once but for the K - 1 rows before a run (and behind it, backward), which come
// from the cache.  (8 channels, 16 bytes of bf16: half the waves for the same runs, 16 ragged
// prompts of some 1000 tokens x 6144 107 us instead of 89.)  Where 64 lanes have channels, a wave
// has one run: its addresses, bounds and conditions are scalars.  Runs cross sequences: they
// are walked in pieces of one sequence each, the rows in the middle of a piece four at a time
// without conditions.  Weight gradients are summed over a thread's run, over the workgroup's runs
// in LDS, and over the workgroups by a second launch, each in a fixed order.
//
// Bound: HBM, forward at 5.3 TB/s (87 us there).  Backward, 8192 tokens x 6144 channels in 75
// us (70 + 5 for the second launch): 302 MB in 60 us at a copy's rate, beside which 45 us of
// vector instructions (28 per element) run, and the ends of the one turn that the workgroups
// take are not covered by others (12 us without the runs' middles).
#include "device_common.h"
#include "internal.h"

namespace onela {
namespace {

constexpr int kRows = 4;  // of x (and dy) in work per thread, and as many on their way

struct Bounds {
  long b, e;
};
// The tokens of sequence n, cut to the tensors.
__device__ inline Bounds bounds_of(const ConvParams& p, int n) {
  if (!p.offsets) return {long(n) * p.L, long(n + 1) * p.L};
  const long b = min(max(long(p.offsets[n]), 0l), p.total);
  return {b, min(max(long(p.offsets[n + 1]), b), p.total)};
}

// A sequence at or before the one that has token t0 (the wave's lowest): the last one that
// begins at or before it, 64 offsets at a time.  Every lane of the wave takes part.
__device__ inline int sequence_at(const ConvParams& p, long t0) {
  if (!p.offsets) return p.L ? int(unsigned(t0) / unsigned(p.L)) : 0;
  const int lane = threadIdx.x & 63;
  int lo = 0, n = p.N;  // it is one of lo .. lo + n - 1
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    const bool before = lane * step < n && (at == 0 || long(p.offsets[at]) <= t0);
    const int last = max(63 - __builtin_clzll(__ballot(before) | 1ull), 0);
    n = min(step, n - last * step);
    lo += last * step;
  }
  return lo;
}

template <int TAPS, int E>
struct Window {  // the last TAPS inputs (or gradients), newest last
  float v[TAPS][E];
  __device__ void push(const float (&x)[E]) {
#pragma unroll
    for (int j = 0; j + 1 < TAPS; ++j)
#pragma unroll
      for (int i = 0; i < E; ++i) v[j][i] = v[j + 1][i];
#pragma unroll
    for (int i = 0; i < E; ++i) v[TAPS - 1][i] = x[i];
  }
};

// Input at place t (before b: in the state) of the E channels from c0 on.
template <int TAPS, bool BF16, int E>
__device__ inline RawN<BF16, E> input_at(const ConvParams& p, const void* state, long row, long b,
                                      long t, unsigned c0) {
  RawN<BF16, E> r;
  if (t >= b)
    r.load(p.x, t * p.xs, c0);
  else if (state)
    r.load(state, (row * (TAPS - 1) + (t - b + TAPS - 1)) * p.C, c0);
  else
    r.clear();
  return r;
}

// The inputs before token t, as they come from memory and as the window (its newest place free).
template <int TAPS, bool BF16, int E>
struct Before {
  RawN<BF16, E> r[TAPS - 1];
  __device__ void load(const ConvParams& p, long n, long b, long t, unsigned c0) {
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i)
      r[i] = input_at<TAPS, BF16, E>(p, p.s_in, n, b, t - (TAPS - 1) + i, c0);
  }
  __device__ void fill(Window<TAPS, E>& win) const {
#pragma unroll
    for (int i = 0; i < TAPS - 1; ++i) r[i].floats(win.v[i + 1]);
  }
};

// kRows rows, `stride` elements apart, those from `count` on zeros.
template <bool BF16, int E>
struct Rows {
  RawN<BF16, E> r[kRows];
  __device__ void load(const void* x, long i, long stride, unsigned c0, int count) {
#pragma unroll
    for (int k = 0; k < kRows; ++k)
      if (k < count)
        r[k].load(x, i + k * stride, c0);
      else
        r[k].clear();
  }
  __device__ void load(const void* x, long i, long stride, unsigned c0) {
#pragma unroll
    for (int k = 0; k < kRows; ++k) r[k].load(x, i + k * stride, c0);
  }
};

template <int TAPS, int E>
struct Weights {
  float w[TAPS][E], b[E];
  __device__ void load(const ConvParams& p, unsigned c0) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
#pragma unroll
      for (int j = 0; j < TAPS; ++j) w[j][i] = p.w[(c0 + i) * TAPS + j];
      b[i] = p.bias ? p.bias[c0 + i] : 0.f;
    }
  }
  __device__ void apply(const Window<TAPS, E>& x, float (&y)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      y[i] = b[i];
#pragma unroll
      for (int j = 0; j < TAPS; ++j) y[i] = fmaf(w[j][i], x.v[j][i], y[i]);
    }
  }
};

template <bool BF16, int E>
__device__ inline void store_output(const ConvParams& p, long i, unsigned c0, float (&y)[E]) {
  if (p.silu)
#pragma unroll
    for (int k = 0; k < E; ++k) y[k] *= sigmoid(y[k]);
  RawN<BF16, E>::of(y).store_once(p.y, i, c0);
}

// The state after sequence n, 4 channels (read before it is stored: it may replace the first).
template <int TAPS, bool BF16, int E>
__device__ inline void last_state(const ConvParams& p, int n, unsigned c0) {
  const Bounds s = bounds_of(p, n);
  RawN<BF16, E> r[TAPS - 1];
#pragma unroll
  for (int i = 0; i < TAPS - 1; ++i)
    r[i] = input_at<TAPS, BF16, E>(p, p.s_in, n, s.b, s.e - (TAPS - 1) + i, c0);
#pragma unroll
  for (int i = 0; i < TAPS - 1; ++i) r[i].store(p.s_out, (long(n) * (TAPS - 1) + i) * p.C, c0);
}

// Zeros in the rows of a run behind the last sequence (p.clear).
template <bool BF16, int E>
__device__ inline void clear_rest(const ConvParams& p, void* out, long t0, long t1, unsigned c0) {
  RawN<BF16, E> zero;
  zero.clear();
  for (long t = max(t0, bounds_of(p, p.N - 1).e); t < t1; ++t) zero.store(out, t * p.C, c0);
}

// Where a thread stands: its channels, its run, and a sequence at or before the run's first token.
// WAVE: the wave's lanes share a run (64 channel groups side by side), and everything
// that depends on it is the same for all of them.
struct Place {
  int c0;
  long t0, t1;
  int n;
  bool in;
};
template <int E, bool WAVE>
__device__ inline Place place_of(const ConvParams& p, int ll, int run, int blocks_c) {
  const int bt = blockIdx.x / blocks_c, bc = blockIdx.x - bt * blocks_c;
  const int c0 = E * ((bc << ll) + int(threadIdx.x & ((1u << ll) - 1)));
  int r = threadIdx.x >> ll;
  if (WAVE) r = __builtin_amdgcn_readfirstlane(r);
  const long t0 = (long(bt) * (kConvThreads >> ll) + r) * run;
  int n = sequence_at(p, WAVE ? t0 : __shfl(t0, 0));
  if (WAVE) n = __builtin_amdgcn_readfirstlane(n);
  return {c0, t0, min(t0 + run, p.total), n, c0 < p.C && t0 < p.total};
}

// The first blocks_c * blocks_t workgroups take the tokens, the others the last states.
template <int TAPS, bool BF16, int E, bool WAVE>
__global__ __launch_bounds__(kConvThreads) void conv_kernel(ConvParams p, int ll, int run,
                                                            int blocks_c, unsigned token_blocks) {
  if (blockIdx.x >= token_blocks) {
    const long i = long(blockIdx.x - token_blocks) * kConvThreads + threadIdx.x;
    const int n = int(i / (p.C / E));
    if (n < p.N) last_state<TAPS, BF16, E>(p, n, E * int(i - long(n) * (p.C / E)));
    return;
  }
  const Place at = place_of<E, WAVE>(p, ll, run, blocks_c);
  if (!at.in) return;
  int n = at.n;
  Weights<TAPS, E> w;
  w.load(p, at.c0);
  for (; n < p.N; ++n) {
    const Bounds s = bounds_of(p, n);
    if (s.b >= at.t1) break;
    const long p0 = max(at.t0, s.b), p1 = min(at.t1, s.e);
    if (p0 >= p1) continue;
    const int own = int(p1 - p0);
    Rows<BF16, E> cur, next;
    // (the first rows are requested before anything is waited for)
    cur.load(p.x, p0 * p.xs, p.xs, at.c0, own);
    Before<TAPS, BF16, E> old;
    old.load(p, n, s.b, p0, at.c0);
    Window<TAPS, E> win;
    old.fill(win);
    auto row = [&](int r, int i) {
      float x[E], y[E];
      cur.r[r].floats(x);
      win.push(x);
      w.apply(win, y);
      store_output<BF16, E>(p, (p0 + i + r) * p.C, at.c0, y);
    };
    int i = 0;
#pragma unroll 1
    for (; i + 2 * kRows <= own; i += kRows) {
      next.load(p.x, (p0 + i + kRows) * p.xs, p.xs, at.c0);
#pragma unroll
      for (int r = 0; r < kRows; ++r) row(r, i);
      cur = next;
    }
#pragma unroll 1
    for (; i < own; i += kRows) {
      next.load(p.x, (p0 + i + kRows) * p.xs, p.xs, at.c0, own - i - kRows);
#pragma unroll
      for (int r = 0; r < kRows; ++r)
        if (i + r < own) row(r, i);
      cur = next;
    }
  }
  if (p.clear) clear_rest<BF16, E>(p, p.y, at.t0, at.t1, at.c0);
}

// (the workgroups that conv_plan takes a compute unit to hold at once)
template <int TAPS, bool BF16, int E, bool WAVE>
__global__ __launch_bounds__(kConvThreads, WAVE ? (BF16 ? 4 : 3) : 2) void conv_backward_kernel(
    ConvParams p, int ll, int run, int blocks_c, unsigned token_blocks) {
  if (blockIdx.x >= token_blocks) {  // sequences without tokens: the state passes through
    const long i = long(blockIdx.x - token_blocks) * kConvThreads + threadIdx.x;
    const int n = int(i / (p.C / E)), c0 = E * int(i - long(n) * (p.C / E));
    if (n >= p.N) return;
    const Bounds s = bounds_of(p, n);
    if (s.b < s.e) return;
#pragma unroll
    for (int j = 0; j < TAPS - 1; ++j) {
      const long o = (long(n) * (TAPS - 1) + j) * p.C + c0;
      RawN<BF16, E> r;
      if (p.ds_in)
        r.load(p.ds_in, o);
      else
        r.clear();
      r.store(p.ds_out, o);
    }
    return;
  }
  __shared__ float acc[TAPS + 1][kConvThreads][E];
  const Place at = place_of<E, WAVE>(p, ll, run, blocks_c);
  int n = at.n;
  float dw[TAPS + 1][E] = {};
  if (at.in) {
    Weights<TAPS, E> w;
    w.load(p, at.c0);
    for (; n < p.N; ++n) {
      const Bounds s = bounds_of(p, n);
      if (s.b >= at.t1) break;
      const long p0 = max(at.t0, s.b), p1 = min(at.t1, s.e);
      if (p0 >= p1) continue;
      // `own` tokens, and TAPS - 1 more, whose gradients the last inputs have a part of (rows behind
      // `end`, the sequence's among them, are zeros); inputs from `last` on are in the last state
      const int own = int(p1 - p0), all = own + TAPS - 1;
      const int end = int(min(p0 + all, s.e) - p0);
      const long last = p.ds_in ? s.e - (TAPS - 1) - p0 : p.total;
      const int low = p0 == s.b && p.ds_out ? 1 - TAPS : 0;  // (below 0: inputs of the first state)
      Rows<BF16, E> cx, cd, nx, nd;
      cx.load(p.x, p0 * p.xs, p.xs, at.c0, end);
      cd.load(p.dy, p0 * p.C, p.C, at.c0, end);
      Before<TAPS, BF16, E> before;
      before.load(p, n, s.b, p0, at.c0);
      Window<TAPS, E> win, gs = {};
      before.fill(win);
      // Row r of those in work: the gradient g before the activation and its share of the
      // weights' (of the run's own tokens), and d of the input TAPS - 1 rows before.
      auto row = [&](int r, bool mine, float(&d)[E]) {
        float x[E], g[E];
        cx.r[r].floats(x);
        cd.r[r].floats(g);
        win.push(x);
        if (p.silu) {
          float y[E];
          w.apply(win, y);
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const float sg = sigmoid(y[k]), t = fmaf(-y[k], sg, y[k]);
            g[k] *= fmaf(sg, t, sg);  // s (1 + y (1 - s))
          }
        }
        gs.push(g);
        if (mine)
#pragma unroll
          for (int k = 0; k < E; ++k) {
#pragma unroll
            for (int j = 0; j < TAPS; ++j) dw[j][k] = fmaf(g[k], win.v[j][k], dw[j][k]);
            dw[TAPS][k] += g[k];
          }
#pragma unroll
        for (int k = 0; k < E; ++k) {
          d[k] = w.w[0][k] * gs.v[TAPS - 1][k];
#pragma unroll
          for (int j = 1; j < TAPS; ++j) d[k] = fmaf(w.w[j][k], gs.v[TAPS - 1 - j][k], d[k]);
        }
      };
      int i = 0;
#pragma unroll 1
      do {
        // the run's beginning and end
        nx.load(p.x, (p0 + i + kRows) * p.xs, p.xs, at.c0, end - i - kRows);
        nd.load(p.dy, (p0 + i + kRows) * p.C, p.C, at.c0, end - i - kRows);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          float d[E];
          row(r, i + r < own, d);
          const int o = i + r - (TAPS - 1);  // the input whose gradient is complete
          if (o < low || o >= own) continue;
          if (o >= last) {
            RawN<BF16, E> f;
            float v[E];
            f.load(p.ds_in, (long(n) * (TAPS - 1) + (o - last)) * p.C, at.c0);
            f.floats(v);
#pragma unroll
            for (int k = 0; k < E; ++k) d[k] += v[k];
          }
          if (o >= 0)
            RawN<BF16, E>::of(d).store_once(p.dx, (p0 + o) * p.C, at.c0);
          else
            RawN<BF16, E>::of(d).store(p.ds_out, (long(n) * (TAPS - 1) + (o + TAPS - 1)) * p.C,
                                       at.c0);
        }
        cx = nx;
        cd = nd;
        // in between: all rows there and the run's own, no input in a state
        static_assert(kRows >= TAPS - 1, "the rows before are behind the first ones");
#pragma unroll 1
        for (i += kRows; i + 2 * kRows <= own; i += kRows) {
          nx.load(p.x, (p0 + i + kRows) * p.xs, p.xs, at.c0);
          nd.load(p.dy, (p0 + i + kRows) * p.C, p.C, at.c0);
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            float d[E];
            row(r, true, d);
            RawN<BF16, E>::of(d).store_once(p.dx, (p0 + i + r - (TAPS - 1)) * p.C, at.c0);
          }
          cx = nx;
          cd = nd;
        }
      } while (i < all);
    }
    if (p.clear) clear_rest<BF16, E>(p, p.dx, at.t0, at.t1, at.c0);
  }
  if (!p.partial) return;
  const int lanes = 1 << ll, c_first = at.c0 - E * (threadIdx.x & (lanes - 1));
  const long bt = blockIdx.x / blocks_c;
  const bool alone = token_blocks == unsigned(blocks_c);  // over the tokens: its sums are the results
#pragma unroll
  for (int j = 0; j <= TAPS; ++j)
#pragma unroll
    for (int k = 0; k < E; ++k) acc[j][threadIdx.x][k] = dw[j][k];
  __syncthreads();
  for (int c = threadIdx.x; c < E * lanes && c_first + c < p.C; c += kConvThreads)
#pragma unroll
    for (int j = 0; j <= TAPS; ++j) {
      float s = 0.f;
      for (int r = c / E; r < kConvThreads; r += lanes) s += acc[j][r][c % E];
      const int ch = c_first + c;
      if (!alone)
        p.partial[(bt * (TAPS + 1) + j) * p.C + ch] = s;
      else if (j < TAPS && p.dw)
        p.dw[long(ch) * TAPS + j] = s;
      else if (j == TAPS && p.db)
        p.db[ch] = s;
    }
}

// The workgroups' sums added up: 16 values of a tap per workgroup, 16 rows at a time.
__global__ __launch_bounds__(256) void conv_weight_kernel(ConvParams p, int taps, long rows) {
  __shared__ float acc[16][17];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
  const long width = long(taps + 1) * p.C;
  for (long first = long(blockIdx.x) * 16; first < width; first += long(gridDim.x) * 16) {
    const long col = first + c;
    float s = 0.f;
    if (col < width)
#pragma unroll 4
      for (long i = g; i < rows; i += 16) s += p.partial[i * width + col];
    __syncthreads();  // (the values before these have been read)
    acc[g][c] = s;
    __syncthreads();
    if (g != 0 || col >= width) continue;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += acc[i][c];
    const int j = int(col / p.C), ch = int(col - long(j) * p.C);
    if (j < taps) {
      if (p.dw) p.dw[long(ch) * taps + j] = s;
    } else if (p.db) {
      p.db[ch] = s;
    }
  }
}

// One thread for 4 channels of a sequence.  512 beams x 6144 channels 11 us: 50 MB (parents' states
// read twice from the cache among them) at 4.6 TB/s; several sequences per thread, which read the
// weights once, were no faster.
template <int TAPS, bool BF16, int E>
__global__ __launch_bounds__(kConvThreads) void conv_step_kernel(ConvParams p) {
  const long i = long(blockIdx.x) * kConvThreads + threadIdx.x;
  const int n = int(i / (p.C / E)), c0 = E * int(i - long(n) * (p.C / E));
  if (n >= p.N) return;
  const Bounds s = bounds_of(p, n);
  if (s.b >= s.e && !p.s_out) return;  // (in another pool the state follows its parent)
  const int from = p.slot ? p.slot[n] : n;
  const int to = p.s_out ? (p.slot_out ? p.slot_out[n] : n) : from;
  const int most = p.s_out ? p.slots_out : p.slots;
  if (from < 0 || from >= p.slots) {  // no state: the sequence's outputs are zeros
    RawN<BF16, E> zero;
    zero.clear();
    for (long t = s.b; t < s.e; ++t) zero.store(p.y, t * p.C + c0);
    return;
  }
  RawN<BF16, E> r[TAPS - 1], x;
  Weights<TAPS, E> w;
#pragma unroll
  for (int j = 0; j < TAPS - 1; ++j)
    r[j].load(p.s_in, (long(from) * (TAPS - 1) + j) * p.C + c0);
  w.load(p, c0);
  Window<TAPS, E> win;
#pragma unroll
  for (int j = 0; j < TAPS - 1; ++j) r[j].floats(win.v[j + 1]);
  for (long t = s.b; t < s.e; ++t) {
    float v[E], y[E];
    x.load(p.x, t * p.xs + c0);
    x.floats(v);
    win.push(v);
    w.apply(win, y);
    store_output<BF16, E>(p, t * p.C, c0, y);
#pragma unroll
    for (int j = 0; j + 2 < TAPS; ++j) r[j] = r[j + 1];
    r[TAPS - 2] = x;
  }
  if (to < 0 || to >= most) return;
  void* const out = p.s_out ? p.s_out : const_cast<void*>(p.s_in);
#pragma unroll
  for (int j = 0; j < TAPS - 1; ++j) r[j].store(out, (long(to) * (TAPS - 1) + j) * p.C + c0);
}

unsigned state_blocks(const ConvParams& p, int channels) {
  return unsigned((long(p.N) * (p.C / channels) + kConvThreads - 1) / kConvThreads);
}

template <int TAPS, bool BF16, bool WAVE>
hipError_t run_forward(const ConvParams& p, const ConvPlan& a, hipStream_t st) {
  constexpr int E = kConvLane;
  const unsigned tokens = unsigned(a.blocks_t * a.blocks_c);
  // a last state that replaces the first one waits until every token has read it
  const bool apart = p.s_out && p.s_out == p.s_in;
  const unsigned states = p.s_out ? state_blocks(p, E) : 0;
  const unsigned with = tokens + (apart ? 0 : states);
  if (with > 0) {
    conv_kernel<TAPS, BF16, E, WAVE>
        <<<with, kConvThreads, 0, st>>>(p, a.lanes_log2, a.run, a.blocks_c, tokens);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (apart)
    conv_kernel<TAPS, BF16, E, WAVE>
        <<<states, kConvThreads, 0, st>>>(p, a.lanes_log2, a.run, a.blocks_c, 0);
  return hipGetLastError();
}

template <int TAPS, bool BF16, bool WAVE>
hipError_t run_backward(const ConvParams& p, const ConvPlan& a, hipStream_t st) {
  constexpr int E = kConvLane;
  const unsigned tokens = unsigned(a.blocks_t * a.blocks_c);
  const unsigned states = p.ds_out ? state_blocks(p, E) : 0;
  if (tokens + states > 0) {
    conv_backward_kernel<TAPS, BF16, E, WAVE>
        <<<tokens + states, kConvThreads, 0, st>>>(p, a.lanes_log2, a.run, a.blocks_c, tokens);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.partial && a.blocks_t != 1)
    conv_weight_kernel<<<conv_weight_blocks(TAPS, p.C), 256, 0, st>>>(p, TAPS, a.blocks_t);
  return hipGetLastError();
}

template <int TAPS, bool BF16>
hipError_t run_step(const ConvParams& p, hipStream_t st) {
  constexpr int E = kConvLane;
  conv_step_kernel<TAPS, BF16, E><<<state_blocks(p, E), kConvThreads, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

#define ONELA_CONV(call)                                                      \
  if (taps == 2) return bf16 ? call(2, true) : call(2, false);                \
  if (taps == 3) return bf16 ? call(3, true) : call(3, false);                \
  return bf16 ? call(4, true) : call(4, false)

hipError_t launch_conv(const ConvParams& p, const ConvPlan& plan, int taps, bool bf16,
                       hipStream_t st) {
#define ONELA_FORWARD(K, B) \
  (plan.lanes_log2 == 6 ? run_forward<K, B, true>(p, plan, st) : run_forward<K, B, false>(p, plan, st))
  ONELA_CONV(ONELA_FORWARD);
#undef ONELA_FORWARD
}

hipError_t launch_conv_backward(const ConvParams& p, const ConvPlan& plan, int taps, bool bf16,
                                hipStream_t st) {
#define ONELA_BACKWARD(K, B)                                  \
  (plan.lanes_log2 == 6 ? run_backward<K, B, true>(p, plan, st) \
                        : run_backward<K, B, false>(p, plan, st))
  ONELA_CONV(ONELA_BACKWARD);
#undef ONELA_BACKWARD
}

hipError_t launch_conv_step(const ConvParams& p, int taps, bool bf16, hipStream_t st) {
#define ONELA_STEP(K, B) run_step<K, B>(p, st)
  ONELA_CONV(ONELA_STEP);
#undef ONELA_STEP
}
#undef ONELA_CONV

}  // namespace onela
