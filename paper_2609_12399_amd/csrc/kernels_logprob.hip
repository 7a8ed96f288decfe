// Log probabilities of tokens from logits: of given tokens, the best ones, the logarithm of the
// sum and the entropy, from one read of a row; and their gradient.
//
// With m the row's largest logit, c the scale, d_v = c (x_v - m):
//   s = sum e^d,  lse = c m + ln s,  logp_v = d_v - ln s,  entropy = ln s - sum e^d d / s.
// Every thread keeps its own m, s and sum e^d d over the columns that it reads (one
// exponential per element, the sums rescaled when m grows); the workgroup joins them at the end.
//
// The best K: the K-th largest of the threads' maxima of the first chunk bounds the K-th best
// from below, so that few elements (some K to 2 K) pass into a list in LDS; the list is
// cut back to its K best by counting, for each, those before it, when it grows over 256, and
// the bound rises to the K-th.  Elements of later chunks have higher columns, so one that
// equals the K-th best then stays out.  The order is by (value, lower column) and does not
// depend on the order of the list.  Masked elements (-inf) never pass: if fewer than K remain,
// the first masked columns fill the rest.
//
// A row belongs to a workgroup (a wave up to 2048 columns), or in parts to several where there
// are few rows, joined by a second launch.  Rows begin anywhere: 16-byte loads need only
// the elements' alignment.  Bound: HBM.
#include "device_common.h"
#include "internal.h"

namespace onela {
namespace {

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr float kNegInf = -__builtin_inff();
// Below e^-200 or 2^-200 an element's share of the entropy or its gradient is 0 in fp32; the bound
// keeps 0 x -inf out of them.
constexpr float kFar = -200.f;

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef unsigned long long u64;

// EV elements (16 bytes) of a row from column c on, those past `end` -inf.
template <bool BF16>
struct Piece {
  static constexpr int EV = BF16 ? 8 : 4;
  u32x4 w;
  __device__ void load(const char* row, int c, int end) {
    constexpr int size = BF16 ? 2 : 4;
    if (c + EV <= end) {
      w = *reinterpret_cast<const u32x4_any*>(row + long(c) * size);
      return;
    }
    unsigned u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        const uint16_t* const q = reinterpret_cast<const uint16_t*>(row) + c + 2 * i;
        const unsigned lo = c + 2 * i < end ? q[0] : 0xff80u;
        const unsigned hi = c + 2 * i + 1 < end ? q[1] : 0xff80u;
        u[i] = lo | hi << 16;
      } else {
        u[i] = c + i < end ? reinterpret_cast<const unsigned*>(row)[c + i] : 0xff800000u;
      }
    }
    w = u32x4{u[0], u[1], u[2], u[3]};
  }
  __device__ void floats(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        x[2 * i] = bf16_lo_to_float(w[i]);
        x[2 * i + 1] = bf16_hi_to_float(w[i]);
      } else {
        x[i] = __uint_as_float(w[i]);
      }
    }
  }
};

template <int G>
__device__ inline float group_max(float x) {
  if constexpr (G >= 2) x = fmaxf(x, dpp<0xB1>(x));
  if constexpr (G >= 4) x = fmaxf(x, dpp<0x4E>(x));
  if constexpr (G >= 8) x = fmaxf(x, dpp<0x141>(x));
  if constexpr (G >= 16) x = fmaxf(x, dpp<0x140>(x));
  if constexpr (G >= 32) x = fmaxf(x, __shfl_xor(x, 16));
  if constexpr (G >= 64) x = fmaxf(x, __shfl_xor(x, 32));
  return x;
}

// A row's sums: m the largest, s = sum e^{c (x - m)}, t = sum of those times log2 of them.
// Nothing but masked elements: m = -inf, s = t = 0.  (s is NaN where an element is NaN or +inf.)
struct Sums {
  float m, s, t;
};
__device__ inline float origin(float m) { return m == kNegInf ? 0.f : m; }
// The sums with another, larger m.
template <bool ENT>
__device__ inline void rebase(Sums& a, float m, float c2) {
  const float d = a.m == kNegInf ? kFar : fmaxf((a.m - origin(m)) * c2, kFar);
  const float f = a.m == m ? 1.f : __builtin_amdgcn_exp2f(d);
  if constexpr (ENT) a.t = f * fmaf(d, a.m == m ? 0.f : a.s, a.t);
  a.s *= f;
  a.m = m;
}

// The workgroup's sums, in every thread.
template <int THREADS, bool ENT>
__device__ inline void join(Sums& a, float c2, float* lds /* [3][THREADS / 64] */) {
  constexpr int W = THREADS / 64;
  float m = group_max<64>(a.m);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) m = fmaxf(m, lds[i]);
  }
  rebase<ENT>(a, m, c2);
  a.s = group_sum<64>(a.s);
  if constexpr (ENT) a.t = group_sum<64>(a.t);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) {
      lds[W + (threadIdx.x >> 6)] = a.s;
      lds[2 * W + (threadIdx.x >> 6)] = a.t;
    }
    __syncthreads();
    a.s = lds[W];
    a.t = lds[2 * W];
#pragma unroll
    for (int i = 1; i < W; ++i) {
      a.s += lds[W + i];
      a.t += lds[2 * W + i];
    }
  }
}

// Candidates in order of preference as whole numbers: the value's order above, lower columns
// first below.  0 is none.
__device__ inline u64 candidate(float x, int col) {
  const unsigned b = __float_as_uint(x + 0.f);  // (-0 becomes 0)
  const unsigned k = b & 0x80000000u ? ~b : b | 0x80000000u;
  return u64(k) << 32 | unsigned(~col);
}
__device__ inline int column_of(u64 c) { return int(~unsigned(c)); }
__device__ inline float value_of(u64 c) {
  const unsigned k = unsigned(c >> 32);
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// The list of candidates of a workgroup.
template <int THREADS, int MORE>
struct List {
  static_assert(THREADS >= kMaxTop, "a thread for each of the best");
  static constexpr int CAP = MORE + kMaxTop;
  u64 c[CAP];
  u64 best[kMaxTop];
  float maxima[THREADS];
  int count;
  float bound;  // of the first chunk

  // Cuts the list to its K best, in order.  Every thread calls it, after a barrier; ends with one.
  __device__ void cut(int K) {
    const int n = count;
    for (int i = threadIdx.x; i < n; i += THREADS) {
      const u64 x = c[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += c[j] > x;
      if (rank < K) best[rank] = x;
    }
    __syncthreads();
    const int m = n < K ? n : K;
    if (int(threadIdx.x) < m) c[threadIdx.x] = best[threadIdx.x];
    if (threadIdx.x == 0) count = m;
    __syncthreads();
  }
};

// Results of a row from its sums and its list (sorted, cut): every thread of the workgroup.
template <int THREADS, bool BF16, bool ENT, bool TOP, typename L>
__device__ inline void finish(const LogprobParams& p, long row, const Sums& a, L* list) {
  constexpr int size = BF16 ? 2 : 4;
  const char* const x = static_cast<const char*>(p.x) + row * p.xs * size;
  const bool gone = a.m == kNegInf && a.s == 0.f;  // (a row of NaN has another s)
  const float o = origin(a.m), logs = kLn2 * __builtin_amdgcn_logf(a.s);
  if (threadIdx.x == 0) {
    // a row of NaN alone has no largest element
    if (p.lse) p.lse[row] = gone ? kNegInf : fmaf(o, p.scale, logs);
    if (ENT && p.entropy) p.entropy[row] = gone ? 0.f : logs - kLn2 * a.t / a.s;
  }
  for (int g = threadIdx.x; g < p.G; g += THREADS) {
    const int v = p.given[row * p.G + g];
    float r = v < 0 ? 0.f : __builtin_nanf("");
    if (v >= 0 && v < p.V)
      r = gone ? kNegInf : fmaf(load1<BF16>(x, v) - o, p.scale, -logs);
    p.logp[row * p.G + g] = r;
  }
  if constexpr (TOP) {
    // fewer than K that are not masked: the first masked columns, then those of NaN
    if (list->count < p.K && threadIdx.x < 64) {
      int at = list->count, nans = 0;
      int nan_col = 0;  // lane i: the column of the i-th NaN
      for (int c = 0; c < p.V && at < p.K; c += 64) {
        const int col = c + int(threadIdx.x);
        const float v = col < p.V ? load1<BF16>(x, col) : 0.f;
        const u64 masked = __ballot(v == kNegInf), nan = __ballot(v != v);
        const u64 below = (1ull << threadIdx.x) - 1;
        if (v == kNegInf) {
          const int i = at + __popcll(masked & below);
          if (i < p.K) list->c[i] = candidate(kNegInf, col);
        }
        at += __popcll(masked);
        if (nan) {  // lane i takes NaN number nans + j from the j-th lane that has one
          const int j = int(threadIdx.x) - nans;
          u64 rest = nan;
          for (int k = 0; k < j && rest; ++k) rest &= rest - 1;
          if (j >= 0 && rest) nan_col = c + __builtin_ctzll(rest);
          nans += __popcll(nan);
        }
      }
      // NaN is last; it keeps the key of none with its column
      if (at < p.K) {
        const int i = at + int(threadIdx.x);
        if (i < p.K && int(threadIdx.x) < nans) list->c[i] = unsigned(~nan_col);
      }
    }
    __syncthreads();
    if (int(threadIdx.x) < p.K) {
      const u64 c = list->c[threadIdx.x];
      const float v = c >> 32 ? value_of(c) : __builtin_nanf("");
      p.top[row * p.K + threadIdx.x] = column_of(c);
      p.top_logp[row * p.K + threadIdx.x] = gone ? kNegInf : fmaf(v - o, p.scale, -logs);
    }
  }
}

// One part of a row per workgroup; with one part, its results.
template <int THREADS, bool BF16, bool ENT, bool TOP>
__global__ __launch_bounds__(THREADS) void logprob_kernel(LogprobParams p, int parts,
                                                          int columns) {
  constexpr int EV = Piece<BF16>::EV, NV = 32 / EV, CH = THREADS * 32;
  __shared__ float red[3 * (THREADS / 64)];
  __shared__ List<THREADS, TOP ? THREADS * EV : 1> list;
  const long row = blockIdx.x / parts;
  const int part = int(blockIdx.x - row * parts), begin = part * columns;
  const int end = min(begin + columns, p.V);
  const char* const x = static_cast<const char*>(p.x) + row * p.xs * (BF16 ? 2 : 4);
  const float c2 = p.scale * kLog2e;
  Sums a{kNegInf, 0.f, 0.f};
  float bound = kNegInf;   // elements above it are candidates,
  bool equal = false;      // and those that equal it
  if (TOP && threadIdx.x == 0) list.count = 0;
  Piece<BF16> next[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
    next[k].load(x, begin + (k * THREADS + int(threadIdx.x)) * EV, end);
  for (int c = begin; c < end; c += CH) {
    float v[32];
#pragma unroll
    for (int k = 0; k < NV; ++k) next[k].floats(v + k * EV);
    if (c + CH < end)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        next[k].load(x, c + CH + (k * THREADS + int(threadIdx.x)) * EV, end);
    float mc = kNegInf;
#pragma unroll
    for (int i = 0; i < 32; ++i) mc = fmaxf(mc, v[i]);
    if (mc > a.m) rebase<ENT>(a, mc, c2);
    const float o = origin(a.m);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float d = (v[i] - o) * c2, e = __builtin_amdgcn_exp2f(d);
      s += e;
      if constexpr (ENT) a.t = fmaf(e, fmaxf(d, kFar), a.t);
    }
    a.s += s;
    if constexpr (TOP) {
      const int K = p.K;
      if (c == begin) {
        // the K-th largest of the threads' maxima
        list.maxima[threadIdx.x] = mc;
        __syncthreads();
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < THREADS; ++j) {
          const float y = list.maxima[j];
          rank += y > mc || (y == mc && j < int(threadIdx.x));
        }
        if (rank == K - 1) list.bound = mc;
        __syncthreads();
        bound = list.bound;
        equal = bound > kNegInf;
      }
      auto passes = [&](float y) { return y > bound || (equal && y == bound); };
      const int before = list.count;
      __syncthreads();
      if (passes(mc)) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) n += passes(v[i]);
        int at = atomicAdd(&list.count, n);
        if (at + n <= list.CAP)
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (passes(v[i])) {
              const int col = c + ((i / EV) * THREADS + int(threadIdx.x)) * EV + i % EV;
              list.c[at++] = candidate(v[i], col);
            }
      }
      __syncthreads();
      const int n = list.count;
      __syncthreads();
      if (n > list.CAP) {
        // many equal elements: again, 16 bytes per thread at a time, cut after each
        if (threadIdx.x == 0) list.count = before;
        __syncthreads();
        if (before > 0) list.cut(K);
#pragma unroll 1
        for (int k = 0; k < NV; ++k) {
          if (list.count >= K) {
            bound = value_of(list.c[K - 1]);
            equal = false;
          }
          __syncthreads();
          float u[EV];
#pragma unroll
          for (int i = 0; i < EV; ++i) {
            u[i] = v[i];
#pragma unroll
            for (int kk = 1; kk < NV; ++kk) u[i] = kk == k ? v[kk * EV + i] : u[i];
          }
#pragma unroll
          for (int i = 0; i < EV; ++i)
            if (passes(u[i]))
              list.c[atomicAdd(&list.count, 1)] =
                  candidate(u[i], c + (k * THREADS + int(threadIdx.x)) * EV + i);
          __syncthreads();
          list.cut(K);
        }
      } else if (n > 256) {
        list.cut(K);
      }
      if (n > 256 && list.count >= K) {
        bound = value_of(list.c[K - 1]);
        equal = false;
      }
    }
  }
  join<THREADS, ENT>(a, c2, red);
  if constexpr (TOP) {
    __syncthreads();
    list.cut(p.K);
  }
  if (parts == 1) {
    finish<THREADS, BF16, ENT, TOP>(p, row, a, &list);
    return;
  }
  const int words = 4 + 2 * p.K;
  float* const out = p.parts + (row * parts + part) * words;
  if (threadIdx.x == 0) {
    out[0] = a.m;
    out[1] = a.s;
    out[2] = a.t;
  }
  if (TOP && int(threadIdx.x) < p.K)
    reinterpret_cast<u64*>(out + 4)[threadIdx.x] =
        int(threadIdx.x) < list.count ? list.c[threadIdx.x] : 0ull;
}

// Joins the parts of a row.
constexpr int kJoinThreads = 256;
template <bool BF16, bool ENT, bool TOP>
__global__ __launch_bounds__(kJoinThreads) void logprob_join_kernel(LogprobParams p, int parts) {
  __shared__ float red[3 * (kJoinThreads / 64)];
  __shared__ List<kJoinThreads, TOP ? 64 * kMaxTop : 1> list;
  const long row = blockIdx.x;
  const int words = 4 + 2 * p.K;
  const float* const in = p.parts + row * parts * words;
  Sums a{kNegInf, 0.f, 0.f};
  if (int(threadIdx.x) < parts) {
    const float* const q = in + long(threadIdx.x) * words;
    a = Sums{q[0], q[1], q[2]};
  }
  if constexpr (TOP) {
    // Each part's best are in order: with q = ceil(K / parts) of every part there are K, so the
    // least of the parts' q-th is a bound.
    if (threadIdx.x == 0) list.count = 0;
    const int q = (p.K + parts - 1) / parts;
    u64 bound = ~0ull;
    for (int i = 0; i < parts; ++i) {
      const u64 y = reinterpret_cast<const u64*>(in + long(i) * words + 4)[q - 1];
      bound = y < bound ? y : bound;
    }
    if (bound == 0) bound = 1;  // (0: none)
    __syncthreads();
    for (int i = threadIdx.x; i < parts * p.K; i += kJoinThreads) {
      const int part = i / p.K;
      const u64 y = reinterpret_cast<const u64*>(in + long(part) * words + 4)[i - part * p.K];
      if (y >= bound) list.c[atomicAdd(&list.count, 1)] = y;
    }
    __syncthreads();
    list.cut(p.K);
  }
  join<kJoinThreads, ENT>(a, p.scale * kLog2e, red);
  finish<kJoinThreads, BF16, ENT, TOP>(p, row, a, &list);
}

// ---- gradient ----------------------------------------------------------------------------
// Every element by itself from lse: p = e^{c x - lse}, dx = c p (a - dH (ln p + H)), with a = dlse
// - sum of the given tokens' gradients; then the given tokens that stand in the workgroup's
// columns are written again with their own gradients added (equal ones all, so
// that it does not matter which thread writes last).
constexpr int kBackThreads = 256;
constexpr int kBackColumns = 4096;  // of a workgroup

template <bool BF16>
__device__ inline void store_any(char* row, int c, int end, const float* x) {
  constexpr int EV = Piece<BF16>::EV;
  if (c + EV <= end) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if constexpr (BF16)
        w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      else
        w[i] = __float_as_uint(x[i]);
    *reinterpret_cast<u32x4_any*>(row + long(c) * (BF16 ? 2 : 4)) = w;
    return;
  }
#pragma unroll
  for (int i = 0; i < EV; ++i)
    if (c + i < end) {
      if constexpr (BF16)
        reinterpret_cast<uint16_t*>(row)[c + i] = uint16_t(pack_bf16x2(x[i], x[i]));
      else
        reinterpret_cast<float*>(row)[c + i] = x[i];
    }
}

template <bool BF16, bool ENT>
__global__ __launch_bounds__(kBackThreads) void logprob_backward_kernel(LogprobParams p,
                                                                        int blocks) {
  constexpr int EV = Piece<BF16>::EV, NV = kBackColumns / (kBackThreads * EV);
  constexpr int size = BF16 ? 2 : 4;
  __shared__ int token[kMaxGiven];
  __shared__ float grad[kMaxGiven];
  const long row = blockIdx.x / blocks;
  const int begin = int(blockIdx.x - row * blocks) * kBackColumns;
  const int end = min(begin + kBackColumns, p.V);
  const char* const x = static_cast<const char*>(p.x) + row * p.xs * size;
  char* const dx = static_cast<char*>(p.dx) + row * p.V * size;
  Piece<BF16> in[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
    in[k].load(x, begin + (k * kBackThreads + int(threadIdx.x)) * EV, end);
  const float lse = p.lse_in[row];
  const bool gone = lse == kNegInf;
  float a = p.dlse ? p.dlse[row] : 0.f;
  const float dh = ENT ? p.dentropy[row] : 0.f, h = ENT ? p.entropy_in[row] : 0.f;
  // the given tokens' gradients; a token past the vocabulary makes the row NaN
  int mine = -1;
  float at_mine = 0.f;
  for (int g = threadIdx.x; g < p.G; g += kBackThreads) {
    const int v = p.given[row * p.G + g];
    token[g] = v;
    grad[g] = v < 0 ? 0.f : v < p.V ? p.dlogp[row * p.G + g] : __builtin_nanf("");
    if (v >= begin && v < end) {
      mine = v;
      at_mine = load1<BF16>(x, v);
    }
  }
  if (p.G > 0) {
    __syncthreads();
    float s = 0.f;
    for (int g = 0; g < p.G; ++g) s += grad[g];
    a -= s;
  }
  auto value = [&](float y) {
    const float l = fmaf(y, p.scale, -lse);
    float f = a;
    if constexpr (ENT) f = fmaf(-dh, fmaxf(l, kFar) + h, a);
    return gone ? 0.f : __builtin_amdgcn_exp2f(l * kLog2e) * f;
  };
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = begin + (k * kBackThreads + int(threadIdx.x)) * EV;
    if (c >= end) break;
    float v[EV];
    in[k].floats(v);
#pragma unroll
    for (int i = 0; i < EV; ++i) v[i] = p.scale * value(v[i]);
    store_any<BF16>(dx, c, end, v);
  }
  if (p.G == 0) return;
  __syncthreads();
  if (mine >= 0) {
    float s = 0.f;
    for (int g = 0; g < p.G; ++g) s += token[g] == mine ? grad[g] : 0.f;
    const float y = gone ? 0.f : p.scale * (value(at_mine) + s);
    if constexpr (BF16)
      reinterpret_cast<uint16_t*>(dx)[mine] = uint16_t(pack_bf16x2(y, y));
    else
      reinterpret_cast<float*>(dx)[mine] = y;
  }
}

template <bool BF16, bool ENT, bool TOP>
hipError_t run(const LogprobParams& p, const LogprobPlan& a, hipStream_t st) {
  const unsigned blocks = unsigned(p.R * a.parts);
  if (a.threads == 64)
    logprob_kernel<64, BF16, ENT, TOP><<<blocks, 64, 0, st>>>(p, a.parts, a.columns);
  else
    logprob_kernel<256, BF16, ENT, TOP><<<blocks, 256, 0, st>>>(p, a.parts, a.columns);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  logprob_join_kernel<BF16, ENT, TOP><<<unsigned(p.R), kJoinThreads, 0, st>>>(p, a.parts);
  return hipGetLastError();
}

template <bool BF16>
hipError_t by_kind(const LogprobParams& p, const LogprobPlan& a, hipStream_t st) {
  if (p.K > 0)
    return p.entropy ? run<BF16, true, true>(p, a, st) : run<BF16, false, true>(p, a, st);
  return p.entropy ? run<BF16, true, false>(p, a, st) : run<BF16, false, false>(p, a, st);
}

}  // namespace

hipError_t launch_logprobs(const LogprobParams& p, const LogprobPlan& plan, bool bf16,
                           hipStream_t st) {
  if (p.R == 0) return hipSuccess;
  return bf16 ? by_kind<true>(p, plan, st) : by_kind<false>(p, plan, st);
}

hipError_t launch_logprobs_backward(const LogprobParams& p, bool bf16, hipStream_t st) {
  if (p.R == 0) return hipSuccess;
  const int blocks = (p.V + kBackColumns - 1) / kBackColumns;
  const unsigned grid = unsigned(p.R * blocks);
#define ONELA_BACK(B, E) \
  logprob_backward_kernel<B, E><<<grid, kBackThreads, 0, st>>>(p, blocks)
  if (bf16) {
    if (p.dentropy)
      ONELA_BACK(true, true);
    else
      ONELA_BACK(true, false);
  } else {
    if (p.dentropy)
      ONELA_BACK(false, true);
    else
      ONELA_BACK(false, false);
  }
#undef ONELA_BACK
  return hipGetLastError();
}

}  // namespace onela
