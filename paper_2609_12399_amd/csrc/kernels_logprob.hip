// Log probabilities of tokens from logits: of given tokens, the best ones, the logarithm of the
// sum and the entropy, from one read of a row; and their gradient.
//
// With m the row's largest logit, c the scale, d_v = c (x_v - m):
//   s = sum e^d,  lse = c m + ln s,  logp_v = d_v - ln s,  entropy = ln s - sum e^d d / s.
// Every thread keeps its own m, s and sum e^d d over the columns that it reads (one
// exponential per element, the sums rescaled when m grows); the workgroup joins them at the end.
//
// The best K: every thread's largest element of the first chunk goes to LDS, and their K-th
// largest (found bit by bit with ballots) bounds the K-th best of the row from below: some K to 2 K
// elements of each chunk pass it into a list in LDS, with no barrier after the first chunk.  At the
// end one wave takes the list's K best, 64 at a time, by counting for each those before it.
// Where a row's order or its ties let more through than the list holds, it is read again in
// smaller pieces with a bound for each.  The order is by (value, lower column) and does not
// depend on the order of the list.  Masked elements (-inf) never pass: if fewer than K remain,
// the first masked columns fill the rest.
//
// A row belongs to a workgroup of one, two or four waves, or in parts to several where there are
// few rows, joined by a second launch.  Rows begin anywhere: 16-byte loads need only the elements'
// alignment.  Bound: HBM without the best (4096 rows of 50001 in bf16 88 us, 4.7 TB/s, with or
// without the entropy).  With the 20 best 105 us, with 64 133: the bound, the list and the choice
// from it are vector instructions, which then keep the units 70% busy, and waits that the other
// workgroups of a compute unit cover in part.  Four waves with chunks of 16 elements per thread
// instead of 32: 104 us with the 20 best, but 137 with 64, and 10.1 instead of 8.0 for 300 rows of
// 8192.  Rows that let more through than the list holds are read twice or more: of 1024 rows of
// 50001 with the 20 best, random ones take 32 us, equal ones 217, rising ones 259, NaN alone
// 326; so does a mask that leaves a range of columns behind those that the bound was last formed
// from (24576 columns, the last third allowed 58 us, the first 17, all 20; 4096 rows, the second
// or last third 160, the first 39, all 49).
#include <type_traits>

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

// Values in order as whole numbers (NaN has none here).
__device__ inline unsigned ordered(float x) {
  const unsigned b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// Candidates in order of preference as whole numbers: the value's order above, lower columns
// first below.  0 is none.
__device__ inline u64 candidate(float x, int col) {
  return u64(ordered(x + 0.f)) << 32 | unsigned(~col);  // (-0 becomes 0)
}
__device__ inline int column_of(u64 c) { return int(~unsigned(c)); }
__device__ inline float value_of(u64 c) {
  const unsigned k = unsigned(c >> 32);
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// The candidates of a workgroup's waves, each in a part of its own (so that finding a place takes
// no exchange), and room for the wave that takes the best of them.
template <int WAVES, int CAPACITY>
struct List {
  static constexpr int CAP = CAPACITY;
  u64 c[WAVES][CAP];
  u64 best[128];
  int count[WAVES];  // of candidates, those that found no room among them

  // Whether one wave had more than its part holds.
  __device__ bool short_of_room() const {
    int n = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) n = max(n, count[w]);
    return n > CAP;
  }
};

// LDS of one wave: what its lanes have written is what they read next.
__device__ inline void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// One wave: the first m <= 128 of `best`, cut to their K best, in order; returns how many.
__device__ inline int in_order(u64* best, int m, int K) {
  const int lane = threadIdx.x & 63;
  const u64 x = lane < m ? best[lane] : 0, y = lane + 64 < m ? best[lane + 64] : 0;
  int rx = 0, ry = 0;
#pragma unroll 4
  for (int j = 0; j < m; ++j) {
    const u64 z = best[j];
    rx += z > x;
    ry += z > y;
  }
  wave_fence();
  if (x && rx < K) best[rx] = x;
  if (y && ry < K) best[ry] = y;
  wave_fence();
  return m < K ? m : K;
}

// One wave: the K best of the candidates in `best`, in order; returns how many there are.  `m`
// of them are there already.
template <int WAVES, int CAP>
__device__ inline int take_best(List<WAVES, CAP>* list, int K, int m = 0) {
  const int lane = threadIdx.x & 63;
  u64 bound = m < K ? 0 : list->best[K - 1];
#pragma unroll 1
  for (int w = 0; w < WAVES; ++w) {
    const int n = list->count[w];
    for (int i = 0; i < n; i += 64) {
      const u64 x = i + lane < n ? list->c[w][i + lane] : 0;
      const u64 pass = __ballot(x > bound);
      if (!pass) continue;
      if (x > bound) list->best[m + __popcll(pass & ((1ull << lane) - 1))] = x;
      m += __popcll(pass);
      wave_fence();
      if (m >= 64) {
        m = in_order(list->best, m, K);
        if (m == K) bound = list->best[K - 1];
      }
    }
  }
  return in_order(list->best, m, K);
}

// A lower bound of the K-th largest of N values per lane over the wave: the upper 16 bits of its
// order, one at a time (exact for bf16), and above -inf.
template <int N>
__device__ inline float kth_largest(const float (&x)[N], int K) {
  unsigned k[N], prefix = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) k[i] = ordered(x[i]);
#pragma unroll 1
  for (unsigned bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
    const unsigned at = prefix | bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __popcll(__ballot(k[i] >= at));
    if (n >= K) prefix = at;
  }
  const unsigned b = prefix & 0x80000000u ? prefix & 0x7fffffffu : ~prefix;
  const float f = __uint_as_float(b);
  return f > -3.40282347e38f ? f : -3.40282347e38f;  // (whatever is no number: everything passes)
}

// Appends the wave's elements from `bound` on to its part of the list, which has `count`; v[i] of a
// lane stands at column(i).  Few pass: one comparison per element finds the lanes that have one,
// and only then is there more to do.
template <int N, typename L, typename C>
__device__ inline void append(L* list, int& count, const float* v, float bound, C column) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const u64 pass = __ballot(v[i] >= bound);
    if (pass == 0) continue;
    const int at = count + __popcll(pass & ((1ull << (threadIdx.x & 63)) - 1));
    if (v[i] >= bound && at < L::CAP) list->c[threadIdx.x >> 6][at] = candidate(v[i], column(i));
    count += __popcll(pass);
  }
}

// The bound of the K-th best from every thread's largest element (in LDS where there are several
// waves).
template <int THREADS>
__device__ inline float bound_of(float mine, int K, volatile float* maxima, bool wait = true) {
  float x[THREADS / 64] = {mine};
  if constexpr (THREADS > 64) {
    maxima[threadIdx.x] = mine;
    if (wait) __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) x[i] = maxima[i * 64 + (threadIdx.x & 63)];
  }
  return kth_largest<THREADS / 64>(x, K);
}

// The K best of a row's columns where the list was too short: pieces of 16 bytes per thread,
// each with a bound of its own, its K best joined to those before it.  Later
// columns that equal the K-th best stay out.
template <int THREADS, bool BF16, typename L>
__device__ __noinline__ int reread(const char* x, int begin, int end, int K, L* list,
                                   float* maxima) {
  constexpr int EV = Piece<BF16>::EV;
  static_assert(64 * EV <= L::CAP, "the list holds a piece");
  int m = 0;
  for (int c = begin; c < end; c += THREADS * EV) {
    const int col = c + int(threadIdx.x) * EV;
    Piece<BF16> in;
    in.load(x, col, end);
    float v[EV], most = kNegInf;
    in.floats(v);
#pragma unroll
    for (int i = 0; i < EV; ++i) most = fmaxf(most, v[i]);
    __syncthreads();  // (the list and the maxima have been read)
    const float bound = bound_of<THREADS>(most, K, maxima);
    int count = 0;
    append<EV>(list, count, v, bound, [&](int i) { return col + i; });
    if ((threadIdx.x & 63) == 0) list->count[threadIdx.x >> 6] = count;
    __syncthreads();
    if (threadIdx.x < 64) m = take_best(list, K, m);
  }
  return m;
}

// Results of a row from its sums; the first wave has the m best of the list in order.
template <int THREADS, bool BF16, bool ENT, bool TOP, typename L>
__device__ inline void finish(const LogprobParams& p, long row, const Sums& a, L* list, int m) {
  constexpr int size = BF16 ? 2 : 4;
  const char* const x = static_cast<const char*>(p.x) + row * p.xs * size;
  const bool gone = a.m == kNegInf && a.s == 0.f;  // (a row of NaN has another s)
  const float o = origin(a.m), logs = kLn2 * __builtin_amdgcn_logf(a.s);
  if (threadIdx.x == 0) {
    if (p.lse) p.lse[row] = gone ? kNegInf : fmaf(o, p.scale, logs);
    if (ENT && p.entropy) {
      const float h = logs - kLn2 * a.t / a.s;
      p.entropy[row] = gone || h < 0.f ? 0.f : h;  // (a rounding below 0)
    }
  }
  for (int g = threadIdx.x; g < p.G; g += THREADS) {
    const int v = p.given[row * p.G + g];
    float r = v < 0 ? 0.f : __builtin_nanf("");
    if (v >= 0 && v < p.V)
      r = gone ? kNegInf : fmaf(load1<BF16>(x, v) - o, p.scale, -logs);
    p.logp[row * p.G + g] = r;
  }
  if constexpr (TOP) {
    if (threadIdx.x >= 64) return;
    const int lane = threadIdx.x;
    if (m < p.K) {
      // fewer than K that are not masked: the first masked columns, then those of NaN
      int at = m, nans = 0;
      int nan_col = 0;  // lane i: the column of the i-th NaN
      for (int c = 0; c < p.V && at < p.K; c += 64) {
        const int col = c + lane;
        const float v = col < p.V ? load1<BF16>(x, col) : 0.f;
        const u64 masked = __ballot(v == kNegInf), nan = __ballot(v != v);
        if (v == kNegInf) {
          const int i = at + __popcll(masked & ((1ull << lane) - 1));
          if (i < p.K) list->best[i] = candidate(kNegInf, col);
        }
        at += __popcll(masked);
        if (nan) {  // lane i takes NaN number nans + j from the j-th lane that has one
          const int j = lane - nans;
          u64 rest = nan;
          for (int k = 0; k < j && rest; ++k) rest &= rest - 1;
          if (j >= 0 && rest) nan_col = c + __builtin_ctzll(rest);
          nans += __popcll(nan);
        }
      }
      // NaN is last; it keeps the key of none with its column
      if (at + lane < p.K && lane < nans) list->best[at + lane] = unsigned(~nan_col);
      wave_fence();
    }
    if (lane < p.K) {
      const u64 c = list->best[lane];
      const float v = c >> 32 ? value_of(c) : __builtin_nanf("");
      p.top[row * p.K + lane] = column_of(c);
      p.top_logp[row * p.K + lane] = gone ? kNegInf : fmaf(v - o, p.scale, -logs);
    }
  }
}

// One part of a row per workgroup, PER columns per thread at a time; with one part, its results.
template <int THREADS, int PER, bool BF16, bool ENT, bool TOP>
__global__ __launch_bounds__(THREADS) void logprob_kernel(LogprobParams p, int parts,
                                                          int columns) {
  constexpr int EV = Piece<BF16>::EV, NV = PER / EV, CH = THREADS * PER;
  __shared__ float red[3 * (THREADS / 64)];
  // (a piece of the second reading fits too)
  __shared__ List<THREADS / 64, TOP ? 512 : 1> list;
  __shared__ float maxima[TOP ? THREADS : 1];
  const long row = blockIdx.x / parts;
  const int part = int(blockIdx.x - row * parts), begin = part * columns;
  const int end = min(begin + columns, p.V);
  const char* const x = static_cast<const char*>(p.x) + row * p.xs * (BF16 ? 2 : 4);
  const float c2 = p.scale * kLog2e;
  Sums a{kNegInf, 0.f, 0.f};
  float bound = kNegInf;
  int count = 0;  // of the wave's candidates
  Piece<BF16> next[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
    next[k].load(x, begin + (k * THREADS + int(threadIdx.x)) * EV, end);
  // n pieces of this thread from column c on, THREADS * EV columns apart
  auto sums = [&](auto n, const float* v, float* mp) {
    float mc = kNegInf;  // (mp: the largest of each piece)
#pragma unroll
    for (int k = 0; k < n(); ++k) {
      mp[k] = v[k * EV];
#pragma unroll
      for (int i = 1; i < EV; ++i) mp[k] = fmaxf(mp[k], v[k * EV + i]);
      mc = fmaxf(mc, mp[k]);
    }
    if (mc > a.m) rebase<ENT>(a, mc, c2);
    const float o = origin(a.m);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < n() * EV; ++i) {
      const float d = (v[i] - o) * c2, e = __builtin_amdgcn_exp2f(d);
      s += e;
      if constexpr (ENT) a.t = fmaf(e, fmaxf(d, kFar), a.t);
    }
    a.s += s;
  };
  auto candidates = [&](auto n, const float* v, const float* mp, int c) {
#pragma unroll
    for (int k = 0; k < n(); ++k)
      if (__ballot(mp[k] >= bound))
        append<EV>(&list, count, v + k * EV, bound, [&](int i) {
          return c + (k * THREADS + int(threadIdx.x)) * EV + i;
        });
  };
  int c = begin;
  do {
    float v[PER], mp[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) next[k].floats(v + k * EV);
    if (c + CH < end)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        next[k].load(x, c + CH + (k * THREADS + int(threadIdx.x)) * EV, end);
    sums(std::integral_constant<int, NV>{}, v, mp);
    if constexpr (TOP) {
      // The threads' largest so far, after 1, 2, 4, ... chunks.  Only the first time do all have to be
      // there: what another wave has not written yet is its largest of before.
      const int done = (c - begin) / CH + 1;
      if ((done & (done - 1)) == 0) bound = bound_of<THREADS>(a.m, p.K, maxima, done == 1);
      candidates(std::integral_constant<int, NV>{}, v, mp, c);
    }
    c += CH;
  } while (c + CH <= end);
  // the rest of the columns, which less than a chunk holds, by pieces: those that a wave has
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int at = c + k * THREADS * EV;
    if (at + wave * 64 * EV >= end) break;
    float v[EV], mp[1];
    next[k].floats(v);
    sums(std::integral_constant<int, 1>{}, v, mp);
    if constexpr (TOP) candidates(std::integral_constant<int, 1>{}, v, mp, at);
  }
  join<THREADS, ENT>(a, c2, red);
  int m = 0;
  if constexpr (TOP) {
    if ((threadIdx.x & 63) == 0) list.count[threadIdx.x >> 6] = count;
    __syncthreads();
    if (list.short_of_room())
      m = reread<THREADS, BF16>(x, begin, end, p.K, &list, maxima);
    else if (threadIdx.x < 64)
      m = take_best(&list, p.K);
  }
  if (parts == 1) {
    finish<THREADS, BF16, ENT, TOP>(p, row, a, &list, m);
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
        int(threadIdx.x) < m ? list.best[threadIdx.x] : 0ull;
}

// Joins the parts of a row.
constexpr int kJoinThreads = 256;
template <bool BF16, bool ENT, bool TOP>
__global__ __launch_bounds__(kJoinThreads) void logprob_join_kernel(LogprobParams p, int parts) {
  __shared__ float red[3 * (kJoinThreads / 64)];
  __shared__ List<1, TOP ? kLogprobParts * kMaxTop : 1> list;
  const long row = blockIdx.x;
  const int words = 4 + 2 * p.K;
  const float* const in = p.parts + row * parts * words;
  Sums a{kNegInf, 0.f, 0.f};
  if (int(threadIdx.x) < parts) {
    const float* const q = in + long(threadIdx.x) * words;
    a = Sums{q[0], q[1], q[2]};
  }
  int m = 0;
  if constexpr (TOP) {
    // Each part's best are in order: with q = ceil(K / parts) of every part there are K, so the
    // least of the parts' q-th is a bound.
    if (threadIdx.x == 0) list.count[0] = 0;
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
      if (y >= bound) list.c[0][atomicAdd(&list.count[0], 1)] = y;
    }
    __syncthreads();
    if (threadIdx.x < 64) m = take_best(&list, p.K);
  }
  join<kJoinThreads, ENT>(a, p.scale * kLog2e, red);
  finish<kJoinThreads, BF16, ENT, TOP>(p, row, a, &list, m);
}

// ---- gradient ----------------------------------------------------------------------------
// With l = ln p and a = dlse - sum of the given tokens' gradients, dx = c p (a - dH (l + H));
// then the given tokens that stand in the workgroup's columns are written again with their own
// gradients added (equal ones all, so that it does not matter which thread writes last).
// A workgroup has kBackColumns columns of a row, a wave up to a quarter of that, every element by
// itself with l = c x - lse.  As one number for c m + ln s, lse is off by half its last place, 4e-6
// up to kNear: less than the sum is.  Beyond (all logits far from 0, a row of a finite mask's
// value, c m past the largest number) ln s is lost in it, and one workgroup has the whole row (which
// may be written over the logits): it forms m and ln s again and takes l = c (x - m) - ln s.
// That is three reads, two from the cache: 8192 x 32768 logits near 4096 592 us in place of 192,
// 300 x 50001 in fp32 72 in place of 20.  (A function of its own for it, not inlined, leaves the other
// rows their registers: inlined, 300 x 50001 with 64 given tokens 25.6 us, so 24.)
constexpr int kBackColumns = 4096;
constexpr float kNear = 128.f;

// m and ln s of a row, in every thread; m = -inf where nothing is left of it.
template <int THREADS, bool BF16>
__device__ inline void row_sums(const char* x, int V, float c2, float& m, float& logs) {
  constexpr int EV = Piece<BF16>::EV, W = THREADS / 64;
  __shared__ float most[W];
  __shared__ double sums[W];
  Piece<BF16> in;
  float v[EV];
  m = kNegInf;
  for (int c = int(threadIdx.x) * EV; c < V; c += THREADS * EV) {
    in.load(x, c, V);
    in.floats(v);
#pragma unroll
    for (int i = 0; i < EV; ++i) m = fmaxf(m, v[i]);
  }
  m = group_max<64>(m);
  if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) m = fmaxf(m, most[i]);
  const float o = origin(m);
  double s = 0.0;  // (one thread's chain may be long)
  for (int c = int(threadIdx.x) * EV; c < V; c += THREADS * EV) {
    in.load(x, c, V);
    in.floats(v);
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < EV; ++i) t += __builtin_amdgcn_exp2f((v[i] - o) * c2);
    s += t;
  }
#pragma unroll
  for (int i = 1; i < 64; i *= 2) s += __shfl_xor(s, i);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int i = 0; i < W; ++i) s += sums[i];
  logs = kLn2 * __builtin_amdgcn_logf(float(s));
}

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
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_any*>(row + long(c) * (BF16 ? 2 : 4)));
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

// What a row's gradients are formed from: dx = scale p (a - dh (l + h)).
struct Slopes {
  float a, dh, h;
};
template <bool ENT>
__device__ inline float slope(const Slopes& d, float l) {
  float f = d.a;
  if constexpr (ENT) f = fmaf(-d.dh, fmaxf(l, kFar) + d.h, d.a);
  return __builtin_amdgcn_exp2f(l * kLog2e) * f;
}
template <bool BF16>
__device__ inline void store_one(char* row, int c, float y) {
  if constexpr (BF16)
    reinterpret_cast<uint16_t*>(row)[c] = uint16_t(pack_bf16x2(y, y));
  else
    reinterpret_cast<float*>(row)[c] = y;
}

// A whole row from its own sums; the given tokens and their gradients are in LDS.
template <int THREADS, bool BF16, bool ENT>
__device__ __noinline__ void far_row(const char* x, char* dx, int V, float scale, Slopes d,
                                     const int* token, const float* grad, int G) {
  constexpr int EV = Piece<BF16>::EV, MINE = kMaxGiven / THREADS;
  float m, ls, at_mine[MINE];
  row_sums<THREADS, BF16>(x, V, scale * kLog2e, m, ls);
  const bool gone = m == kNegInf;
  m = origin(m);
  auto value = [&](float y) { return gone ? 0.f : slope<ENT>(d, fmaf(y - m, scale, -ls)); };
#pragma unroll
  for (int i = 0; i < MINE; ++i) {
    const int g = i * THREADS + int(threadIdx.x), v = g < G ? token[g] : -1;
    if (v >= 0 && v < V) at_mine[i] = load1<BF16>(x, v);
  }
  __syncthreads();  // (read before anything is stored: dx may be x)
#pragma unroll 1
  for (int c = int(threadIdx.x) * EV; c < V; c += THREADS * EV) {
    Piece<BF16> in;
    float v[EV];
    in.load(x, c, V);
    in.floats(v);
#pragma unroll
    for (int i = 0; i < EV; ++i) v[i] = scale * value(v[i]);
    store_any<BF16>(dx, c, V, v);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < MINE; ++i) {
    const int g = i * THREADS + int(threadIdx.x), t = g < G ? token[g] : -1;
    if (t < 0 || t >= V) continue;
    float s = 0.f;
    for (int j = 0; j < G; ++j) s += token[j] == t ? grad[j] : 0.f;
    store_one<BF16>(dx, t, gone ? 0.f : scale * (value(at_mine[i]) + s));
  }
}

template <int THREADS, bool BF16, bool ENT>
__global__ __launch_bounds__(THREADS) void logprob_backward_kernel(LogprobParams p, int blocks) {
  constexpr int EV = Piece<BF16>::EV, NV = kBackColumns / (256 * EV), MINE = kMaxGiven / THREADS;
  constexpr int size = BF16 ? 2 : 4;
  __shared__ int token[kMaxGiven];
  __shared__ float grad[kMaxGiven];
  const long row = blockIdx.x / blocks;
  const int begin = int(blockIdx.x - row * blocks) * (THREADS * EV * NV);
  const int end = min(begin + THREADS * EV * NV, p.V);
  const char* const x = static_cast<const char*>(p.x) + row * p.xs * size;
  char* const dx = static_cast<char*>(p.dx) + row * p.V * size;
  Piece<BF16> in[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k)
    in[k].load(x, begin + (k * THREADS + int(threadIdx.x)) * EV, end);
  const float lse = p.lse_in[row];
  Slopes d{p.dlse ? p.dlse[row] : 0.f, ENT ? p.dentropy[row] : 0.f, ENT ? p.entropy_in[row] : 0.f};
  // the given tokens' gradients; a token past the vocabulary makes the row NaN
  int mine[MINE];
  float at_mine[MINE];
#pragma unroll
  for (int i = 0; i < MINE; ++i) {
    const int g = i * THREADS + int(threadIdx.x);
    mine[i] = -1;
    if (g >= p.G) continue;
    const int v = p.given[row * p.G + g];
    token[g] = v;
    grad[g] = v < 0 ? 0.f : v < p.V ? p.dlogp[row * p.G + g] : __builtin_nanf("");
    if (v >= begin && v < end) {  // (read before anything is stored: dx may be x)
      mine[i] = v;
      at_mine[i] = load1<BF16>(x, v);
    }
  }
  if (p.G > 0) {
    __syncthreads();
    float s = 0.f;
    for (int g = 0; g < p.G; ++g) s += grad[g];
    d.a -= s;
  }
  // (with scale <= 1 no row of numbers has an lse of -inf)
  const bool gone = lse == kNegInf && p.scale <= 1.f;
  if (fabsf(lse) > kNear && !gone) {
    // (another one from row to row: neighbouring workgroups are on different XCDs)
    if (begin == int(row % blocks) * (THREADS * EV * NV))
      far_row<THREADS, BF16, ENT>(x, dx, p.V, p.scale, d, token, grad, p.G);
    return;
  }
  auto value = [&](float y) { return gone ? 0.f : slope<ENT>(d, fmaf(y, p.scale, -lse)); };
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = begin + (k * THREADS + int(threadIdx.x)) * EV;
    if (c >= end) break;
    float v[EV];
    in[k].floats(v);
#pragma unroll
    for (int i = 0; i < EV; ++i) v[i] = p.scale * value(v[i]);
    store_any<BF16>(dx, c, end, v);
  }
  if (p.G == 0) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < MINE; ++i) {
    if (mine[i] < 0) continue;
    float s = 0.f;
    for (int g = 0; g < p.G; ++g) s += token[g] == mine[i] ? grad[g] : 0.f;
    store_one<BF16>(dx, mine[i], gone ? 0.f : p.scale * (value(at_mine[i]) + s));
  }
}

template <bool BF16, bool ENT, bool TOP>
hipError_t run(const LogprobParams& p, const LogprobPlan& a, hipStream_t st) {
  const unsigned blocks = unsigned(p.R * a.parts);
#define ONELA_ROWS(T, PER) \
  logprob_kernel<T, PER, BF16, ENT, TOP><<<blocks, T, 0, st>>>(p, a.parts, a.columns)
  // (8192 rows of 500 with the 5 best 10.6 us, by the last of the first three 14.1)
  if (a.threads == 64 && p.V <= 64 * 8)
    ONELA_ROWS(64, 8);
  else if (a.threads == 64 && p.V <= 64 * 16)
    ONELA_ROWS(64, 16);
  else if (a.threads == 64)
    ONELA_ROWS(64, 32);
  else if (a.threads == 128)
    ONELA_ROWS(128, 32);
  else
    ONELA_ROWS(256, 32);
#undef ONELA_ROWS
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
  const bool wave = p.V <= kBackColumns / 4;
  const int blocks = wave ? 1 : (p.V + kBackColumns - 1) / kBackColumns;
  const unsigned grid = unsigned(p.R * blocks);
#define ONELA_BACK(B, E)                                                          \
  if (wave)                                                                       \
    logprob_backward_kernel<64, B, E><<<grid, 64, 0, st>>>(p, blocks);            \
  else                                                                            \
    logprob_backward_kernel<256, B, E><<<grid, 256, 0, st>>>(p, blocks)
  if (bf16 && p.dentropy) {
    ONELA_BACK(true, true);
  } else if (bf16) {
    ONELA_BACK(true, false);
  } else if (p.dentropy) {
    ONELA_BACK(false, true);
  } else {
    ONELA_BACK(false, false);
  }
#undef ONELA_BACK
  return hipGetLastError();
}

}  // namespace onela
