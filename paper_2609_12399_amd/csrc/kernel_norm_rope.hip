// Norms of queries and keys per head with the position rotation in the same pass, and
// their gradients.
//
// A row x of D columns (one token's head): y = w x r, r = (sum x^2 / n + eps)^-1/2 with
// n = D (RMS) or 1 (L2); then the pairs (y_i, y_{i + rot / 2}), or (y_2i, y_{2i + 1})
// interleaved, i < rot / 2, are turned by the angle of the token's position, whose
// cosine and sine come from a table.  Backward: dy is dz turned back,
//   dw = sum over rows of dy x r,   dx = r (w dy - x r^2 (w dy . x) / n).
// All in fp32, rounded once on the store.
//
// A row is held by G lanes of 8 columns (G the power of two from D / 8 up, the lanes past
// D idle); the partner columns of a half-turn pair are another lane's 8 and
// come by a lane exchange.  Queries and keys are one list of rows, so that one launch
// takes both.  Bound: HBM; 16384 tokens x 32 heads of 128 in bf16 take 40 us, 6.7 TB/s (part of
// it from the memory-side cache), 80 rows 4.2 us of latency.
#include "device_common.h"
#include "internal.h"

namespace onela {
namespace {

constexpr int kNormThreads = 256;
// A grid has fewer than 2^32 threads: past that the runtime starts what is left of the number
// in 32 bits, without an error.
constexpr long kNormLaunch = (1l << 32) / kNormThreads - 1;

// Turns this lane's 8 columns (from c0) of a row by the table's row cs (SIGN -1:
// back).  Every lane of the row's group takes part.
template <int G>
__device__ inline void turn(float (&y)[8], const float* cs, int c0, int rot, bool pairs,
                            float sign) {
  const int half = rot / 2;
  if (pairs) {
    if (c0 >= rot) return;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float c = cs[(c0 + j) / 2], s = sign * cs[half + (c0 + j) / 2];
      const float a = y[j], b = y[j + 1];
      y[j] = a * c - b * s;
      y[j + 1] = fmaf(b, c, a * s);
    }
    return;
  }
  // half is a multiple of 8: the partner columns are those of the lane half / 8 away
  const bool upper = c0 >= half;
  const int lane = threadIdx.x & 63;
  const int from = c0 < rot ? (upper ? lane - half / 8 : lane + half / 8) : lane;
  float o[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = __shfl(y[j], from);
  if (c0 >= rot) return;
  const int i0 = upper ? c0 - half : c0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float c = cs[i0 + j], s = sign * cs[half + i0 + j];
    y[j] = fmaf(y[j], c, upper ? o[j] * s : -(o[j] * s));
  }
}

struct Row {
  const void* x;
  long at, out;  // element offsets of the row in x and in the dense output
  const float* w;
  bool key;
};
__device__ inline Row row_of(const NormParams& p, long r) {
  const int H = p.HQ + p.HK;
  const long t = r / H;
  const int h = int(r - t * H);
  if (h < p.HQ) return {p.q, t * p.qs + long(h) * p.D, (t * p.HQ + h) * p.D, p.wq, false};
  return {p.k, t * p.ks + long(h - p.HQ) * p.D, (t * p.HK + (h - p.HQ)) * p.D, p.wk, true};
}

// The table's row of token t; null where the position is outside the table.
__device__ inline const float* angle_of(const NormParams& p, long t) {
  const int pos = p.positions ? p.positions[t] : int(t);
  return pos >= 0 && pos < p.table ? p.cos_sin + long(pos) * p.rot : nullptr;
}

// Rows from `first` on: one launch takes kNormLaunch workgroups at most.
template <int G, bool BF16>
__global__ __launch_bounds__(kNormThreads) void norm_rope_kernel(NormParams p, long first) {
  const int sub = threadIdx.x % G, c0 = 8 * sub;
  const long r = first + long(blockIdx.x) * (kNormThreads / G) + threadIdx.x / G;
  if (r >= p.rows) return;  // (whole groups)
  const bool in = c0 < p.D;
  const Row row = row_of(p, r);
  float x[8] = {};
  if (in) load8<BF16>(row.x, row.at + c0, x);
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) s = fmaf(x[j], x[j], s);
  s = group_sum<G>(s);
  const float rn = 1.f / sqrtf(s * p.inv_n + p.eps);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = x[j] * rn * (row.w && in ? row.w[c0 + j] : 1.f);
  if (p.rot) {
    const float* cs = angle_of(p, r / (p.HQ + p.HK));
    if (cs) {
      turn<G>(x, cs, c0, p.rot, p.pairs, 1.f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __builtin_nanf("");
    }
  }
  if (in) store8<BF16>(row.key ? p.ko : p.qo, row.out + c0, x);
}

// The first workgroups take the queries' rows, the others the keys', in proportion; each
// walks its rows in a fixed order and adds up their weight gradients, so that the sums
// do not depend on timing.  kRows rows per lane group are in flight at once: with one,
// 8191 tokens x 32 heads of 128 took 81 us, with two 47 (4.4 TB/s).
constexpr int kRows = 2;

template <int G, bool BF16>
__global__ __launch_bounds__(kNormThreads) void norm_rope_backward_kernel(NormParams p,
                                                                         int q_blocks) {
  constexpr int RW = kNormThreads / G;
  __shared__ float acc[RW][8 * G];
  const int sub = threadIdx.x % G, g = threadIdx.x / G, c0 = 8 * sub;
  const bool in = c0 < p.D, key = int(blockIdx.x) >= q_blocks;
  const int H = key ? p.HK : p.HQ;
  const int block = key ? blockIdx.x - q_blocks : blockIdx.x;
  const int blocks = key ? gridDim.x - q_blocks : q_blocks;
  const void* const xs = key ? p.k : p.q;
  const void* const ds = key ? p.dko : p.dqo;
  void* const os = key ? p.dk : p.dq;
  const float* const ws = key ? p.wk : p.wq;
  const long stride = key ? p.ks : p.qs, rows = p.rows / (p.HQ + p.HK) * H;
  float w[8], dw[8] = {};
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = ws && in ? ws[c0 + j] : 1.f;
  for (long r0 = long(block) * RW + g; r0 < rows; r0 += long(blocks) * RW * kRows) {
    float x[kRows][8] = {}, d[kRows][8] = {};
    long t[kRows];
    bool here[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const long r = r0 + long(blocks) * RW * i;
      here[i] = r < rows;  // (whole groups)
      t[i] = here[i] ? r / H : 0;
      if (here[i] && in) {
        load8<BF16>(xs, t[i] * stride + (r - t[i] * H) * p.D + c0, x[i]);
        load8<BF16>(ds, r * p.D + c0, d[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (!here[i]) break;
      if (p.rot) {
        const float* cs = angle_of(p, t[i]);
        if (cs) {
          turn<G>(d[i], cs, c0, p.rot, p.pairs, -1.f);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) d[i][j] = __builtin_nanf("");
        }
      }
      float s = 0.f, u = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s = fmaf(x[i][j], x[i][j], s);
        u = fmaf(x[i][j], w[j] * d[i][j], u);
      }
      s = group_sum<G>(s);
      u = group_sum<G>(u);
      const float rn = 1.f / sqrtf(s * p.inv_n + p.eps);
      const float f = u * p.inv_n * rn * rn;
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = rn * (w[j] * d[i][j] - x[i][j] * f);
        dw[j] = fmaf(d[i][j], x[i][j] * rn, dw[j]);
      }
      if (in) store8<BF16>(os, (r0 + long(blocks) * RW * i) * p.D + c0, o);
    }
  }
  if (!p.partial) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[g][c0 + j] = dw[j];
  __syncthreads();
  for (int c = threadIdx.x; c < p.D; c += kNormThreads) {
    float s = 0.f;
    for (int i = 0; i < RW; ++i) s += acc[i][c];
    p.partial[long(blockIdx.x) * p.D + c] = s;
  }
}

// The workgroups' sums added up: 16 columns of one weight per workgroup, 64 rows of
// partial sums at a time.
__global__ __launch_bounds__(1024) void norm_weight_kernel(NormParams p, int q_blocks, int blocks) {
  __shared__ float acc[64][17];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int cols = (p.D + 15) / 16, col = int(blockIdx.x) % cols * 16 + c;
  const bool key = int(blockIdx.x) >= cols;
  float* const out = key ? p.dwk : p.dwq;
  if (!out) return;
  const int end = key ? blocks : q_blocks;
  float s = 0.f;
  if (col < p.D)
#pragma unroll 4
    for (int i = (key ? q_blocks : 0) + g; i < end; i += 64) s += p.partial[long(i) * p.D + col];
  acc[g][c] = s;
  __syncthreads();
  if (g == 0 && col < p.D) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) s += acc[i][c];
    out[col] = s;
  }
}

template <int G, bool BF16>
hipError_t run(const NormParams& p, bool backward, hipStream_t st) {
  constexpr int RW = kNormThreads / G;
  if (!backward) {
    const long groups = (p.rows + RW - 1) / RW;
    hipError_t e = hipSuccess;
    for (long g = 0; g < groups && e == hipSuccess; g += kNormLaunch) {
      const long n = groups - g < kNormLaunch ? groups - g : kNormLaunch;
      norm_rope_kernel<G, BF16><<<unsigned(n), kNormThreads, 0, st>>>(p, g * RW);
      e = hipGetLastError();
    }
    return e;
  }
  // workgroups for the queries' and the keys' rows, kRows rows per group and turn
  const long T = p.rows / (p.HQ + p.HK), per = RW * kRows;
  const long need_q = (T * p.HQ + per - 1) / per, need_k = (T * p.HK + per - 1) / per;
  long bq = need_q, bk = need_k;
  if (bq + bk > kNormBlocks) {
    bk = need_k * kNormBlocks / (need_q + need_k);
    if (bk < 1 && need_k > 0) bk = 1;
    bq = kNormBlocks - bk;
  }
  if (bq + bk > 0) {
    norm_rope_backward_kernel<G, BF16><<<unsigned(bq + bk), kNormThreads, 0, st>>>(p, int(bq));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.partial)
    norm_weight_kernel<<<unsigned(2 * ((p.D + 15) / 16)), 1024, 0, st>>>(p, int(bq), int(bq + bk));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rope(const NormParams& p, bool bf16, bool backward, hipStream_t st) {
  if (!backward && p.rows == 0) return hipSuccess;
#define ONELA_NORM(G) return bf16 ? run<G, true>(p, backward, st) : run<G, false>(p, backward, st)
  if (p.D <= 8) ONELA_NORM(1);
  if (p.D <= 16) ONELA_NORM(2);
  if (p.D <= 32) ONELA_NORM(4);
  if (p.D <= 64) ONELA_NORM(8);
  if (p.D <= 128) ONELA_NORM(16);
  if (p.D <= 256) ONELA_NORM(32);
  ONELA_NORM(64);
#undef ONELA_NORM
}

}  // namespace onela
