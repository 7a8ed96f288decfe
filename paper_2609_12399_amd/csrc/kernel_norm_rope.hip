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
// takes both.  Bound: HBM.
#include "device_common.h"
#include "internal.h"

namespace onela {
namespace {

constexpr int kNormThreads = 256;

template <bool BF16>
__device__ inline void get8(const void* base, long i, float (&x)[8]) {
  if constexpr (BF16) {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + i);
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = bf16_lo_to_float(w[j]);
      x[2 * j + 1] = bf16_hi_to_float(w[j]);
    }
  } else {
    const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + i);
    const f32x4 a = q[0], b = q[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = a[j];
      x[4 + j] = b[j];
    }
  }
}

template <bool BF16>
__device__ inline void put8(void* base, long i, const float (&x)[8]) {
  if constexpr (BF16) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + i) =
        make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                   pack_bf16x2(x[6], x[7]));
  } else {
    f32x4* const q = reinterpret_cast<f32x4*>(static_cast<float*>(base) + i);
    q[0] = f32x4{x[0], x[1], x[2], x[3]};
    q[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
}

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

template <int G, bool BF16>
__global__ __launch_bounds__(kNormThreads) void norm_rope_kernel(NormParams p) {
  const int sub = threadIdx.x % G, c0 = 8 * sub;
  const long r = long(blockIdx.x) * (kNormThreads / G) + threadIdx.x / G;
  if (r >= p.rows) return;  // (whole groups)
  const bool in = c0 < p.D;
  const Row row = row_of(p, r);
  float x[8] = {};
  if (in) get8<BF16>(row.x, row.at + c0, x);
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
  if (in) put8<BF16>(row.key ? p.ko : p.qo, row.out + c0, x);
}

// Rows are dealt out to the workgroups in a fixed order and each adds up its rows' weight
// gradients, so that the sums do not depend on timing.
template <int G, bool BF16>
__global__ __launch_bounds__(kNormThreads) void norm_rope_backward_kernel(NormParams p) {
  constexpr int RW = kNormThreads / G;
  __shared__ float acc[2][RW][8 * G];
  const int sub = threadIdx.x % G, g = threadIdx.x / G, c0 = 8 * sub;
  const bool in = c0 < p.D;
  float dw[2][8] = {};
  for (long r = long(blockIdx.x) * RW + g; r < p.rows; r += long(gridDim.x) * RW) {
    const Row row = row_of(p, r);
    float x[8] = {}, d[8] = {}, w[8];
    if (in) {
      get8<BF16>(row.x, row.at + c0, x);
      get8<BF16>(row.key ? p.dko : p.dqo, row.out + c0, d);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = row.w && in ? row.w[c0 + j] : 1.f;
    if (p.rot) {
      const float* cs = angle_of(p, r / (p.HQ + p.HK));
      if (cs) {
        turn<G>(d, cs, c0, p.rot, p.pairs, -1.f);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = __builtin_nanf("");
      }
    }
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s = fmaf(x[j], x[j], s);
      u = fmaf(x[j], w[j] * d[j], u);
    }
    s = group_sum<G>(s);
    u = group_sum<G>(u);
    const float rn = 1.f / sqrtf(s * p.inv_n + p.eps);
    const float f = u * p.inv_n * rn * rn;
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      o[j] = rn * (w[j] * d[j] - x[j] * f);
      const float t = d[j] * (x[j] * rn);
      dw[0][j] += row.key ? 0.f : t;
      dw[1][j] += row.key ? t : 0.f;
    }
    if (in) put8<BF16>(row.key ? p.dk : p.dq, row.out + c0, o);
  }
  if (!p.partial) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    acc[0][g][c0 + j] = dw[0][j];
    acc[1][g][c0 + j] = dw[1][j];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * p.D; e += kNormThreads) {
    const int which = e / p.D, c = e - which * p.D;
    float s = 0.f;
    for (int i = 0; i < RW; ++i) s += acc[which][i][c];
    p.partial[long(blockIdx.x) * (2 * p.D) + e] = s;
  }
}

// The workgroups' sums added up, one column per wave.
__global__ __launch_bounds__(64) void norm_weight_kernel(NormParams p, int parts) {
  const int e = blockIdx.x, which = e / p.D, c = e - which * p.D;
  float* const out = which ? p.dwk : p.dwq;
  if (!out) return;
  float s = 0.f;
  for (int i = threadIdx.x; i < parts; i += 64) s += p.partial[long(i) * (2 * p.D) + e];
  s = group_sum<64>(s);
  if (threadIdx.x == 0) out[c] = s;
}

template <int G, bool BF16>
hipError_t run(const NormParams& p, bool backward, hipStream_t st) {
  constexpr int RW = kNormThreads / G;
  const long groups = (p.rows + RW - 1) / RW;
  if (!backward) {
    norm_rope_kernel<G, BF16><<<unsigned(groups), kNormThreads, 0, st>>>(p);
    return hipGetLastError();
  }
  const unsigned blocks = unsigned(groups < kNormBlocks ? groups : kNormBlocks);
  if (blocks) {
    norm_rope_backward_kernel<G, BF16><<<blocks, kNormThreads, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.partial) norm_weight_kernel<<<unsigned(2 * p.D), 64, 0, st>>>(p, int(blocks));
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
