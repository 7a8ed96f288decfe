// Norms before and after a block with its gate and residual scale, and their gradients: from a
// block's output x to the next block's input y and the residual stream h, in one pass.
//
//   n = x r(x),  u = wa n act(g),  h = res + s cs u,  y = wb h r(h),  r(v) = (mean v^2 + eps)^-1/2
// Backward, with dh the gradient of h as an output:
//   dh += r(h) (wb dy - h r(h)^2 mean(wb dy h)),   dwb = sum dy h r(h),   dres = dh,
//   dcs = s sum dh u,   du = s cs dh,   dg = du wa n act'(g),   dn = du act(g),
//   dwa = sum dn n,   dx = r(x) (wa dn - x r(x)^2 mean(wa dn x)).
// All in fp32; h and y are rounded once, at their stores (y is formed from the unrounded h).
//
// A row is held by LANES lanes with NV times 8 columns each: a part of a wave, or a whole
// workgroup whose waves exchange their sums through LDS (two buffers in turn, so that one
// barrier per sum is enough).  Workgroups stay and walk over rows, with the weights in registers
// and the next row on its way while this one is worked on.  Bound: HBM.
#include "device_common.h"
#include "internal.h"

namespace onela {
namespace {

// Sum over the LANES lanes of a row, in every one of them; `turn` counts the calls.
template <int LANES>
__device__ inline float row_sum(float x, int& turn) {
  if constexpr (LANES <= 64) {
    return group_sum<LANES>(x);
  } else {
    constexpr int W = LANES / 64;
    __shared__ float part[2][W];
    x = group_sum<64>(x);
    float* const b = part[turn & 1];
    ++turn;
    if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = x;
    __syncthreads();
    x = b[0];
#pragma unroll
    for (int i = 1; i < W; ++i) x += b[i];
    return x;
  }
}

// Two sums at once.
template <int LANES>
__device__ inline void row_sum2(float& x, float& y, int& turn) {
  if constexpr (LANES <= 64) {
    x = group_sum<LANES>(x);
    y = group_sum<LANES>(y);
  } else {
    constexpr int W = LANES / 64;
    __shared__ float2 part[2][W];
    x = group_sum<64>(x);
    y = group_sum<64>(y);
    float2* const b = part[turn & 1];
    ++turn;
    if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = make_float2(x, y);
    __syncthreads();
    x = b[0].x;
    y = b[0].y;
#pragma unroll
    for (int i = 1; i < W; ++i) {
      x += b[i].x;
      y += b[i].y;
    }
  }
}

__device__ inline void vector8(const float* w, int c0, bool in, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = w && in ? w[c0 + j] : 1.f;
}

// Rows first, first + step, ... with their tokens and heads (divisions once).
struct Walk {
  long row, t, step, dt;
  int h, dh;
  __device__ Walk(long first, long by, int H) : row(first), step(by) {
    t = first / H;
    h = int(first - t * H);
    dt = by / H;
    dh = int(by - dt * H);
  }
  __device__ void next(int H) {
    row += step;
    t += dt;
    h += dh;
    if (h >= H) {
      h -= H;
      ++t;
    }
  }
};

// What a lane reads of a row.
template <int NV, bool BF16, bool RES_BF16>
struct RowIn {
  Raw8<BF16> x[NV], g[NV];
  Raw8<RES_BF16> r[NV];
  __device__ void load(const BlockNormParams& p, const Walk& w, const int (&c0)[NV]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (c0[v] >= p.D) continue;
      const long c = long(w.h) * p.D + c0[v];
      x[v].load(p.x, w.t * p.xs + c);
      if (p.gate) g[v].load(p.gate, w.t * p.gs + c);
      if (p.res) r[v].load(p.res, w.row * p.D + c0[v]);
    }
  }
};

__device__ inline float act(float g, bool silu) {
  const float s = sigmoid(g);
  return silu ? g * s : s;
}

template <int LANES, int NV, bool BF16, bool RES_BF16>
__global__ __launch_bounds__(LANES > 64 ? LANES : 256) void block_norm_kernel(BlockNormParams p) {
  constexpr int RW = LANES > 64 ? 1 : 256 / LANES;
  const int sub = threadIdx.x % LANES;
  const float inv_d = 1.f / float(p.D);
  int c0[NV], turn = 0;
  bool in[NV];
  float wa[NV][8], wb[NV][8], cs[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    c0[v] = 8 * (v * LANES + sub);
    in[v] = c0[v] < p.D;
    vector8(p.wa, c0[v], in[v], wa[v]);
    vector8(p.wb, c0[v], in[v], wb[v]);
    vector8(p.cs, c0[v], in[v], cs[v]);
#pragma unroll
    for (int j = 0; j < 8; ++j) cs[v][j] *= p.scale;
  }
  Walk ahead(long(blockIdx.x) * RW + threadIdx.x / LANES, long(gridDim.x) * RW, p.H);
  RowIn<NV, BF16, RES_BF16> cur, next;
  if (ahead.row < p.rows) cur.load(p, ahead, c0);
  for (long row = ahead.row; row < p.rows; row += ahead.step) {  // (whole rows of lanes)
    ahead.next(p.H);
    if (ahead.row < p.rows) next.load(p, ahead, c0);
    float h[NV][8];
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (in[v]) {
        cur.x[v].floats(h[v]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) h[v][j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(h[v][j], h[v][j], s);
    }
    float rn = 1.f;
    if (p.after) rn = 1.f / sqrtf(row_sum<LANES>(s, turn) * inv_d + p.eps);
    s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (!in[v]) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) h[v][j] *= rn * wa[v][j];
      if (p.gate) {
        float g[8];
        cur.g[v].floats(g);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[v][j] *= act(g[j], p.silu);
      }
      float r[8] = {};
      if (p.res) cur.r[v].floats(r);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[v][j] = fmaf(cs[v][j], h[v][j], r[j]);
        s = fmaf(h[v][j], h[v][j], s);
      }
      if (p.h) store8<RES_BF16>(p.h, row * p.D + c0[v], h[v]);
    }
    if (p.y) {
      float rh = 1.f;
      if (p.before) rh = 1.f / sqrtf(row_sum<LANES>(s, turn) * inv_d + p.eps);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if (!in[v]) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[v][j] *= rh * wb[v][j];
        store8<BF16>(p.y, row * p.D + c0[v], h[v]);
      }
    }
    cur = next;
  }
}

template <int NV, bool BF16, bool RES_BF16>
struct GradIn {
  Raw8<BF16> y[NV];
  Raw8<RES_BF16> h[NV];
  __device__ void load(const BlockNormParams& p, long row, const int (&c0)[NV]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (c0[v] >= p.D) continue;
      if (p.dy) y[v].load(p.dy, row * p.D + c0[v]);
      if (p.dh) h[v].load(p.dh, row * p.D + c0[v]);
    }
  }
};

// Every workgroup walks its rows in a fixed order and leaves the sums of the three weights'
// gradients over them.
template <int LANES, int NV, bool BF16, bool RES_BF16>
__global__ __launch_bounds__(LANES > 64 ? LANES : 256) void block_norm_backward_kernel(
    BlockNormParams p) {
  constexpr int RW = LANES > 64 ? 1 : 256 / LANES;
  __shared__ float acc[RW > 1 ? RW : 1][RW > 1 ? 8 * LANES * NV : 1];
  const int sub = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const float inv_d = 1.f / float(p.D);
  int c0[NV], turn = 0;
  bool in[NV];
  float wa[NV][8], wb[NV][8], cs[NV][8], da[NV][8] = {}, db[NV][8] = {}, dc[NV][8] = {};
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    c0[v] = 8 * (v * LANES + sub);
    in[v] = c0[v] < p.D;
    vector8(p.wa, c0[v], in[v], wa[v]);
    vector8(p.wb, c0[v], in[v], wb[v]);
    vector8(p.cs, c0[v], in[v], cs[v]);
  }
  Walk ahead(long(blockIdx.x) * RW + group, long(gridDim.x) * RW, p.H);
  RowIn<NV, BF16, RES_BF16> cur, next;
  GradIn<NV, BF16, RES_BF16> gcur, gnext;
  if (ahead.row < p.rows) {
    cur.load(p, ahead, c0);
    gcur.load(p, ahead.row, c0);
  }
  for (long row = ahead.row; row < p.rows; row += ahead.step) {
    ahead.next(p.H);
    if (ahead.row < p.rows) {
      next.load(p, ahead, c0);
      gnext.load(p, ahead.row, c0);
    }
    float x[NV][8], g[NV][8], h[NV][8], dy[NV][8], d[NV][8];
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[v][j] = g[v][j] = h[v][j] = dy[v][j] = d[v][j] = 0.f;
      if (!in[v]) continue;
      cur.x[v].floats(x[v]);
      if (p.gate) cur.g[v].floats(g[v]);
      if (p.res) cur.r[v].floats(h[v]);
      if (p.dy) gcur.y[v].floats(dy[v]);
      if (p.dh) gcur.h[v].floats(d[v]);
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(x[v][j], x[v][j], s);
    }
    float rx = 1.f;
    if (p.after) rx = 1.f / sqrtf(row_sum<LANES>(s, turn) * inv_d + p.eps);
    // h, and the two sums of its norm
    float hh = 0.f, hd = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float u = x[v][j] * rx * wa[v][j];
        if (p.gate) u *= act(g[v][j], p.silu);
        h[v][j] = fmaf(p.scale * cs[v][j], u, h[v][j]);
        hh = fmaf(h[v][j], h[v][j], hh);
        hd = fmaf(wb[v][j] * dy[v][j], h[v][j], hd);
      }
    if (p.before) {
      row_sum2<LANES>(hh, hd, turn);
      const float rh = 1.f / sqrtf(hh * inv_d + p.eps), f = hd * inv_d * rh * rh;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          db[v][j] = fmaf(dy[v][j], h[v][j] * rh, db[v][j]);
          d[v][j] = fmaf(rh, wb[v][j] * dy[v][j] - h[v][j] * f, d[v][j]);
        }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) d[v][j] += dy[v][j];
    }
    s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (!in[v]) continue;
      if (p.dres) store8<RES_BF16>(p.dres, row * p.D + c0[v], d[v]);
      float dg[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = x[v][j] * rx, un = n * wa[v][j];
        float du = p.scale * cs[v][j] * d[v][j], a = 1.f;
        if (p.gate) {
          const float sg = sigmoid(g[v][j]);
          a = p.silu ? g[v][j] * sg : sg;
          const float slope = p.silu ? sg * fmaf(g[v][j], 1.f - sg, 1.f) : sg * (1.f - sg);
          dg[j] = du * un * slope;
        }
        dc[v][j] = fmaf(p.scale * d[v][j], un * a, dc[v][j]);
        du *= a;
        da[v][j] = fmaf(du, n, da[v][j]);
        d[v][j] = du * wa[v][j];
        s = fmaf(d[v][j], x[v][j], s);
      }
      if (p.gate && p.dgate) store8<BF16>(p.dgate, row * p.D + c0[v], dg);
    }
    float f = 0.f;
    if (p.after) f = row_sum<LANES>(s, turn) * inv_d * rx * rx;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (!in[v]) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) d[v][j] = rx * (d[v][j] - x[v][j] * f);
      store8<BF16>(p.dx, row * p.D + c0[v], d[v]);
    }
    cur = next;
    gcur = gnext;
  }
  if (!p.partial) return;
  float* const out = p.partial + long(blockIdx.x) * 3 * p.D;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const auto& sum = k == 0 ? da : k == 1 ? db : dc;
    if constexpr (RW == 1) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (in[v]) store8<false>(out, long(k) * p.D + c0[v], sum[v]);
    } else {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[group][8 * (v * LANES + sub) + j] = sum[v][j];
      __syncthreads();
      for (int c = threadIdx.x; c < p.D; c += 256) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < RW; ++i) t += acc[i][c];
        out[long(k) * p.D + c] = t;
      }
    }
  }
}

// The workgroups' sums added up: 16 columns per workgroup, 64 rows of partial sums at a time.
__global__ __launch_bounds__(1024) void block_norm_weight_kernel(BlockNormParams p, int blocks) {
  __shared__ float acc[64][17];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int cols = (p.D + 15) / 16, k = blockIdx.x / cols, col = (blockIdx.x - k * cols) * 16 + c;
  float* const out = k == 0 ? p.dwa : k == 1 ? p.dwb : p.dcs;
  if (!out) return;
  float s = 0.f;
  if (col < p.D)
#pragma unroll 4
    for (int i = g; i < blocks; i += 64) s += p.partial[(long(i) * 3 + k) * p.D + col];
  acc[g][c] = s;
  __syncthreads();
  if (g == 0 && col < p.D) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) s += acc[i][c];
    out[col] = s;
  }
}

template <int LANES, int NV, bool BF16, bool RES_BF16>
hipError_t run(const BlockNormParams& p, bool backward, int cus, hipStream_t st) {
  constexpr int RW = LANES > 64 ? 1 : 256 / LANES, threads = LANES > 64 ? LANES : 256;
  const long need = (p.rows + RW - 1) / RW;
  if (!backward) {
    // as many workgroups as the compute units hold
    const long most = long(cus > 0 ? cus : 256) * (2048 / threads);
    block_norm_kernel<LANES, NV, BF16, RES_BF16>
        <<<unsigned(need < most ? need : most), threads, 0, st>>>(p);
    return hipGetLastError();
  }
  const long blocks = need < kBlockNormBlocks ? need : kBlockNormBlocks;
  if (blocks > 0) {
    block_norm_backward_kernel<LANES, NV, BF16, RES_BF16><<<unsigned(blocks), threads, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.partial)
    block_norm_weight_kernel<<<unsigned(3 * ((p.D + 15) / 16)), 1024, 0, st>>>(p, int(blocks));
  return hipGetLastError();
}

template <bool BF16, bool RES_BF16>
hipError_t by_width(const BlockNormParams& p, bool backward, int cus, hipStream_t st) {
#define ONELA_NORM(L, NV) return run<L, NV, BF16, RES_BF16>(p, backward, cus, st)
  if (p.D <= 32) ONELA_NORM(4, 1);
  if (p.D <= 64) ONELA_NORM(8, 1);
  if (p.D <= 128) ONELA_NORM(16, 1);
  if (p.D <= 256) ONELA_NORM(32, 1);
  if (p.D <= 512) ONELA_NORM(64, 1);
  if (p.D <= 1024) ONELA_NORM(128, 1);
  if (p.D <= 2048) ONELA_NORM(256, 1);
  if (p.D <= 4096) ONELA_NORM(512, 1);
  if (p.D <= 8192) ONELA_NORM(1024, 1);
  ONELA_NORM(1024, 2);
#undef ONELA_NORM
}

hipError_t by_type(const BlockNormParams& p, bool bf16, bool res_bf16, bool backward, int cus,
                   hipStream_t st) {
  if (bf16)
    return res_bf16 ? by_width<true, true>(p, backward, cus, st)
                    : by_width<true, false>(p, backward, cus, st);
  return res_bf16 ? by_width<false, true>(p, backward, cus, st)
                  : by_width<false, false>(p, backward, cus, st);
}

}  // namespace

hipError_t launch_block_norm(const BlockNormParams& p, bool bf16, bool res_bf16, int cus,
                             hipStream_t st) {
  return p.rows == 0 ? hipSuccess : by_type(p, bf16, res_bf16, false, cus, st);
}

hipError_t launch_block_norm_backward(const BlockNormParams& p, bool bf16, bool res_bf16, int cus,
                                      hipStream_t st) {
  return by_type(p, bf16, res_bf16, true, cus, st);
}

}  // namespace onela
