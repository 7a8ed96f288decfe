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
// A row is held by LANES lanes with 8 columns each: a part of a wave, or a whole workgroup whose
// waves exchange their sums through LDS (two buffers in turn, so that one barrier per sum is
// enough).  Workgroups stay and walk over rows, with the weights in registers and the next row on
// its way while this one is worked on.  Bound: HBM.  16384 rows of 2048 with an fp32 residual
// stream 83 us (403 MB, 4.9 TB/s), 262144 gated heads of 128 38.5 us (201 MB, 5.2 TB/s); backward,
// 8191 rows of 2048 with everything, 51 us (269 MB, 5.2 TB/s) and 6 for the second launch, which
// sums the workgroups' weight gradients.
#include "device_common.h"
#include "internal.h"

namespace onela {
namespace {

constexpr int E = 8;  // columns of a lane

// Sum over the wave, in every lane: within rows of 16 lanes as group_sum, then row 0 to 1 and 2 to
// 3, then lane 31 to the upper half (no exchange through LDS).
__device__ inline float wave_sum(float x) {
  x = group_sum<16>(x);
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x142,
                                                             0xa, 0xf, false));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x143,
                                                             0xc, 0xf, false));
  return __builtin_bit_cast(float,
                            __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// Sums over the LANES lanes of a row, in every one of them; `turn` counts the calls.
template <int LANES, int N>
__device__ inline void row_sums(float (&x)[N], int& turn) {
  if constexpr (LANES < 64) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = group_sum<LANES>(x[k]);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = wave_sum(x[k]);
  }
  if constexpr (LANES > 64) {
    constexpr int W = LANES / 64;
    __shared__ float part[2][N][W];
    float(*const b)[W] = part[turn & 1];
    ++turn;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) b[k][threadIdx.x >> 6] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      x[k] = b[k][0];
#pragma unroll
      for (int i = 1; i < W; ++i) x[k] += b[k][i];
    }
  }
}
template <int LANES>
__device__ inline float row_sum(float x, int& turn) {
  float v[1] = {x};
  row_sums<LANES>(v, turn);
  return v[0];
}

__device__ inline void vector_of(const float* w, int c0, bool in, float (&x)[E]) {
#pragma unroll
  for (int j = 0; j < E; ++j) x[j] = w && in ? w[c0 + j] : 1.f;
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
template <bool BF16, bool RES_BF16>
struct RowIn {
  RawN<BF16, E> x, g;
  RawN<RES_BF16, E> r;
  __device__ void load(const BlockNormParams& p, const Walk& w, int c0) {
    if (c0 >= p.D) return;
    const long c = long(w.h) * p.D + c0;
    x.load_once(p.x, w.t * p.xs + c);
    if (p.gate) g.load_once(p.gate, w.t * p.gs + c);
    if (p.res) r.load_once(p.res, w.row * p.D + c0);
  }
};

template <int LANES, bool BF16, bool RES_BF16>
__global__ __launch_bounds__(LANES > 64 ? LANES : 256) void block_norm_kernel(BlockNormParams p) {
  constexpr int RW = LANES > 64 ? 1 : 256 / LANES;
  const float inv_d = 1.f / float(p.D);
  const int c0 = E * int(threadIdx.x % LANES);
  const bool in = c0 < p.D;
  int turn = 0;
  float wa[E], wb[E], cs[E];
  vector_of(p.wa, c0, in, wa);
  vector_of(p.wb, c0, in, wb);
  vector_of(p.cs, c0, in, cs);
#pragma unroll
  for (int j = 0; j < E; ++j) cs[j] *= p.scale;
  Walk ahead(long(blockIdx.x) * RW + threadIdx.x / LANES, long(gridDim.x) * RW, p.H);
  RowIn<BF16, RES_BF16> cur, next;
  if (ahead.row < p.rows) cur.load(p, ahead, c0);
  for (long row = ahead.row; row < p.rows; row += ahead.step) {  // (whole rows of lanes)
    ahead.next(p.H);
    if (ahead.row < p.rows) next.load(p, ahead, c0);
    float h[E] = {};
    if (in) cur.x.floats(h);
    float rn = 1.f;
    if (p.after) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < E; ++j) s = fmaf(h[j], h[j], s);
      rn = 1.f / sqrtf(row_sum<LANES>(s, turn) * inv_d + p.eps);
    }
    float s = 0.f;
    if (in) {
#pragma unroll
      for (int j = 0; j < E; ++j) h[j] *= rn * wa[j];
      if (p.gate) {
        float g[E];
        cur.g.floats(g);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const float sg = sigmoid(g[j]);
          h[j] *= p.silu ? g[j] * sg : sg;
        }
      }
      float r[E] = {};
      if (p.res) cur.r.floats(r);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        h[j] = fmaf(cs[j], h[j], r[j]);
        s = fmaf(h[j], h[j], s);
      }
      if (p.h) RawN<RES_BF16, E>::of(h).store_once(p.h, row * p.D + c0);
    }
    if (p.y) {
      float rh = 1.f;
      if (p.before) rh = 1.f / sqrtf(row_sum<LANES>(s, turn) * inv_d + p.eps);
      if (in) {
#pragma unroll
        for (int j = 0; j < E; ++j) h[j] *= rh * wb[j];
        RawN<BF16, E>::of(h).store_once(p.y, row * p.D + c0);
      }
    }
    cur = next;
  }
}

template <bool BF16, bool RES_BF16>
struct GradIn {
  RawN<BF16, E> y;
  RawN<RES_BF16, E> h;
  __device__ void load(const BlockNormParams& p, long row, int c0) {
    if (c0 >= p.D) return;
    if (p.dy) y.load_once(p.dy, row * p.D + c0);
    if (p.dh) h.load_once(p.dh, row * p.D + c0);
  }
};

// A lane's sums of one weight's gradient, in registers or in LDS (16 bytes of each lane side by
// side).
template <bool KEEP, int LANES>
struct Sum {
  float v[KEEP ? E : 1] = {};
  f32x4* at = nullptr;
  __device__ void set(f32x4* lds) {
    at = lds + threadIdx.x;
    at[0] = at[LANES] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ void add(const float (&x)[E], const float (&y)[E]) {
    if constexpr (KEEP) {
#pragma unroll
      for (int j = 0; j < E; ++j) v[j] = fmaf(x[j], y[j], v[j]);
    } else {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        f32x4 s = at[i * LANES];
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = fmaf(x[4 * i + j], y[4 * i + j], s[j]);
        at[i * LANES] = s;
      }
    }
  }
  __device__ float get(int j) const {
    if constexpr (KEEP) return v[j];
    else return at[j / 4 * LANES][j % 4];
  }
};

// Every workgroup walks its rows in a fixed order and leaves the sums of the three weights'
// gradients over them.  1024 lanes (more than 4096 columns) have half the registers of fewer: there
// the sums are in LDS, the weights are read at their uses in every row (from the cache), the gate
// and the normed x are formed again for the second half, and no row is requested ahead (2047 rows
// of 8192 with everything in bf16 97 us, in fp32 202; with sums in registers 188 and 326; with a row
// ahead, spilled, 99 and 251).  4095 rows of 4096 take 58 us.
template <int LANES, bool BF16, bool RES_BF16>
__global__ __launch_bounds__(LANES > 64 ? LANES : 256) void block_norm_backward_kernel(
    BlockNormParams p) {
  constexpr int RW = LANES > 64 ? 1 : 256 / LANES;
  constexpr bool KEEP = LANES < 1024;
  __shared__ float acc[RW][RW > 1 ? E * LANES : 1];
  const int group = threadIdx.x / LANES, c0 = E * int(threadIdx.x % LANES);
  const float inv_d = 1.f / float(p.D);
  const bool in = c0 < p.D;
  int turn = 0;
  float wa[E], wb[E], cs[E];
  Sum<KEEP, LANES> da, db, dc;
  if constexpr (!KEEP) {
    __shared__ f32x4 lds[3 * E / 4 * LANES];
    da.set(lds);
    db.set(lds + E / 4 * LANES);
    dc.set(lds + 2 * E / 4 * LANES);
  }
  auto inner = [&] {
    vector_of(p.wa, c0, in, wa);
    vector_of(p.cs, c0, in, cs);
#pragma unroll
    for (int j = 0; j < E; ++j) cs[j] *= p.scale;
  };
  if constexpr (KEEP) {
    inner();
    vector_of(p.wb, c0, in, wb);
  }
  Walk ahead(long(blockIdx.x) * RW + group, long(gridDim.x) * RW, p.H);
  RowIn<BF16, RES_BF16> cur, next;
  GradIn<BF16, RES_BF16> gcur, gnext;
  if (ahead.row < p.rows) {
    cur.load(p, ahead, c0);
    gcur.load(p, ahead.row, c0);
  }
  for (long row = ahead.row; row < p.rows; row += ahead.step) {
    if constexpr (KEEP) {
      ahead.next(p.H);
      if (ahead.row < p.rows) {
        next.load(p, ahead, c0);
        gnext.load(p, ahead.row, c0);
      }
    } else {
      cur.load(p, ahead, c0);
      gcur.load(p, ahead.row, c0);
      ahead.next(p.H);
    }
    // a: the gate's activation, slope: its derivative; un: x normed and weighted
    float x[E] = {}, a[E], slope[E], h[E] = {}, dy[E] = {}, d[E] = {}, un[E];
    float s = 0.f, rx = 1.f;
    auto open = [&] {
      if (in) cur.x.floats(x);
#pragma unroll
      for (int j = 0; j < E; ++j) a[j] = 1.f;
      if (p.gate) {
        float g[E] = {};
        if (in) cur.g.floats(g);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const float sg = sigmoid(g[j]), z = p.silu ? g[j] : 1.f;
          a[j] = sg * z;
          // s (1 + g (1 - s)), or s (1 - s); 1 - s first: g + 1 would lose the 1 beside a large g
          slope[j] = fmaf(sg, fmaf(-z, sg, z), p.silu ? sg : 0.f);
        }
      }
    };
    auto weigh = [&](float r) {
      if constexpr (!KEEP) {
        asm volatile("" ::: "memory");  // (the weights are read here, each time)
        inner();
      }
#pragma unroll
      for (int j = 0; j < E; ++j) un[j] = x[j] * r * wa[j];
    };
    open();
    if (in) {
      if (p.res) cur.r.floats(h);
      if (p.dy) gcur.y.floats(dy);
      if (p.dh) gcur.h.floats(d);
    }
    if (p.after) {
#pragma unroll
      for (int j = 0; j < E; ++j) s = fmaf(x[j], x[j], s);
      rx = 1.f / sqrtf(row_sum<LANES>(s, turn) * inv_d + p.eps);
    }
    weigh(rx);
#pragma unroll
    for (int j = 0; j < E; ++j) h[j] = fmaf(cs[j], un[j] * a[j], h[j]);
    if (p.before) {
      float both[2] = {0.f, 0.f};
      if constexpr (!KEEP) vector_of(p.wb, c0, in, wb);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        both[0] = fmaf(h[j], h[j], both[0]);
        both[1] = fmaf(wb[j] * dy[j], h[j], both[1]);
      }
      row_sums<LANES>(both, turn);
      const float rh = 1.f / sqrtf(both[0] * inv_d + p.eps);
      const float f = both[1] * inv_d * rh * rh * rh;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        d[j] = fmaf(rh, wb[j] * dy[j], fmaf(-f, h[j], d[j]));
        h[j] *= rh;
      }
      db.add(dy, h);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) d[j] += dy[j];
    }
    if (p.dres && in) RawN<RES_BF16, E>::of(d).store_once(p.dres, row * p.D + c0);
    if constexpr (!KEEP) {  // (formed again, not held since then)
      cur.x.opaque();
      cur.g.opaque();
      open();
      weigh(rx);
    }
    s = 0.f;
    float dg[E], t[E], n[E];
#pragma unroll
    for (int j = 0; j < E; ++j) t[j] = un[j] * a[j];
    dc.add(d, t);
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const float du = cs[j] * d[j], dn = du * a[j];
      if (p.gate) dg[j] = du * un[j] * slope[j];
      t[j] = dn * x[j];
      n[j] = rx;
      s = fmaf(t[j], wa[j], s);
      d[j] = dn * wa[j];
    }
    da.add(t, n);
    if (p.gate && p.dgate && in) RawN<BF16, E>::of(dg).store_once(p.dgate, row * p.D + c0);
    if (p.after) {
      const float f = row_sum<LANES>(s, turn) * inv_d * rx * rx * rx;
#pragma unroll
      for (int j = 0; j < E; ++j) d[j] = fmaf(rx, d[j], -f * x[j]);
    }
    if (in) RawN<BF16, E>::of(d).store_once(p.dx, row * p.D + c0);
    if constexpr (KEEP) {
      cur = next;
      gcur = gnext;
    }
  }
  if (!p.partial) return;
  const bool alone = gridDim.x == 1;  // (its sums are the results)
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const auto& sum = k == 0 ? da : k == 1 ? db : dc;
    const float f = k == 2 ? p.scale : 1.f;
    float* const out = !alone   ? p.partial + (long(blockIdx.x) * 3 + k) * p.D
                       : k == 0 ? p.dwa
                       : k == 1 ? p.dwb
                                : p.dcs;
    if (!out) continue;
    if constexpr (RW == 1) {
      if (!in) continue;
#pragma unroll
      for (int j = 0; j < E; ++j) out[c0 + j] = f * sum.get(j);
    } else {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < E; ++j) acc[group][c0 + j] = f * sum.get(j);
      __syncthreads();
      for (int c = threadIdx.x; c < p.D; c += 256) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < RW; ++i) t += acc[i][c];
        out[c] = t;
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

// Workgroups that the compute units hold, for walks over `need` of them.
unsigned walkers(long need, int per_cu, int cus) {
  const long most = long(cus > 0 ? cus : 256) * per_cu;
  return unsigned(need < most ? need : most);
}

template <int LANES, bool BF16, bool RES_BF16>
hipError_t run(const BlockNormParams& p, bool backward, int cus, hipStream_t st) {
  constexpr int RW = LANES > 64 ? 1 : 256 / LANES, threads = LANES > 64 ? LANES : 256;
  const long need = (p.rows + RW - 1) / RW;
  if (!backward) {
    block_norm_kernel<LANES, BF16, RES_BF16>
        <<<walkers(need, 2048 / threads, cus), threads, 0, st>>>(p);
    return hipGetLastError();
  }
  // 512 threads of this kernel's registers on a compute unit
  unsigned blocks = walkers(need, threads < 512 ? 512 / threads : 1, cus);
  if (blocks > unsigned(kBlockNormBlocks)) blocks = kBlockNormBlocks;
  if (blocks > 0) {
    block_norm_backward_kernel<LANES, BF16, RES_BF16><<<blocks, threads, 0, st>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.partial && blocks != 1)
    block_norm_weight_kernel<<<unsigned(3 * ((p.D + 15) / 16)), 1024, 0, st>>>(p, int(blocks));
  return hipGetLastError();
}

template <bool BF16, bool RES_BF16>
hipError_t by_width(const BlockNormParams& p, bool backward, int cus, hipStream_t st) {
#define ONELA_NORM(L) return run<L, BF16, RES_BF16>(p, backward, cus, st)
  if (p.D <= 32) ONELA_NORM(4);
  if (p.D <= 64) ONELA_NORM(8);
  if (p.D <= 128) ONELA_NORM(16);
  if (p.D <= 256) ONELA_NORM(32);
  if (p.D <= 512) ONELA_NORM(64);
  if (p.D <= 1024) ONELA_NORM(128);
  if (p.D <= 2048) ONELA_NORM(256);
  if (p.D <= 4096) ONELA_NORM(512);
  ONELA_NORM(1024);
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
