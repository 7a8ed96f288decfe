// The delta rule's chain over the chunks (see kernels_delta.hip).
#include "delta_tiles.h"

namespace onela {
namespace {

// Waves of a scan workgroup: 32 state rows each, at most 128 per workgroup.
template <int DV>
constexpr int kScanWaves = DV / 32 < 4 ? DV / 32 : 4;

// The chain over the chunks of one (sequence, value head) with its outputs: up to 128 rows of
// the state per workgroup, 32 per wave as two column tiles of S^T (tile u, lane lr: row 2 lr
// + u), which stay in registers.  Per chunk
//   Y = K S^T, X = V - gamma Y, e = T X, O = scale gamma Q S^T + P e, S^T <- g S^T + K^T (beta sigma e)
// with all products chained in registers: the order of tokens and columns within a
// 32-deep step is that of the accumulators.
//
// Operands come to LDS straight from memory in the layout that is read there: the next
// chunk's keys and queries during T X and P e, its T, P and gates during the update.
//
// Scales (powers of two).  Each lane's two rows are kept as st = sc S with a bound on
// their largest value; the bound grows with every update by what 64 tokens can add at
// most, and where it leaves [2^8, 2^15] the rows are scaled anew.  The true values are some
// 2^7 below the bound, far inside what two fp16 parts hold to 22 bits of the largest.
//
// Segments.  One chain per 128 rows leaves most of the chip idle for few heads, so a
// sequence can be cut into segments of p.cps chunks that run at once: S_out = S_in A + B.
// With SEG the kernel forms, without outputs, for every segment but the sequence's last
// the state that it leaves: of the first the true one, of the others B (from S_in =
// 0) and, by the same code on the rows of the identity and V = 0, A.
// delta_combine_kernel chains them, and then every segment starts from its true state.
template <int DK, int DV, int NP, bool SEG>
__global__ __launch_bounds__(64 * kScanWaves<DV>, DK >= 256 || NP == 2 ? 1 : 2)
void delta_forward_kernel(DeltaParams p) {
  constexpr int NW = kScanWaves<DV>, GB = DV / (32 * NW);
  constexpr int GA = SEG ? DK / (32 * NW) : 0;
  constexpr int NB = DK / 16;
  constexpr int PS = NB / 2 < 4 ? NB / 2 : 4;
  auto t0 = [](int h) constexpr { return h / PS * (2 * PS) + h % PS; };
  constexpr int kIo = NP == 1 ? 2 : 4;
  constexpr int kImage = sizeof(Swz<DK>) * NP, kFrags = 6 * 2 * 1024;
  constexpr int kGateBytes = kDeltaGates * kC * 4;
  __shared__ __align__(16) Swz<DK> sK[2][NP];
  __shared__ __align__(16) Swz<DK> sQ[SEG ? 1 : NP];
  __shared__ __align__(16) uint4 sT[kFrags / 16];
  __shared__ __align__(16) uint4 sP[SEG ? 1 : kFrags / 16];
  __shared__ __align__(16) float sG[kDeltaGates][kC];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int item = int(blockIdx.x % (GB + GA));
  const bool ident = SEG && item >= GB;  // rows of A
  const int grp = ident ? item - GB : item;
  const long su = blockIdx.x / (GB + GA);  // segment slot and value head
  const int hv = int(su % p.HV), hk = hv / (p.HV / p.HK);
  const Segment sg = segment_of(p, su / p.HV);
  if (sg.j < 0 || (SEG && (sg.j + 1 == sg.nseg || (ident && sg.j == 0)))) return;
  const Seq& sq = sg.sq;
  const int row0 = 32 * (NW * grp + w) + 2 * lr;  // this lane's rows: row0, row0 + 1
  const int nch = sg.ce;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};

  // st[u][b][i] = sc S(row0 + u, 16 b + 4 lq + i)
  f32x4 st[2][NB];
  float sc = 1.f, bound = 0.f;
  const long rows = long(row0) * DK + 4 * lq;
  const float* from = sg.j == 0 ? p.s_in : SEG ? nullptr : p.segs + (su - p.HV) * (DV * DK);
  if (sg.j == 0 && from) from += (long(sg.n) * p.HV + hv) * (DV * DK);
  auto rescale = [&](float f) __attribute__((always_inline)) {
    const float to = fminf(fmaxf(sc * f, 0x1p-100f), 0x1p100f);
    f = to * inverse_pow2(sc);
    sc = to;
    bound *= f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int b = 0; b < NB; ++b) st[u][b] *= f;
  };
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      st[u][b] = from ? *reinterpret_cast<const f32x4*>(from + rows + u * DK + 16 * b) : z;
      if (ident)
#pragma unroll
        for (int i = 0; i < 4; ++i) st[u][b][i] = 16 * b + 4 * lq + i == row0 + u ? 1.f : 0.f;
      bound = max4abs(bound, st[u][b]);
    }
  bound = max_over_rows(bound);
  if (from || ident) rescale(bound > 0.f ? scale_for(bound) : 1.f);

  auto load_kq = [&](int c) __attribute__((always_inline)) {
    const long at = ((sq.slot + c) * p.HK + hk) * (kImage / 16);
    dma<kImage, NW>(p.kimg + at, sK[c & 1], w, lane);
    if constexpr (!SEG) dma<kImage, NW>(p.qimg + at, sQ, w, lane);
  };
  auto load_tp = [&](int c) __attribute__((always_inline)) {
    const long cu = (sq.slot + c) * p.HV + hv;
    dma<kFrags, NW>(p.tp + cu * (kFrags / 16), sT, w, lane);
    if constexpr (!SEG) dma<kFrags, NW>(p.pf + cu * (kFrags / 16), sP, w, lane);
    dma<kGateBytes, NW>(p.gates + cu * (kDeltaGates * kC), sG, w, lane);
  };
  // values V(t = 16 a + 4 lq + i, row0 + u), raw
  const unsigned vs = unsigned(p.vs) * kIo;
  unsigned vr[16][NP];
  auto load_v = [&](int c) __attribute__((always_inline)) {
    const int m = ident ? 0 : min(kC, sq.len - c * kC);  // (A: no values)
    const auto rs = rows_buffer(p.v, ((sq.t0 + long(c) * kC) * p.vs + hv * DV) * kIo, DV * kIo, vs, m);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const unsigned o = unsigned(4 * lq) * vs + row0 * kIo, so = (16 * (i >> 2) + (i & 3)) * vs;
      if constexpr (NP == 1) {
        vr[i][0] = __builtin_amdgcn_raw_buffer_load_b32(rs, o, so, 0);
      } else {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(rs, o, so, 0);
        vr[i][0] = x[0];
        vr[i][1] = x[1];
      }
    }
  };
  auto value = [&](int i, int u) {
    if constexpr (NP == 1)
      return u ? bf16_hi_to_float(vr[i][0]) : bf16_lo_to_float(vr[i][0]);
    else
      return __uint_as_float(vr[i][u]);
  };
  auto gate = [&](int row, int a) { return *reinterpret_cast<const f32x4*>(&sG[row][16 * a + 4 * lq]); };
  const int kb = Swz<DK>::off(lr, lq), tb = Swz<DK>::off(4 * lq + (lr >> 2), lr & 3);
  constexpr int KR = 32 * Swz<DK>::LD;  // bytes of 16 rows
  // acc[u][a] += F x[u] over a lower triangular 64 x 64 matrix in two parts, F's fragments in LDS
  auto triangle = [&](const uint4* F, const uint4 (&x)[2][2][2], f32x4 (&acc)[2][4])
      __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 f[4][2];
#pragma unroll
      for (int a = 2 * h; a < 4; ++a)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          f[a][i] = F[((a < 2 ? a : 2 * a - 2 + h) * 2 + i) * 64 + lane];
      for_products<2, 2>([&](int i, int j) {
#pragma unroll
        for (int a = 2 * h; a < 4; ++a)
#pragma unroll
          for (int u = 0; u < 2; ++u) acc[u][a] = mfma_f16(f[a][i], x[u][h][j], acc[u][a]);
      });
    }
  };

  if (sg.cb < nch) {
    load_kq(sg.cb);
    load_tp(sg.cb);
    load_v(sg.cb);
  }
  for (int c = sg.cb; c < nch; ++c) {
    const Swz<DK>* const K = sK[c & 1];
    dma_wait();
    __syncthreads();  // this chunk's operands are in LDS
    const float inv = inverse_pow2(sc);
    // Y = K S^T and Q S^T
    f32x4 y[2][4], o[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int a = 0; a < 4; ++a) y[u][a] = o[u][a] = z;
#pragma unroll
    for (int h = 0; h < DK / 32; ++h) {
      uint4 sp[2][2], kf[4][NP], qf[4][NP];
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          kf[a][i] = row_frag(K[i], kb, t0(h), t0(h) + PS, KR * a);
          if constexpr (!SEG) qf[a][i] = row_frag(sQ[i], kb, t0(h), t0(h) + PS, KR * a);
        }
#pragma unroll
      for (int u = 0; u < 2; ++u) parts8(st[u][t0(h)], st[u][t0(h) + PS], sp[u]);
      for_products<NP, 2>([&](int i, int j) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int a = 0; a < 4; ++a) y[u][a] = mfma_f16(kf[a][i], sp[u][j], y[u][a]);
        if constexpr (!SEG)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int a = 0; a < 4; ++a) o[u][a] = mfma_f16(qf[a][i], sp[u][j], o[u][a]);
      });
    }
    // X = V - gamma Y, scaled for the lane's two rows
    uint4 xp[2][2][2];
    float ix;
    {
      f32x4 x[2][4];
      float m = 0.f;
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 g = gate(kGateY, a) * inv;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[u][a][i] = fmaf(g[i], y[u][a][i], value(4 * a + i, u));
          m = max4abs(m, x[u][a]);
        }
      }
      const float s = scale_for(max_over_rows(m));
      ix = inverse_pow2(s);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        parts8<2>(x[u][0], x[u][1], s, xp[u][0]);
        parts8<2>(x[u][2], x[u][3], s, xp[u][1]);
      }
    }
    __syncthreads();  // all have read the queries, and the last chunk's keys
    if (c + 1 < nch) load_kq(c + 1);
    // e = T X (each token's row times its scale of T: the gates undo it)
    f32x4 e[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int a = 0; a < 4; ++a) e[u][a] = z;
    triangle(sT, xp, e);
    uint4 ep[2][2][2], zp[2][2][2];
    float ie;
    const float g = sG[kGateOne][0];
    {
      float m = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int a = 0; a < 4; ++a) m = max4abs(m, e[u][a]);
      m = max_over_rows(m);
      const float s = scale_for(m);
      ie = inverse_pow2(s) * ix;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        parts8<2>(e[u][0], e[u][1], s, ep[u][0]);
        parts8<2>(e[u][2], e[u][3], s, ep[u][1]);
      }
      // what the update adds, in units of sc, and the rows' bound after it
      const float most = m * ix * (sG[kGateOne][1] * sG[kGateOne][2]);
      float next = fmaf(g, bound, 0x1p13f * most * sc);
      const bool off = !(next <= 32768.f && next >= 256.f) && next > 0.f;
      if (__any(off)) {
        const float was = sc;
        rescale(off ? scale_for(next) : 1.f);
        next *= sc * inverse_pow2(was);
      }
      bound = next;
      const float cz = ix * sc * sG[kGateOne][2];
      f32x4 gz[4];
#pragma unroll
      for (int a = 0; a < 4; ++a) gz[a] = gate(kGateZ, a) * cz;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        parts8(e[u][0], e[u][1], gz[0], gz[1], zp[u][0]);
        parts8(e[u][2], e[u][3], gz[2], gz[3], zp[u][1]);
      }
    }
    // P e, and the outputs
    if constexpr (!SEG) {
      f32x4 q[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int a = 0; a < 4; ++a) q[u][a] = z;
      triangle(sP, ep, q);
      const int m = min(kC, sq.len - c * kC);
      const unsigned os = unsigned(p.HV) * (DV * kIo);
      // a buffer that ends with the sequence's last token: stores past it are dropped
      const auto rs = rows_buffer(p.o, ((sq.t0 + long(c) * kC) * p.HV + hv) * (DV * kIo), DV * kIo,
                                  os, m);
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 go = gate(kGateO, a) * inv, gp = gate(kGateP, a) * ie;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x0 = fmaf(go[i], o[0][a][i], gp[i] * q[0][a][i]);
          const float x1 = fmaf(go[i], o[1][a][i], gp[i] * q[1][a][i]);
          const unsigned at = unsigned(4 * lq) * os + row0 * kIo, so = (16 * a + i) * os;
          if constexpr (NP == 1) {
            __builtin_amdgcn_raw_buffer_store_b32(pack_bf16x2(x0, x1), rs, at, so, 0);
          } else {
            typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
            __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(x0), __float_as_uint(x1)},
                                                  rs, at, so, 0);
          }
        }
      }
    }
    __syncthreads();  // all have read T, P and the gates
    if (c + 1 < nch) {
      load_tp(c + 1);
      load_v(c + 1);
    }
    // S^T <- g S^T + K^T (beta sigma e)
    constexpr int NG = NB < 4 ? NB : 4;
#pragma unroll
    for (int b0 = 0; b0 < NB; b0 += NG) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int b = 0; b < NG; ++b) st[u][b0 + b] *= g;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 kt[NG][NP];
#pragma unroll
        for (int b = 0; b < NG; ++b)
#pragma unroll
          for (int i = 0; i < NP; ++i) kt[b][i] = col_frag(K[i], tb, b0 + b, 2 * KR * h);
        for_products<NP, 2>([&](int i, int j) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int b = 0; b < NG; ++b)
              st[u][b0 + b] = mfma_f16(kt[b][i], zp[u][h][j], st[u][b0 + b]);
        });
      }
    }
  }
  float* to = nullptr;
  if constexpr (SEG)
    to = ident ? p.sega + su * (DK * DK) : p.segs + su * (DV * DK);
  else if (p.s_out && sg.j + 1 == sg.nseg)
    to = p.s_out + (long(sg.n) * p.HV + hv) * (DV * DK);
  if (to) {
    const float inv = inverse_pow2(sc);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *reinterpret_cast<f32x4*>(to + rows + u * DK + 16 * b) = inv * st[u][b];
  }
}

// The true states after the segments of one (sequence, value head, 16 state rows): S_0 as
// it is, then S_j = S_{j-1} A_j + B_j, in B_j's place.  Wave w holds the columns 16 w ..
// 16 w + 15 as an accumulator tile of S^T; the tiles, cut into three bf16 parts, are exchanged
// through LDS as operands (one barrier per segment), A_j's rows come from memory, requested one
// segment ahead.  Bound: latency of the chain over the segments.
template <int DK, int DV>
__global__ __launch_bounds__(4 * DK) void delta_combine_kernel(DeltaParams p) {
  constexpr int NH = DK / 32, NRB = DV / 16;
  __shared__ uint4 xs[2][NH][3][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int unit = blockIdx.x / NRB, rb = blockIdx.x % NRB;
  const int n = unit / p.HV, hv = unit - n * p.HV;
  const Seq sq = seq_of(p, n);
  const long slot0 = first_segment(p, sq, n);
  const int last = segments_of(p, sq) - 2;  // the last segment that leaves a state
  if (last < 1) return;
  const long at = long(16 * rb + lr) * DK + 16 * w + 4 * lq;
  auto state = [&](int j) { return p.segs + ((slot0 + j) * p.HV + hv) * (DV * DK) + at; };
  f32x4 st = *reinterpret_cast<const f32x4*>(state(0));
  // A^T(16 w + lr, k): slots k = 32 h + 4 lq + i and 32 h + 16 + 4 lq + i
  f32x4 a[NH][2];
  auto load = [&](int j, int h) {
    const float* q = p.sega + ((slot0 + min(j, last)) * p.HV + hv) * (DK * DK) +
                     (32 * h + 4 * lq) * DK + 16 * w + lr;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) a[h][u][i] = q[(16 * u + i) * DK];
  };
  f32x4 bn = *reinterpret_cast<const f32x4*>(state(1));
#pragma unroll
  for (int h = 0; h < NH; ++h) load(1, h);
  for (int j = 1; j <= last; ++j) {
    const int x = j & 1;
    uint4 d[3];
    cut3(st, st, d[0], d[1], d[2]);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      reinterpret_cast<uint2*>(&xs[x][w >> 1][i][lane])[w & 1] = make_uint2(d[i].x, d[i].y);
    __syncthreads();
    f32x4 hi[2] = {}, lo[4] = {};
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const uint4 dh = xs[x][h][0][lane], dm = xs[x][h][1][lane], dl = xs[x][h][2][lane];
      uint4 t[3];
      cut3(a[h][0], a[h][1], t[0], t[1], t[2]);
      load(j + 1, h);  // (into the registers just read)
      const int e = h & 1;
      hi[e] = mfma_bf16(t[0], dh, hi[e]);
      lo[e] = mfma_bf16(t[2], dh, lo[e]);
      lo[2 + e] = mfma_bf16(t[1], dm, lo[2 + e]);
      lo[e] = mfma_bf16(t[0], dl, lo[e]);
      lo[2 + e] = mfma_bf16(t[1], dh, lo[2 + e]);
      lo[e] = mfma_bf16(t[0], dm, lo[e]);
    }
    st = bn + ((hi[0] + hi[1]) + ((lo[0] + lo[1]) + (lo[2] + lo[3])));
    bn = *reinterpret_cast<const f32x4*>(state(min(j + 1, last)));
    *reinterpret_cast<f32x4*>(state(j)) = st;
  }
}

template <int DK, int DV, int NP>
hipError_t run(const DeltaParams& p, hipStream_t st) {
  constexpr int NW = kScanWaves<DV>, GB = DV / (32 * NW), GA = DK / (32 * NW);
  const unsigned units = unsigned(p.seg_slots) * unsigned(p.HV);
  if (p.sega) {
    delta_forward_kernel<DK, DV, NP, true><<<units * (GB + GA), 64 * NW, 0, st>>>(p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    delta_combine_kernel<DK, DV>
        <<<unsigned(p.N) * unsigned(p.HV) * (DV / 16), 4 * DK, 0, st>>>(p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  delta_forward_kernel<DK, DV, NP, false><<<units * GB, 64 * NW, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_forward(const DeltaShape& s, const DeltaParams& p, hipStream_t st) {
#define ONELA_DELTA_SCAN(DK, DV, NP) \
  if (s.dk == DK && s.dv == DV && s.bf16 == (NP == 1)) return run<DK, DV, NP>(p, st);
  ONELA_DELTA_SCAN(32, 32, 1)
  ONELA_DELTA_SCAN(64, 64, 1)
  ONELA_DELTA_SCAN(128, 128, 1)
  ONELA_DELTA_SCAN(128, 256, 1)
  ONELA_DELTA_SCAN(128, 512, 1)
  ONELA_DELTA_SCAN(256, 256, 1)
  ONELA_DELTA_SCAN(256, 512, 1)
  ONELA_DELTA_SCAN(32, 32, 2)
  ONELA_DELTA_SCAN(64, 64, 2)
  ONELA_DELTA_SCAN(128, 128, 2)
#undef ONELA_DELTA_SCAN
  return hipErrorInvalidValue;
}

}  // namespace onela
