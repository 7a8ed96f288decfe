// The delta rule's chain over the chunks in reverse, for the gradients (see
// kernels_delta.hip).
#include "delta_chain.h"

namespace onela {
namespace {

// The adjoint's chain over the chunks of one (sequence, value head), as delta_forward_kernel
// with the tokens of a chunk in reverse order (t' = 63 - t) and S the adjoint of the state
// after the chunk.  Per chunk
//   Y = K S^T, X = P^T dO + beta sigma Y, dV = T^T X,
//   S^T <- g S^T - K^T (gamma dV) + Q^T (scale gamma dO);
// it leaves dV (as a tensor and in fp32 for the gradients) and the adjoint before each
// update.  SEG: segments, counted from the sequence's end, as there (p.ds_out may be p.ds_in).
//   Bound: as there, and the stores of the adjoints.  16 x 1024 tokens x 32 heads of 128 take
// 302 us (3.1 TB/s written; 318 with a state's rows stored 64 bytes at a time in place of
// whole lines, 355 with those as non-temporal stores).
template <int DK, int DV, int NP, bool SEG>
__global__ __launch_bounds__(64 * kChainWaves<DV>, DK >= 256 || NP == 2 ? 1 : 2)
void delta_reverse_kernel(DeltaParams p) {
  constexpr int NW = kChainWaves<DV>, GB = DV / (32 * NW);
  constexpr int GA = SEG ? DK / (32 * NW) : 0;
  constexpr int kIo = NP == 1 ? 2 : 4;
  constexpr int kImage = sizeof(Swz<DK>) * NP;
  // tokens in reverse order: rows of K and Q are read from the other end of their tiles
  __shared__ __align__(16) Swz<DK> sK[2][NP];
  __shared__ __align__(16) Swz<DK> sQ[NP];
  __shared__ __align__(16) uint4 sT[kFragBytes / 16];
  __shared__ __align__(16) uint4 sP[kFragBytes / 16];
  __shared__ __align__(16) float sG[kGateStage][kC];
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
  const int all = delta_chunks(sq.len);           // the walk's step s is the chunk all - 1 - s
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};

  ChainState<DK> s;
  const long rows = long(row0) * DK + 4 * lq;
  {
    const float* from = start_of<DK, DV, SEG>(p, sg, su, hv, p.ds_in);
    s.init(from ? from + rows : nullptr,
           SEG && from ? kept_start<DK, DV>(p, sg, su) + rows : nullptr, ident, row0, lq);
  }
  auto image_at = [&](int c) { return ((sq.slot + c) * p.HK + hk) * (kImage / 16); };
  auto load_tp = [&](int c) __attribute__((always_inline)) {
    const long cu = (sq.slot + c) * p.HV + hv;
    dma<kFragBytes, NW>(p.tr + cu * (kFragBytes / 16), sT, w, lane);
    dma<kFragBytes, NW>(p.pr + cu * (kFragBytes / 16), sP, w, lane);
    dma<kGateStage * kC * 4, NW>(p.gates + (cu * p.gate_rows + kGateStage) * kC, sG, w, lane);
  };
  const unsigned os = unsigned(p.HV) * (DV * kIo);
  auto rows_of = [&](const void* t, int c, int m) {  // a dense tensor's rows of the chunk
    return rows_buffer(t, ((sq.t0 + long(c) * kC) * p.HV + hv) * (DV * kIo), DV * kIo, os, m);
  };
  Columns<NP, true> v;
  auto load_v = [&](int c) __attribute__((always_inline)) {
    v.load(rows_of(p.d_o, c, ident ? 0 : min(kC, sq.len - c * kC)), os, lq, row0 * kIo);
  };
  // gates by t': the lane's four tokens from the other end
  auto back = [](const f32x4& x) { return f32x4{x.w, x.z, x.y, x.x}; };
  auto gate = [&](int row, int a) {
    return back(*reinterpret_cast<const f32x4*>(&sG[row - kGateStage][60 - 16 * a - 4 * lq]));
  };
  auto one = [&](int i) { return sG[kRevOne - kGateStage][i]; };
  // K's and Q's tiles hold the tokens in order: row 16 a + lr of the walk is row 16 (3 - a) + 15 - lr
  const int kb = Swz<DK>::off(15 - lr, lq);
  constexpr int KR = ChainState<DK>::KR, PS = ChainState<DK>::PS;

  if (sg.cb < sg.ce) {
    const int c = all - 1 - sg.cb;
    dma<kImage, NW>(p.kimg + image_at(c), sK[sg.cb & 1], w, lane);
    load_tp(c);
    load_v(c);
  }
  for (int step = sg.cb; step < sg.ce; ++step) {
    const int c = all - 1 - step;
    const Swz<DK>* const K = sK[step & 1];
    const bool more = step + 1 < sg.ce;
    if (!SEG || (step - sg.cb) % kTighten == kTighten - 1) s.tighten();
    dma_wait();
    __syncthreads();  // this chunk's keys, T, P and gates are in LDS; all have left the last update
    dma<kImage, NW>(p.qimg + image_at(c), sQ, w, lane);
    const long cu = (sq.slot + c) * p.HV + hv;
    const float inv[2] = {inverse_pow2(s.sc[0]), inverse_pow2(s.sc[1])};
    const float before = max_bits(s.bound[0], s.bound[1]);
    if constexpr (!SEG)
      s.template store_tiles<DV>(p.dsws + cu * (DV * DK), NW * grp + w, lane);
    // Y = K S^T
    f32x4 y[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int a = 0; a < 4; ++a) y[u][a] = z;
#pragma unroll
    for (int h = 0; h < DK / 32; ++h) {
      constexpr auto t0 = ChainState<DK>::t0;
      uint4 sp[2][2], kf[4][NP];
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int i = 0; i < NP; ++i)
          kf[a][i] = row_frag(K[i], kb, t0(h), t0(h) + PS, KR * (3 - a));
#pragma unroll
      for (int u = 0; u < 2; ++u) parts8(s.st[u][t0(h)], s.st[u][t0(h) + PS], sp[u]);
      for_products<NP, 2>([&](int i, int j) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int a = 0; a < 4; ++a) y[u][a] = mfma_f16(kf[a][i], sp[u][j], y[u][a]);
      });
    }
    // P^T dO
    f32x4 q[2][4];
    float mo[2], fo[2];
    {
      uint4 op[2][2][NP];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        mo[u] = 0.f;
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          q[u][a] = z;
          mo[u] = max4abs(mo[u], v.tile(a, u));
        }
        fo[u] = scale_for(max_over_rows(mo[u]));
#pragma unroll
        for (int h = 0; h < 2; ++h)
          parts8<NP>(v.tile(2 * h, u), v.tile(2 * h + 1, u), fo[u], op[u][h]);
      }
      triangle(sP, op, q, lane);
    }
    // X = P^T dO + beta sigma Y, each row with a scale of its own
    uint4 xp[2][2][2];
    float ix[2];
    {
      f32x4 x[2][4];
      float m[2] = {0.f, 0.f};
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 gy = gate(kRevY, a), gp = gate(kRevP, a);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const f32x4 yi = y[u][a] * inv[u], qi = q[u][a] * inverse_pow2(fo[u]);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[u][a][i] = fmaf(gy[i], yi[i], gp[i] * qi[i]);
          m[u] = max4abs(m[u], x[u][a]);
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float f = scale_for(max_over_rows(m[u]));
        ix[u] = inverse_pow2(f);
        parts8<2>(x[u][0], x[u][1], f, xp[u][0]);
        parts8<2>(x[u][2], x[u][3], f, xp[u][1]);
      }
    }
    dma_wait();       // the queries
    __syncthreads();  // (and all have left the last chunk's keys)
    if (more) dma<kImage, NW>(p.kimg + image_at(c - 1), sK[(step + 1) & 1], w, lane);
    // dV = T^T X, times T's scale
    f32x4 e[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int a = 0; a < 4; ++a) e[u][a] = z;
    triangle(sT, xp, e, lane);
    uint4 zp[2][2][2], op[2][2][2];
    float g[2];
    {
      const float f[2] = {one(kRevIT) * ix[0], one(kRevIT) * ix[1]};
      if constexpr (!SEG) {
        f32x4* const d = reinterpret_cast<f32x4*>(p.hws + cu * (DV * kC)) +
                         512 * (NW * grp + w) + 4 * lr + (3 - lq);
        const auto rs = rows_of(p.dv, c, min(kC, sq.len - c * kC));
        float m = 0.f;
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const f32x4 x0 = f[0] * e[0][a], x1 = f[1] * e[1][a];
          m = max4abs(max4abs(m, x0), x1);
          d[128 * (3 - a)] = back(x0);
          d[128 * (3 - a) + 64] = back(x1);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            store_columns<NP, true>(rs, os, lq, row0 * kIo, 4 * a + i, x0[i], x1[i]);
        }
        static_assert(kMaxV == kMaxD + 1 && kMaxO == kMaxD + 2, "");
        note_max<3>(p.gates + (cu * p.gate_rows + kRevOne) * kC + kMaxD,
                    {before, m, max_bits(mo[0], mo[1])}, lane);
      }
      // gamma dV and gamma dO, negative
      f32x4 od[2][4];
      float mz[2] = {0.f, 0.f}, md[2] = {0.f, 0.f};
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 ng = gate(kRevZ, a);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          mz[u] = max4abs(mz[u], e[u][a] *= ng);
          md[u] = max4abs(md[u], od[u][a] = v.tile(a, u) * ng);
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float cz = f[u] * one(kRevK), co = -p.scale * one(kRevQ);
        g[u] = s.make_room(u, one(kRevG),
                           max_over_rows(mz[u]) * cz + max_over_rows(md[u]) * fabsf(co));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // (back to front within fours, the order of the update's column operands)
          parts8<2>(back(e[u][2 * h]), back(e[u][2 * h + 1]), cz * s.sc[u], zp[u][h]);
          parts8<2>(back(od[u][2 * h]), back(od[u][2 * h + 1]), co * s.sc[u], op[u][h]);
        }
      }
    }
    __syncthreads();  // all have read T, P and the gates
    if (more) {
      load_tp(c - 1);
      load_v(c - 1);
    }
    // S^T <- S^T diag(g) - K^T (gamma dV) + Q^T (scale gamma dO)
    {
      constexpr int NB = DK / 16, NG = NB < 4 ? NB : 4;
      // slots 0..3 of a column operand are the walk's rows 32 h + 4 lq + 3 - i, the tile's
      // rows 60 - 32 h - 4 lq + i
      const int tb = Swz<DK>::off(12 - 4 * lq + (lr >> 2), lr & 3);
      auto col = [&](const Swz<DK>& t, int b, int h) {
        const uint2 x = lds_tr4(t.template at<uint16_t>(tb, b, KR * (3 - 2 * h)));
        const uint2 x2 = lds_tr4(t.template at<uint16_t>(tb, b, KR * (2 - 2 * h)));
        return make_uint4(x.x, x.y, x2.x, x2.y);
      };
#pragma unroll
      for (int b0 = 0; b0 < NB; b0 += NG) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int b = 0; b < NG; ++b) s.st[u][b0 + b] *= g[u];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 kt[NG][NP];
          auto add = [&](const Swz<DK>* T, const uint4 (&x)[2][2][2]) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < NG; ++b)
#pragma unroll
              for (int i = 0; i < NP; ++i) kt[b][i] = col(T[i], b0 + b, h);
            for_products<NP, 2>([&](int i, int j) {
#pragma unroll
              for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int b = 0; b < NG; ++b)
                  s.st[u][b0 + b] = mfma_f16(kt[b][i], x[u][h][j], s.st[u][b0 + b]);
            });
          };
          add(K, zp);
          add(sQ, op);
        }
      }
    }
  }
  if (SEG && ident)
    store_matrix<DK>(s, reinterpret_cast<SegmentMatrix<DK>*>(p.sega) + su, NW * grp + w, lane);
  else if (SEG)
    s.store(p.segs + su * (DV * DK) + rows);
  else if (p.ds_out && sg.j + 1 == sg.nseg)
    s.store(p.ds_out + (long(sg.n) * p.HV + hv) * (DV * DK) + rows);
}

template <int DK, int DV, int NP>
hipError_t run(const DeltaShape& s, const DeltaParams& p, hipStream_t st) {
  constexpr int NW = kChainWaves<DV>, GB = DV / (32 * NW), GA = DK / (32 * NW);
  const unsigned units = unsigned(p.seg_slots) * unsigned(p.HV);
  if (p.sega) {
    delta_reverse_kernel<DK, DV, NP, true><<<units * (GB + GA), 64 * NW, 0, st>>>(p);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = launch_delta_combine(s, p, st);
    if (e != hipSuccess) return e;
  }
  delta_reverse_kernel<DK, DV, NP, false><<<units * GB, 64 * NW, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_reverse(const DeltaShape& s, const DeltaParams& p, hipStream_t st) {
#define ONELA_DELTA_REVERSE(DK, DV, NP) \
  if (s.dk == DK && s.dv == DV && s.bf16 == (NP == 1)) return run<DK, DV, NP>(s, p, st);
  ONELA_DELTA_REVERSE(32, 32, 1)
  ONELA_DELTA_REVERSE(64, 64, 1)
  ONELA_DELTA_REVERSE(128, 128, 1)
  ONELA_DELTA_REVERSE(128, 256, 1)
  ONELA_DELTA_REVERSE(128, 512, 1)
  ONELA_DELTA_REVERSE(256, 256, 1)
  ONELA_DELTA_REVERSE(256, 512, 1)
  ONELA_DELTA_REVERSE(32, 32, 2)
  ONELA_DELTA_REVERSE(64, 64, 2)
  ONELA_DELTA_REVERSE(128, 128, 2)
#undef ONELA_DELTA_REVERSE
  return hipErrorInvalidValue;
}

}  // namespace onela
