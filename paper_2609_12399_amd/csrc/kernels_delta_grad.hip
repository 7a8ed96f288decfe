// The delta rule's gradients, chunk by chunk (see kernels_delta.hip).
#include "delta_tiles.h"

namespace onela {
namespace {

constexpr int kNB = 32;  // columns of the values taken at a time

// 64 rows of 64 fp16 elements that are written in pieces of 4 and read by rows (padded by 8
// bytes: 16 rows' pieces in 16 different places of the 128-byte bank row).
struct Square {
  uint16_t x[kC][kC + 4];
};

// The lower triangle's tile x (of 10): row block a, column block b <= a.
__device__ inline void tile_of(int x, int& a, int& b) {
  a = (x >= 1) + (x >= 3) + (x >= 6);
  b = x - a * (a + 1) / 2;
}

// [columns][tokens], only read transposed.
using Columns32 = Swz<kC, kNB, 15>;

template <int NP>
struct GradStage {
  Columns32 e[2], dv[2];           // two parts
  uint16_t dO[NP][kC][kNB + 4];   // [tokens][columns]
};

template <int DK, int NP>
struct GradLds {
  Swz<DK> K[NP], Q[NP];
  union {
    GradStage<NP> s[2];
    struct {
      Square l[2], lt[2], m[2];  // L, its transpose, M + M^T
    } p;
  };
  alignas(16) float gates[kGateStage][kC];
  float dots[8][3][kC];    // per wave: q . (dO S), k . (dV S), k . (e dS)
  float zrow[4][kC];       // sums of Z over a column block
  float zcol[4][kC], bcol[4][kC];  // sums over a row block: Z; P X - B N
  float ss[8], most[8];
};

// A lane's place that the compiler has not seen before: what is addressed by it is formed where
// it is used, and not held in registers throughout the loops before.
struct Lane {
  int lr, lq;
};
__device__ inline Lane unseen(int lane) {
  asm("" : "+v"(lane));
  return {lane & 15, lane >> 4};
}

// Gradients of one chunk and one query/key head (the value heads of its group in
// turn, their dQ and dK summed in registers).  Wave w holds the key columns 16 CT w ..
// of dQ and dK; the tiles of the token by token products are dealt out to the waves.
// The values' columns come 32 at a time, e, dV and dO through LDS (the next ones
// requested a block ahead), the states' rows straight into operands.
//   Bound: latency of its phases, one workgroup per compute unit (256 registers, 86 KB of LDS
// at d_k = 128).  The registers do not hold all of it: the compiler spills 10 at d_k = 128 (fp32 19),
// 175 at 256.  16 x 1024 tokens x 32 heads of 128 take 0.82 ms (2.5 TB/s; matrix
// cores 11% busy, vector units 31%); per chunk and head the four column blocks are 13 us, near
// the rate at which their states can arrive, and the products of tokens with tokens, the
// rows' sums and the last products with Q and K another 13, no part above 2.  Writing L and
// M + M^T both ways or reading them transposed, and the next head's gates ahead of its
// first block, measured the same; non-temporal loads of the states 2% slower.
template <int DK, int NP, int NW>
__global__ __launch_bounds__(64 * NW, 1) void delta_grad_kernel(DeltaParams p) {
  constexpr int TH = 64 * NW, CT = DK / (16 * NW), MT = (10 + NW - 1) / NW;
  constexpr int kIo = NP == 1 ? 2 : 4;
  constexpr int kImage = sizeof(Swz<DK>) * NP;
  using Lds = GradLds<DK, NP>;
  extern __shared__ __align__(16) unsigned char smem[];
  Lds& sh = *reinterpret_cast<Lds*>(smem);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const long slot = blockIdx.x / p.HK;
  const int hk = int(blockIdx.x - slot * p.HK), G = p.HV / p.HK;
  const Chunk ch = chunk_of(p, slot);
  if (ch.n <= 0) return;
  const unsigned os = unsigned(p.HV) * p.DV * kIo;
  dma<kImage, NW>(p.kimg + (slot * p.HK + hk) * (kImage / 16), sh.K, w, lane);
  dma<kImage, NW>(p.qimg + (slot * p.HK + hk) * (kImage / 16), sh.Q, w, lane);
  const int eb = Columns32::off(4 * lq + (lr >> 2), lr & 3);
  constexpr int KR = 32 * Swz<DK>::LD;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};
  f32x4 aq[4][CT], ak[4][CT];  // dQ, dK(t = 16 a + 4 lq + i, 16 (CT w + c) + lr)
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int c = 0; c < CT; ++c) aq[a][c] = ak[a][c] = z;
  const int blocks = p.DV / kNB;

  // the next 32 columns of the values: e and dV, dO, and this lane's operands of the
  // states, S(n, k = 16 (CT w + c) + lr) at the places n0 + 4 lq + i and n0 + 16 + 4 lq + i
  // (place 16 u + m of 32 columns is column 2 m + u, the order in which the chains leave them)
  constexpr int NE = kNB * kC / 4 / TH, NO = (kC * kNB / 8 + TH - 1) / TH;
  f32x4 re[NE], rd[NE], s0[CT][2], d0[CT][2];
  u32x4 ro[NO][NP];
  auto load = [&](long cu, int hv, int nb) __attribute__((always_inline)) {
    const int n0 = nb * kNB;
    const auto er = buffer(p.ews + cu * (p.DV * kC), p.DV * (kC * 4)),
               vr = buffer(p.hws + cu * (p.DV * kC), p.DV * (kC * 4));
#pragma unroll
    for (int q = 0; q < NE; ++q) {
      const unsigned so = unsigned(n0) * (kC * 4) + q * TH * 16;
      re[q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(er, tid * 16, so, 0));
      rd[q] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(vr, tid * 16, so, 0));
    }
    const auto rs = rows_buffer(p.d_o, ((ch.t0 * p.HV + hv) * p.DV + n0) * kIo, kNB * kIo, os, ch.n);
#pragma unroll
    for (int q = 0; q < NO; ++q) {
      const int e = tid + q * TH;
      if (NO * TH > kC * kNB / 8 && e >= kC * kNB / 8) break;
#pragma unroll
      for (int i = 0; i < NP; ++i)
        ro[q][i] = __builtin_amdgcn_raw_buffer_load_b128(
            rs, unsigned(e / (kNB / 8)) * os + (e % (kNB / 8)) * (8 * kIo) + 16 * i, 0, 0);
    }
    const auto sr = buffer(p.sws + cu * (p.DV * DK), p.DV * (DK * 4)),
               dr = buffer(p.dsws + cu * (p.DV * DK), p.DV * (DK * 4));
    const unsigned at = unsigned(16 * CT * w * p.DV + 64 * lq + lr) * 4;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned so = unsigned(c * p.DV + n0 + 16 * u + i) * 64;
          s0[c][u][i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sr, at, so, 0));
          d0[c][u][i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(dr, at, so, 0));
        }
  };

  load(slot * p.HV + hk * G, hk * G, 0);
  for (int hg = 0; hg < G; ++hg) {
    const int hv = hk * G + hg;
    const long cu = slot * p.HV + hv;
    if (hg > 0) __syncthreads();  // (the last head's readers are done)
    int at0 = tid;
    asm("" : "+v"(at0));
    for (int i = at0; i < kGateStage * kC; i += TH)
      (&sh.gates[0][0])[i] = p.gates[(cu * p.gate_rows + kGateStage) * kC + i];
    auto gate = [&](int row) { return sh.gates[row - kGateStage]; };
    // scales, from the bounds that the chains left (the same for every lane)
    float sS, sD, sE, sV, sO;
    {
      const float* one = p.gates + (cu * p.gate_rows + kRevOne) * kC;
      sS = scale_for(one[kMaxS]);
      sD = scale_for(one[kMaxD]);
      sE = scale_for(one[kMaxE]);
      sV = scale_for(one[kMaxV]);
      sO = scale_for(one[kMaxO]);
    }
    f32x4 xs[MT], ns[MT];  // tiles of X = dO e^T and N = dV e^T
#pragma unroll
    for (int m = 0; m < MT; ++m) xs[m] = ns[m] = z;
    f32x4 qS[4][CT], kS[4][CT], eD[4][CT];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int c = 0; c < CT; ++c) qS[a][c] = kS[a][c] = eD[a][c] = z;
    float ss = 0.f;
    for (int nb = 0; nb < blocks; ++nb) {
      GradStage<NP>& x = sh.s[nb & 1];
      // (this buffer's last readers passed the barrier of the block before)
#pragma unroll
      for (int q = 0; q < NE; ++q) {
        const int e = tid + q * TH, o = Columns32::off(e / 4 % 32, e / 128 * 4 + e % 4);
        unsigned u[2], v[2];
        auto put = [&](const f32x4& y, float s, Columns32* to) {
          parts2<2>(y.x, y.y, s, u);
          parts2<2>(y.z, y.w, s, v);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            *reinterpret_cast<uint2*>(reinterpret_cast<char*>(to[i].x) + o) = make_uint2(u[i], v[i]);
        };
        put(re[q], sE, x.e);
        put(rd[q], sV, x.dv);
      }
#pragma unroll
      for (int q = 0; q < NO; ++q) {
        const int e = tid + q * TH;
        if (NO * TH > kC * kNB / 8 && e >= kC * kNB / 8) break;
        f32x4 y0, y1;
        if constexpr (NP == 1) {
          const u32x4 y = ro[q][0];
          y0 = f32x4{bf16_lo_to_float(y.x), bf16_hi_to_float(y.x), bf16_lo_to_float(y.y),
                     bf16_hi_to_float(y.y)};
          y1 = f32x4{bf16_lo_to_float(y.z), bf16_hi_to_float(y.z), bf16_lo_to_float(y.w),
                     bf16_hi_to_float(y.w)};
        } else {
          y0 = __builtin_bit_cast(f32x4, ro[q][0]);
          y1 = __builtin_bit_cast(f32x4, ro[q][1]);
        }
        uint4 part[NP];  // even columns and odd ones
        parts8<NP>(f32x4{y0.x, y0.z, y1.x, y1.z}, f32x4{y0.y, y0.w, y1.y, y1.w}, sO, part);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          uint16_t* const to = &x.dO[i][e / (kNB / 8)][4 * (e % (kNB / 8))];
          *reinterpret_cast<uint2*>(to) = make_uint2(part[i].x, part[i].y);
          *reinterpret_cast<uint2*>(to + 16) = make_uint2(part[i].z, part[i].w);
        }
      }
      uint4 sp[CT][2], dp[CT][2];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        parts8<2>(s0[c][0], s0[c][1], sS, sp[c]);
        parts8<2>(d0[c][0], d0[c][1], sD, dp[c]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) ss = fmaf(s0[c][u][i], d0[c][u][i], ss);
      }
      if (nb + 1 < blocks)
        load(cu, hv, nb + 1);
      else if (hg + 1 < G)
        load(cu + 1, hv + 1, 0);
      if (hg == 0 && nb == 0) __builtin_amdgcn_s_waitcnt(0x0f70);  // keys and queries
      __syncthreads();
      auto of = [&](int i, int a) {
        const uint16_t* r = x.dO[i][16 * a + lr] + 4 * lq;
        const uint2 y0 = *reinterpret_cast<const uint2*>(r),
                    y1 = *reinterpret_cast<const uint2*>(r + 16);
        return make_uint4(y0.x, y0.y, y1.x, y1.y);
      };
      // X and N
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int t = w + m * NW;
        if (t >= 10) break;
        int a, b;
        tile_of(t, a, b);
        uint4 ef[2], df[2], og[NP];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ef[i] = col_frag(x.e[i], eb, b, 0);
          df[i] = col_frag(x.dv[i], eb, a, 0);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) og[i] = of(i, a);
        for_products<NP, 2>([&](int i, int j) { xs[m] = mfma_f16(og[i], ef[j], xs[m]); });
        for_products<2, 2>([&](int i, int j) { ns[m] = mfma_f16(df[i], ef[j], ns[m]); });
      }
      // products with the states
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        uint4 ef[2], df[2], og[NP];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ef[i] = col_frag(x.e[i], eb, a, 0);
          df[i] = col_frag(x.dv[i], eb, a, 0);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) og[i] = of(i, a);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          for_products<2, 2>([&](int i, int j) {
            kS[a][c] = mfma_f16(df[i], sp[c][j], kS[a][c]);
            eD[a][c] = mfma_f16(ef[i], dp[c][j], eD[a][c]);
          });
          for_products<NP, 2>([&](int i, int j) { qS[a][c] = mfma_f16(og[i], sp[c][j], qS[a][c]); });
        }
      }
    }
    // rows' dot products with q and k, and the parts of dQ and dK from the states
    ss = group_sum<64>(ss);
    if (lane == 0) sh.ss[w] = ss;
    const float ik = gate(kRevOne)[kRevK], iq = gate(kRevOne)[kRevQ];
    {
      const Lane l = unseen(lane);
      const int lr = l.lr, lq = l.lq, tb = Swz<DK>::off(4 * lq + (lr >> 2), lr & 3);
      const float iS = inverse_pow2(sS), iV = inverse_pow2(sV), iE = inverse_pow2(sE),
                  iO = inverse_pow2(sO), iD = inverse_pow2(sD);
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int t0 = 16 * a + 4 * lq;
        const f32x4 ga = *reinterpret_cast<const f32x4*>(&gate(kRevZ)[t0]);
        const f32x4 gb = *reinterpret_cast<const f32x4*>(&gate(kRevBS)[t0]);
        f32x4 dots[3] = {z, z, z};
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          qS[a][c] *= iO * iS;
          kS[a][c] *= iV * iS;
          eD[a][c] *= iE * iD;
          // q and k of this lane's tokens and column: a transposed read gives all four
          f32x4 qv = z, kv = z;
#pragma unroll
          for (int u = NP - 1; u >= 0; --u) {
            auto four = [&](const Swz<DK>& t) {
              const uint2 x = lds_tr4(t.template at<uint16_t>(tb, CT * w + c, KR * a));
              const half2v lo = __builtin_bit_cast(half2v, x.x), hi = __builtin_bit_cast(half2v, x.y);
              return f32x4{float(lo.x), float(lo.y), float(hi.x), float(hi.y)};
            };
            qv += four(sh.Q[u]);
            kv += four(sh.K[u]);
          }
          dots[0] += qv * qS[a][c];
          dots[1] += kv * kS[a][c];
          dots[2] += kv * eD[a][c];
          aq[a][c] += (-p.scale * ga) * qS[a][c];
          ak[a][c] += gb * eD[a][c] + ga * kS[a][c];
        }
        // lane lr keeps the sum lr = 4 u + i of the 16 lanes
        float mine = 0.f;
#pragma unroll
        for (int u = 0; u < 3; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float s = group_sum<16>(dots[u][i]);
            mine = lr == 4 * u + i ? s : mine;
          }
        if (lr < 12) sh.dots[w][lr >> 2][t0 + (lr & 3)] = mine * (lr < 4 ? iq : ik);
      }
    }
    // the tiles of L and M and their sums
    f32x4 lt[MT], mt[MT];
    float most = 0.f;
    const float ix = inverse_pow2(sO) * inverse_pow2(sE), in = inverse_pow2(sV) * inverse_pow2(sE);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int x = w + m * NW;
      if (x >= 10) break;
      const Lane l = unseen(lane);
      const int lr = l.lr, lq = l.lq, kb = Swz<DK>::off(lr, lq);
      int a, b;
      tile_of(x, a, b);
      f32x4 qk = z, kk = z;
#pragma unroll
      for (int h = 0; h < DK / 32; ++h) {
        uint4 qf[NP], ka[NP], kf[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          qf[i] = row_frag(sh.Q[i], kb, Steps<DK>::t0(h), Steps<DK>::t0(h) + Steps<DK>::PS, KR * a);
          ka[i] = row_frag(sh.K[i], kb, Steps<DK>::t0(h), Steps<DK>::t0(h) + Steps<DK>::PS, KR * a);
          kf[i] = row_frag(sh.K[i], kb, Steps<DK>::t0(h), Steps<DK>::t0(h) + Steps<DK>::PS, KR * b);
        }
        for_products<NP, NP>([&](int i, int j) {
          qk = mfma_f16(qf[i], kf[j], qk);
          kk = mfma_f16(ka[i], kf[j], kk);
        });
      }
      qk *= iq * ik;
      kk *= ik * ik;
      const int j = 16 * b + lr;
      const float hj = gate(kRevHi)[j], lj = gate(kRevLo)[j], bj = gate(kRevBeta)[j];
      float cz = 0.f, cb = 0.f, mine = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = 16 * a + 4 * lq + q;
        const float d = (gate(kRevHi)[i] - hj) + (gate(kRevLo)[i] - lj);
        const float g = j <= i ? exp2_fast(d) : 0.f, gs = j < i ? g : 0.f;
        const float px = p.scale * g * (xs[m][q] * ix), nx = gs * (ns[m][q] * in);
        lt[m][q] = px * bj;
        mt[m][q] = -nx * bj;
        const float zz = j < i ? lt[m][q] * qk[q] + mt[m][q] * kk[q] : 0.f;
        cb += px * qk[q] - nx * kk[q];
        cz += zz;
        const float rz = group_sum<16>(zz);
        mine = lr == q ? rz : mine;
      }
      if (lr < 4) sh.zrow[b][16 * a + 4 * lq + lr] = mine;
      most = max4abs(max4abs(most, lt[m]), mt[m]);
      cz = sum_over_rows(cz);
      cb = sum_over_rows(cb);
      if (lq == 0) {
        sh.zcol[a][j] = cz;
        sh.bcol[a][j] = cb;
      }
    }
    most = wave_max(most);
    if (lane == 0) sh.most[w] = most;
    lds_barrier();  // (all have read the last columns)
#pragma unroll
    for (int i = 0; i < NW; ++i) most = fmaxf(most, sh.most[i]);
    const float sl = scale_for(most);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int x = w + m * NW;
      if (x >= 10) break;
      const Lane ln = unseen(lane);
      const int lr = ln.lr, lq = ln.lq;
      int a, b;
      tile_of(x, a, b);
      unsigned l0[2], l1[2], m0[2], m1[2];
      parts2<2>(lt[m].x, lt[m].y, sl, l0);
      parts2<2>(lt[m].z, lt[m].w, sl, l1);
      parts2<2>(mt[m].x, mt[m].y, sl, m0);
      parts2<2>(mt[m].z, mt[m].w, sl, m1);
      const int r0 = 16 * a + 4 * lq, cc = 16 * b + lr;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint16_t le[4] = {uint16_t(l0[i]), uint16_t(l0[i] >> 16), uint16_t(l1[i]),
                                uint16_t(l1[i] >> 16)};
        const uint16_t me[4] = {uint16_t(m0[i]), uint16_t(m0[i] >> 16), uint16_t(m1[i]),
                                uint16_t(m1[i] >> 16)};
        *reinterpret_cast<uint2*>(&sh.p.lt[i].x[cc][r0]) = make_uint2(l0[i], l1[i]);
        if (a != b) *reinterpret_cast<uint2*>(&sh.p.m[i].x[cc][r0]) = make_uint2(m0[i], m1[i]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          sh.p.l[i].x[r0 + q][cc] = le[q];
          if (a != b) {
            sh.p.m[i].x[r0 + q][cc] = me[q];
          } else if (cc <= r0 + q) {  // both triangles of a diagonal block
            sh.p.m[i].x[r0 + q][cc] = me[q];
            sh.p.m[i].x[cc][r0 + q] = me[q];
          }
        }
      }
    }
    // the blocks past the diagonal that a 32-deep step covers: (0, 1), (2, 3) of L, (1, 0),
    // (3, 2) of its transpose
    for (int e = tid; e < 8 * 64; e += TH) {
      const int i = e >> 8, tr = (e >> 7) & 1, a = 2 * ((e >> 6) & 1), l = e & 63;
      const int r = 16 * (tr ? a + 1 : a) + (l & 15), c = 16 * (tr ? a : a + 1) + 4 * (l >> 4);
      *reinterpret_cast<uint2*>(&(tr ? sh.p.lt : sh.p.l)[i].x[r][c]) = make_uint2(0u, 0u);
    }
    lds_barrier();
    // dQ += L K, dK += L^T Q + (M + M^T) K
    {
      const float il = inverse_pow2(sl);
      const Lane l = unseen(lane);
      const int lr = l.lr, lq = l.lq, tb = Swz<DK>::off(4 * lq + (lr >> 2), lr & 3);
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        f32x4 x0[CT], x1[CT], x2[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) x0[c] = x1[c] = x2[c] = z;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          auto sq = [&](const Square& t) {
            const uint16_t* r = t.x[16 * a + lr] + 32 * h + 4 * lq;
            const uint2 y0 = *reinterpret_cast<const uint2*>(r),
                        y1 = *reinterpret_cast<const uint2*>(r + 16);
            return make_uint4(y0.x, y0.y, y1.x, y1.y);
          };
          uint4 lf[2], tf[2], mf[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (a >= 2 * h) lf[i] = sq(sh.p.l[i]);       // L: columns up to the row
            if (a < 2 * h + 2) tf[i] = sq(sh.p.lt[i]);   // L^T: columns from the row on
            mf[i] = sq(sh.p.m[i]);
          }
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            uint4 kf[NP], qf[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
              kf[i] = col_frag(sh.K[i], tb, CT * w + c, 2 * KR * h);
              qf[i] = col_frag(sh.Q[i], tb, CT * w + c, 2 * KR * h);
            }
            for_products<2, NP>([&](int i, int j) {
              if (a >= 2 * h) x0[c] = mfma_f16(lf[i], kf[j], x0[c]);
              if (a < 2 * h + 2) x1[c] = mfma_f16(tf[i], qf[j], x1[c]);
              x2[c] = mfma_f16(mf[i], kf[j], x2[c]);
            });
          }
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          aq[a][c] += (il * ik) * x0[c];
          ak[a][c] += (il * iq) * x1[c] + (il * ik) * x2[c];
        }
      }
    }
    // dbeta and dlog_alpha (the dot products and sums passed the barriers above)
    if (w == 0) {
      int t = lane;
      asm("" : "+v"(t));
      float dt[3] = {0.f, 0.f, 0.f};
      for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int u = 0; u < 3; ++u) dt[u] += sh.dots[i][u][t];
      float zr = 0.f, zc = 0.f, bc = 0.f, all = 0.f;
      const int blk = t >> 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i <= blk) zr += sh.zrow[i][t];
        if (i >= blk) {
          zc += sh.zcol[i][t];
          bc += sh.bcol[i][t];
        }
      }
      for (int i = 0; i < NW; ++i) all += sh.ss[i];
      const float gam = -gate(kRevZ)[t], bs = gate(kRevBS)[t];
      const float sg = exp2_fast((gate(kRevHi)[63] - gate(kRevHi)[t]) +
                                 (gate(kRevLo)[63] - gate(kRevLo)[t]));
      const float kd = bs * dt[2];
      float suf = gam * (p.scale * dt[0] - dt[1]) + (zr - zc) - kd;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {  // sums from t to the end
        const float u = __shfl_down(suf, d);
        if (t + d < 64) suf += u;
      }
      const float last = __shfl(gam, 63) * all + group_sum<64>(kd);
      if (t < ch.n) {
        const long at = (ch.t0 + t) * p.HV + hv;
        p.db[at] = fmaf(sg, dt[2], bc);
        p.dla[at] = p.la[at] < -1e5f ? 0.f : suf + last;
      }
    }
  }
  // (buffers that end with the last token: stores past it are dropped)
  const unsigned ds = unsigned(p.HK) * (DK * kIo);
  const long first = (ch.t0 * p.HK + hk) * (DK * kIo);
  const auto qr = rows_buffer(p.dq, first, DK * kIo, ds, ch.n),
             kr = rows_buffer(p.dk, first, DK * kIo, ds, ch.n);
  const Lane l = unseen(lane);
  const unsigned at = unsigned(4 * l.lq) * ds + (16 * CT * w + l.lr) * kIo;
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const unsigned so = unsigned(16 * a + i) * ds + 16 * c * kIo;
        if constexpr (NP == 1) {
          const unsigned u = pack_bf16x2(aq[a][c][i], ak[a][c][i]);
          __builtin_amdgcn_raw_buffer_store_b16(uint16_t(u), qr, at, so, 0);
          __builtin_amdgcn_raw_buffer_store_b16(uint16_t(u >> 16), kr, at, so, 0);
        } else {
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(aq[a][c][i]), qr, at, so, 0);
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(ak[a][c][i]), kr, at, so, 0);
        }
      }
}

template <int DK, int NP>
hipError_t run(const DeltaParams& p, hipStream_t st) {
  constexpr int NW = DK / 16 < 8 ? DK / 16 : 8;
  auto grad = delta_grad_kernel<DK, NP, NW>;
  constexpr size_t lds = sizeof(GradLds<DK, NP>);
  static_assert(lds <= 160 * 1024, "one workgroup's LDS");
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(grad),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
  if (e != hipSuccess) return e;
  grad<<<unsigned(p.slots) * unsigned(p.HK), 64 * NW, lds, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_grad(const DeltaShape& s, const DeltaParams& p, hipStream_t st) {
  if (!p.slots) return hipSuccess;
#define ONELA_DELTA_GRAD(DK, NP) \
  if (s.dk == DK && s.bf16 == (NP == 1)) return run<DK, NP>(p, st);
  ONELA_DELTA_GRAD(32, 1)
  ONELA_DELTA_GRAD(64, 1)
  ONELA_DELTA_GRAD(128, 1)
  ONELA_DELTA_GRAD(256, 1)
  ONELA_DELTA_GRAD(32, 2)
  ONELA_DELTA_GRAD(64, 2)
  ONELA_DELTA_GRAD(128, 2)
#undef ONELA_DELTA_GRAD
  return hipErrorInvalidValue;
}

}  // namespace onela
