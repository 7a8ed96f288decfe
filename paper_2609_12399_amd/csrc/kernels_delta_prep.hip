// The delta rule's chunks, first launch (see kernels_delta.hip): what the chain over the
// chunks needs of each and that no chunk needs of another.
#include "delta_tiles.h"

namespace onela {
namespace {

constexpr int kThreads = 256;

// 8-element pieces of rows [64][DK] of one head on their way: the tensor's own bits.
template <int DK, int NP>
struct Pieces {
  static constexpr int NV = (kC * DK / 8) / kThreads;
  u32x4 r[NV][NP];
  __device__ void load(const void* base, long at, long stride, int n, int tid) {
    constexpr int kIo = NP == 1 ? 2 : 4;
    const unsigned st = unsigned(stride) * kIo;
    const auto rs = rows_buffer(base, at * kIo, DK * kIo, st, n);
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int e = tid + q * kThreads;
      const unsigned o = unsigned(e / (DK / 8)) * st + (e % (DK / 8)) * (8 * kIo);
#pragma unroll
      for (int i = 0; i < NP; ++i)
        r[q][i] = __builtin_amdgcn_raw_buffer_load_b128(rs, o + 16 * i, 0, 0);
    }
  }
  // largest magnitude of this thread's elements
  __device__ float largest() const {
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    if constexpr (NP == 1) {
      us2 m = {0, 0};
#pragma unroll
      for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          m = __builtin_elementwise_max(m, __builtin_bit_cast(us2, r[q][0][j] & 0x7fff7fffu));
      return __uint_as_float(unsigned(max(m.x, m.y)) << 16);
    } else {
      unsigned m = 0;
#pragma unroll
      for (int q = 0; q < NV; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, r[q][j >> 2][j & 3] & 0x7fffffffu);
      return __uint_as_float(m);
    }
  }
  // the elements times s as fp16 parts into LDS tiles
  template <typename Tile>
  __device__ void store(Tile* tile, float s, int tid) const {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int e = tid + q * kThreads;
      f32x4 x, y;
      if constexpr (NP == 1) {
        const u32x4 v = r[q][0];
        x = f32x4{bf16_lo_to_float(v.x), bf16_hi_to_float(v.x), bf16_lo_to_float(v.y),
                  bf16_hi_to_float(v.y)};
        y = f32x4{bf16_lo_to_float(v.z), bf16_hi_to_float(v.z), bf16_lo_to_float(v.w),
                  bf16_hi_to_float(v.w)};
      } else {
        x = __builtin_bit_cast(f32x4, r[q][0]);
        y = __builtin_bit_cast(f32x4, r[q][1]);
      }
      uint4 p[NP];
      parts8<NP>(x, y, s, p);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        tile[i].put(e / (DK / 8), e % (DK / 8), __builtin_bit_cast(u32x4, p[i]));
      }
    }
  }
};

template <int DK, int NP>
struct PrepLds {
  struct KQ {
    Swz<DK> K[NP], Q[NP];  // fp16 parts
  };
  struct MT {
    float T[kC][kC + 4];
    float M[kC][kC + 4];  // B diag(beta); its diagonal blocks then hold those of T
  };
  union {
    KQ kq;
    MT mt;  // after the products of keys and queries
  };
  alignas(16) float gh[kC], gl[kC];          // sums of log2(alpha) as hi + lo
  alignas(16) float be[kC], bs[kC], ip[kC];  // beta, beta sigma, inverse scales of P's rows
  float most[4][4];  // per wave: the largest key, query, element of T, row sum of it
};

// Zeros in rows of `width` bytes, `stride` bytes apart.
__device__ inline void clear_rows(void* base, long rows, unsigned width, long stride) {
  const unsigned pieces = width / 16;
  for (long i = threadIdx.x; i < rows * pieces; i += kThreads) {
    const long r = i / pieces;
    *reinterpret_cast<uint4*>(static_cast<char*>(base) + r * stride + (i - r * pieces) * 16) =
        make_uint4(0, 0, 0, 0);
  }
}

// The rows behind the last sequence, of 64 tokens and a value head (slots are 64 tokens each at
// least, whatever sequences' chunks they hold): outputs, or gradients.
template <int DK, int NP, bool BWD>
__device__ inline void clear_rest(const DeltaParams& p, long slot, int hv) {
  constexpr int kIo = NP == 1 ? 2 : 4;
  const Seq last = seq_of(p, p.N - 1);
  const long b = max(slot * kC, last.t0 + last.len), n = min(slot * kC + kC, p.total) - b;
  if (n <= 0) return;
  const unsigned width = unsigned(p.DV) * kIo;
  const long at = b * p.HV + hv;
  clear_rows(static_cast<char*>(BWD ? p.dv : p.o) + at * width, n, width, long(p.HV) * width);
  if constexpr (BWD) {
    const int G = p.HV / p.HK;
    if (hv % G == 0) {
      const long row = (b * p.HK + hv / G) * (DK * kIo), stride = long(p.HK) * (DK * kIo);
      clear_rows(static_cast<char*>(p.dq) + row, n, DK * kIo, stride);
      clear_rows(static_cast<char*>(p.dk) + row, n, DK * kIo, stride);
    }
    if (threadIdx.x < n) p.dla[at + long(threadIdx.x) * p.HV] = p.db[at + long(threadIdx.x) * p.HV] = 0.f;
  }
}

// One chunk of one value head: the fp16 images of its keys and queries, T = (I + B
// diag(beta))^-1 and P in the fragment order of the chain, and the gates; for the backward
// pass, in P's place, T and P transposed with their tokens in reverse order.  Four waves.
//   The inverse goes by 16-token blocks: the four diagonal blocks by forward
// substitution, one per wave with a column per lane, then each wave the blocks below
// the diagonal block of its block column, T_ij = -T_ii sum_k M_ik T_kj, in fp32 matrix
// instructions with T_kj in the accumulator layout as the next operand.
//   Bound: HBM for many chunks, mostly what it leaves for the chain: 8192 chunks and value heads
// of 128 (two to a key head) take 106 us, 4.7 TB/s; for few the latency of the inverse.  Vector
// units 57% busy at four workgroups per compute unit, to which the LDS (36 KB up to d_k
// = 128) and the registers are held.  With decays from 64-bit differences behind branches 7%
// more, with operands whose pieces no one read fetches 3%.
template <int DK, int NP, bool BWD>
__global__ __launch_bounds__(kThreads, DK * NP >= 256 ? 2 : 4) void delta_prep_kernel(DeltaParams p) {
  __shared__ __align__(16) PrepLds<DK, NP> sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const long slot = blockIdx.x / p.HV;
  const int hv = int(blockIdx.x - slot * p.HV), G = p.HV / p.HK, hk = hv / G;
  const Chunk ch = chunk_of(p, slot);
  if (p.clear) clear_rest<DK, NP, BWD>(p, slot, hv);
  if (ch.n <= 0) return;
  const long cu = long(blockIdx.x);
  float* const gt = p.gates + cu * (p.gate_rows * kC);
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};
  float sk, sq;
  {
    Pieces<DK, NP> rk, rq;
    rk.load(p.k, ch.t0 * p.ks + hk * DK, p.ks, ch.n, tid);
    rq.load(p.q, ch.t0 * p.qs + hk * DK, p.qs, ch.n, tid);
    if (w == 0) {  // lane t holds token t
      const long ti = (ch.t0 + min(lane, ch.n - 1)) * p.HV + hv;
      float la = p.la[ti];
      float be = p.beta[ti];
      la = la < -1e5f ? -1e5f : la;
      double g = lane < ch.n ? double(la) * 1.4426950408889634 : 0.0;
      be = lane < ch.n ? be : 0.f;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const double u = __shfl_up(g, d);
        if (lane >= d) g += u;
      }
      sh.gh[lane] = float(g);
      sh.gl[lane] = float(g - double(float(g)));
      sh.be[lane] = be;
      sh.bs[lane] = be * exp2_fast(float(__shfl(g, 63) - g));
    }
    const float mk = wave_max(rk.largest()), mq = wave_max(rq.largest());
    if (lane == 0) {
      sh.most[w][0] = mk;
      sh.most[w][1] = mq;
    }
    lds_barrier();
    sk = scale_for_rows(fmaxf(fmaxf(sh.most[0][0], sh.most[1][0]),
                              fmaxf(sh.most[2][0], sh.most[3][0])));
    sq = scale_for_rows(fmaxf(fmaxf(sh.most[0][1], sh.most[1][1]),
                              fmaxf(sh.most[2][1], sh.most[3][1])));
    rk.store(sh.kq.K, sk, tid);
    rq.store(sh.kq.Q, sq, tid);
  }
  const float ik = inverse_pow2(sk), iq = inverse_pow2(sq);
  lds_barrier();
  if (hv == hk * G) {  // one of the group's heads keeps the images, as they stand in LDS
    constexpr int NI = sizeof(sh.kq.K) / 16;
    uint4* const ki = p.kimg + (slot * p.HK + hk) * NI;
    uint4* const qi = p.qimg + (slot * p.HK + hk) * NI;
    for (int e = tid; e < NI; e += kThreads) {
      ki[e] = reinterpret_cast<const uint4*>(sh.kq.K)[e];
      qi[e] = reinterpret_cast<const uint4*>(sh.kq.Q)[e];
    }
  }
  const int kb = Swz<DK>::off(lr, lq);
  constexpr int KR = 32 * Swz<DK>::LD;
  auto four = [&](const float* x) { return *reinterpret_cast<const f32x4*>(x); };
  // rows x of a against rows y of b, 16 each: lane (lr, lq) holds (16 a + 4 lq + i, 16 b + lr)
  // (base: the lane's first piece of row lr, or of row 15 - lr for rows in reverse order)
  auto dots = [&](const Swz<DK>* x, int a, const Swz<DK>* y, int b, int base) {
    f32x4 acc = z;
#pragma unroll
    for (int h = 0; h < DK / 32; ++h) {
      uint4 u[NP], v[NP];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        u[i] = row_frag(x[i], base, Steps<DK>::t0(h), Steps<DK>::t0(h) + Steps<DK>::PS, KR * a);
        v[i] = row_frag(y[i], base, Steps<DK>::t0(h), Steps<DK>::t0(h) + Steps<DK>::PS, KR * b);
      }
      for_products<NP, NP>([&](int i, int j) { acc = mfma_f16(u[i], v[j], acc); });
    }
    return acc;
  };
  {
    // P(t, j) = scale Gamma(t, j) (q_t . k_j) beta_j, j <= t, of 16 tokens t per wave (the
    // longer rows to the waves with fewer tiles of M): a lane holds four neighbouring j
    // of one token, half a fragment; backward of 16 tokens j and four neighbouring t
    const int pa = w == 0 ? 2 : w == 1 ? 1 : w == 2 ? 3 : 0;
    const int t = BWD ? kC - 1 - 16 * pa - lr : 16 * pa + lr;  // backward: the token j
    const float hq = sh.gh[t], lo = sh.gl[t];
    const float c = p.scale * (ik * iq) * (BWD ? sh.be[t] : 1.f);
    f32x4 x[4];
    float most = 0.f;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      x[b] = z;
      if (b > pa) continue;
      if constexpr (!BWD) {
        const f32x4 acc = dots(sh.kq.K, b, sh.kq.Q, pa, kb);
        const int j0 = 16 * b + 4 * lq;
        const f32x4 be = four(&sh.be[j0]), h = four(&sh.gh[j0]), l = four(&sh.gl[j0]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float y = c * exp2_fast((hq - h[q]) + (lo - l[q])) * be[q] * acc[q];
          x[b][q] = j0 + q <= t ? y : 0.f;
        }
      } else {
        const f32x4 acc = dots(sh.kq.Q, 3 - b, sh.kq.K, 3 - pa, Swz<DK>::off(15 - lr, lq));
        const int i0 = kC - 4 - 16 * b - 4 * lq;
        const f32x4 h = four(&sh.gh[i0]), l = four(&sh.gl[i0]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float y = c * exp2_fast((h[3 - q] - hq) + (l[3 - q] - lo)) * acc[q];
          x[b][q] = t <= i0 + 3 - q ? y : 0.f;
        }
      }
      most = max4abs(most, x[b]);
    }
    const float s = scale_for(max_over_rows(most));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h > 0 && pa < 2) break;
      const int f = pa < 2 ? pa : 2 * pa - 2 + h;
      uint4 part[2];
      parts8<2>(x[2 * h], x[2 * h + 1], s, part);
#pragma unroll
      for (int i = 0; i < 2; ++i) (BWD ? p.pr : p.pf)[(cu * 6 + f) * 128 + i * 64 + lane] = part[i];
    }
    if (lq == 0) sh.ip[t] = inverse_pow2(s);
  }
  {
    // M(i, j) = Gamma(i, j) (k_i . k_j) beta_j, 0 on and above the diagonal: the tiles (1, 0),
    // (2, 0), (2, 1), (3, 0); (3, 1), (3, 2); the diagonal block w
    f32x4 m[3];
    auto tile = [&](int a, int b) {
      f32x4 acc = dots(sh.kq.K, a, sh.kq.K, b, kb);
      const int j = 16 * b + lr, i0 = 16 * a + 4 * lq;
      const float hj = sh.gh[j], lj = sh.gl[j];
      const f32x4 h = four(&sh.gh[i0]), l = four(&sh.gl[i0]);
      const float bk = sh.be[j] * ik * ik;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float y = exp2_fast((h[q] - hj) + (l[q] - lj)) * bk * acc[q];
        acc[q] = j < i0 + q ? y : 0.f;
      }
      return acc;
    };
    const int a0 = w == 0 ? 1 : w < 3 ? 2 : 3, b0 = w == 2 ? 1 : 0;
    m[0] = tile(a0, b0);
    m[1] = tile(w, w);
    if (w < 2) m[2] = tile(3, w + 1);
    lds_barrier();  // keys and queries are not read any more: M and T take their place
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sh.mt.M[16 * a0 + 4 * lq + q][16 * b0 + lr] = m[0][q];
      sh.mt.M[16 * w + 4 * lq + q][16 * w + lr] = m[1][q];
      if (w < 2) sh.mt.M[48 + 4 * lq + q][16 * (w + 1) + lr] = m[2][q];
    }
  }
  auto& M = sh.mt.M;
  auto& T = sh.mt.T;
  f32x4 tc[4];  // blocks (w + d, w) of T, rows 4 lq + component, column lr
  {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i == lr ? 1.f : 0.f;
    // row i of the inverse from the rows before it
#pragma unroll
    for (int i = 1; i < 16; ++i) {
      f32x4 m[4];
#pragma unroll
      for (int q = 0; q < (i + 3) / 4; ++q)
        m[q] = *reinterpret_cast<const f32x4*>(&M[16 * w + i][16 * w + 4 * q]);
      float s0 = x[i], s1 = 0.f;
#pragma unroll
      for (int j = 0; j < i; ++j) {
        float& s = (j & 1) ? s1 : s0;
        s = fmaf(-m[j >> 2][j & 3], x[j], s);
      }
      x[i] = s0 + s1;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      tc[0][q] = lq == 0 ? x[q] : lq == 1 ? x[4 + q] : lq == 2 ? x[8 + q] : x[12 + q];
      M[16 * w + 4 * lq + q][16 * w + lr] = tc[0][q];
    }
  }
  lds_barrier();
#pragma unroll
  for (int d = 1; d < 4; ++d) {
    if (w + d >= 4) break;
    const int i = w + d;
    f32x4 a0 = z, a1 = z;
#pragma unroll
    for (int e = 0; e < d; ++e) {
      const f32x4 mm = *reinterpret_cast<const f32x4*>(&M[16 * i + lr][16 * (w + e) + 4 * lq]);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        f32x4& acc = (s & 1) ? a1 : a0;
        acc = mfma4(mm[s], tc[e][s], acc);
      }
    }
    const f32x4 pr = a0 + a1;
    const f32x4 tt = *reinterpret_cast<const f32x4*>(&M[16 * i + lr][16 * i + 4 * lq]);
    f32x4 b0 = z, b1 = z;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      f32x4& acc = (s & 1) ? b1 : b0;
      acc = mfma4(tt[s], pr[s], acc);
    }
    tc[d] = -(b0 + b1);
  }
  {
    float most = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      if (w + d >= 4) break;
      most = max4abs(most, tc[d]);
#pragma unroll
      for (int q = 0; q < 4; ++q) T[16 * (w + d) + 4 * lq + q][16 * w + lr] = tc[d][q];
    }
    most = wave_max(most);
    if (lane == 0) sh.most[w][2] = most;
#pragma unroll
    for (int q = 0; q < 4; ++q)  // the blocks above the diagonal that a 32-token step covers
      if (w & 1) T[16 * (w - 1) + 4 * lq + q][16 * w + lr] = 0.f;
  }
  lds_barrier();
  const float s = scale_for(fmaxf(fmaxf(sh.most[0][2], sh.most[1][2]),
                                  fmaxf(sh.most[2][2], sh.most[3][2])));
  // T fragments of row tile w: a lane holds row 16 w + lr and the columns 32 h + 4 lq +
  // 0..3 and 32 h + 16 + 4 lq + 0..3, the order in which the chain's accumulators hold
  // the tokens; transposed and reversed, rows and columns count from the chunk's end and
  // change places
  {
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h > 0 && w < 2) break;
      const int f = w < 2 ? w : 2 * w - 2 + h, t = 16 * w + lr, c0 = 32 * h + 4 * lq;
      f32x4 x[2][2];
      x[0][0] = *reinterpret_cast<const f32x4*>(&T[t][c0]);
      x[0][1] = *reinterpret_cast<const f32x4*>(&T[t][c0 + 16]);
      if constexpr (BWD)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[1][0][j] = T[kC - 1 - (c0 + j)][kC - 1 - t];
          x[1][1][j] = T[kC - 1 - (c0 + 16 + j)][kC - 1 - t];
        }
#pragma unroll
      for (int r = 0; r < (BWD ? 2 : 1); ++r) {
        uint4 part[2];
        parts8<2>(x[r][0], x[r][1], s, part);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          (r ? p.tr : p.tp)[(cu * 6 + f) * 128 + i * 64 + lane] = part[i];
      }
      if constexpr (!BWD)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += fabsf(x[0][0][i]) + fabsf(x[0][1][i]);
    }
    if constexpr (!BWD) {
      sum = wave_max(sum_over_rows(sum));
      if (lane == 0) sh.most[w][3] = sum;
    }
  }
  lds_barrier();
  if (w == 0) {
    const float it = inverse_pow2(s), gam = exp2_fast(sh.gh[lane]), bs = sh.bs[lane];
    const float all = exp2_fast(sh.gh[63]);
    // (X is scaled below 2^14)
    const float se = BWD ? 1.f
                         : scale_for(fmaxf(fmaxf(sh.most[0][3], sh.most[1][3]),
                                           fmaxf(sh.most[2][3], sh.most[3][3])) * s * 0x1p14f);
    gt[kGateY * kC + lane] = -gam * ik;
    gt[kGateO * kC + lane] = p.scale * gam * iq;
    gt[kGateZ * kC + lane] = bs * it;
    gt[kGateP * kC + lane] = BWD ? 0.f : sh.ip[lane] * it * inverse_pow2(se);
    gt[kGateOne * kC + lane] = lane == kOneG ? all : lane == kOneK ? ik : lane == kOneE ? se : it;
    if constexpr (BWD) {
      gt[kRevY * kC + lane] = bs * ik;
      gt[kRevP * kC + lane] = sh.ip[lane];
      gt[kRevZ * kC + lane] = -gam;
      gt[kRevBS * kC + lane] = bs;
      gt[kRevBeta * kC + lane] = sh.be[lane];
      gt[kRevHi * kC + lane] = sh.gh[lane];
      gt[kRevLo * kC + lane] = sh.gl[lane];
      gt[kRevOne * kC + lane] = lane == kRevG ? all : lane == kRevK ? ik : lane == kRevQ ? iq
                              : lane == kRevIT ? it : 0.f;
    }
  }
}

}  // namespace

hipError_t launch_delta_prep(const DeltaShape& s, const DeltaParams& p, bool backward,
                             hipStream_t st) {
  const unsigned cus = unsigned(p.slots) * unsigned(p.HV);
  if (!cus) return hipSuccess;
#define ONELA_DELTA_PREP(DK, NP)                                   \
  if (s.dk == DK && s.bf16 == (NP == 1)) {                         \
    if (backward)                                                  \
      delta_prep_kernel<DK, NP, true><<<cus, kThreads, 0, st>>>(p);  \
    else                                                           \
      delta_prep_kernel<DK, NP, false><<<cus, kThreads, 0, st>>>(p); \
    return hipGetLastError();                                      \
  }
  ONELA_DELTA_PREP(32, 1)
  ONELA_DELTA_PREP(64, 1)
  ONELA_DELTA_PREP(128, 1)
  ONELA_DELTA_PREP(256, 1)
  ONELA_DELTA_PREP(32, 2)
  ONELA_DELTA_PREP(64, 2)
  ONELA_DELTA_PREP(128, 2)
#undef ONELA_DELTA_PREP
  return hipErrorInvalidValue;
}

}  // namespace onela
