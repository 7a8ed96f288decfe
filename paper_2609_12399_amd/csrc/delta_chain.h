// The state's rows of one wave in the delta rule's chains (kernels_delta_scan.hip,
// kernels_delta_reverse.hip) and the products they take part in.
#pragma once

#include "delta_tiles.h"

namespace onela {

// Waves of a chain's workgroup: 32 state rows each, at most 128 per workgroup.
template <int DV>
constexpr int kChainWaves = DV / 32 < 4 ? DV / 32 : 4;

// Chunks after which a state's bound is taken from its rows (which costs some 50 vector
// instructions at d_k = 128, of 900 per chunk).
constexpr int kTighten = 8;

// Bytes of a triangular matrix's fragments, and of a chunk's gates.
constexpr int kFragBytes = 6 * 2 * 1024;

// 32 rows of the state per wave as two column tiles of S^T (tile u, lane lr: row row0 + u,
// row0 = 32 w + 2 lr), in registers: st[u][b][i] = sc[u] S(row0 + u, 16 b + 4 lq + i).
//
// Scales (powers of two).  sc[u] keeps the row inside what two fp16 parts hold, by a bound on
// its largest value; the bound grows with every update by what 64 tokens of the
// largest size among them can add at most (the values of the update are measured, so that tokens
// that add nothing leave it), and where it leaves [2^12, 2^15] in the row's scale it is
// scaled anew.  What the tokens of a chunk add is some 2^7 below that; over many chunks without
// decay the bound alone would rise and rise while the delta rule keeps the state where it is, so
// it is taken from the row itself every kTighten chunks (2^10 below at worst; before every chunk
// where the largest value is kept for the gradients anyway).  Parts lose bits only below 2^-3,
// 2^15 below the bound.  Every row is a recurrence of its own, and nothing that is
// scaled by a row is shared with another: small channels keep their bits beside large ones, and
// what is not finite stays in its own.
template <int DK>
struct ChainState {
  static constexpr int NB = DK / 16;
  static constexpr int PS = Steps<DK>::PS;
  static constexpr int t0(int h) { return Steps<DK>::t0(h); }
  static constexpr int KR = 32 * Swz<DK>::LD;  // bytes of 16 rows of an operand tile

  f32x4 st[2][NB];
  float sc[2], bound[2];  // bound: of the true values

  // The scale for rows of at most `most` > 0, no further from 1 than products with it can be.
  __device__ static float row_scale(float most) {
    return fminf(fmaxf(scale_for(fminf(most, 0x1p126f)), 0x1p-112f), 0x1p100f);
  }
  // from: the lane's first row (null: zeros), or the rows of the identity; keep: where the rows are
  // stored as they came (or null)
  __device__ void init(const float* from, float* keep, bool ident, int row0, int lq) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float m = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        st[u][b] = from ? *reinterpret_cast<const f32x4*>(from + u * DK + 16 * b)
                        : f32x4{0.f, 0.f, 0.f, 0.f};
        if (ident)
#pragma unroll
          for (int i = 0; i < 4; ++i) st[u][b][i] = 16 * b + 4 * lq + i == row0 + u ? 1.f : 0.f;
        m = max4abs(m, st[u][b]);
      }
      bound[u] = max_over_rows(m);
      sc[u] = bound[u] > 0.f ? row_scale(bound[u]) : 1.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if (keep) *reinterpret_cast<f32x4*>(keep + u * DK + 16 * b) = st[u][b];
        st[u][b] *= sc[u];
      }
    }
  }
  __device__ void store(float* to) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float inv = inverse_pow2(sc[u]);
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *reinterpret_cast<f32x4*>(to + u * DK + 16 * b) = inv * st[u][b];
    }
  }
  // The same for the gradients (DeltaParams::sws), whole lines at a time, the rows of the state's
  // wave w.  Through buffers, which take one register of addresses, each with a base of its own:
  // with the base's part in the instruction's scalar offset the compiler leaves no wait
  // between a 16-byte store and the next write to its data registers, and some of what was
  // stored was the next write's.
  template <int DV>
  __device__ void store_tiles(float* to, int w, int lane) const {
    const unsigned off = 64 * (lane & 15) + 16 * (lane >> 4);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float inv = inverse_pow2(sc[u]);
#pragma unroll
      for (int b = 0; b < NB; ++b)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, inv * st[u][b]),
                                               buffer(to + 512 * w + 16 * DV * b + 256 * u, 1024),
                                               off, 0, 0);
    }
  }
  // Bounds from the rows themselves.
  __device__ void tighten() {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float m = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) m = max4abs(m, st[u][b]);
      bound[u] = fminf(bound[u], max_over_rows(m) * inverse_pow2(sc[u]));
    }
  }
  // Makes room in row u for an update S <- g S + (64 tokens' keys times values of at most
  // `most`; keys are scaled below 2^3): the factor that the row takes in it, g and the change of
  // its scale in one (by itself the change could overflow where g undoes it: a state of 1e30
  // forgotten for values of 1e-30).
  __device__ float make_room(int u, float g, float most) {
    bound[u] = fmaf(g, bound[u], 0x1p9f * most);
    const float at = bound[u] * sc[u], fit = row_scale(bound[u]);
    const bool off = (bound[u] > 0.f) & !((at <= 32768.f) & (at >= 4096.f));  // (no branch)
    const float to = off ? fit : sc[u];
    g = ldexpf(g, (__float_as_int(to) - __float_as_int(sc[u])) >> 23);
    sc[u] = to;
    return g;
  }
};

// Where a chain's first segment of several keeps the state that it starts from (kernels_delta_scan.hip):
// the last segment's place, su being the first's (segment slot and value head).
template <int DK, int DV>
__device__ inline float* kept_start(const DeltaParams& p, const Segment& sg, long su) {
  return p.segs + (su + long(sg.nseg - 1) * p.HV) * (DV * DK);
}
// The state of a value head that a segment starts from (null: zeros): of a sequence's first the
// caller's (given: [N][HV][DV][DK] or null), of the others none while the segments' own states are
// formed (SEG), and then what the segment before leaves.
template <int DK, int DV, bool SEG>
__device__ inline const float* start_of(const DeltaParams& p, const Segment& sg, long su, int hv,
                                        const float* given) {
  if (sg.j > 0) return SEG ? nullptr : p.segs + (su - p.HV) * (DV * DK);
  if (!given) return nullptr;
  if (!SEG && sg.nseg > 1) return kept_start<DK, DV>(p, sg, su);
  return given + (long(sg.n) * p.HV + hv) * (DV * DK);
}

// The transition matrix A of a segment in memory, as operands of A^T S^T: two fp16 parts of
// A^T(16 b + lr, k), of the lanes' slots k = 32 h + 4 lq + i and 32 h + 16 + 4 lq + i; and the
// scale that the rows k of every h carry.
template <int DK>
struct SegmentMatrix {
  uint4 x[DK / 16][DK / 32][2][64];
  float scale[64];
};

// Stores the rows of A that the wave holds as its state (rows 32 h .. 32 h + 31 of A).
template <int DK>
__device__ inline void store_matrix(const ChainState<DK>& s, SegmentMatrix<DK>* to, int h,
                                    int lane) {
  static_assert(sizeof(SegmentMatrix<DK>) == delta_matrix_bytes(DK), "");
  const int lr = lane & 15, lq = lane >> 4;
  float g[2], most = 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    float m = 0.f;
#pragma unroll
    for (int b = 0; b < ChainState<DK>::NB; ++b) m = max4abs(m, s.st[u][b]);
    g[u] = inverse_pow2(s.sc[u]);
    most = fmaxf(most, m * g[u]);
  }
  const float f = scale_for(wave_max(most));
  if (lane == 0) to->scale[h] = f;
  g[0] *= f;
  g[1] *= f;
#pragma unroll
  for (int b = 0; b < ChainState<DK>::NB; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // rows 32 h + 2 lr + u, u < 2: two neighbouring slots
      unsigned p[2];
      parts2(s.st[0][b][i], s.st[1][b][i], g[0], g[1], p);
#pragma unroll
      for (int q = 0; q < 2; ++q)
        reinterpret_cast<unsigned*>(&to->x[b][h][q][16 * ((lr & 7) >> 1) + 4 * lq + i])
            [(lr & 1) + 2 * (lr >> 3)] = p[q];
    }
}

// y[u][a] += rows of A (16 a ..) times S^T, and with TWO the same of B into o: the operand
// tiles have NP parts, the state two.
template <int DK, int NP, bool TWO>
__device__ __attribute__((always_inline)) inline void rows_times_state(
    const Swz<DK>* A, const Swz<DK>* B, const ChainState<DK>& s, int kb, f32x4 (&y)[2][4],
    f32x4 (&o)[2][4]) {
  using C = ChainState<DK>;
#pragma unroll
  for (int h = 0; h < DK / 32; ++h) {
    uint4 sp[2][2], af[4][NP], bf[4][NP];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        af[a][i] = row_frag(A[i], kb, C::t0(h), C::t0(h) + C::PS, C::KR * a);
        if constexpr (TWO) bf[a][i] = row_frag(B[i], kb, C::t0(h), C::t0(h) + C::PS, C::KR * a);
      }
#pragma unroll
    for (int u = 0; u < 2; ++u) parts8(s.st[u][C::t0(h)], s.st[u][C::t0(h) + C::PS], sp[u]);
    // (the wave in its products goes before the one beside it: 512 workgroups of 16 chunks
    // 201 -> 193 us)
    __builtin_amdgcn_s_setprio(1);
    for_products<NP, 2>([&](int i, int j) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int a = 0; a < 4; ++a) y[u][a] = mfma_f16(af[a][i], sp[u][j], y[u][a]);
      if constexpr (TWO)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int a = 0; a < 4; ++a) o[u][a] = mfma_f16(bf[a][i], sp[u][j], o[u][a]);
    });
    __builtin_amdgcn_s_setprio(0);
  }
}

// acc[u][a] += F x[u], F a lower triangular 64 x 64 matrix in two parts whose fragments are in
// LDS, x in NX parts (tokens 32 h .. of column tile u: x[u][h]).
template <int NX>
__device__ __attribute__((always_inline)) inline void triangle(const uint4* F,
                                                               const uint4 (&x)[2][2][NX],
                                                               f32x4 (&acc)[2][4], int lane) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint4 f[4][2];
#pragma unroll
    for (int a = 2 * h; a < 4; ++a)
#pragma unroll
      for (int i = 0; i < 2; ++i) f[a][i] = F[((a < 2 ? a : 2 * a - 2 + h) * 2 + i) * 64 + lane];
    for_products<2, NX>([&](int i, int j) {
#pragma unroll
      for (int a = 2 * h; a < 4; ++a)
#pragma unroll
        for (int u = 0; u < 2; ++u) acc[u][a] = mfma_f16(f[a][i], x[u][h][j], acc[u][a]);
    });
  }
}

// S^T <- S^T diag(g) + A^T x: A an operand tile in NP parts, x in two.
template <int DK, int NP>
__device__ __attribute__((always_inline)) inline void update_state(
    ChainState<DK>& s, const float (&g)[2], const Swz<DK>* A, const uint4 (&x)[2][2][2], int tb) {
  using C = ChainState<DK>;
  constexpr int NG = C::NB < 4 ? C::NB : 4;
#pragma unroll
  for (int b0 = 0; b0 < C::NB; b0 += NG) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int b = 0; b < NG; ++b) s.st[u][b0 + b] *= g[u];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 kt[NG][NP];
#pragma unroll
      for (int b = 0; b < NG; ++b)
#pragma unroll
        for (int i = 0; i < NP; ++i) kt[b][i] = col_frag(A[i], tb, b0 + b, 2 * C::KR * h);
      for_products<NP, 2>([&](int i, int j) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int b = 0; b < NG; ++b)
            s.st[u][b0 + b] = mfma_f16(kt[b][i], x[u][h][j], s.st[u][b0 + b]);
      });
    }
  }
}

// Two neighbouring columns of the 16 tokens t(i) = 16 (i / 4) + 4 lq + i % 4 of a lane, raw.
// REV: of token 63 - t.
template <int NP, bool REV = false>
struct Columns {
  unsigned r[16][NP];
  __device__ void load(__amdgpu_buffer_rsrc_t rs, unsigned stride, int lq, unsigned at) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const unsigned t = 16 * (i >> 2) + (i & 3);
      const unsigned o = unsigned(REV ? 12 - 4 * lq : 4 * lq) * stride + at,
                     so = (REV ? 51 - t : t) * stride;
      if constexpr (NP == 1) {
        r[i][0] = __builtin_amdgcn_raw_buffer_load_b32(rs, o, so, 0);
      } else {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(rs, o, so, 0);
        r[i][0] = x[0];
        r[i][1] = x[1];
      }
    }
  }
  __device__ float get(int i, int u) const {
    if constexpr (NP == 1)
      return u ? bf16_hi_to_float(r[i][0]) : bf16_lo_to_float(r[i][0]);
    else
      return __uint_as_float(r[i][u]);
  }
  __device__ f32x4 tile(int a, int u) const {
    return f32x4{get(4 * a, u), get(4 * a + 1, u), get(4 * a + 2, u), get(4 * a + 3, u)};
  }
};
// The same stored, rounded to the tensor's type.
template <int NP, bool REV = false>
__device__ inline void store_columns(__amdgpu_buffer_rsrc_t rs, unsigned stride, int lq, unsigned at,
                                     int i, float x0, float x1) {
  const unsigned t = 16 * (i >> 2) + (i & 3);
  const unsigned o = unsigned(REV ? 12 - 4 * lq : 4 * lq) * stride + at,
                 so = (REV ? 51 - t : t) * stride;
  if constexpr (NP == 1) {
    __builtin_amdgcn_raw_buffer_store_b32(pack_bf16x2(x0, x1), rs, o, so, 0);
  } else {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(x0), __float_as_uint(x1)}, rs, o,
                                          so, 0);
  }
}

}  // namespace onela
