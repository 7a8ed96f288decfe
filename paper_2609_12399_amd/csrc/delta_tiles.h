// Device helpers of the delta-rule kernels (kernels_delta*.hip): sequences and
// chunks of packed tokens, fp32 operands as fp16 parts, and operand loads.
#pragma once

#include <type_traits>

#include "delta_params.h"
#include "device_common.h"
#include "internal.h"
#include "split_tiles.h"

namespace onela {

constexpr int kC = kDeltaChunk;

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- sequences and chunks --------------------------------------------------------

// A sequence's tokens and its first chunk slot.  Slots of sequence n start at
// floor(first token / 64) + n: no two sequences share one, and total / 64 + N are
// enough.  Offsets out of order are cut to [0, total]: wrong sequences, but no
// access outside the tensors.
struct Seq {
  long t0;
  int len;
  long slot;
};
__device__ inline Seq seq_of(const DeltaParams& p, int n) {
  if (!p.offsets) return {long(n) * p.L, p.L, long(n) * p.nch_l};
  const long a = min(max(long(p.offsets[n]), 0l), p.total);
  const long b = min(max(long(p.offsets[n + 1]), a), p.total);
  return {a, int(b - a), a / kC + n};
}

// The last sequence whose first item (first(token offset, n), rising with n) is not past
// `item`.  Every lane of the wave takes part.
template <typename First>
__device__ inline int find_seq(const DeltaParams& p, long item, First&& first) {
  const int lane = threadIdx.x & 63;
  int count = 0;
  for (int b = 0; b < p.N; b += 64) {
    const int n = b + lane;
    const long o = n < p.N ? min(max(long(p.offsets[n]), 0l), p.total) : 0;
    const unsigned long long m = __ballot(n < p.N && first(o, n) <= item);
    count += __popcll(m);
    if (m != ~0ull) break;
  }
  return __builtin_amdgcn_readfirstlane(max(count - 1, 0));
}

// The chunk of a slot: its first token and how many it has (0: the slot is empty).
struct Chunk {
  long t0;
  int n;
};
__device__ inline Chunk chunk_of(const DeltaParams& p, long slot) {
  if (!p.offsets) {
    const int n = int(slot / p.nch_l), c = int(slot - long(n) * p.nch_l);
    return {long(n) * p.L + long(c) * kC, min(kC, p.L - c * kC)};
  }
  const Seq s = seq_of(p, find_seq(p, slot, [](long o, int n) { return o / kC + n; }));
  const long c = slot - s.slot;
  if (c < 0 || c * kC >= s.len) return {0, 0};
  return {s.t0 + c * kC, int(min(long(kC), s.len - c * kC))};
}

// Segments: stretches of p.cps chunks that run at once, slots as for chunks (without
// segments p.cps is larger than any sequence and slot n is sequence n).
struct Segment {
  int n, j, nseg;  // sequence, number within it (no segment outside [0, nseg)), how many it has
  Seq sq;
  int cb, ce;      // chunks
};
__device__ inline int segments_of(const DeltaParams& p, const Seq& sq) {
  return max((delta_chunks(sq.len) + p.cps - 1) / p.cps, 1);
}
__device__ inline long first_segment(const DeltaParams& p, const Seq& sq, int n) {
  return p.offsets ? sq.slot / p.cps + n : long(n) * p.nseg_l;
}
__device__ inline Segment segment_of(const DeltaParams& p, long slot) {
  Segment s;
  s.n = p.offsets ? find_seq(p, slot, [&](long o, int n) { return (o / kC + n) / p.cps + n; })
                  : int(slot / p.nseg_l);
  s.sq = seq_of(p, s.n);
  s.nseg = segments_of(p, s.sq);
  const long j = slot - first_segment(p, s.sq, s.n);
  s.j = j >= 0 && j < s.nseg ? int(j) : -1;
  s.cb = s.j * p.cps;
  s.ce = int(min(long(s.cb) + p.cps, long(delta_chunks(s.sq.len))));
  return s;
}

// ---- memory ------------------------------------------------------------------------

__device__ inline __amdgpu_buffer_rsrc_t buffer(const void* base, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), static_cast<short>(0),
                                           int(bytes), 0x00020000);
}

// Rows of one head of n tokens: a buffer that ends with the last one's row, so that
// rows past it read as zeros.  row: bytes of a row, stride: bytes between tokens.
__device__ inline __amdgpu_buffer_rsrc_t rows_buffer(const void* base, long at, unsigned row,
                                                     unsigned stride, int n) {
  return buffer(static_cast<const char*>(base) + at, n > 0 ? unsigned(n - 1) * stride + row : 0u);
}

// BYTES (a multiple of 1 KiB) from memory straight into LDS, dealt out to NW waves.  In
// flight until the wave's vector memory counter says otherwise: dma_wait, then a barrier,
// before anyone reads them.
template <int BYTES, int NW>
__device__ inline void dma(const void* from, void* to, int w, int lane) {
  static_assert(BYTES % 1024 == 0, "whole wave loads");
#pragma unroll
  for (int q = 0; q < (BYTES / 1024 + NW - 1) / NW; ++q) {
    const int b = w + q * NW;
    if (BYTES / 1024 % NW == 0 || b < BYTES / 1024)
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(static_cast<const char*>(from) +
                                                          b * 1024 + lane * 16),
          (__attribute__((address_space(3))) void*)(static_cast<char*>(to) + b * 1024), 16, 0, 0);
  }
}
// Barrier for what the waves exchange through LDS by ordinary reads and writes: loads and
// stores of memory stay in flight across it (__syncthreads waits for all stores).
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ inline void dma_wait() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt(0)

// The 32-deep step h of a contraction over DK columns covers the tiles t0(h) and t0(h) + PS
// of 16: PS = 4 puts a row operand's two pieces 128 bytes apart (one two-address read).
template <int DK>
struct Steps {
  static constexpr int PS = DK / 32 < 4 ? DK / 32 : 4;
  static constexpr int t0(int h) { return h / PS * (2 * PS) + h % PS; }
};

// Row operand of a tile of 16 rows (lane row lr, first piece lq): the two pieces
// at column blocks b0 and b1 of 16, i.e. slots 0..3 are the columns 16 b0 + 4 lq
// + i and slots 4..7 the columns 16 b1 + 4 lq + i.
template <typename Tile>
__device__ inline uint4 row_frag(const Tile& t, int base, int b0, int b1, int rest) {
  const uint2 x = *t.template at<uint2>(base, b0, rest);
  const uint2 y = *t.template at<uint2>(base, b1, rest);
  return make_uint4(x.x, x.y, y.x, y.y);
}
// Column operand, contracted over rows: columns 16 b + lr, slots 0..3 the rows r0
// + 4 lq + i and 4..7 the rows r0 + 16 + 4 lq + i (base: off(4 lq + lr / 4, lr % 4),
// rest: bytes of r0 rows).
template <typename Tile>
__device__ inline uint4 col_frag(const Tile& t, int base, int b, int rest) {
  const uint2 x = lds_tr4(t.template at<uint16_t>(base, b, rest));
  const uint2 y = lds_tr4(t.template at<uint16_t>(base, b, rest + 32 * Tile::LD));
  return make_uint4(x.x, x.y, y.x, y.y);
}

// ---- fp32 operands as fp16 parts ---------------------------------------------------
//
// x = (hi + lo) / s with s a power of two that puts the largest magnitude of a row
// (or tile) at [2^13, 2^14): hi = fp16(s x), lo = fp16(s x - hi), together 22 bits of the
// largest values; small ones keep an error of 2^-39 of the largest.  Products of two
// such operands leave out lo lo (2^-22).  bf16 values are exact in hi alone down to 2^-28
// of the largest.

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

__device__ inline f32x4 mfma_f16(const uint4& a, const uint4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a),
                                                __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// The power of two that brings magnitude m to [2^13, 2^14) (within what a float can
// hold; of 0, infinity and NaN: 2^14).
__device__ inline float scale_for(float m) {
  return ldexpf(1.f, min(14 - __builtin_amdgcn_frexp_expf(m), 100));
}
// 1 / s of a power of two.
__device__ inline float inverse_pow2(float s) {
  return __uint_as_float(0x7f000000u - __float_as_uint(s));
}

// The same to [2^2, 2^3), for keys and queries: bf16 values stay exact down to 2^-16 of the
// largest, with an error of 2^-28 of it below, and the values that products with them add
// to a state stay large where the state's bound (delta_chain.h) limits their sum.
__device__ inline float scale_for_rows(float m) { return scale_for(m) * 0x1p-11f; }

__device__ inline unsigned pack_f16x2(float a, float b) {
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, half2v));
}

// a s and b s as one or two fp16 parts.
template <int NP>
__device__ inline void parts2(float a, float b, float s, unsigned (&p)[NP]) {
  p[0] = pack_f16x2(a * s, b * s);
  if constexpr (NP == 2) {
    const half2v h = __builtin_bit_cast(half2v, p[0]);
    p[1] = pack_f16x2(fmaf(a, s, -float(h.x)), fmaf(b, s, -float(h.y)));
  }
}

// The same, each with a scale of its own.
__device__ inline void parts2(float a, float b, float s, float t, unsigned (&p)[2]) {
  p[0] = pack_f16x2(a * s, b * t);
  const half2v h = __builtin_bit_cast(half2v, p[0]);
  p[1] = pack_f16x2(fmaf(a, s, -float(h.x)), fmaf(b, t, -float(h.y)));
}
// The same without a scale.
__device__ inline void parts2(float a, float b, unsigned (&p)[2]) {
  p[0] = pack_f16x2(a, b);
  const half2v h = __builtin_bit_cast(half2v, p[0]);
  float one = 1.f;
  asm("" : "+v"(one));  // (unseen, so that each difference is one mixed multiply-add)
  p[1] = pack_f16x2(fmaf(a, one, -float(h.x)), fmaf(b, one, -float(h.y)));
}
__device__ inline void parts8(const f32x4& x, const f32x4& y, uint4 (&p)[2]) {
  unsigned u[4][2];
  parts2(x.x, x.y, u[0]);
  parts2(x.z, x.w, u[1]);
  parts2(y.x, y.y, u[2]);
  parts2(y.z, y.w, u[3]);
#pragma unroll
  for (int i = 0; i < 2; ++i) p[i] = make_uint4(u[0][i], u[1][i], u[2][i], u[3][i]);
}
// Eight values (two accumulator tiles of four) as parts of an operand.
template <int NP>
__device__ inline void parts8(const f32x4& x, const f32x4& y, float s, uint4 (&p)[NP]) {
  unsigned u[4][NP];
  parts2<NP>(x.x, x.y, s, u[0]);
  parts2<NP>(x.z, x.w, s, u[1]);
  parts2<NP>(y.x, y.y, s, u[2]);
  parts2<NP>(y.z, y.w, s, u[3]);
#pragma unroll
  for (int i = 0; i < NP; ++i) p[i] = make_uint4(u[0][i], u[1][i], u[2][i], u[3][i]);
}

// The parts (a, b) of a product of NA and NB part operands, smallest first: all but lo lo.
template <int NA, int NB, typename F>
__device__ inline void for_products(F&& f) {
  if constexpr (NA == 2) f(1, 0);
  if constexpr (NB == 2) f(0, 1);
  f(0, 0);
}

// max(m, |x|) of values m >= 0: three instructions, as medians and integers (fmaxf would first make
// each operand canonical, and a median with an infinity that the compiler sees is fmaxf to it:
// eight).  NaN counts as nothing beside a number.
__device__ inline float max4abs(float m, const f32x4& x) {
  float inf = __builtin_inff();
  asm("" : "+s"(inf));
  const unsigned a = __float_as_uint(__builtin_amdgcn_fmed3f(fabsf(x.x), fabsf(x.y), inf));
  const unsigned b = __float_as_uint(__builtin_amdgcn_fmed3f(fabsf(x.z), fabsf(x.w), inf));
  return __uint_as_float(max(__float_as_uint(m), max(a, b)));
}

// max(a, b) of values >= 0, whose bits rise with them (NaN is the largest).
__device__ inline float max_bits(float a, float b) {
  return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
}
// Maximum of values m >= 0 over the wave, in every lane.
__device__ inline float max_over_rows(float m);
__device__ inline float wave_max(float m) {
  m = max_bits(m, dpp<0xB1>(m));   // quad_perm [1,0,3,2]
  m = max_bits(m, dpp<0x4E>(m));   // quad_perm [2,3,0,1]
  m = max_bits(m, dpp<0x141>(m));  // row_half_mirror
  m = max_bits(m, dpp<0x140>(m));  // row_mirror
  return max_over_rows(m);
}

// Maximum (of values m >= 0) and sum over the four lanes lr, lr + 16, lr + 32, lr + 48.
__device__ inline float max_over_rows(float m) {
  const unsigned v = __float_as_uint(m);
  const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const unsigned u = max(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(max(q[0], q[1]));
}
__device__ inline float sum_over_rows(float m) {
  const unsigned v = __float_as_uint(m);
  const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  m = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  const unsigned u = __float_as_uint(m);
  const auto q = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// Raises to[i] (>= 0, in memory) to the wave's largest m[i] >= 0.  Bits of floats >= 0 rise with
// them, and a maximum does not depend on the order.
template <int N>
__device__ inline void note_max(float* to, const float (&m)[N], int lane) {
  float mine = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float x = wave_max(m[i]);
    mine = lane == i ? x : mine;
  }
  if (lane < N) atomicMax(reinterpret_cast<unsigned*>(to) + lane, __float_as_uint(mine));
}

}  // namespace onela
