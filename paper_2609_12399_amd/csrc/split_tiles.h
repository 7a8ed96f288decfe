// Device helpers of the chunked recurrences (prefill and the delta rule over
// sequences): fp32 values as sums of bf16 parts for the bf16 matrix
// instructions, and bf16 tiles in LDS that are read by rows and transposed.
#pragma once

#include "device_common.h"

namespace onela {

__device__ inline f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// x = hi + mid + lo (8 floats, three bf16 vectors; exact for normal x).
__device__ inline void split3(const float* x, uint4& hi, uint4& mid, uint4& lo) {
  unsigned h[4], m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    const float r0 = x[2 * i] - bf16_lo_to_float(h[i]);
    const float r1 = x[2 * i + 1] - bf16_hi_to_float(h[i]);
    m[i] = pack_bf16x2(r0, r1);
    l[i] = pack_bf16x2(r0 - bf16_lo_to_float(m[i]), r1 - bf16_hi_to_float(m[i]));
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  mid = make_uint4(m[0], m[1], m[2], m[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}

__device__ inline void split3(const f32x4& x0, const f32x4& x1, uint4& hi, uint4& mid, uint4& lo) {
  const float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
  split3(x, hi, mid, lo);
}

// x = hi + mid + lo exactly by truncation (8 of the 24 significant bits each),
// for products that use all three parts.  Byte permutes and masks in place of
// the conversions.
__device__ inline void cut3(const f32x4& x0, const f32x4& x1, uint4& hi, uint4& mid, uint4& lo) {
  const float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
  unsigned h[4], m[4], l[4];
  auto top2 = [](float a, float b) {  // the upper halves, a's in the low half
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  };
  auto top = [](float a) { return __uint_as_float(__float_as_uint(a) & 0xffff0000u); };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x[2 * i], b = x[2 * i + 1];
    const float a1 = a - top(a), b1 = b - top(b);
    h[i] = top2(a, b);
    m[i] = top2(a1, b1);
    l[i] = top2(a1 - top(a1), b1 - top(b1));
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  mid = make_uint4(m[0], m[1], m[2], m[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// 16 bytes on their way through registers, as a native vector: arrays of the
// header's uint4 (a class) that are moved under a condition stay in memory
// (scratch, or LDS that the compiler adds).
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ inline u32x4 keep(u32x4 v, bool in) {
  return in ? v : u32x4{0u, 0u, 0u, 0u};
}

// x of the lane N places back (forward) in the row of 16 lanes; 1 past its end.
template <int CTRL>
__device__ inline float row_shift1(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, 1.f),
                                                               __builtin_bit_cast(int, x), CTRL,
                                                               0xF, 0xF, false));
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Transposed LDS read: the 16 lanes of a group address four rows of four
// 8-byte pieces (lane s: row s / 4, piece s % 4); lane j receives element j of
// the 16 of each row.
__device__ inline uint2 lds_tr4(const uint16_t* a) {
  return __builtin_bit_cast(
      uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                 (__attribute__((address_space(3))) s16x4*)(const_cast<uint16_t*>(a))));
}

// ROWS (64) rows of COLS bf16 elements in LDS, addressed in pieces of 4 elements (8
// bytes).  The scan reads the keys in two ways: pieces of 16 consecutive rows
// (16 lanes, one piece column), and transposed, 4 rows x 4 neighbouring pieces
// (16 lanes, rows from a multiple of 4).  From 16 pieces per row on, the piece
// index is XORed with f(row) = the row's bits 1:0 above its bits 3:2, which gives
// the 16 lanes of either read 16 different slots of the 128-byte bank row
// (LDS bank conflicts of the scan: 12.6 M -> 2.4 M cycles at 16 requests x 1000
// tokens against padded rows; with 16 pieces per row only f's low 3 bits are used, so
// that the two pieces of a key operand stay a constant apart).  Narrower rows
// are padded instead.
// Tiles that are only read transposed take all four bits from 16 pieces on (MASK).
template <int COLS, int ROWS = 64, int MASK = COLS >= 128 ? 15 : 7>
struct Swz {
  static constexpr bool kXor = COLS >= 64;
  static constexpr int LD = kXor ? COLS : COLS + 16;
  uint16_t x[ROWS * LD];
  __device__ static int f(int row) {
    return (((row & 3) << 2) | ((row >> 2) & 3)) & MASK;
  }
  // Byte offset of (row, piece): f(row) has the four low bits, so the pieces
  // 4 j + m of one lane are the XOR of its piece m with 4 j, j < 4, and the rest
  // of the address is a constant.
  __device__ static int off(int row, int piece) {
    return 2 * LD * row + 8 * (kXor ? piece ^ f(row) : piece);
  }
  template <typename T>
  __device__ const T* at(int base, int j, int rest) const {
    return reinterpret_cast<const T*>(reinterpret_cast<const char*>(x) +
                                      (kXor ? base ^ (32 * (j & 3)) : base + 32 * (j & 3)) +
                                      128 * (j >> 2) + rest);
  }
  // stores the pieces 2 i and 2 i + 1 of a row
  __device__ void put(int row, int i, u32x4 v) {
    if constexpr (kXor) {
      typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
      char* const b = reinterpret_cast<char*>(x);
      *reinterpret_cast<u32x2*>(b + off(row, 2 * i)) = v.xy;
      *reinterpret_cast<u32x2*>(b + off(row, 2 * i + 1)) = v.zw;
    } else {
      *reinterpret_cast<u32x4*>(x + row * LD + 8 * i) = v;
    }
  }
};

}  // namespace onela
