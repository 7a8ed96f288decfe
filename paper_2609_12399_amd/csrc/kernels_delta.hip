// The gated delta rule over whole sequences, forward and backward, in chunks of
// C = 64 tokens (Eq. 1 of Sec. 2.2 with outputs, states to start from and gradients).
//
// With alpha_t = exp(log_alpha_t), inside a chunk that starts from state S_0
// let gamma_i = alpha_0 ... alpha_i, Gamma(i, j) = alpha_{j+1} ... alpha_i (i >= j),
// sigma_j = Gamma(C - 1, j), and e_i = v_i - alpha_i S_{i-1} k_i the error that Eq. 1
// corrects (the paper's delta_i is beta_i e_i).  Unrolling Eq. 1,
//   S_i = gamma_i S_0 + sum_{j<=i} Gamma(i, j) beta_j e_j k_j^T,
// and with B(i, j) = Gamma(i, j) (k_i . k_j) for j < i and T = (I + B diag(beta))^-1
// (unit lower triangular), P(i, j) = scale Gamma(i, j) (q_i . k_j) for j <= i,
//   e   = T (V - diag(gamma) K S_0^T)
//   O   = scale diag(gamma) Q S_0^T + P diag(beta) e
//   S_C = gamma_{C-1} S_0 + (diag(beta sigma) e)^T K.
// Reversed, with dS the adjoint of S_C (dD = the adjoint of beta e):
//   dD   = P^T dO + diag(sigma) K dS^T
//   dV   = T^T diag(beta) dD
//   dS_0 = gamma_{C-1} dS + scale (diag(gamma) dO)^T Q - (diag(gamma) dV)^T K,
// which is the forward step over the chunk with its tokens in reverse order (T^T
// reversed is lower triangular again) and one more term, so that one kernel walks
// both.  Then, chunk by chunk on its own, with X = dO e^T and N = dV e^T,
//   L = scale Gamma . (X diag(beta)) (j <= i),  M = -Gamma . (N diag(beta)) (j < i),
//   dQ = scale diag(gamma) dO S_0 + L K
//   dK = L^T Q + (M + M^T) K + diag(beta sigma) e dS - diag(gamma) dV S_0
//   dbeta_j = sum_i P(i, j) X(i, j) - sum_i B(i, j) N(i, j) + sigma_j k_j . (dS^T e_j)
//   dlog_alpha_t = sum_{i>=t>j} Z(i, j)
//     + sum_{i>=t} gamma_i (scale q_i . (S_0^T dO_i) - k_i . (S_0^T dV_i))
//     + gamma_{C-1} <S_0, dS> + sum_{j<t} beta_j sigma_j k_j . (dS^T e_j),
// Z = L . (Q K^T) + M . (K K^T).
//
// Launches.  Forward: delta_factor_kernel (T, decays; one workgroup per chunk and
// value head), delta_scan_kernel (the chain over the chunks; 16 state rows per wave),
// delta_out_kernel (one workgroup per chunk and value head).  Backward: the
// first two again (the states are not kept from the forward call), delta_intra_kernel
// (P^T dO), the scan in reverse, delta_grad_kernel.
//
// Precision.  States, e, T, decays and sums are fp32.  Every product runs on
// v_mfma_f32_16x16x32_bf16 with its fp32 operands as the sum of three bf16 parts
// (exact; products of parts below 2^-24 are left out) and bf16 tensors as they
// stand, NP = 1; fp32 tensors are three parts too, NP = 3.  Where a result is
// only rounded to a bf16 tensor, fp32 operands take two parts (2^-17 of the operand
// against the 2^-9 of the rounding).  Decays are exp2 of differences of in-chunk sums of
// log2(alpha), which are kept to 48 bits (a float pair), so that a vanishing decay
// does not blur the ones after it; log_alpha below -1e5, -inf among it, is an exact 0.
//
// Tokens past a sequence's end read as k = v = q = 0, beta = 0, alpha = 1: they
// leave the state as it is and give zeros.
#include <type_traits>

#include "delta_params.h"
#include "device_common.h"
#include "internal.h"
#include "split_tiles.h"

namespace onela {
namespace {

constexpr int kC = kDeltaChunk;
constexpr int kTFrags = 6;  // 16 x 32 fragments of a lower triangular 64 x 64 matrix
constexpr int kTChunk = kTFrags * 3 * 64;
static_assert(kTChunk * 16 == kDeltaFactorBytes, "");
constexpr int kThreads = 256;

// Rows of a chunk's gates in the workspace.
enum { kGateA, kGateB, kGateBeta, kGateHi, kGateLo };  // -gamma, beta sigma, beta, log2 sums

// The parts of a product of NA and NB part operands, largest first: a + b <= 2.
template <int NA, int NB, typename F>
__device__ inline void for_parts(F&& f) {
#pragma unroll
  for (int s = (NA - 1) + (NB - 1) < 2 ? (NA - 1) + (NB - 1) : 2; s >= 0; --s)
#pragma unroll
    for (int a = 0; a < NA; ++a)
      if (s - a >= 0 && s - a < NB) f(a, s - a);
}

// x as NPART bf16 parts: three by truncation (exact), two rounded.
template <int NPART>
__device__ inline void parts_of(const f32x4& x0, const f32x4& x1, uint4 (&p)[NPART]) {
  static_assert(NPART == 2 || NPART == 3, "");
  if constexpr (NPART == 3) {
    cut3(x0, x1, p[0], p[1], p[2]);
  } else {
    const float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
    split8(x, p[0], p[1]);
  }
}

// Four floats as NPART parts of 8 bytes.
template <int NPART>
__device__ inline void parts4(const f32x4& x, uint2 (&p)[NPART]) {
  if constexpr (NPART == 1) {
    p[0] = make_uint2(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w));
  } else {
    const f32x4 z = {0.f, 0.f, 0.f, 0.f};
    uint4 y[NPART];
    parts_of<NPART>(x, z, y);
#pragma unroll
    for (int i = 0; i < NPART; ++i) p[i] = make_uint2(y[i].x, y[i].y);
  }
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

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
  // the last sequence whose first slot is not past this one (first slots rise)
  const int lane = threadIdx.x & 63;
  int count = 0;
  for (int b = 0; b < p.N; b += 64) {
    const int n = b + lane;
    const long o = n < p.N ? min(max(long(p.offsets[n]), 0l), p.total) : 0;
    const unsigned long long m = __ballot(n < p.N && o / kC + n <= slot);
    count += __popcll(m);
    if (m != ~0ull) break;
  }
  const int n = __builtin_amdgcn_readfirstlane(max(count - 1, 0));
  const Seq s = seq_of(p, n);
  const long c = slot - s.slot;
  if (c < 0 || c * kC >= s.len) return {0, 0};
  return {s.t0 + c * kC, int(min(long(kC), s.len - c * kC))};
}

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

// Rows [64][COLS] of a tensor on their way into LDS as NP bf16 planes: bf16 as it
// stands, fp32 cut into three parts.  REV: row r holds token 63 - r.
template <int COLS, int NP, int TH, bool REV = false>
struct RowStage {
  static constexpr int NV = (kC * COLS / 8 + TH - 1) / TH;  // pieces of 8 elements per thread
  static constexpr bool kEven = kC * COLS / 8 % TH == 0;
  u32x4 r[NV][NP == 1 ? 1 : 2];
  // each lane's piece q of thread tid
  __device__ void load(__amdgpu_buffer_rsrc_t rs, unsigned stride, int tid) {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int e = tid + q * TH, row = e / (COLS / 8), c = e % (COLS / 8);
      const unsigned o = unsigned(REV ? kC - 1 - row : row) * stride + c * (NP == 1 ? 16 : 32);
      if (!kEven && row >= kC) continue;
      r[q][0] = __builtin_amdgcn_raw_buffer_load_b128(rs, o, 0, 0);
      if constexpr (NP == 3) r[q][1] = __builtin_amdgcn_raw_buffer_load_b128(rs, o + 16, 0, 0);
    }
  }
  template <typename Tile>
  __device__ void store(Tile* pl, int tid) const {
#pragma unroll
    for (int q = 0; q < NV; ++q) {
      const int e = tid + q * TH, row = e / (COLS / 8), c = e % (COLS / 8);
      if (!kEven && row >= kC) continue;
      if constexpr (NP == 1) {
        pl[0].put(row, c, r[q][0]);
      } else {
        uint4 x[3];
        cut3(__builtin_bit_cast(f32x4, r[q][0]), __builtin_bit_cast(f32x4, r[q][1]), x[0], x[1],
             x[2]);
#pragma unroll
        for (int i = 0; i < 3; ++i) pl[i].put(row, c, __builtin_bit_cast(u32x4, x[i]));
      }
    }
  }
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

// The lower triangle's tile x (of 10): row block a, column block b <= a.
__device__ inline void tile_of(int x, int& a, int& b) {
  a = (x >= 1) + (x >= 3) + (x >= 6);
  b = x - a * (a + 1) / 2;
}

// ---- factors of the chunks ---------------------------------------------------

template <int DK, int NP>
struct FactorLds {
  union {
    Swz<DK> K[NP];        // the chunk's keys
    float T[kC][kC + 4];  // then T
  };
  float M[kC][kC + 4];  // B diag(beta); its diagonal blocks then hold those of T
  double g[kC];         // sums of log2(alpha)
  float be[kC];
};

// T = (I + B diag(beta))^-1 and the gates of one chunk of one value head.  Four waves.
// The inverse goes by 16-token blocks: the four diagonal blocks by forward
// substitution, one per wave with a column per lane, then each wave the blocks below
// the diagonal block of its block column, T_ij = -T_ii sum_k M_ik T_kj, in fp32 matrix
// instructions with T_kj in the accumulator layout as the next operand.
//   Bound: latency of that chain; several workgroups share a compute unit.
template <int DK, int NP, bool BWD>
__global__ __launch_bounds__(kThreads) void delta_factor_kernel(DeltaParams p) {
  __shared__ __align__(16) FactorLds<DK, NP> sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const long slot = blockIdx.x / p.HV;
  const int hv = int(blockIdx.x - slot * p.HV), hk = hv / (p.HV / p.HK);
  const Chunk ch = chunk_of(p, slot);
  if (ch.n <= 0) return;
  const long cu = long(blockIdx.x);
  constexpr int kIo = NP == 1 ? 2 : 4;
  RowStage<DK, NP, kThreads> ks;
  ks.load(rows_buffer(p.k, (ch.t0 * p.ks + hk * DK) * kIo, DK * kIo, unsigned(p.ks) * kIo, ch.n),
          unsigned(p.ks) * kIo, tid);
  if (w == 0) {  // lane t holds token t
    const long ti = (ch.t0 + min(lane, ch.n - 1)) * p.HV + hv;
    float la = p.la[ti], be = p.beta[ti];
    la = la < -1e5f ? -1e5f : la;
    double g = lane < ch.n ? double(la) * 1.4426950408889634 : 0.0;
    be = lane < ch.n ? be : 0.f;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double u = __shfl_up(g, d);
      if (lane >= d) g += u;
    }
    const double last = __shfl(g, 63);
    sh.g[lane] = g;
    sh.be[lane] = be;
    float* const gt = p.gates + cu * (kDeltaGates * kC) + lane;
    const float hi = float(g);
    gt[kGateA * kC] = -exp2_fast(hi);
    gt[kGateB * kC] = be * exp2_fast(float(last - g));
    gt[kGateBeta * kC] = be;
    gt[kGateHi * kC] = hi;
    gt[kGateLo * kC] = float(g - double(hi));
  }
  ks.store(sh.K, tid);
  __syncthreads();
  const int kb = Swz<DK>::off(lr, lq);
  constexpr int KR = 32 * Swz<DK>::LD;
  // M(i, j) = Gamma(i, j) (k_i . k_j) beta_j of a tile, 0 on and above the diagonal
  auto tile = [&](int a, int b) {
    f32x4 hi = {0.f, 0.f, 0.f, 0.f}, lo = hi;
#pragma unroll
    for (int h = 0; h < DK / 32; ++h) {
      uint4 x[NP], y[NP];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        x[i] = row_frag(sh.K[i], kb, 2 * h, 2 * h + 1, KR * a);
        y[i] = row_frag(sh.K[i], kb, 2 * h, 2 * h + 1, KR * b);
      }
      for_parts<NP, NP>([&](int i, int j) {
        f32x4& acc = i + j == 0 ? hi : lo;
        acc = mfma_bf16(x[i], y[j], acc);
      });
    }
    const f32x4 acc = hi + lo;
    const int j = 16 * b + lr;
    const double gj = sh.g[j];
    const float be = sh.be[j];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int i = 16 * a + 4 * lq + q;
      sh.M[i][j] = j < i ? exp2_fast(float(sh.g[i] - gj)) * be * acc[q] : 0.f;
    }
  };
  // (1, 0), (2, 0), (2, 1), (3, 0); (3, 1), (3, 2); the diagonal block w
  tile(w == 0 ? 1 : w < 3 ? 2 : 3, w == 2 ? 1 : 0);
  if (w < 2) tile(3, w + 1);
  tile(w, w);
  f32x4 tc[4];  // blocks (w + d, w) of T, rows 4 lq + component, column lr
  {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float x[16];
    f32x4 m[16][4];
#pragma unroll
    for (int i = 1; i < 16; ++i)
#pragma unroll
      for (int q = 0; q < (i + 3) / 4; ++q)
        m[i][q] = *reinterpret_cast<const f32x4*>(&sh.M[16 * w + i][16 * w + 4 * q]);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i == lr ? 1.f : 0.f;
#pragma unroll
    for (int j = 0; j < 15; ++j)
#pragma unroll
      for (int i = j + 1; i < 16; ++i) x[i] = fmaf(-m[i][j >> 2][j & 3], x[j], x[i]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      tc[0][q] = lq == 0 ? x[q] : lq == 1 ? x[4 + q] : lq == 2 ? x[8 + q] : x[12 + q];
      sh.M[16 * w + 4 * lq + q][16 * w + lr] = tc[0][q];
    }
  }
  __syncthreads();  // (the keys are not read any more: T takes their place)
#pragma unroll
  for (int d = 1; d < 4; ++d) {
    if (w + d >= 4) break;
    const int i = w + d;
    f32x4 a0 = {0.f, 0.f, 0.f, 0.f}, a1 = a0;
#pragma unroll
    for (int e = 0; e < d; ++e) {
      const f32x4 mm = *reinterpret_cast<const f32x4*>(&sh.M[16 * i + lr][16 * (w + e) + 4 * lq]);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        f32x4& acc = (s & 1) ? a1 : a0;
        acc = mfma4(mm[s], tc[e][s], acc);
      }
    }
    const f32x4 pr = a0 + a1;
    const f32x4 tt = *reinterpret_cast<const f32x4*>(&sh.M[16 * i + lr][16 * i + 4 * lq]);
    f32x4 b0 = {0.f, 0.f, 0.f, 0.f}, b1 = b0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      f32x4& acc = (s & 1) ? b1 : b0;
      acc = mfma4(tt[s], pr[s], acc);
    }
    tc[d] = -(b0 + b1);
#pragma unroll
    for (int q = 0; q < 4; ++q) sh.T[16 * i + 4 * lq + q][16 * w + lr] = tc[d][q];
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    sh.T[16 * w + 4 * lq + q][16 * w + lr] = tc[0][q];
    // the blocks above the diagonal that a 32-token step covers
    if (w & 1) sh.T[16 * (w - 1) + 4 * lq + q][16 * w + lr] = 0.f;
  }
  __syncthreads();
  // T fragments: lane (lr, lq) of (row tile a, step h) holds row 16 a + lr and the
  // columns 32 h + 4 lq + 0..3 and 32 h + 16 + 4 lq + 0..3, the order in which the
  // scan's accumulators hold the tokens; reversed, rows and columns count from
  // the chunk's end and change places
  for (int f = w; f < kTFrags; f += 4) {
    const int a = f < 2 ? f : f < 4 ? 2 : 3, h = f < 2 ? 0 : f & 1;
    const int t = 16 * a + lr, s0 = 32 * h + 4 * lq;
    uint4 x[3];
    split3(*reinterpret_cast<const f32x4*>(&sh.T[t][s0]),
           *reinterpret_cast<const f32x4*>(&sh.T[t][s0 + 16]), x[0], x[1], x[2]);
#pragma unroll
    for (int i = 0; i < 3; ++i) p.tf[cu * kTChunk + (f * 3 + i) * 64 + lane] = x[i];
    if constexpr (BWD) {
      f32x4 y0, y1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y0[j] = sh.T[kC - 1 - (s0 + j)][kC - 1 - t];
        y1[j] = sh.T[kC - 1 - (s0 + 16 + j)][kC - 1 - t];
      }
      split3(y0, y1, x[0], x[1], x[2]);
#pragma unroll
      for (int i = 0; i < 3; ++i) p.tr[cu * kTChunk + (f * 3 + i) * 64 + lane] = x[i];
    }
  }
}

// ---- the chain over the chunks -------------------------------------------------

// Waves of a scan workgroup (16 state rows each) of a head of DV rows.
template <int DV>
constexpr int kScanWaves = DV / 16 < 8 ? DV / 16 : 8;

template <int DK, int NP, int NW, bool REV>
struct ScanLds {
  struct Buf {
    alignas(16) Swz<DK> K[NP * (REV ? 2 : 1)];  // keys, reversed: then queries
    alignas(16) std::conditional_t<NP == 1, Swz<16 * NW>, char> V;  // values / dO
    alignas(16) u32x4 T[kTChunk];
    alignas(16) float ga[kC], gb[kC];
  };
  static constexpr int kBufs = 2 * sizeof(Buf) <= 160 * 1024 ? 2 : 1;
  Buf b[kBufs];
};

// The chain over the chunks of one (sequence, value head), 16 NW rows of the state
// per workgroup, 16 per wave: S^T in DK / 16 accumulator tiles that stay in registers.
// Forward, per chunk:
//   Y = K S^T, X = V - gamma Y, e = T X, S^T <- g S^T + K^T (beta sigma e);
// in reverse (tokens counted from the chunk's end, S the adjoint):
//   Y = K S^T, X = H + beta sigma Y, dV = T' X, S^T <- g S^T - K^T (gamma dV) + Q^T (scale gamma dO).
// The state at the chunk's entry and e (dV) go to the workspace.  All products
// chain in registers: the order of tokens and columns within a 32-deep step is that
// of the accumulators.
template <int DK, int DV, int NP, bool REV>
__global__ __launch_bounds__(64 * kScanWaves<DV>) void delta_scan_kernel(DeltaParams p) {
  constexpr int NW = kScanWaves<DV>, TH = 64 * NW, GB = DV / (16 * NW);
  constexpr int NB = DK / 16;
  constexpr int PS = NB / 2 < 4 ? NB / 2 : 4;
  auto t0 = [](int h) constexpr { return h / PS * (2 * PS) + h % PS; };
  constexpr int kIo = NP == 1 ? 2 : 4;
  constexpr int NT = (kTChunk + TH - 1) / TH;
  using Lds = ScanLds<DK, NP, NW, REV>;
  constexpr int kBufs = Lds::kBufs;
  __shared__ __align__(16) Lds buf;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int grp = blockIdx.x % GB, unit = blockIdx.x / GB;
  const int n = unit / p.HV, hv = unit - n * p.HV, hk = hv / (p.HV / p.HK);
  const int row0 = 16 * NW * grp + 16 * w;  // this wave's rows
  const Seq sq = seq_of(p, n);
  const int nch = (sq.len + kC - 1) / kC;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};

  f32x4 st[NB];  // st[b][i] = S^T(16 b + 4 lq + i, lr) = S(row0 + lr, 16 b + 4 lq + i)
  const float* const from = REV ? p.ds_in : p.s_in;
  const long sat = (long(unit) * DV + row0 + lr) * DK + 4 * lq;
#pragma unroll
  for (int b = 0; b < NB; ++b)
    st[b] = from ? *reinterpret_cast<const f32x4*>(from + sat + 16 * b) : z;

  // operands of the next chunk, on their way
  RowStage<DK, NP, TH, REV> rk, rq;
  RowStage<16 * NW, 1, TH, REV> rv;
  u32x4 rt[NT];
  float rga = 0.f, rgb = 0.f, rvf[NP == 1 ? 1 : 16];
  f32x4 rh[4];
  const unsigned ks = unsigned(p.ks) * kIo, qs = unsigned(p.qs) * kIo;
  const unsigned vs = REV ? unsigned(p.HV) * (DV * kIo) : unsigned(p.vs) * kIo;
  const int vcol = hv * DV + 16 * NW * grp;
  auto cu_of = [&](int c) { return (sq.slot + c) * p.HV + hv; };
  auto chunk = [&](int s) {  // the s-th chunk of the walk (past its end: the last)
    s = min(s, nch - 1);
    return REV ? nch - 1 - s : s;
  };
  auto load = [&](int s) __attribute__((always_inline)) {
    const int c = chunk(s), m = min(kC, sq.len - c * kC);
    const long tok = sq.t0 + long(c) * kC, cu = cu_of(c);
    rk.load(rows_buffer(p.k, (tok * p.ks + hk * DK) * kIo, DK * kIo, ks, m), ks, tid);
    if constexpr (REV)
      rq.load(rows_buffer(p.q, (tok * p.qs + hk * DK) * kIo, DK * kIo, qs, m), qs, tid);
    const auto vr = rows_buffer(REV ? p.d_o : p.v,
                                (tok * (REV ? long(p.HV) * DV : p.vs) + vcol) * kIo,
                                16 * NW * kIo, vs, m);
    if constexpr (NP == 1) {
      rv.load(vr, vs, tid);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = 16 * (i >> 2) + 4 * lq + (i & 3);
        rvf[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
            vr, unsigned(REV ? kC - 1 - t : t) * vs + (16 * w + lr) * 4, 0, 0));
      }
    }
    if constexpr (REV) {
      const float* h = p.hws + (cu * DV + row0 + lr) * kC + 60 - 4 * lq;
#pragma unroll
      for (int a = 0; a < 4; ++a) rh[a] = *reinterpret_cast<const f32x4*>(h - 16 * a);
    }
    const auto tr = buffer((REV ? p.tr : p.tf) + cu * kTChunk, kTChunk * 16);
#pragma unroll
    for (int q = 0; q < NT; ++q)
      rt[q] = __builtin_amdgcn_raw_buffer_load_b128(tr, tid * 16, q * TH * 16, 0);
    const float* g = p.gates + cu * (kDeltaGates * kC) + (REV ? kC - 1 - (tid & 63) : tid & 63);
    rga = g[(REV ? kGateB : kGateA) * kC];
    rgb = g[(REV ? kGateA : kGateB) * kC];
  };
  auto store = [&](int x) __attribute__((always_inline)) {
    auto& b = buf.b[x];
    rk.store(b.K, tid);
    if constexpr (REV) rq.store(b.K + NP, tid);
    if constexpr (NP == 1) rv.store(&b.V, tid);
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      const int e = tid + q * TH;
      if (kTChunk % TH == 0 || e < kTChunk) b.T[e] = rt[q];
    }
    if (tid < kC) {
      b.ga[tid] = rga;
      b.gb[tid] = rgb;
    }
  };
  const int kb = Swz<DK>::off(lr, lq), tb = Swz<DK>::off(4 * lq + (lr >> 2), lr & 3),
            vb = Swz<16 * NW>::off(4 * lq + (lr >> 2), 4 * w + (lr & 3));
  constexpr int KR = 32 * Swz<DK>::LD, VR = 32 * Swz<16 * NW>::LD;  // bytes of 16 rows
  auto step = [&](int c, int x, const f32x4(&hb)[4], const float* vf) __attribute__((always_inline)) {
    const auto& b = buf.b[x];
    const long cu = cu_of(c);
    {  // the state at the chunk's entry
      float* const d = (REV ? p.dsws : p.sws) + (cu * DV + row0 + lr) * DK + 4 * lq;
#pragma unroll
      for (int i = 0; i < NB; ++i) *reinterpret_cast<f32x4*>(d + 16 * i) = st[i];
    }
    // Y = K S^T
    f32x4 yh[4], yl[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) yh[a] = yl[a] = z;
#pragma unroll
    for (int h = 0; h < DK / 32; ++h) {
      uint4 kf[NP][4], sp[3];
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int a = 0; a < 4; ++a) kf[i][a] = row_frag(b.K[i], kb, t0(h), t0(h) + PS, KR * a);
      parts_of<3>(st[t0(h)], st[t0(h) + PS], sp);
      for_parts<NP, 3>([&](int i, int j) {
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          f32x4& acc = i + j == 0 ? yh[a] : yl[a];
          acc = mfma_bf16(kf[i][a], sp[j], acc);
        }
      });
    }
    // values (forward) or output gradients (reverse) of this lane: t = 16 a + 4 lq + i, n = lr
    f32x4 vv[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      if constexpr (NP == 1) {
        const uint2 u = lds_tr4(b.V.template at<uint16_t>(vb, 0, VR * a));
        vv[a] = f32x4{bf16_lo_to_float(u.x), bf16_hi_to_float(u.x), bf16_lo_to_float(u.y),
                      bf16_hi_to_float(u.y)};
      } else {
        vv[a] = f32x4{vf[4 * a], vf[4 * a + 1], vf[4 * a + 2], vf[4 * a + 3]};
      }
    }
    uint4 xp[2][3];
    {
      f32x4 xx[4];
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 g = *reinterpret_cast<const f32x4*>(&b.ga[16 * a + 4 * lq]);
        const f32x4 y = yh[a] + yl[a];
        f32x4 base = vv[a];
        if constexpr (REV) base = f32x4{hb[a].w, hb[a].z, hb[a].y, hb[a].x};
#pragma unroll
        for (int i = 0; i < 4; ++i) xx[a][i] = fmaf(g[i], y[i], base[i]);
      }
      parts_of<3>(xx[0], xx[1], xp[0]);
      parts_of<3>(xx[2], xx[3], xp[1]);
    }
    // e = T X
    f32x4 eh[4], el[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) eh[a] = el[a] = z;
#pragma unroll
    for (int f = 0; f < kTFrags; ++f) {
      const int a = f < 2 ? f : f < 4 ? 2 : 3, h = f < 2 ? 0 : f & 1;
      uint4 tf[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) tf[i] = __builtin_bit_cast(uint4, b.T[(f * 3 + i) * 64 + lane]);
      for_parts<3, 3>([&](int i, int j) {
        f32x4& acc = i + j == 0 ? eh[a] : el[a];
        acc = mfma_bf16(tf[i], xp[h][j], acc);
      });
    }
    uint4 ep[2][3], op[REV ? 2 : 1][3];
    {
      float* const d = (REV ? p.hws : p.ews) + (cu * DV + row0 + lr) * kC + (REV ? 60 - 4 * lq : 4 * lq);
      f32x4 ee[4];
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 e = eh[a] + el[a];
        const f32x4 g = *reinterpret_cast<const f32x4*>(&b.gb[16 * a + 4 * lq]);
        if constexpr (REV) {
          *reinterpret_cast<f32x4*>(d - 16 * a) = f32x4{e.w, e.z, e.y, e.x};
          vv[a] = (-p.scale * g) * vv[a];
        } else {
          *reinterpret_cast<f32x4*>(d + 16 * a) = e;
        }
        ee[a] = g * e;
      }
      parts_of<3>(ee[0], ee[1], ep[0]);
      parts_of<3>(ee[2], ee[3], ep[1]);
      if constexpr (REV) {
        parts_of<3>(vv[0], vv[1], op[0]);
        parts_of<3>(vv[2], vv[3], op[1]);
      }
    }
    // S^T <- g S^T + K^T (.)
    const float gc = REV ? -b.gb[0] : -b.ga[kC - 1];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      f32x4 hi = z, lo = z;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 kt[NP];
#pragma unroll
        for (int u = 0; u < NP; ++u) kt[u] = col_frag(b.K[u], tb, i, 2 * KR * h);
        for_parts<NP, 3>([&](int u, int j) {
          f32x4& acc = u + j == 0 ? hi : lo;
          acc = mfma_bf16(kt[u], ep[h][j], acc);
        });
        if constexpr (REV) {
#pragma unroll
          for (int u = 0; u < NP; ++u) kt[u] = col_frag(b.K[NP + u], tb, i, 2 * KR * h);
          for_parts<NP, 3>([&](int u, int j) {
            f32x4& acc = u + j == 0 ? hi : lo;
            acc = mfma_bf16(kt[u], op[h][j], acc);
          });
        }
      }
      st[i] = gc * st[i] + (hi + lo);
    }
  };
  if (nch > 0) {
    load(0);
    store(0);
    f32x4 hb[4] = {rh[0], rh[1], rh[2], rh[3]};
    float vf[NP == 1 ? 1 : 16];
#pragma unroll
    for (int i = 0; i < (NP == 1 ? 1 : 16); ++i) vf[i] = NP == 1 ? 0.f : rvf[i];
    __syncthreads();
    for (int s = 0; s < nch; ++s) {
      const int x = kBufs == 2 ? s & 1 : 0;
      __builtin_amdgcn_sched_barrier(0);
      load(s + 1);
      __builtin_amdgcn_sched_barrier(0);
      step(chunk(s), x, hb, vf);
      if constexpr (kBufs == 1) __syncthreads();
      store(kBufs == 2 ? x ^ 1 : 0);
#pragma unroll
      for (int a = 0; a < 4; ++a) hb[a] = rh[a];
      if constexpr (NP == 3) {
#pragma unroll
        for (int i = 0; i < 16; ++i) vf[i] = rvf[i];
      }
      __syncthreads();
    }
  }
  float* const to = REV ? p.ds_out : p.s_out;
  if (to) {
#pragma unroll
    for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4*>(to + sat + 16 * b) = st[b];
  }
}

// ---- the chunk's own products ----------------------------------------------------

// 64 rows of 64 bf16 elements that are written in pieces of 4 and read by rows
// (padded by 16 bytes).
struct Square {
  uint16_t x[kC][kC + 8];
};

// scale Gamma(i, j) (q_i . k_j) of the lower triangle as NQ parts, times beta_j: by
// rows i (TR = false) or by rows j (TR = true), with the blocks above (below) the
// diagonal that a 32-deep step covers zero.  Four waves.
template <int DK, int NP, int NQ, bool TR>
__device__ inline void scores(const Swz<DK>* Q, const Swz<DK>* K, Square* out, const float* gates,
                              float scale, int w, int lane) {
  const int lr = lane & 15, lq = lane >> 4;
  const int kb = Swz<DK>::off(lr, lq);
  constexpr int KR = 32 * Swz<DK>::LD;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};
  for (int x = w; x < 12; x += 4) {
    if (x >= 10) {  // (0, 1) and (2, 3), above the diagonal
      const int a = 2 * (x - 10), b = a + 1;
      const int r = TR ? 16 * b + lr : 16 * a + lr, c = TR ? 16 * a : 16 * b;
#pragma unroll
      for (int i = 0; i < NQ; ++i)
        *reinterpret_cast<uint2*>(&out[i].x[r][c + 4 * lq]) = make_uint2(0u, 0u);
      continue;
    }
    int a, b;
    tile_of(x, a, b);
    f32x4 hi = z, lo = z;
#pragma unroll
    for (int h = 0; h < DK / 32; ++h) {
      uint4 qf[NP], kf[NP];
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        qf[i] = row_frag(Q[i], kb, 2 * h, 2 * h + 1, KR * a);
        kf[i] = row_frag(K[i], kb, 2 * h, 2 * h + 1, KR * b);
      }
      for_parts<NP, NP>([&](int i, int j) {
        f32x4& acc = i + j == 0 ? hi : lo;
        acc = TR ? mfma_bf16(qf[i], kf[j], acc) : mfma_bf16(kf[i], qf[j], acc);
      });
    }
    f32x4 s = hi + lo;  // TR: rows 4 lq + i of q, column lr of k; else the other way round
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 16 * a + (TR ? 4 * lq + e : lr), j = 16 * b + (TR ? lr : 4 * lq + e);
      const float d = (gates[kGateHi * kC + i] - gates[kGateHi * kC + j]) +
                      (gates[kGateLo * kC + i] - gates[kGateLo * kC + j]);
      s[e] = j <= i ? scale * exp2_fast(d) * gates[kGateBeta * kC + j] * s[e] : 0.f;
    }
    uint2 part[NQ];
    parts4<NQ>(s, part);
    const int r = TR ? 16 * b + lr : 16 * a + lr, c = TR ? 16 * a : 16 * b;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
      *reinterpret_cast<uint2*>(&out[i].x[r][c + 4 * lq]) = part[i];
  }
}

template <int DK, int NP>
struct OutLds {
  Swz<DK> Q[NP], K[NP];
  Square P[NP == 1 ? 2 : 3];
  alignas(16) float gates[kDeltaGates * kC];
};

// O = scale diag(gamma) Q S^T + P diag(beta) e of one chunk of one value head, up to 128
// rows of the state per workgroup, 32 per wave, as O^T: the state's and e's
// rows go from memory straight into operands, each once.  Bound: HBM (the state).
template <int DK, int NP>
__global__ __launch_bounds__(kThreads) void delta_out_kernel(DeltaParams p) {
  constexpr int kIo = NP == 1 ? 2 : 4, NQ = NP == 1 ? 2 : 3;
  __shared__ __align__(16) OutLds<DK, NP> sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int groups = (p.DV + 127) / 128;
  const int grp = blockIdx.x % groups;
  const long cu = blockIdx.x / groups, slot = cu / p.HV;
  const int hv = int(cu - slot * p.HV), hk = hv / (p.HV / p.HK);
  const Chunk ch = chunk_of(p, slot);
  if (ch.n <= 0) return;
  const unsigned ks = unsigned(p.ks) * kIo, qs = unsigned(p.qs) * kIo;
  RowStage<DK, NP, kThreads> rk, rq;
  rk.load(rows_buffer(p.k, (ch.t0 * p.ks + hk * DK) * kIo, DK * kIo, ks, ch.n), ks, tid);
  rq.load(rows_buffer(p.q, (ch.t0 * p.qs + hk * DK) * kIo, DK * kIo, qs, ch.n), qs, tid);
  for (int i = tid; i < kDeltaGates * kC; i += kThreads)
    sh.gates[i] = p.gates[cu * (kDeltaGates * kC) + i];
  rk.store(sh.K, tid);
  rq.store(sh.Q, tid);
  __syncthreads();
  scores<DK, NP, NQ, false>(sh.Q, sh.K, sh.P, sh.gates, p.scale, w, lane);
  __syncthreads();
  const int kb = Swz<DK>::off(lr, lq);
  constexpr int KR = 32 * Swz<DK>::LD;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};
  const int n0 = 128 * grp + 32 * w;
  if (n0 >= p.DV) return;
  // row r of tile u is the state row n0 + 8 (r / 4) + 4 u + r % 4, so that a lane ends
  // with 8 neighbouring rows of a token
  f32x4 acc[2][4], lo[2][4];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int a = 0; a < 4; ++a) acc[u][a] = lo[u][a] = z;
  const int nr = n0 + 8 * (lr >> 2) + (lr & 3);
  const float* const sp = p.sws + (cu * p.DV + nr) * DK + 4 * lq;
#pragma unroll
  for (int h = 0; h < DK / 32; ++h) {
    uint4 s[2][NQ];
#pragma unroll
    for (int u = 0; u < 2; ++u)
      parts_of<NQ>(*reinterpret_cast<const f32x4*>(sp + 4 * u * DK + 32 * h),
                   *reinterpret_cast<const f32x4*>(sp + 4 * u * DK + 32 * h + 16), s[u]);
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      uint4 qf[NP];
#pragma unroll
      for (int i = 0; i < NP; ++i) qf[i] = row_frag(sh.Q[i], kb, 2 * h, 2 * h + 1, KR * a);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        for_parts<NQ, NP>([&](int i, int j) {
          f32x4& c = i + j == 0 ? acc[u][a] : lo[u][a];
          c = mfma_bf16(s[u][i], qf[j], c);
        });
    }
  }
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const float g = -p.scale * sh.gates[kGateA * kC + 16 * a + lr];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      acc[u][a] = g * (acc[u][a] + lo[u][a]);
      lo[u][a] = z;
    }
  }
  const float* const ep = p.ews + (cu * p.DV + nr) * kC + 8 * lq;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint4 e[2][NQ];
#pragma unroll
    for (int u = 0; u < 2; ++u)
      parts_of<NQ>(*reinterpret_cast<const f32x4*>(ep + 4 * u * kC + 32 * h),
                   *reinterpret_cast<const f32x4*>(ep + 4 * u * kC + 32 * h + 4), e[u]);
#pragma unroll
    for (int a = 2 * h; a < 4; ++a) {
      uint4 pf[NQ];
#pragma unroll
      for (int i = 0; i < NQ; ++i)
        pf[i] = *reinterpret_cast<const uint4*>(&sh.P[i].x[16 * a + lr][32 * h + 8 * lq]);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        for_parts<NQ, NQ>([&](int i, int j) {
          if (NQ == 2 && i + j == 2) return;
          f32x4& c = i + j == 0 ? acc[u][a] : lo[u][a];
          c = mfma_bf16(e[u][i], pf[j], c);
        });
    }
  }
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int t = 16 * a + lr;
    if (t >= ch.n) continue;
    const f32x4 x = acc[0][a] + lo[0][a], y = acc[1][a] + lo[1][a];
    const long at = ((ch.t0 + t) * p.HV + hv) * p.DV + n0 + 8 * lq;
    if constexpr (NP == 1) {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.o) + at) =
          make_uint4(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w), pack_bf16x2(y.x, y.y),
                     pack_bf16x2(y.z, y.w));
    } else {
      float* const o = static_cast<float*>(p.o) + at;
      *reinterpret_cast<f32x4*>(o) = x;
      *reinterpret_cast<f32x4*>(o + 4) = y;
    }
  }
}

// ---- backward: the chunk's own part of dD -----------------------------------------

template <int DK, int NP, int DVB>
struct IntraLds {
  union {
    struct {
      Swz<DK> Q[NP], K[NP];
    } qk;
    Swz<DVB> dO[NP];  // after the scores
  };
  Square P[3];
  alignas(16) float gates[kDeltaGates * kC];
};

// H = diag(beta) P^T dO of one chunk of one value head, DVB columns per workgroup (at
// most 128), 16 per wave and turn; stored as H^T.
template <int DK, int NP, int DVB>
__global__ __launch_bounds__(kThreads) void delta_intra_kernel(DeltaParams p) {
  constexpr int kIo = NP == 1 ? 2 : 4;
  __shared__ __align__(16) IntraLds<DK, NP, DVB> sh;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int groups = p.DV / DVB, grp = blockIdx.x % groups;
  const long cu = blockIdx.x / groups, slot = cu / p.HV;
  const int hv = int(cu - slot * p.HV), hk = hv / (p.HV / p.HK);
  const Chunk ch = chunk_of(p, slot);
  if (ch.n <= 0) return;
  const unsigned ks = unsigned(p.ks) * kIo, qs = unsigned(p.qs) * kIo;
  const unsigned os = unsigned(p.HV) * p.DV * kIo;
  RowStage<DK, NP, kThreads> rk, rq;
  RowStage<DVB, NP, kThreads> ro;
  rk.load(rows_buffer(p.k, (ch.t0 * p.ks + hk * DK) * kIo, DK * kIo, ks, ch.n), ks, tid);
  rq.load(rows_buffer(p.q, (ch.t0 * p.qs + hk * DK) * kIo, DK * kIo, qs, ch.n), qs, tid);
  for (int i = tid; i < kDeltaGates * kC; i += kThreads)
    sh.gates[i] = p.gates[cu * (kDeltaGates * kC) + i];
  rk.store(sh.qk.K, tid);
  rq.store(sh.qk.Q, tid);
  ro.load(rows_buffer(p.d_o, ((ch.t0 * p.HV + hv) * p.DV + grp * DVB) * kIo, DVB * kIo, os, ch.n),
          os, tid);
  __syncthreads();
  scores<DK, NP, 3, true>(sh.qk.Q, sh.qk.K, sh.P, sh.gates, p.scale, w, lane);
  __syncthreads();
  ro.store(sh.dO, tid);
  __syncthreads();
  const int ob = Swz<DVB>::off(4 * lq + (lr >> 2), lr & 3);
  constexpr int OR = 32 * Swz<DVB>::LD;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};
  for (int nb = w; nb < DVB / 16; nb += 4) {
    uint4 of[2][NP];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < NP; ++i) of[h][i] = col_frag(sh.dO[i], ob, nb, 2 * OR * h);
    float* const dst = p.hws + (cu * p.DV + grp * DVB + 16 * nb + lr) * kC + 4 * lq;
#pragma unroll
    for (int a = 0; a < 4; ++a) {  // tokens j = 16 a + ..
      f32x4 hi = z, lo = z;
#pragma unroll
      for (int h = a >> 1; h < 2; ++h) {
        uint4 pf[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const uint16_t* r = sh.P[i].x[16 * a + lr] + 32 * h + 4 * lq;
          const uint2 x = *reinterpret_cast<const uint2*>(r),
                      y = *reinterpret_cast<const uint2*>(r + 16);
          pf[i] = make_uint4(x.x, x.y, y.x, y.y);
        }
        for_parts<3, NP>([&](int i, int j) {
          f32x4& acc = i + j == 0 ? hi : lo;
          acc = mfma_bf16(pf[i], of[h][j], acc);
        });
      }
      *reinterpret_cast<f32x4*>(dst + 16 * a) = hi + lo;
    }
  }
}

// ---- backward: gradients of the chunk ----------------------------------------------

constexpr int kNB = 32;  // columns of the values taken at a time

template <int DK, int NP>
struct GradLds {
  static constexpr int NQ = NP == 1 ? 2 : 3;
  Swz<DK> Q[NP], K[NP];
  union {
    struct {
      Swz<kC, kNB> e[3], dv[3];        // [columns][tokens]
      uint16_t dO[NP][kC][kNB + 16];   // [tokens][columns]
    } s;
    Square P[NQ];  // L, then its transpose, then M + M^T
  };
  alignas(16) float gates[kDeltaGates * kC];
  float dots[8][3][kC];    // per wave: q . (dO S), k . (dV S), k . (e dS)
  float zrow[4][kC];       // sums of Z over a column block
  float zcol[4][kC], bcol[4][kC];  // sums over a row block: Z; P X - B N
  float ss[8];
};

// Gradients of one chunk and one query/key head (the value heads of its group in
// turn, their dQ and dK summed in registers).  Wave w holds the key columns 16 CT w ..
// of dQ and dK; the tiles of the token by token products are dealt out to the waves.
template <int DK, int NP, int NW>
__global__ __launch_bounds__(64 * NW) void delta_grad_kernel(DeltaParams p) {
  constexpr int TH = 64 * NW, CT = DK / (16 * NW), MT = (10 + NW - 1) / NW;
  constexpr int kIo = NP == 1 ? 2 : 4;
  using Lds = GradLds<DK, NP>;
  constexpr int NQ = Lds::NQ;
  extern __shared__ __align__(16) unsigned char smem[];
  Lds& sh = *reinterpret_cast<Lds*>(smem);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const long slot = blockIdx.x / p.HK;
  const int hk = int(blockIdx.x - slot * p.HK), G = p.HV / p.HK;
  const Chunk ch = chunk_of(p, slot);
  if (ch.n <= 0) return;
  const unsigned ks = unsigned(p.ks) * kIo, qs = unsigned(p.qs) * kIo;
  const unsigned os = unsigned(p.HV) * p.DV * kIo;
  {
    RowStage<DK, NP, TH> rk, rq;
    rk.load(rows_buffer(p.k, (ch.t0 * p.ks + hk * DK) * kIo, DK * kIo, ks, ch.n), ks, tid);
    rq.load(rows_buffer(p.q, (ch.t0 * p.qs + hk * DK) * kIo, DK * kIo, qs, ch.n), qs, tid);
    rk.store(sh.K, tid);
    rq.store(sh.Q, tid);
  }
  const int kb = Swz<DK>::off(lr, lq), tb = Swz<DK>::off(4 * lq + (lr >> 2), lr & 3);
  const int eb = Swz<kC, kNB>::off(4 * lq + (lr >> 2), lr & 3);
  constexpr int KR = 32 * Swz<DK>::LD;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};
  f32x4 aq[4][CT], ak[4][CT];  // dQ, dK(t = 16 a + 4 lq + i, 16 (CT w + c) + lr)
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int c = 0; c < CT; ++c) aq[a][c] = ak[a][c] = z;

  for (int hg = 0; hg < G; ++hg) {
    const int hv = hk * G + hg;
    const long cu = slot * p.HV + hv;
    __syncthreads();  // (the last head's readers are done)
    for (int i = tid; i < kDeltaGates * kC; i += TH)
      sh.gates[i] = p.gates[cu * (kDeltaGates * kC) + i];
    f32x4 xs[MT], ns[MT];  // tiles of X = dO e^T and N = dV e^T
#pragma unroll
    for (int m = 0; m < MT; ++m) xs[m] = ns[m] = z;
    f32x4 qS[4][CT], kS[4][CT], eD[4][CT];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int c = 0; c < CT; ++c) qS[a][c] = kS[a][c] = eD[a][c] = z;
    float ss = 0.f;
    for (int nb = 0; nb < p.DV / kNB; ++nb) {
      const int n0 = nb * kNB;
      // e and dV [columns][tokens] and dO [tokens][columns] into LDS
      constexpr int NE = kNB * kC / 4 / TH;
      static_assert(NE >= 1, "");
      f32x4 re[NE], rd[NE];
#pragma unroll
      for (int q = 0; q < NE; ++q) {
        const int e = tid + q * TH;
        re[q] = *reinterpret_cast<const f32x4*>(p.ews + (cu * p.DV + n0) * kC + 4 * e);
        rd[q] = *reinterpret_cast<const f32x4*>(p.hws + (cu * p.DV + n0) * kC + 4 * e);
      }
      RowStage<kNB, NP, TH> ro;
      ro.load(rows_buffer(p.d_o, ((ch.t0 * p.HV + hv) * p.DV + n0) * kIo, kNB * kIo, os, ch.n), os,
              tid);
      // this lane's operands of the states: S(n, k = 16 (CT w + c) + lr) at n = n0 + 4 lq
      // + i and n0 + 16 + 4 lq + i
      f32x4 s0[CT][2], d0[CT][2];
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const long at = (cu * p.DV + n0 + 16 * u + 4 * lq + i) * DK + 16 * (CT * w + c) + lr;
            s0[c][u][i] = p.sws[at];
            d0[c][u][i] = p.dsws[at];
          }
      __syncthreads();  // (the last columns' readers are done)
#pragma unroll
      for (int q = 0; q < NE; ++q) {
        const int e = tid + q * TH, row = e / 16, pc = e % 16;
        uint2 x[3];
        parts4<3>(re[q], x);
        const int o = Swz<kC, kNB>::off(row, pc);
#pragma unroll
        for (int i = 0; i < 3; ++i)
          *reinterpret_cast<uint2*>(reinterpret_cast<char*>(sh.s.e[i].x) + o) = x[i];
        parts4<3>(rd[q], x);
#pragma unroll
        for (int i = 0; i < 3; ++i)
          *reinterpret_cast<uint2*>(reinterpret_cast<char*>(sh.s.dv[i].x) + o) = x[i];
      }
      {
        struct Tile {
          uint16_t x[kC][kNB + 16];
          __device__ void put(int row, int c, u32x4 v) {
            *reinterpret_cast<u32x4*>(&x[row][8 * c]) = v;
          }
        };
        ro.store(reinterpret_cast<Tile*>(sh.s.dO), tid);
      }
      __syncthreads();
      // dV as a tensor: 4 columns of a token per thread
      for (int e = tid; e < kC * kNB / 4; e += TH) {
        const int t = e / (kNB / 4), c = e % (kNB / 4);
        if (t < ch.n) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int o = Swz<kC, kNB>::off(4 * c + i, t >> 2) + 2 * (t & 3);
            x[i] = 0.f;
#pragma unroll
            for (int u = 2; u >= 0; --u)
              x[i] += __uint_as_float(
                  unsigned(*reinterpret_cast<const uint16_t*>(
                      reinterpret_cast<const char*>(sh.s.dv[u].x) + o)) << 16);
          }
          const long at = ((ch.t0 + t) * p.HV + hv) * p.DV + n0 + 4 * c;
          if constexpr (NP == 1) {
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.dv) + at) =
                make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
          } else {
            *reinterpret_cast<f32x4*>(static_cast<float*>(p.dv) + at) =
                f32x4{x[0], x[1], x[2], x[3]};
          }
        }
      }
      auto of = [&](int i, int a) {
        const uint16_t* r = sh.s.dO[i][16 * a + lr] + 4 * lq;
        const uint2 x = *reinterpret_cast<const uint2*>(r),
                    y = *reinterpret_cast<const uint2*>(r + 16);
        return make_uint4(x.x, x.y, y.x, y.y);
      };
      // X and N
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int x = w + m * NW;
        if (x >= 10) break;
        int a, b;
        tile_of(x, a, b);
        uint4 ef[3], df[3], og[NP];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          ef[i] = col_frag(sh.s.e[i], eb, b, 0);
          df[i] = col_frag(sh.s.dv[i], eb, a, 0);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) og[i] = of(i, a);
        for_parts<NP, 3>([&](int i, int j) { xs[m] = mfma_bf16(og[i], ef[j], xs[m]); });
        for_parts<3, 3>([&](int i, int j) { ns[m] = mfma_bf16(df[i], ef[j], ns[m]); });
      }
      // products with the states
      uint4 sp[CT][3], dp[CT][3];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        parts_of<3>(s0[c][0], s0[c][1], sp[c]);
        parts_of<3>(d0[c][0], d0[c][1], dp[c]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) ss = fmaf(s0[c][u][i], d0[c][u][i], ss);
      }
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        uint4 ef[3], df[3], og[NP];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          ef[i] = col_frag(sh.s.e[i], eb, a, 0);
          df[i] = col_frag(sh.s.dv[i], eb, a, 0);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) og[i] = of(i, a);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          for_parts<NP, 3>([&](int i, int j) { qS[a][c] = mfma_bf16(og[i], sp[c][j], qS[a][c]); });
          for_parts<3, 3>([&](int i, int j) { kS[a][c] = mfma_bf16(df[i], sp[c][j], kS[a][c]); });
          for_parts<3, 3>([&](int i, int j) { eD[a][c] = mfma_bf16(ef[i], dp[c][j], eD[a][c]); });
        }
      }
    }
    // rows' dot products with q and k, and the parts of dQ and dK from the states
    ss = group_sum<64>(ss);
    if (lane == 0) sh.ss[w] = ss;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int t0 = 16 * a + 4 * lq;
      const f32x4 ga = *reinterpret_cast<const f32x4*>(&sh.gates[kGateA * kC + t0]);
      const f32x4 gb = *reinterpret_cast<const f32x4*>(&sh.gates[kGateB * kC + t0]);
      f32x4 dots[3] = {z, z, z};
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const int col = 16 * (CT * w + c) + lr;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int o = Swz<DK>::off(t0 + i, col >> 2) + 2 * (col & 3);
          float qv = 0.f, kv = 0.f;
#pragma unroll
          for (int u = NP - 1; u >= 0; --u) {
            auto el = [&](const Swz<DK>& x) {
              return __uint_as_float(unsigned(*reinterpret_cast<const uint16_t*>(
                                         reinterpret_cast<const char*>(x.x) + o)) << 16);
            };
            qv += el(sh.Q[u]);
            kv += el(sh.K[u]);
          }
          dots[0][i] = fmaf(qv, qS[a][c][i], dots[0][i]);
          dots[1][i] = fmaf(kv, kS[a][c][i], dots[1][i]);
          dots[2][i] = fmaf(kv, eD[a][c][i], dots[2][i]);
        }
        aq[a][c] += (-p.scale * ga) * qS[a][c];
        ak[a][c] += gb * eD[a][c] + ga * kS[a][c];
      }
#pragma unroll
      for (int u = 0; u < 3; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = group_sum<16>(dots[u][i]);
          if (lr == 0) sh.dots[w][u][t0 + i] = s;
        }
    }
    // the tiles of L and M, their sums, and the products with Q and K
    f32x4 lt[MT], mt[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int x = w + m * NW;
      if (x >= 10) break;
      int a, b;
      tile_of(x, a, b);
      f32x4 qh = z, ql = z, kh = z, kl = z;
#pragma unroll
      for (int h = 0; h < DK / 32; ++h) {
        uint4 qf[NP], ka[NP], kf[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          qf[i] = row_frag(sh.Q[i], kb, 2 * h, 2 * h + 1, KR * a);
          ka[i] = row_frag(sh.K[i], kb, 2 * h, 2 * h + 1, KR * a);
          kf[i] = row_frag(sh.K[i], kb, 2 * h, 2 * h + 1, KR * b);
        }
        for_parts<NP, NP>([&](int i, int j) {
          f32x4& c = i + j == 0 ? qh : ql;
          c = mfma_bf16(qf[i], kf[j], c);
          f32x4& d = i + j == 0 ? kh : kl;
          d = mfma_bf16(ka[i], kf[j], d);
        });
      }
      const f32x4 qk = qh + ql, kk = kh + kl;
      const int j = 16 * b + lr;
      const float hj = sh.gates[kGateHi * kC + j], lj = sh.gates[kGateLo * kC + j],
                  bj = sh.gates[kGateBeta * kC + j];
      float cz = 0.f, cb = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = 16 * a + 4 * lq + q;
        const float d = (sh.gates[kGateHi * kC + i] - hj) + (sh.gates[kGateLo * kC + i] - lj);
        const float g = j <= i ? exp2_fast(d) : 0.f, gs = j < i ? g : 0.f;
        const float px = p.scale * g * xs[m][q], nx = gs * ns[m][q];
        lt[m][q] = px * bj;
        mt[m][q] = -nx * bj;
        const float zz = j < i ? lt[m][q] * qk[q] + mt[m][q] * kk[q] : 0.f;
        cb += px * qk[q] - nx * kk[q];
        cz += zz;
        const float rz = group_sum<16>(zz);
        if (lr == 0) sh.zrow[b][i] = rz;
      }
      cz += __shfl_xor(cz, 16);
      cb += __shfl_xor(cb, 16);
      cz += __shfl_xor(cz, 32);
      cb += __shfl_xor(cb, 32);
      if (lq == 0) {
        sh.zcol[a][j] = cz;
        sh.bcol[a][j] = cb;
      }
    }
    // three matrices of 64 x 64 in turn: dQ += L K, dK += L^T Q, dK += (M + M^T) K
#pragma unroll
    for (int turn = 0; turn < 3; ++turn) {
      __syncthreads();  // (readers of the columns, or of the last matrix, are done)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int x = w + m * NW;
        if (x >= 10) break;
        int a, b;
        tile_of(x, a, b);
        const f32x4 v = turn == 2 ? mt[m] : lt[m];
        uint2 part[NQ];
        parts4<NQ>(v, part);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          if (turn >= 1) {  // rows j = 16 b + lr, columns 16 a + 4 lq ..; M + M^T on the
                            // diagonal block: both triangles
            if (turn == 1 || a != b)
              *reinterpret_cast<uint2*>(&sh.P[i].x[16 * b + lr][16 * a + 4 * lq]) = part[i];
          }
          if (turn == 0 || turn == 2) {
            const uint16_t e4[4] = {uint16_t(part[i].x), uint16_t(part[i].x >> 16),
                                    uint16_t(part[i].y), uint16_t(part[i].y >> 16)};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int r = 16 * a + 4 * lq + q, cc = 16 * b + lr;
              if (turn == 0 || a != b) {
                sh.P[i].x[r][cc] = e4[q];
              } else if (cc <= r) {
                sh.P[i].x[r][cc] = e4[q];
                sh.P[i].x[cc][r] = e4[q];
              }
            }
          }
        }
      }
      if (turn < 2) {  // the blocks past the diagonal that a 32-deep step covers
        for (int e = tid; e < 2 * 64 * NQ; e += TH) {
          const int i = e / 128, blk = (e / 64) & 1, l = e & 63;
          const int a = 2 * blk, b = a + 1;  // (a, b) above the diagonal
          const int r = 16 * (turn == 0 ? a : b) + (l & 15), c = 16 * (turn == 0 ? b : a) + 4 * (l >> 4);
          *reinterpret_cast<uint2*>(&sh.P[i].x[r][c]) = make_uint2(0u, 0u);
        }
      }
      __syncthreads();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint4 bf[CT][NP];
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int i = 0; i < NP; ++i)
            bf[c][i] = col_frag(turn == 1 ? sh.Q[i] : sh.K[i], tb, CT * w + c, 2 * KR * h);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          if (turn == 0 && a < 2 * h) continue;     // L: columns up to the row
          if (turn == 1 && a >= 2 * h + 2) continue;  // L^T: columns from the row on
          uint4 pf[NQ];
#pragma unroll
          for (int i = 0; i < NQ; ++i) {
            const uint16_t* r = sh.P[i].x[16 * a + lr] + 32 * h + 4 * lq;
            const uint2 x = *reinterpret_cast<const uint2*>(r),
                        y = *reinterpret_cast<const uint2*>(r + 16);
            pf[i] = make_uint4(x.x, x.y, y.x, y.y);
          }
#pragma unroll
          for (int c = 0; c < CT; ++c)
            for_parts<NQ, NP>([&](int i, int j) {
              f32x4& acc = turn == 0 ? aq[a][c] : ak[a][c];
              acc = mfma_bf16(pf[i], bf[c][j], acc);
            });
        }
      }
    }
    // dbeta and dlog_alpha (the dot products and sums passed the barriers above)
    if (w == 0) {
      const int t = lane;
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
      const float gam = -sh.gates[kGateA * kC + t], bs = sh.gates[kGateB * kC + t];
      const float sg = exp2_fast((sh.gates[kGateHi * kC + 63] - sh.gates[kGateHi * kC + t]) +
                                 (sh.gates[kGateLo * kC + 63] - sh.gates[kGateLo * kC + t]));
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
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 16 * a + 4 * lq + i;
      if (t >= ch.n) continue;
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const long at = ((ch.t0 + t) * p.HK + hk) * DK + 16 * (CT * w + c) + lr;
        if constexpr (NP == 1) {
          const unsigned u = pack_bf16x2(aq[a][c][i], ak[a][c][i]);
          static_cast<uint16_t*>(p.dq)[at] = uint16_t(u);
          static_cast<uint16_t*>(p.dk)[at] = uint16_t(u >> 16);
        } else {
          static_cast<float*>(p.dq)[at] = aq[a][c][i];
          static_cast<float*>(p.dk)[at] = ak[a][c][i];
        }
      }
    }
}

template <int DK, int DV, int NP, bool BWD>
hipError_t run(const DeltaParams& p, hipStream_t st) {
  const unsigned cus = unsigned(p.slots) * unsigned(p.HV);
  hipError_t e;
#define ONELA_CHECK_LAUNCH()                             \
  if ((e = hipGetLastError()) != hipSuccess) return e
  if (cus) {
    delta_factor_kernel<DK, NP, BWD><<<cus, kThreads, 0, st>>>(p);
    ONELA_CHECK_LAUNCH();
  }
  constexpr int NW = kScanWaves<DV>;
  const unsigned scans = unsigned(p.N) * unsigned(p.HV) * (DV / (16 * NW));
  delta_scan_kernel<DK, DV, NP, false><<<scans, 64 * NW, 0, st>>>(p);
  ONELA_CHECK_LAUNCH();
  if constexpr (!BWD) {
    if (!cus) return hipSuccess;
    delta_out_kernel<DK, NP><<<cus * unsigned((DV + 127) / 128), kThreads, 0, st>>>(p);
    return hipGetLastError();
  } else {
    constexpr int DVB = DV < 128 ? DV : 128;
    if (cus) {
      delta_intra_kernel<DK, NP, DVB><<<cus * unsigned(DV / DVB), kThreads, 0, st>>>(p);
      ONELA_CHECK_LAUNCH();
    }
    delta_scan_kernel<DK, DV, NP, true><<<scans, 64 * NW, 0, st>>>(p);
    ONELA_CHECK_LAUNCH();
    if (!cus) return hipSuccess;
    constexpr int NG = DK / 16 < 8 ? DK / 16 : 8;
    auto grad = delta_grad_kernel<DK, NP, NG>;
    const size_t lds = sizeof(GradLds<DK, NP>);
    static_assert(sizeof(GradLds<DK, NP>) <= 160 * 1024, "one workgroup's LDS");
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(grad),
                            hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
    if (e != hipSuccess) return e;
    grad<<<unsigned(p.slots) * unsigned(p.HK), 64 * NG, lds, st>>>(p);
    return hipGetLastError();
  }
#undef ONELA_CHECK_LAUNCH
}

}  // namespace

hipError_t launch_delta_rule(const DeltaShape& s, DeltaParams p, bool backward, void* workspace,
                             hipStream_t st) {
  const size_t cus = size_t(s.slots) * s.HV;
  char* at = static_cast<char*>(workspace);
  auto take = [&](size_t bytes) {
    char* const x = at;
    at += bytes;
    return x;
  };
  if (!backward) {
    const size_t np = s.bf16 ? 1 : 2, image = size_t(s.slots) * s.HK * np * delta_image_bytes(s.dk);
    p.kimg = reinterpret_cast<uint4*>(take(image));
    p.qimg = reinterpret_cast<uint4*>(take(image));
    p.tp = reinterpret_cast<uint4*>(take(cus * 6 * 2 * 1024));
    p.pf = reinterpret_cast<uint4*>(take(cus * 6 * 2 * 1024));
    p.gates = reinterpret_cast<float*>(take(cus * kDeltaGates * kC * 4));
    const DeltaSegments sg = delta_segments(s, p.offsets != nullptr);
    p.cps = sg.cps;
    p.nseg_l = sg.nseg_l;
    p.seg_slots = sg.slots;
    if (sg.many) {
      p.segs = reinterpret_cast<float*>(take(size_t(sg.slots) * s.HV * s.dv * s.dk * 4));
      p.sega = reinterpret_cast<float*>(take(size_t(sg.slots) * s.HV * s.dk * s.dk * 4));
    }
    const hipError_t e = launch_delta_prep(s, p, st);
    return e == hipSuccess ? launch_delta_forward(s, p, st) : e;
  }
  p.tf = reinterpret_cast<uint4*>(take(cus * kDeltaFactorBytes));
  p.gates = reinterpret_cast<float*>(take(cus * kDeltaGates * kC * 4));
  p.sws = reinterpret_cast<float*>(take(cus * s.dv * s.dk * 4));
  p.ews = reinterpret_cast<float*>(take(cus * s.dv * kC * 4));
  p.tr = reinterpret_cast<uint4*>(take(cus * kDeltaFactorBytes));
  p.dsws = reinterpret_cast<float*>(take(cus * s.dv * s.dk * 4));
  p.hws = reinterpret_cast<float*>(take(cus * s.dv * kC * 4));
#define ONELA_DELTA_SHAPE(DK, DV, NP)                      \
  if (s.dk == DK && s.dv == DV && s.bf16 == (NP == 1))     \
    return run<DK, DV, NP, true>(p, st);
  ONELA_DELTA_SHAPE(32, 32, 1)
  ONELA_DELTA_SHAPE(64, 64, 1)
  ONELA_DELTA_SHAPE(128, 128, 1)
  ONELA_DELTA_SHAPE(128, 256, 1)
  ONELA_DELTA_SHAPE(128, 512, 1)
  ONELA_DELTA_SHAPE(256, 256, 1)
  ONELA_DELTA_SHAPE(256, 512, 1)
  ONELA_DELTA_SHAPE(32, 32, 3)
  ONELA_DELTA_SHAPE(64, 64, 3)
  ONELA_DELTA_SHAPE(128, 128, 3)
#undef ONELA_DELTA_SHAPE
  return hipErrorInvalidValue;
}

}  // namespace onela
