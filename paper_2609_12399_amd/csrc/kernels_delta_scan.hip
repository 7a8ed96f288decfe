// The delta rule's chain over the chunks, forward (see kernels_delta.hip), and the chain over
// the segments of either direction.
#include "delta_chain.h"

namespace onela {
namespace {

// What a walk over the chunks leaves: the outputs and the last state; the state after a
// segment; or for the backward pass the state before and e of every chunk.
enum { kOutputs, kSegment, kSave };

// The chain over the chunks of one (sequence, value head): up to 128 rows of the state per
// workgroup, 32 per wave, in registers (ChainState).  Per chunk
//   Y = K S^T, X = V - gamma Y, e = T X, O = scale gamma Q S^T + P e, S^T <- g S^T + K^T (beta sigma e)
// with all products chained in registers: the order of tokens and columns within a
// 32-deep step is that of the accumulators.
//
// Operands come to LDS straight from memory in the layout that is read there: the next
// chunk's keys and queries during T X and P e, its T, P and gates during the update.
//
// Segments.  One chain per 128 rows leaves most of the chip idle for few heads, so a
// sequence can be cut into segments of p.cps chunks that run at once: S_out = S_in A + B.
// kSegment forms, without outputs, for every segment but the sequence's last the
// state that it leaves: of the first the true one, of the others B (from S_in = 0)
// and, by the same code on the rows of the identity and V = 0, A.
// delta_combine_kernel chains them, and then every segment starts from its true state.
// The last state may be stored where the state to start from is (p.s_out == p.s_in), and in
// that last launch nothing orders the workgroup of a sequence's first segment, which would
// read it, before that of its last, which stores it.  So kSegment's first segment keeps
// the rows that it starts from in the last segment's place of p.segs, which holds nothing
// else, and the last launch reads them there.
//
// Bound: vector and matrix instructions (about 4 and 16 cycles each) take turns.  16 x 1024
// tokens x 32 heads of 128 (512 workgroups of 16 chunks) with outputs 173 us, 818 TFLOP/s of
// fp16 products: matrix cores 36% busy, vector units 43%, waves waiting 22%;
// kSave 244 us (3.3 TB/s written), kSegment 37 us for 16 segments of 4096 tokens x 16 heads.
// (Scales per row and measured updates, with two rows to a scale and a bound instead: 170 us, and
// small channels beside large ones lost.)  The outputs go before the update's values, whose
// largest is waited for while the stores leave: 16 segments 31.6 us, the other way round 33.6.
// Barriers that leave the stores in flight, operand reads a step ahead and one wave per SIMD
// with 512 registers were all slower.
template <int DK, int DV, int NP, int KIND>
__global__ __launch_bounds__(64 * kChainWaves<DV>, DK >= 256 || NP == 2 ? 1 : 2)
void delta_forward_kernel(DeltaParams p) {
  constexpr bool SEG = KIND == kSegment, OUT = KIND == kOutputs;
  constexpr int NW = kChainWaves<DV>, GB = DV / (32 * NW);
  constexpr int GA = SEG ? DK / (32 * NW) : 0;
  constexpr int kIo = NP == 1 ? 2 : 4;
  constexpr int kImage = sizeof(Swz<DK>) * NP;
  __shared__ __align__(16) Swz<DK> sK[2][NP];
  __shared__ __align__(16) Swz<DK> sQ[OUT ? NP : 1];
  __shared__ __align__(16) uint4 sT[kFragBytes / 16];
  __shared__ __align__(16) uint4 sP[OUT ? kFragBytes / 16 : 1];
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
  const int nch = sg.ce;
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};

  ChainState<DK> s;
  const long rows = long(row0) * DK + 4 * lq;
  {
    const float* from = start_of<DK, DV, SEG>(p, sg, su, hv, p.s_in);
    s.init(from ? from + rows : nullptr,
           SEG && from ? kept_start<DK, DV>(p, sg, su) + rows : nullptr, ident, row0, lq);
  }
  auto load_kq = [&](int c) __attribute__((always_inline)) {
    const long at = ((sq.slot + c) * p.HK + hk) * (kImage / 16);
    dma<kImage, NW>(p.kimg + at, sK[c & 1], w, lane);
    if constexpr (OUT) dma<kImage, NW>(p.qimg + at, sQ, w, lane);
  };
  auto load_tp = [&](int c) __attribute__((always_inline)) {
    const long cu = (sq.slot + c) * p.HV + hv;
    dma<kFragBytes, NW>(p.tp + cu * (kFragBytes / 16), sT, w, lane);
    if constexpr (OUT) dma<kFragBytes, NW>(p.pf + cu * (kFragBytes / 16), sP, w, lane);
    dma<kGateStage * kC * 4, NW>(p.gates + cu * (p.gate_rows * kC), sG, w, lane);
  };
  const unsigned vs = unsigned(p.vs) * kIo;
  Columns<NP> v;
  auto load_v = [&](int c) __attribute__((always_inline)) {
    const int m = ident ? 0 : min(kC, sq.len - c * kC);  // (A: no values)
    v.load(rows_buffer(p.v, ((sq.t0 + long(c) * kC) * p.vs + hv * DV) * kIo, DV * kIo, vs, m), vs,
           lq, row0 * kIo);
  };
  auto gate = [&](int row, int a) { return *reinterpret_cast<const f32x4*>(&sG[row][16 * a + 4 * lq]); };
  const int kb = Swz<DK>::off(lr, lq), tb = Swz<DK>::off(4 * lq + (lr >> 2), lr & 3);

  if (sg.cb < nch) {
    load_kq(sg.cb);
    load_tp(sg.cb);
    load_v(sg.cb);
  }
  for (int c = sg.cb; c < nch; ++c) {
    const Swz<DK>* const K = sK[c & 1];
    if (KIND == kSave || (c - sg.cb) % kTighten == kTighten - 1) s.tighten();
    dma_wait();
    __syncthreads();  // this chunk's operands are in LDS
    const long cu = (sq.slot + c) * p.HV + hv;
    const float inv[2] = {inverse_pow2(s.sc[0]), inverse_pow2(s.sc[1])};
    const float before = max_bits(s.bound[0], s.bound[1]);
    if constexpr (KIND == kSave)
      s.template store_tiles<DV>(p.sws + cu * (DV * DK), NW * grp + w, lane);
    // Y = K S^T and Q S^T
    f32x4 y[2][4], o[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int a = 0; a < 4; ++a) y[u][a] = o[u][a] = z;
    rows_times_state<DK, NP, OUT>(K, sQ, s, kb, y, o);
    // X = V - gamma Y, each row with a scale of its own
    uint4 xp[2][2][2];
    float ix[2];
    {
      f32x4 x[2][4];
      float m[2] = {0.f, 0.f};
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 g = gate(kGateY, a);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const f32x4 gi = g * inv[u];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[u][a][i] = fmaf(gi[i], y[u][a][i], v.get(4 * a + i, u));
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
    __syncthreads();  // all have read the queries, and the last chunk's keys
    if (c + 1 < nch) load_kq(c + 1);
    // e = T X, times T's scale: the gates undo it
    f32x4 e[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int a = 0; a < 4; ++a) e[u][a] = z;
    triangle(sT, xp, e, lane);
    uint4 ep[2][2][2], zp[2][2][2];
    if constexpr (OUT) {
      const float f = sG[kGateOne][kOneE];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        parts8<2>(e[u][0], e[u][1], f, ep[u][0]);
        parts8<2>(e[u][2], e[u][3], f, ep[u][1]);
      }
    }
    if constexpr (KIND == kSave) {
      const float f[2] = {sG[kGateOne][kOneIT] * ix[0], sG[kGateOne][kOneIT] * ix[1]};
      f32x4* const d =
          reinterpret_cast<f32x4*>(p.ews + cu * (DV * kC)) + 512 * (NW * grp + w) + 4 * lr + lq;
      float m = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const f32x4 x = f[u] * e[u][a];
          m = max4abs(m, x);
          d[128 * a + 64 * u] = x;
        }
      static_assert(kMaxE == kMaxS + 1, "");
      note_max<2>(p.gates + (cu * p.gate_rows + kRevOne) * kC + kMaxS, {before, m}, lane);
    }
    if constexpr (OUT) {
      // P e, and the outputs
      f32x4 q[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int a = 0; a < 4; ++a) q[u][a] = z;
      triangle(sP, ep, q, lane);
      const int m = min(kC, sq.len - c * kC);
      const unsigned os = unsigned(p.HV) * (DV * kIo);
      // a buffer that ends with the sequence's last token: stores past it are dropped
      const auto rs = rows_buffer(p.o, ((sq.t0 + long(c) * kC) * p.HV + hv) * (DV * kIo), DV * kIo,
                                  os, m);
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 go = gate(kGateO, a), gp = gate(kGateP, a);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          o[u][a] *= inv[u];
          q[u][a] *= ix[u];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          store_columns<NP>(rs, os, lq, row0 * kIo, 4 * a + i,
                            fmaf(go[i], o[0][a][i], gp[i] * q[0][a][i]),
                            fmaf(go[i], o[1][a][i], gp[i] * q[1][a][i]));
      }
    }
    // beta sigma e, in the place of e
    float g[2];
    {
      float m[2] = {0.f, 0.f};
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 gz = gate(kGateZ, a);
#pragma unroll
        for (int u = 0; u < 2; ++u) m[u] = max4abs(m[u], e[u][a] *= gz);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float f = ix[u] * sG[kGateOne][kOneK];
        g[u] = s.make_room(u, sG[kGateOne][kOneG], max_over_rows(m[u]) * f);
        parts8<2>(e[u][0], e[u][1], f * s.sc[u], zp[u][0]);
        parts8<2>(e[u][2], e[u][3], f * s.sc[u], zp[u][1]);
      }
    }
    __syncthreads();  // all have read T, P and the gates
    if (c + 1 < nch) {
      load_tp(c + 1);
      load_v(c + 1);
    }
    update_state<DK, NP>(s, g, K, zp, tb);
  }
  if (SEG && ident)
    store_matrix<DK>(s, reinterpret_cast<SegmentMatrix<DK>*>(p.sega) + su, NW * grp + w, lane);
  else if (SEG)
    s.store(p.segs + su * (DV * DK) + rows);
  else if (p.s_out && sg.j + 1 == sg.nseg)
    s.store(p.s_out + (long(sg.n) * p.HV + hv) * (DV * DK) + rows);
}

// The true states after the segments of one (sequence, value head, 16 state rows): S_0 as
// it is, then S_j = S_{j-1} A_j + B_j, in B_j's place.  Wave w holds the columns 32 w ..
// 32 w + 31 as two accumulator tiles of S^T; as two fp16 parts under a scale per row they are
// exchanged through LDS (one barrier per segment), A_j's operands come straight from
// memory, requested ahead.  A head's workgroups are a multiple of 8 apart where the heads
// are, so that they share an L2.  Bound: latency of the chain over the segments (1.5 us each
// for 16 heads of 128, 2.6 for 8 of 256: A_j's operands, 64 and 256 KB per workgroup).  With A in
// fp32 rows, cut into bf16 parts by every workgroup, 2.6 and 5.5; through LDS tiles 3.2 and 2.7.
template <int DK, int DV>
__global__ __launch_bounds__(2 * DK) void delta_combine_kernel(DeltaParams p) {
  constexpr int NH = DK / 32;
  using A = SegmentMatrix<DK>;
  __shared__ uint4 xs[2][NH][2][64];
  __shared__ float xi[2][NH][16];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lq = lane >> 4;
  const int units = p.N * p.HV, rb = blockIdx.x / units, unit = blockIdx.x - rb * units;
  const int n = unit / p.HV, hv = unit - n * p.HV;
  const Seq sq = seq_of(p, n);
  const long slot0 = first_segment(p, sq, n);
  const int last = segments_of(p, sq) - 2;  // the last segment that leaves a state
  if (last < 1) return;
  const long at = long(16 * rb + lr) * DK + 32 * w + 4 * lq;
  auto state = [&](int j) { return p.segs + ((slot0 + j) * p.HV + hv) * (DV * DK) + at; };
  const f32x4 z = {0.f, 0.f, 0.f, 0.f};
  f32x4 st[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) st[t] = *reinterpret_cast<const f32x4*>(state(0) + 16 * t);
  // segments ahead: two but for d_k = 256, whose eight waves' registers hold one
  constexpr int AHEAD = DK < 256 ? 2 : 1;
  u32x4 a[AHEAD][NH][2][2];
  f32x4 bn[AHEAD][2];
  float as[AHEAD][NH];
  auto load = [&](int j, int e, int h) __attribute__((always_inline)) {
    const A* const m =
        reinterpret_cast<const A*>(p.sega) + (slot0 + min(j, last)) * p.HV + hv;
    as[e][h] = m->scale[h];
    const auto rs = buffer(m, sizeof(A));
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        a[e][h][t][i] = __builtin_amdgcn_raw_buffer_load_b128(
            rs, 16 * lane, unsigned(((2 * w + t) * NH + h) * 2 + i) * 1024, 0);
  };
  auto load_next = [&](int j, int e) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      bn[e][t] = *reinterpret_cast<const f32x4*>(state(min(j, last)) + 16 * t);
  };
  auto step = [&](int j, int e) __attribute__((always_inline)) {
    const int x = j & 1;
    {
      uint4 d[2];
      const float s = scale_for(max_over_rows(max4abs(max4abs(0.f, st[0]), st[1])));
      parts8<2>(st[0], st[1], s, d);
      xs[x][w][0][lane] = d[0];
      xs[x][w][1][lane] = d[1];
      if (lq == 0) xi[x][w][lr] = inverse_pow2(s);
    }
    lds_barrier();
    f32x4 y[2] = {bn[e][0], bn[e][1]};
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const uint4 d[2] = {xs[x][h][0][lane], xs[x][h][1][lane]};
      const float inv = xi[x][h][lr] * inverse_pow2(as[e][h]);
      f32x4 acc[2] = {z, z};
      for_products<2, 2>([&](int i, int q) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
          acc[t] = mfma_f16(__builtin_bit_cast(uint4, a[e][h][t][i]), d[q], acc[t]);
      });
      load(j + AHEAD, e, h);  // (into the registers just read)
#pragma unroll
      for (int t = 0; t < 2; ++t) y[t] += inv * acc[t];
    }
    load_next(j + AHEAD, e);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      st[t] = y[t];
      *reinterpret_cast<f32x4*>(state(j) + 16 * t) = y[t];
    }
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
#pragma unroll
    for (int h = 0; h < NH; ++h) load(1 + i, i, h);
    load_next(1 + i, i);
  }
  for (int j = 1; j <= last; j += AHEAD) {
    step(j, 0);
    if constexpr (AHEAD == 2) {
      if (j + 1 > last) break;
      step(j + 1, 1);
    }
  }
}

template <int DK, int DV, int NP>
hipError_t run(const DeltaParams& p, bool save, hipStream_t st) {
  constexpr int NW = kChainWaves<DV>, GB = DV / (32 * NW), GA = DK / (32 * NW);
  const unsigned units = unsigned(p.seg_slots) * unsigned(p.HV);
  if (p.sega) {
    delta_forward_kernel<DK, DV, NP, kSegment><<<units * (GB + GA), 64 * NW, 0, st>>>(p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    delta_combine_kernel<DK, DV>
        <<<unsigned(p.N) * unsigned(p.HV) * (DV / 16), 2 * DK, 0, st>>>(p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (save)
    delta_forward_kernel<DK, DV, NP, kSave><<<units * GB, 64 * NW, 0, st>>>(p);
  else
    delta_forward_kernel<DK, DV, NP, kOutputs><<<units * GB, 64 * NW, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_forward(const DeltaShape& s, const DeltaParams& p, bool save,
                                hipStream_t st) {
#define ONELA_DELTA_SCAN(DK, DV, NP) \
  if (s.dk == DK && s.dv == DV && s.bf16 == (NP == 1)) return run<DK, DV, NP>(p, save, st);
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

hipError_t launch_delta_combine(const DeltaShape& s, const DeltaParams& p, hipStream_t st) {
  const unsigned wgs = unsigned(p.N) * unsigned(p.HV) * unsigned(s.dv / 16);
#define ONELA_DELTA_COMBINE(DK, DV)                         \
  if (s.dk == DK && s.dv == DV) {                           \
    delta_combine_kernel<DK, DV><<<wgs, 2 * DK, 0, st>>>(p); \
    return hipGetLastError();                               \
  }
  ONELA_DELTA_COMBINE(32, 32)
  ONELA_DELTA_COMBINE(64, 64)
  ONELA_DELTA_COMBINE(128, 128)
  ONELA_DELTA_COMBINE(128, 256)
  ONELA_DELTA_COMBINE(128, 512)
  ONELA_DELTA_COMBINE(256, 256)
  ONELA_DELTA_COMBINE(256, 512)
#undef ONELA_DELTA_COMBINE
  return hipErrorInvalidValue;
}

}  // namespace onela
