// The gated delta rule token by token on a pool of states (Eq. 1 of Sec. 2.2): per
// token S <- alpha S, e = v - S k, S <- S + beta e k^T, o = scale S q, with the
// state's rows in registers over the tokens of a call and written back in place.
//
// Both products of a token share one pass over the state: with the old, decayed
// state, S k and S q are formed together and o = scale (S q + beta e (k . q)).
// Everything is fp32; bf16 tensors are exact in it.
//
// A workgroup is one wave with NPASS times 512 / DK state rows, DK / 8 lanes to a row with 8
// columns each; rows are independent, so the state is split over as many workgroups as
// there are row blocks.  Bound: HBM, each state is read and written once: 256 states of 32
// heads of 128 x 128 210 us, 5.1 TB/s, as a large copy.  One state of 16 heads: latency, 4.0 us.
#include "delta_params.h"
#include "device_common.h"
#include "internal.h"

namespace onela {
namespace {

template <bool BF16>
__device__ inline void store1(void* base, long i, float x) {
  if constexpr (BF16)
    static_cast<uint16_t*>(base)[i] = uint16_t(pack_bf16x2(x, x));
  else
    static_cast<float*>(base)[i] = x;
}

// NPASS passes of 64 / (DK / 8) rows per wave.
template <int DK, bool BF16, int NPASS>
__global__ __launch_bounds__(64) void delta_step_kernel(DeltaParams p) {
  constexpr int LPR = DK / 8, RPW = 64 / LPR;  // lanes to a row, rows to a pass
  const int lane = threadIdx.x, sub = lane % LPR, rr = lane / LPR;
  const int blocks = p.DV / (RPW * NPASS);
  const int blk = blockIdx.x % blocks, unit = blockIdx.x / blocks;
  const int n = unit / p.HV, hv = unit - n * p.HV, hk = hv / (p.HV / p.HK);
  long t0, t1;
  if (p.offsets) {
    t0 = min(max(long(p.offsets[n]), 0l), p.total);
    t1 = min(max(long(p.offsets[n + 1]), t0), p.total);
  } else {
    t0 = long(n) * p.L;
    t1 = t0 + p.L;
  }
  if (t0 == t1) return;
  const int slot = p.slot ? p.slot[n] : n;
  const int row0 = blk * RPW * NPASS + rr;
  if (slot < 0 || slot >= p.num_slots) {  // no state: the sequence's outputs are zeros
    for (long t = t0; t < t1; ++t)
      if (sub == 0)
#pragma unroll
        for (int i = 0; i < NPASS; ++i)
          store1<BF16>(p.o, (t * p.HV + hv) * p.DV + row0 + i * RPW, 0.f);
    return;
  }
  float* const sp = p.pool + ((long(slot) * p.HV + hv) * p.DV + row0) * DK + 8 * sub;
  f32x4 st[NPASS][2];
#pragma unroll
  for (int i = 0; i < NPASS; ++i) {
    st[i][0] = *reinterpret_cast<const f32x4*>(sp + i * RPW * DK);
    st[i][1] = *reinterpret_cast<const f32x4*>(sp + i * RPW * DK + 4);
  }
  for (long t = t0; t < t1; ++t) {
    float q[8], k[8], v[NPASS];
    load8<BF16>(p.k, t * p.ks + hk * DK + 8 * sub, k);
    load8<BF16>(p.q, t * p.qs + hk * DK + 8 * sub, q);
#pragma unroll
    for (int i = 0; i < NPASS; ++i) v[i] = load1<BF16>(p.v, t * p.vs + hv * p.DV + row0 + i * RPW);
    const float be = p.beta[t * p.HV + hv];
    const float al = expf(p.la[t * p.HV + hv]);
    float kq = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) kq = fmaf(k[j], q[j], kq);
    kq = group_sum<LPR>(kq);
#pragma unroll
    for (int i = 0; i < NPASS; ++i) {
      float sk = 0.f, sq = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float& s = reinterpret_cast<float*>(&st[i][j >> 2])[j & 3];
        s *= al;
        sk = fmaf(s, k[j], sk);
        sq = fmaf(s, q[j], sq);
      }
      sk = group_sum<LPR>(sk);
      sq = group_sum<LPR>(sq);
      const float d = be * (v[i] - sk);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float& s = reinterpret_cast<float*>(&st[i][j >> 2])[j & 3];
        s = fmaf(d, k[j], s);
      }
      if (sub == 0)
        store1<BF16>(p.o, (t * p.HV + hv) * p.DV + row0 + i * RPW, p.scale * fmaf(d, kq, sq));
    }
  }
#pragma unroll
  for (int i = 0; i < NPASS; ++i) {
    *reinterpret_cast<f32x4*>(sp + i * RPW * DK) = st[i][0];
    *reinterpret_cast<f32x4*>(sp + i * RPW * DK + 4) = st[i][1];
  }
}

template <int DK, bool BF16>
hipError_t run(const DeltaShape& s, const DeltaParams& p, hipStream_t st) {
  constexpr int RPW = 64 / (DK / 8), NPASS = 4;
  const unsigned blocks = unsigned(s.N) * unsigned(s.HV) * unsigned(s.dv / (RPW * NPASS));
  delta_step_kernel<DK, BF16, NPASS><<<blocks, 64, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_step(const DeltaShape& s, const DeltaParams& p, hipStream_t st) {
  if (s.dk == 32) {  // 16 rows to a pass
    constexpr int RPW = 16;
    const unsigned blocks = unsigned(s.N) * unsigned(s.HV) * unsigned(s.dv / RPW);
    if (s.bf16)
      delta_step_kernel<32, true, 1><<<blocks, 64, 0, st>>>(p);
    else
      delta_step_kernel<32, false, 1><<<blocks, 64, 0, st>>>(p);
    return hipGetLastError();
  }
  if (s.dk == 64) return s.bf16 ? run<64, true>(s, p, st) : run<64, false>(s, p, st);
  if (s.dk == 128) return s.bf16 ? run<128, true>(s, p, st) : run<128, false>(s, p, st);
  if (s.dk == 256 && s.bf16) return run<256, true>(s, p, st);
  return hipErrorInvalidValue;
}

}  // namespace onela
