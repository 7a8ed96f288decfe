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
// Launches.  Forward: delta_prep_kernel (T, P, decays; one workgroup per chunk and value
// head), delta_forward_kernel (the chain over the chunks with the outputs; few heads: in
// segments, with delta_combine_kernel between).  Backward: the same two for the states
// (nothing is kept from the forward call), delta_reverse_kernel (the chain in reverse),
// delta_grad_kernel (one workgroup per chunk and query/key head).
//
// Precision.  States, e, T, decays and sums are fp32.  Every product runs on
// v_mfma_f32_16x16x32_f16 with its fp32 operands as the sum of two fp16 parts under a
// power-of-two scale (22 bits of the largest element that shares the scale, products of two low
// parts left out; delta_tiles.h) and bf16 tensors as one part, in which they are exact
// (NP = 1); fp32 tensors are two parts too (NP = 2).  What shares a scale: in the chains a row of
// a state, or a chunk's tokens in one channel of X, e, dO and dV, so that every value channel is
// right to some 3e-7 of its own largest value (1e-5 beside 1 too; 32768 tokens without decay
// too); keys and queries of a chunk and head (fp32 ones: 2^-27 of their largest element), T, and
// in the gradients a chunk's S, dS, e, dV and dO of a head (2^-38 of each one's largest).  With
// three bf16 parts, which are exact,
// the same chain took 1.4 times as long (16 x 1000 tokens x 32 heads of 128) for an error of
// 1e-7 in place of 1.5e-7 of the state's norm.  Decays are exp2 of differences of
// in-chunk sums of log2(alpha) in 64 bits (a float pair where they are stored), so that a
// vanishing decay does not blur the ones after it; log_alpha below -1e5, -inf among it,
// is an exact 0.
//
// Tokens past a sequence's end read as k = v = q = 0, beta = 0, alpha = 1: they
// leave the state as it is and give zeros.
#include <type_traits>

#include "delta_params.h"
#include "internal.h"

namespace onela {

hipError_t launch_delta_rule(const DeltaShape& s, DeltaParams p, bool backward, void* workspace,
                             hipStream_t st) {
  const size_t cus = size_t(s.slots) * s.HV;
  const size_t image = size_t(s.slots) * s.HK * (s.bf16 ? 1 : 2) * delta_image_bytes(s.dk);
  char* at = static_cast<char*>(workspace);
  auto take = [&](auto*& to, size_t bytes) {
    to = reinterpret_cast<std::remove_reference_t<decltype(to)>>(at);
    at += bytes;
  };
  take(p.kimg, image);
  take(p.qimg, image);
  take(p.tp, cus * kDeltaFragBytes);
  p.gate_rows = kDeltaGates * (backward ? 2 : 1);
  take(p.gates, cus * p.gate_rows * kDeltaChunk * 4);
  const DeltaSegments sg = delta_segments(s, p.offsets != nullptr);
  p.cps = sg.cps;
  p.nseg_l = sg.nseg_l;
  p.seg_slots = sg.slots;
  if (sg.many) {
    take(p.segs, size_t(sg.slots) * s.HV * s.dv * s.dk * 4);
    take(p.sega, size_t(sg.slots) * s.HV * delta_matrix_bytes(s.dk));
  }
  if (!backward) {
    take(p.pf, cus * kDeltaFragBytes);
  } else {
    take(p.tr, cus * kDeltaFragBytes);
    take(p.pr, cus * kDeltaFragBytes);
    take(p.sws, cus * s.dv * s.dk * 4);
    take(p.ews, cus * s.dv * kDeltaChunk * 4);
    take(p.dsws, cus * s.dv * s.dk * 4);
    take(p.hws, cus * s.dv * kDeltaChunk * 4);
  }
  hipError_t e = launch_delta_prep(s, p, backward, st);
  if (e == hipSuccess) e = launch_delta_forward(s, p, backward, st);
  if (!backward || e != hipSuccess) return e;
  e = launch_delta_reverse(s, p, st);
  return e == hipSuccess ? launch_delta_grad(s, p, st) : e;
}

}  // namespace onela
