// Arguments of the delta-rule kernels (kernels_delta.hip, kernel_delta_step.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "host_plan.h"

namespace onela {

// Rows of a chunk's gates in the workspace, 64 values each (operands' scales undone in
// each).  Forward: factors of K S^T in X (-gamma), of T X in the state's update (beta sigma), of
// Q S^T and of P e in the outputs; single values.  Backward: factors of K dS^T (beta sigma)
// and of P^T dO in X; -gamma; beta sigma; beta; sums of log2(alpha) as float pairs; single values.
enum {
  kGateY, kGateZ, kGateO, kGateP, kGateOne, kGateStage = 8,
  kRevY = 8, kRevP, kRevZ, kRevBS, kRevBeta, kRevHi, kRevLo, kRevOne
};
// Single values.  Forward: gamma_{C-1}; the keys' inverse scale; the scale of T X; T's inverse scale.
enum { kOneG, kOneK, kOneE, kOneIT };
// Backward: gamma_{C-1}; the keys' and queries' inverse scales; T's inverse scale; then, as they
// come, the largest magnitudes of the state, e, the adjoint, dV and dO.
enum { kRevG, kRevK, kRevQ, kRevIT, kMaxS = 8, kMaxE, kMaxD, kMaxV, kMaxO };

struct DeltaParams {
  const void *q, *k, *v;    // [total][heads][d], token strides qs, ks, vs
  const void* d_o;          // [total][HV][DV] io dtype (backward)
  const float *la, *beta;   // [total][HV]
  const float *s_in;        // [N][HV][DV][DK] or null
  const float *ds_in;       // gradient of the final state, or null (backward)
  float *s_out, *ds_out;    // final state / gradient of the initial state, or null
  void *o;                  // [total][HV][DV] io dtype
  void *dq, *dk, *dv;       // dense, io dtype
  float *dla, *db;          // [total][HV]
  const int* offsets;       // [N + 1] or null: N sequences of L tokens
  long total, qs, ks, vs;
  float scale;
  int N, HK, HV, DV, L, nch_l;  // nch_l: chunks of a sequence of L tokens (no offsets)
  long slots;               // chunk slots
  // workspace, per (chunk slot, value head)
  float* gates;  // [gate_rows][64]
  int gate_rows; // kDeltaGates, backward twice that
  uint4* tr;     // as tp and pf, of T and P transposed with their tokens in reverse order
  uint4* pr;     // (backward)
  // Backward: what the chains leave, place 32 g + 16 u + m of the values' columns being column
  // 32 g + 2 m + u (a wave's store then covers whole lines)
  float* sws;    // [DK/16][DV places][16]  state before the chunk
  float* ews;    // [DV/32][4][32 places][16 tokens]  e
  float* dsws;   // as sws: adjoint of the state after the chunk
  float* hws;    // as ews: dV
  uint4 *kimg, *qimg;  // per (slot, query/key head): the LDS image Swz<DK>[NP] of the fp16
                       // parts of keys and queries
  uint4* tp;     // T fragments, two fp16 parts [6][2][64]
  uint4* pf;     // P fragments, two fp16 parts [6][2][64]
  // segments of the chain
  int cps, nseg_l;     // chunks per segment; segments of a sequence of L tokens
  long seg_slots;
  float* segs;         // [slot][HV][DV][DK]  the state after each segment but a sequence's last; in
                       // the last one's place the state that the sequence starts from
  char* sega;          // [slot][HV]  transition matrices of the segments between (SegmentMatrix)
  // recurrent step
  float* pool;       // [num_slots][HV][DV][DK]
  const int* slot;   // [N] or null
  int num_slots;
};

}  // namespace onela
