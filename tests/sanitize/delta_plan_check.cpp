// Host-only exercise of the delta rule's and the norm's configuration, workspace and segment
// plans (host_plan.cpp), built with the address and undefined-behaviour sanitizers by
// tests/test_delta_sanitizers.py.  Exits non-zero on a violated expectation; the
// sanitizers abort on their own.
#include <climits>
#include <cmath>
#include <cstdio>
#include <limits>
#include <random>

#include "../../paper_2609_12399_amd/csrc/host_plan.h"

using namespace onela;

static int failures = 0;
#define EXPECT(c)                                                          \
  do {                                                                     \
    if (!(c)) {                                                            \
      std::fprintf(stderr, "%s:%d: expectation failed: %s\n", __FILE__,   \
                   __LINE__, #c);                                          \
      ++failures;                                                          \
    }                                                                      \
  } while (0)

// The segments of a shape: every chunk is in one, and they fit the workspace's share.
static void check_segments(const DeltaShape& s, bool ragged) {
  for (int cus : {0, 1, 104, 256, 304}) {
    DeltaShape d = s;
    d.cus = cus;
    const DeltaSegments g = delta_segments(d, ragged);
    if (!g.many) {
      EXPECT(g.cps == 1 << 30 && g.nseg_l == 1 && g.slots == d.N);
      continue;
    }
    EXPECT(cus > 0 && g.cps >= 2 && g.nseg_l >= 2);
    if (!ragged) {
      const long nch = delta_chunks(d.L);
      EXPECT(long(g.cps) * g.nseg_l >= nch && long(g.cps) * (g.nseg_l - 1) < nch);
      EXPECT(g.slots == long(d.N) * g.nseg_l);
    } else {
      // a sequence of n chunks has ceil(n / cps) segments, all together at most this many
      EXPECT(g.slots >= d.slots / g.cps + d.N);
    }
    const size_t state = size_t(d.HV) * d.dk * d.dv * 4;
    const size_t matrix = size_t(d.HV) * delta_matrix_bytes(d.dk);
    DeltaShape none = d;  // what the workspace holds without segments
    EXPECT(delta_workspace_bytes(none, false) >= size_t(g.slots) * (state + matrix));
  }
}

static void shapes() {
  const int64_t limits[] = {INT64_MIN, -1, 0, 1, 63, 64, 65, 1000, 4096, INT32_MAX,
                            int64_t(INT32_MAX) + 1, INT64_MAX};
  const int heads[][2] = {{16, 16}, {16, 32}, {2, 3}, {0, 4}, {4, 0}, {-1, 4}, {1, INT_MAX}};
  const int dims[][2] = {{32, 32}, {64, 64}, {128, 128}, {128, 512}, {256, 256}, {256, 512},
                         {100, 100}, {0, 0}, {-128, 128}, {INT_MAX, INT_MAX}};
  const int64_t strides[] = {0, 128, 4096, 4100, INT32_MAX, INT64_MAX, -8};
  int ok = 0;
  for (int N : {INT_MIN, 0, 1, 7, 1000, INT_MAX})
    for (auto& h : heads)
      for (auto& d : dims)
        for (int64_t total : limits)
          for (int io = -1; io < 3; ++io)
            for (int64_t st : strides)
              for (bool ragged : {false, true}) {
                onela_delta_config_t c{};
                c.num_seqs = N;
                c.num_qk_heads = h[0];
                c.num_v_heads = h[1];
                c.d_k = d[0];
                c.d_v = d[1];
                c.io_dtype = io;
                c.total_tokens = total;
                c.q_stride = c.v_stride = st;
                c.scale = 1.f;
                DeltaShape s{};
                const onela_status_t rc = delta_shape_of(&c, ragged, &s);
                EXPECT(rc == ONELA_OK || rc == ONELA_EINVAL);
                if (rc != ONELA_OK) continue;
                ++ok;
                EXPECT(s.N >= 1 && s.HV % s.HK == 0 && s.total >= 0);
                EXPECT(s.qs >= long(s.HK) * s.dk && s.vs >= long(s.HV) * s.dv);
                EXPECT(s.slots >= s.total / kDeltaChunk);
                EXPECT(ragged || long(s.L) * s.N == s.total);
                const size_t f = delta_workspace_bytes(s, false), b = delta_workspace_bytes(s, true);
                EXPECT(f % 256 == 0 && b % 256 == 0 && b >= f);
                check_segments(s, ragged);
              }
  EXPECT(ok > 100);
  EXPECT(delta_shape_of(nullptr, true, nullptr) == ONELA_EINVAL);
}

static void random_shapes() {
  std::mt19937 rng(5);
  auto pick = [&](int lo, int hi) { return int(lo + rng() % unsigned(hi - lo + 1)); };
  const int dims[][2] = {{32, 32}, {64, 64}, {128, 128}, {128, 256}, {256, 256}};
  for (int i = 0; i < 20000; ++i) {
    const auto& d = dims[rng() % 5];
    onela_delta_config_t c{};
    c.num_seqs = pick(1, 64);
    c.num_qk_heads = pick(1, 16);
    c.num_v_heads = c.num_qk_heads * pick(1, 4);
    c.d_k = d[0];
    c.d_v = d[1];
    c.io_dtype = d[0] <= 128 && d[1] <= 128 ? pick(0, 1) : ONELA_BF16;
    const bool ragged = rng() & 1;
    c.total_tokens = ragged ? pick(0, 70000) : int64_t(c.num_seqs) * pick(0, 9000);
    DeltaShape s{};
    EXPECT(delta_shape_of(&c, ragged, &s) == ONELA_OK);
    check_segments(s, ragged);
  }
}

static void norms() {
  const int64_t tokens[] = {INT64_MIN, -1, 0, 1, 8191, INT32_MAX, INT64_MAX};
  const float eps[] = {0.f, 1e-6f, -1.f, std::numeric_limits<float>::quiet_NaN(),
                       std::numeric_limits<float>::infinity()};
  int ok = 0;
  for (int64_t t : tokens)
    for (int hq : {INT_MIN, 0, 1, 16, INT_MAX})
      for (int hk : {INT_MIN, 0, 2, INT_MAX})
        for (int D : {INT_MIN, 0, 8, 96, 512, 520, INT_MAX})
          for (int rot : {INT_MIN, 0, 16, 96, INT_MAX})
            for (int64_t st : {int64_t(0), int64_t(1536), INT64_MIN, INT64_MAX})
              for (float e : eps) {
                onela_norm_config_t c{};
                c.num_tokens = t;
                c.num_q_heads = hq;
                c.num_k_heads = hk;
                c.head_dim = D;
                c.rotary_dim = rot;
                c.table_rows = rot > 0 ? 64 : 0;
                c.io_dtype = ONELA_BF16;
                c.norm = ONELA_NORM_RMS;
                c.rotation = ONELA_ROTATE_HALVES;
                c.q_stride = c.k_stride = st;
                c.eps = e;
                const onela_status_t rc = check_norm(&c);
                EXPECT(rc == ONELA_OK || rc == ONELA_EINVAL);
                const size_t n = norm_workspace_bytes(&c);
                if (rc == ONELA_OK) {
                  ++ok;
                  EXPECT(n >= size_t(D) * 8);
                }
              }
  EXPECT(ok > 20);
  EXPECT(check_norm(nullptr) == ONELA_EINVAL);
}

int main() {
  shapes();
  random_shapes();
  norms();
  if (failures) {
    std::fprintf(stderr, "%d expectation(s) failed\n", failures);
    return 1;
  }
  std::printf("delta plan checks: ok\n");
  return 0;
}
