// Host-only exercise of the plans of the short convolution, the norms around a block and the log
// probabilities (host_plan.cpp), built with the address and undefined-behaviour sanitizers by
// tests/test_model_sanitizers.py.  Exits non-zero on a violated expectation; the sanitizers
// abort on their own.
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

// Every token and channel belongs to one run, the grid fits, and the workspace holds a row
// of sums for every workgroup over the tokens.
static void conv(const onela_conv_config_t& c) {
  for (bool ragged : {false, true}) {
    if (check_conv(&c, ragged) != ONELA_OK) continue;
    for (bool backward : {false, true}) {
      const ConvPlan a = conv_plan(&c, backward);
      EXPECT(a.lanes_log2 >= 0 && a.lanes_log2 <= 6 && a.run >= 1 && a.blocks_c >= 1);
      EXPECT((long(a.blocks_c) << a.lanes_log2) * 8 >= c.channels);
      const double covered = double(a.blocks_t) * a.run * (kConvThreads >> a.lanes_log2);
      EXPECT(covered >= double(c.total_tokens));
      const double states = (double(c.num_seqs) * (c.channels / kConvLane) + kConvThreads) / kConvThreads;
      EXPECT((double(a.blocks_t) * a.blocks_c + states) * kConvThreads < kGridThreads);
      if (backward)
        EXPECT(conv_workspace_bytes(&c) >=
               size_t(a.blocks_t) * size_t(c.taps + 1) * size_t(c.channels) * 4);
    }
  }
}

static void norm(const onela_block_norm_config_t& c) {
  if (check_block_norm(&c) != ONELA_OK) return;
  EXPECT(block_norm_workspace_bytes(&c) == size_t(3) * kBlockNormBlocks * size_t(c.width) * 4);
}

// The parts cover the vocabulary, none is empty, and the workspace holds them.
static void logprob(const onela_logprob_config_t& c) {
  if (check_logprob(&c) != ONELA_OK) return;
  const LogprobPlan a = logprob_plan(&c);
  EXPECT(a.threads >= kMaxTop && a.parts >= 1 && a.parts <= kLogprobParts && a.columns >= 1);
  EXPECT(double(a.parts) * a.columns >= c.vocab && double(a.parts - 1) * a.columns < c.vocab);
  EXPECT(double(c.num_rows) * a.parts * a.threads < kGridThreads);
  const size_t n = logprob_workspace_bytes(&c);
  EXPECT(n >= 256 && n % 256 == 0);
  if (a.parts > 1)
    EXPECT(n >= size_t(c.num_rows) * a.parts * (4 + 2 * size_t(c.num_top)) * 4);
}

int main() {
  std::mt19937_64 rng(7);
  const int64_t wide[] = {INT64_MIN, -1, 0, 1, 7, 8, 63, 64, 65, 1000, 4096, 100000, 1 << 24,
                          INT32_MAX, int64_t(INT32_MAX) + 1, int64_t(1) << 40, INT64_MAX};
  const int32_t some[] = {INT32_MIN, -1, 0, 1, 2, 3, 4, 5, 8, 40, 64, 65, 257, 2048, 6144, 16384,
                          16392, 50001, 131072, 1 << 20, (1 << 28) - 1, 1 << 28, INT32_MAX - 7,
                          INT32_MAX};
  auto w = [&] { return wide[rng() % (sizeof(wide) / sizeof(*wide))]; };
  auto s = [&] {
    const int32_t v = some[rng() % (sizeof(some) / sizeof(*some))];
    return rng() % 2 ? v : int32_t(rng() % 70000);
  };
  const float f[] = {0.f, 1.f, 0.5f, -1.f, 1e30f, INFINITY, NAN};
  for (int i = 0; i < 400000; ++i) {
    const int32_t io = int32_t(rng() % 8) ? int32_t(rng() % 2) : s();
    conv({rng() % 2 ? int32_t(1 + rng() % 9) : s(), rng() % 2 ? int32_t(8 * (1 + rng() % 1024)) : s(),
          int32_t(rng() % 6), io, int32_t(rng() % 4) - 1, rng() % 2 ? int64_t(rng() % 100000) : w(),
          rng() % 2 ? 0 : w()});
    norm({w(), s(), rng() % 2 ? int32_t(8 * (1 + rng() % 2100)) : s(), io, int32_t(rng() % 3),
          int32_t(rng() % 3), int32_t(rng() % 3), int32_t(rng() % 5) - 1, rng() % 2 ? 0 : w(),
          rng() % 2 ? 0 : w(), f[rng() % 7], f[rng() % 7]});
    logprob({rng() % 2 ? int64_t(rng() % 2000) : w(), s(), int32_t(rng() % 300) - 9,
             int32_t(rng() % 80) - 9, io, rng() % 2 ? 0 : w(), f[rng() % 7]});
  }
  EXPECT(check_conv(nullptr, true) == ONELA_EINVAL);
  EXPECT(check_block_norm(nullptr) == ONELA_EINVAL);
  EXPECT(check_logprob(nullptr) == ONELA_EINVAL);
  char block[64];
  EXPECT(overlap(block, 32, block + 31, 1) && !overlap(block, 32, block + 32, 32));
  EXPECT(overlap(block + 31, 8, block, 32) && !overlap(block + 32, 8, block, 32));
  EXPECT(!overlap(nullptr, 32, block, 32) && !overlap(block, 0, block, 32));
  if (failures) return 1;
  std::printf("model plan checks: ok\n");
  return 0;
}
