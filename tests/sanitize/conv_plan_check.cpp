// Host-only check that the plans of the short convolution (host_plan.cpp) give every token and
// channel to exactly one thread's run, built with the address and undefined-behaviour sanitizers
// by tests/test_conv_plan.py.  Exits non-zero on a violated expectation.
#include <cstdio>
#include <random>
#include <vector>

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

static onela_conv_config_t config(int channels, int taps, long tokens, int io) {
  onela_conv_config_t c{};
  c.num_seqs = 1;
  c.channels = channels;
  c.taps = taps;
  c.io_dtype = io;
  c.total_tokens = tokens;
  return c;
}

// Thread by thread, as the kernels place them.
static void count(const onela_conv_config_t& c, bool backward) {
  const ConvPlan a = conv_plan(&c, backward);
  const int lanes = 1 << a.lanes_log2, runs = kConvThreads / lanes;
  std::vector<int> seen(size_t(c.total_tokens) * (c.channels / kConvLane));
  for (long bt = 0; bt < a.blocks_t; ++bt)
    for (int bc = 0; bc < a.blocks_c; ++bc)
      for (int t = 0; t < kConvThreads; ++t) {
        const long group = long(bc) * lanes + t % lanes, t0 = (bt * runs + t / lanes) * a.run;
        if (group >= c.channels / kConvLane) continue;
        for (long i = t0; i < t0 + a.run && i < c.total_tokens; ++i)
          ++seen[size_t(i) * (c.channels / kConvLane) + size_t(group)];
      }
  for (int n : seen) EXPECT(n == 1);
}

// The same by its products, for any sizes.
static void cover(const onela_conv_config_t& c, bool backward) {
  if (check_conv(&c, true) != ONELA_OK) return;
  const ConvPlan a = conv_plan(&c, backward);
  EXPECT(a.lanes_log2 >= 0 && a.lanes_log2 <= 6 && a.run >= 1);
  const long channels = (long(a.blocks_c) << a.lanes_log2) * kConvLane;
  EXPECT(channels >= c.channels);
  EXPECT(channels - c.channels < long(kConvLane) << a.lanes_log2);
  const long tokens = (kConvThreads >> a.lanes_log2) * long(a.run);
  EXPECT(a.blocks_t * tokens >= c.total_tokens);
  EXPECT((a.blocks_t - 1) * tokens < c.total_tokens || c.total_tokens == 0);
}

// The launch that adds up the weights' gradients is within a grid for every size that is taken.
static void weights(int channels, int taps) {
  const onela_conv_config_t c = config(channels, taps, 0, 0);
  EXPECT(check_conv(&c, true) == ONELA_OK);
  const unsigned n = conv_weight_blocks(taps, channels);
  EXPECT(n >= 1 && double(n) * 256 < kGridThreads);
  EXPECT(n == (1u << 20) || double(n) * 16 >= double(taps + 1) * channels);
}

int main() {
  std::mt19937 rng(11);
  for (int i = 0; i < 300; ++i) {
    const onela_conv_config_t c = config(8 * int(1 + rng() % 160), 2 + int(rng() % 3),
                                         long(rng() % 700), int(rng() % 2));
    EXPECT(check_conv(&c, true) == ONELA_OK);
    for (bool backward : {false, true}) count(c, backward);
  }
  for (int i = 0; i < 200000; ++i) {
    const int shift = int(rng() % 24);
    const onela_conv_config_t c = config(8 * int(1 + (rng() % (1 << 23)) / (1u << shift)),
                                         2 + int(rng() % 3), long(rng() % (1u << (1 + rng() % 31))),
                                         int(rng() % 2));
    for (bool backward : {false, true}) cover(c, backward);
  }
  for (int taps = 2; taps <= 4; ++taps)
    for (int channels : {8, 64, 6144, 1 << 20, 1 << 25, (1 << 26) - 8, 1 << 26}) weights(channels, taps);
  if (failures) return 1;
  std::printf("convolution plan checks: ok\n");
  return 0;
}
