// Host-side check of the choice that a step with shared prefixes is planned by, built by
// tests/test_shared_choice_cpu.py with optimisation: what it costs, and where it shares. Prints "ok" and returns 0.
#include <algorithm>
#include <chrono>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "plan.h"

using namespace ppas;

namespace {

int g_failures = 0;

struct Step {
  std::vector<ppas_seq> seqs;
  std::vector<ppas_prefix> prefixes;
  int32_t rows = 0;
  void add(int32_t n, int32_t cached) {
    seqs.push_back(ppas_seq{rows, n, cached});
    rows += n;
  }
};

Plan plan_of(const Step& s, bool share, int hkv = 2) {
  ppas_shape sh{8 * hkv, hkv, 128, 16, 1 << 20, 0.1f};
  Plan plan;
  make_plan(sh, s.seqs.data(), int32_t(s.seqs.size()), 256, PlanOpts{}, plan, s.prefixes.data(),
            share ? int32_t(s.prefixes.size()) : 0);
  return plan;
}

double microseconds(const Step& s, bool share) {
  double best = 1e30;
  for (int k = 0; k < 5; ++k) {
    const auto t = std::chrono::steady_clock::now();
    const Plan plan = plan_of(s, share);
    best = std::min(best, std::chrono::duration<double, std::micro>(std::chrono::steady_clock::now() - t).count());
    if (plan.items.empty()) ++g_failures;
  }
  return best;
}

// Many short chunks, each with a length of its own: the choice takes no more than a few times
// the plan apart, which walks the same requests (one lot per request: 17 to 50 times).
void check_time(int requests, int rows) {
  Step s;
  uint32_t z = 1;
  for (int i = 0; i < requests; ++i) {
    z = z * 1664525u + 1013904223u;
    s.add(rows, 8192 + int32_t((z >> 8) % 4000));
  }
  s.prefixes = {ppas_prefix{0, requests, 8192}};
  const double apart = microseconds(s, false), shared = microseconds(s, true);
  if (shared > 12 * apart + 200) {
    std::fprintf(stderr, "%d requests of %d rows: %.0f us, apart %.0f\n", requests, rows, shared, apart);
    ++g_failures;
  }
}

Step group(int requests, int rows, int prefix, int own) {
  Step s;
  for (int i = 0; i < requests; ++i) s.add(rows, prefix + own * (i % 3));
  s.prefixes = {ppas_prefix{0, requests, prefix}};
  return s;
}

bool same_plan(const Step& s) {
  const Plan a = plan_of(s, false), b = plan_of(s, true);
  return a.items.size() == b.items.size() && a.part_slots == b.part_slots && a.combine.size() == b.combine.size() &&
         a.tile_pos == b.tile_pos && b.rows.empty();
}

void check_shares(int requests, int rows, int prefix, bool want) {
  for (int own : {0, 50}) {
    if (same_plan(group(requests, rows, prefix, own)) != want) continue;
    std::fprintf(stderr, "%d requests of %d rows behind %d: %s\n", requests, rows, prefix, want ? "apart" : "shared");
    ++g_failures;
  }
}

}  // namespace

int main() {
  // whole tiles of rows share their keys already: together they are as many tiles
  for (int requests : {2, 4, 8, 16, 64, 128})
    for (int rows : {16, 32, 48, 64})
      for (int prefix : {512, 1024, 2048, 4096, 8192}) check_shares(requests, rows, prefix, false);
  // a few tiles saved, and the partials of every row for it
  check_shares(128, 17, 512, false);
  check_shares(128, 33, 512, false);
  check_shares(128, 17, 1024, false);
  check_shares(64, 33, 1024, false);
  // many saved
  check_shares(64, 1, 8192, true);
  check_shares(256, 1, 24576, true);
  check_shares(64, 2, 8192, true);
  check_shares(128, 8, 8192, true);
  check_shares(64, 33, 16384, true);
  check_time(256, 2);
  check_time(1024, 2);
  check_time(2048, 33);
  check_time(2048, 17);
  if (g_failures) return 1;
  std::printf("ok\n");
  return 0;
}
