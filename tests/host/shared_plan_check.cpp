// Host-side check of plans with shared prefixes, built with g++ under
// AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_shared_plan_cpu.py.
// It fuzzes steps with groups and checks that every (row, KV head) sees each of its
// keys exactly once, that shared items take whole unmasked blocks, and that every
// partial is written once and merged for the right rows. Prints "ok" and returns 0.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <utility>
#include <vector>

#include "plan.h"

using namespace ppas;

namespace {

int g_failures = 0;
#define CHECK(cond)                                                              \
  do {                                                                           \
    if (!(cond)) {                                                               \
      std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
      if (++g_failures > 20) std::exit(1);                                       \
    }                                                                            \
  } while (0)

struct Rng {
  uint64_t s;
  uint64_t next() {
    uint64_t z = (s += 0x9E3779B97F4A7C15ull);
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
  }
  int uniform(int lo, int hi) { return lo + int(next() % uint64_t(hi - lo + 1)); }   // inclusive
};

struct Step {
  std::vector<ppas_seq> seqs;
  std::vector<ppas_prefix> prefixes;
  std::vector<int32_t> len;   // per request: its group's prefix
};

Step random_step(Rng& g) {
  Step st;
  int32_t row = 0;
  auto add = [&](int n, int cached, int len) {
    st.seqs.push_back(ppas_seq{row, n, cached});
    st.len.push_back(len);
    row += n;
  };
  auto rows = [&]() { return g.uniform(0, 2) ? 1 : g.uniform(0, 3) ? g.uniform(2, 70) : g.uniform(60, 400); };
  const int groups = g.uniform(0, 4);
  for (int k = 0; k <= groups; ++k) {
    for (int i = g.uniform(0, 2); i > 0; --i) add(rows(), g.uniform(0, 3000), 0);
    if (k == groups) break;
    const int n = g.uniform(0, 4) ? g.uniform(1, 12) : g.uniform(30, 150);
    const int len = 16 * (g.uniform(0, 3) ? g.uniform(0, 60) : g.uniform(0, 2000));
    st.prefixes.push_back(ppas_prefix{int32_t(st.seqs.size()), n, len});
    for (int i = 0; i < n; ++i) add(rows(), len + (g.uniform(0, 2) ? g.uniform(0, 2000) : 0), len);
  }
  return st;
}

void check(const Step& st, const Plan& plan, int hkv) {
  // by first slot of each item: which rows of the step its partials hold
  std::vector<int64_t> slot_row(size_t(plan.part_slots), -1);   // (row * hkv + head group) * 8 + head
  std::vector<std::pair<int32_t, int32_t>> slot_keys(size_t(plan.part_slots));
  std::vector<char> merged(size_t(plan.part_slots), 0);
  std::map<std::pair<int64_t, int>, std::vector<std::pair<int64_t, int64_t>>> seen;   // whole rows
  std::vector<int64_t> pos_of, seq_of;
  for (size_t s = 0; s < st.seqs.size(); ++s)
    for (int i = 0; i < st.seqs[s].n_query; ++i) {
      pos_of.push_back(int64_t(st.seqs[s].cached_len) + i);
      seq_of.push_back(int64_t(s));
    }
  std::vector<WorkItem> items = plan.items;
  items.insert(items.end(), plan.rows.begin(), plan.rows.end());
  for (const WorkItem& r : plan.rows)
    CHECK(r.npos_kind == (1 | kKindDecode << 16) && r.key_hi - r.key_lo <= kRowMaxKeys && r.key_hi == r.pos0 + 1);
  CHECK(plan.off_rows >= plan.items.size() * sizeof(WorkItem) && plan.off_rows % 256 == 0);
  CHECK(plan.off_combine >= plan.off_rows + plan.rows.size() * sizeof(WorkItem) && plan.off_combine % 256 == 0);
  CHECK(plan.list_bytes == plan.off_combine + plan.combine.size() * sizeof(CombineItem));
  for (const WorkItem& it : items) {
    const int npos = it.npos_kind & 0xffff, kind = it.npos_kind >> 16;
    CHECK(it.key_lo >= 0 && it.key_lo < it.key_hi && npos >= 1 && npos <= plan.tile_pos);
    CHECK(it.row0 >= 0 && size_t(it.row0 + npos) <= pos_of.size());
    if (kind == kKindDecode) CHECK(npos == 1 && it.key_hi - it.key_lo <= kDecodeMaxKeys && it.key_lo % kDecodeBlock == 0);
    else CHECK(it.key_lo % kPrefillBlock == 0);
    const bool shared = it.pos0 != pos_of[size_t(it.row0)] || it.pos0 + npos - 1 != pos_of[size_t(it.row0 + npos - 1)] ||
                        seq_of[size_t(it.row0)] != it.seq || seq_of[size_t(it.row0 + npos - 1)] != it.seq;
    for (int i = 0; i < npos; ++i) {
      const size_t r = size_t(it.row0 + i);
      const int64_t s = seq_of[r];
      if (shared) {
        // every key of the item is in the group's prefix, in whole blocks below the item's position
        CHECK(kind == kKindPrefill && it.part >= 0);
        CHECK(it.key_hi <= st.len[size_t(s)] && it.key_hi % kPrefillBlock == 0 && it.key_hi <= it.pos0);
        const bool member = [&] {
          for (const auto& p : st.prefixes)
            if (p.first_seq == it.seq) return s >= p.first_seq && s < p.first_seq + p.n_seqs;
          return false;
        }();
        CHECK(member);
      } else {
        CHECK(s == it.seq && it.key_lo <= it.pos0 + i);
      }
      const int64_t hi = shared ? it.key_hi : std::min<int64_t>(it.key_hi, pos_of[r] + 1);
      CHECK(it.key_lo < hi);
      if (it.part < 0) {
        seen[{int64_t(r), it.kvh}].push_back({it.key_lo, hi});
      } else {
        for (int h = 0; h < kGroup; ++h) {
          const size_t slot = size_t(it.part) + size_t(i * kGroup + h);
          CHECK(slot < slot_row.size() && slot_row[slot] == -1);
          if (slot >= slot_row.size()) continue;
          slot_row[slot] = (int64_t(r) * hkv + it.kvh) * kGroup + h;
          slot_keys[slot] = {it.key_lo, int32_t(hi)};
        }
      }
    }
  }
  for (int64_t r : slot_row) CHECK(r >= 0);
  for (const CombineItem& c : plan.combine) {
    CHECK(c.npos >= 1 && c.npos <= plan.combine_pos && c.nsplit >= 1 && c.nsplit + c.pre_nsplit >= 2);
    for (int i = 0; i < c.npos; ++i)
      for (int h = 0; h < kGroup; ++h) {
        std::vector<std::pair<int64_t, int64_t>> keys;
        auto take = [&](int part, int stride, int n) {
          for (int k = 0; k < n; ++k) {
            const size_t slot = size_t(part) + size_t(k) * size_t(stride) + size_t(i * kGroup + h);
            CHECK(slot < slot_row.size());
            if (slot >= slot_row.size()) return;
            CHECK(slot_row[slot] == (int64_t(c.row0 + i) * hkv + c.kvh) * kGroup + h);
            CHECK(!merged[slot]);
            merged[slot] = 1;
            keys.push_back(slot_keys[slot]);
          }
        };
        take(c.pre_part, c.strides >> 16, c.pre_nsplit);
        take(c.part, c.strides & 0xffff, c.nsplit);
        // in key order, so that the merge's order is that of the keys
        CHECK(std::is_sorted(keys.begin(), keys.end()));
        if (h == 0) seen[{int64_t(c.row0 + i), c.kvh}].insert(seen[{int64_t(c.row0 + i), c.kvh}].end(), keys.begin(), keys.end());
      }
  }
  for (char m : merged) CHECK(m);
  CHECK(seen.size() == pos_of.size() * size_t(hkv));
  for (auto& [row, keys] : seen) {
    std::sort(keys.begin(), keys.end());
    CHECK(keys.front().first == 0 && keys.back().second == pos_of[size_t(row.first)] + 1);
    for (size_t k = 1; k < keys.size(); ++k) CHECK(keys[k].first == keys[k - 1].second);
  }
  CHECK(plan.total >= plan.off_acc + size_t(plan.part_slots) * kHeadDim * 4);
}

}  // namespace

int main() {
  Rng g{99};
  const int cus[] = {1, 8, 256, 304};
  const int32_t splits[][2] = {{0, 0}, {64, 32}, {128, 96}, {4096, 1 << 20}};
  for (int t = 0; t < 400; ++t) {
    const Step st = random_step(g);
    const int hkv = t % 2 ? 2 : 1;
    ppas_shape sh{8 * hkv, hkv, 128, 16, 1 << 20, 0.1f};
    const int32_t n = int32_t(st.seqs.size()), np = int32_t(st.prefixes.size());
    CHECK(validate(&sh, st.seqs.data(), n, nullptr, INT32_MAX, false) == PPAS_OK);
    CHECK(validate_prefixes(st.seqs.data(), n, nullptr, INT32_MAX, st.prefixes.data(), np) == PPAS_OK);
    PlanOpts o;
    o.prefill_split = splits[t % 4][0];
    o.decode_split = splits[t % 4][1];
    o.tile_pos = (t / 4) % 3 == 0 ? 0 : (t / 4) % 3 == 1 ? kTilePosSmall : kTilePosLarge;
    Plan plan;
    make_plan(sh, st.seqs.data(), n, cus[(t / 3) % 4], o, plan, st.prefixes.data(), np);
    check(st, plan, hkv);
  }
  // own ranges around multiples of the longest decode item, cut as long as can be
  for (int keys : {16384, 16385, 32767, 32768, 32769, 49151, 65535}) {
    Step st;
    st.seqs = {ppas_seq{0, 1, 1024 + keys - 1}, ppas_seq{1, 1, 1024 + keys - 1}, ppas_seq{2, 1, 1024}};
    st.len = {1024, 1024, 1024};
    st.prefixes = {ppas_prefix{0, 3, 1024}};
    ppas_shape sh{8, 1, 128, 16, 1 << 20, 0.1f};
    CHECK(validate(&sh, st.seqs.data(), 3, nullptr, INT32_MAX, false) == PPAS_OK);
    PlanOpts o;
    o.prefill_split = 1024;
    o.decode_split = 1 << 20;
    Plan plan;
    make_plan(sh, st.seqs.data(), 3, 256, o, plan, st.prefixes.data(), 1);
    check(st, plan, 1);
  }
  if (g_failures) return 1;
  std::printf("ok\n");
  return 0;
}
