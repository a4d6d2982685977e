// Host-side validation and work planning for one mixed step (pure C++, no HIP).
#include "plan.h"

#include <algorithm>
#include <cmath>
#include <limits>
#include <numeric>

namespace ppas {

namespace {
size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// decode cost / prefill cost above which the two kinds are interleaved
#ifndef PPAS_INTERLEAVE_RATIO
#define PPAS_INTERLEAVE_RATIO 0.5
#endif
constexpr double kInterleaveRatio = PPAS_INTERLEAVE_RATIO;
// largest decode cost, relative to the prefill cost, at which a step may use
// 32-position prefill tiles
#ifndef PPAS_LARGE_TILE_DECODE_SHARE
#define PPAS_LARGE_TILE_DECODE_SHARE 0.05
#endif
constexpr double kLargeTileDecodeShare = PPAS_LARGE_TILE_DECODE_SHARE;
// when interleaving, prefill advances at this multiple of the decode fraction
#ifndef PPAS_INTERLEAVE_BIAS
#define PPAS_INTERLEAVE_BIAS 1.0
#endif
// prefill items aimed at per compute unit when tiles need key splits
#ifndef PPAS_PREFILL_ITEMS_PER_CU
#define PPAS_PREFILL_ITEMS_PER_CU 2
#endif
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
}  // namespace

ppas_status validate(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                     const int32_t* bt_host, int32_t bt_stride, bool check_overlap) {
  if (!shape) return PPAS_EINVAL;
  const ppas_shape& s = *shape;
  if (s.n_q_heads <= 0 || s.n_kv_heads <= 0 || s.head_dim <= 0 || s.page_size <= 0 || s.num_pages <= 0)
    return PPAS_EINVAL;
  if (!std::isfinite(s.scale) || !(s.scale > 0.f)) return PPAS_EINVAL;
  if (s.n_q_heads % s.n_kv_heads != 0) return PPAS_EINVAL;
  if (s.n_q_heads / s.n_kv_heads != kGroup || s.head_dim != kHeadDim || s.page_size != kPage)
    return PPAS_EUNSUPPORTED;
  if (n_seqs < 0) return PPAS_EINVAL;
  if (n_seqs == 0) return PPAS_OK;
  if (!seqs) return PPAS_EINVAL;
  if (bt_stride <= 0) return PPAS_EINVAL;
  int64_t qs = 0;
  for (int32_t i = 0; i < n_seqs; ++i) {
    const ppas_seq& q = seqs[i];
    if (q.n_query < 1 || q.cached_len < 0) return PPAS_EINVAL;
    if (q.query_start != qs) return PPAS_EINVAL;
    const int64_t len = int64_t(q.cached_len) + q.n_query;
    if (len > INT32_MAX - 64) return PPAS_ERANGE;
    qs += q.n_query;
    if (qs > INT32_MAX) return PPAS_ERANGE;
    if (ceil_div(len, kPage) > bt_stride) return PPAS_EINVAL;
  }
  if (!bt_host) return PPAS_OK;
  for (int32_t i = 0; i < n_seqs; ++i) {
    const int64_t pages = ceil_div(int64_t(seqs[i].cached_len) + seqs[i].n_query, kPage);
    const int32_t* row = bt_host + int64_t(i) * bt_stride;
    for (int64_t j = 0; j < pages; ++j)
      if (row[j] < 0 || row[j] >= s.num_pages) return PPAS_ERANGE;
  }
  if (check_overlap) {
    // No (page, slot) may be written by two requests of the step. A request's new
    // positions form one run of slots per page it touches; sorting those runs by
    // (page, first slot) puts any two that share a page side by side, so the cost
    // follows the pages the step writes, not the size of the pool.
    struct Run {
      int32_t page, lo, hi;   // slots lo..hi of the page
    };
    std::vector<Run> runs;
    for (int32_t i = 0; i < n_seqs; ++i) {
      const int32_t* row = bt_host + int64_t(i) * bt_stride;
      const int64_t end = int64_t(seqs[i].cached_len) + seqs[i].n_query;
      for (int64_t p = seqs[i].cached_len; p < end;) {
        const int64_t lp = p / kPage;
        const int64_t stop = std::min(end, (lp + 1) * kPage);
        runs.push_back(Run{row[lp], int32_t(p % kPage), int32_t((stop - 1) % kPage)});
        p = stop;
      }
    }
    std::sort(runs.begin(), runs.end(),
              [](const Run& a, const Run& b) { return a.page != b.page ? a.page < b.page : a.lo < b.lo; });
    for (size_t k = 1; k < runs.size(); ++k)
      if (runs[k].page == runs[k - 1].page && runs[k].lo <= runs[k - 1].hi) return PPAS_EINVAL;
  }
  return PPAS_OK;
}

ppas_status validate_prefixes(const ppas_seq* seqs, int32_t n_seqs, const int32_t* bt_host, int32_t bt_stride,
                              const ppas_prefix* prefixes, int32_t n_prefixes) {
  if (n_prefixes < 0 || (n_prefixes > 0 && !prefixes)) return PPAS_EINVAL;
  int32_t at = 0;   // requests before this one belong to earlier prefixes
  for (int32_t k = 0; k < n_prefixes; ++k) {
    const ppas_prefix& p = prefixes[k];
    if (p.first_seq < at || p.n_seqs < 1 || p.first_seq >= n_seqs || p.n_seqs > n_seqs - p.first_seq) return PPAS_EINVAL;
    if (p.len < 0 || p.len % kPage != 0) return PPAS_EINVAL;
    at = p.first_seq + p.n_seqs;
    for (int32_t s = p.first_seq; s < at; ++s)
      if (p.len > seqs[s].cached_len) return PPAS_EINVAL;
    if (!bt_host) continue;
    const int32_t* first = bt_host + int64_t(p.first_seq) * bt_stride;
    for (int32_t s = p.first_seq + 1; s < at; ++s)
      if (!std::equal(first, first + p.len / kPage, bt_host + int64_t(s) * bt_stride)) return PPAS_EINVAL;
  }
  return PPAS_OK;
}

namespace {

// Most new tokens of a request whose rows share their prefix's tiles with other
// requests' rows; the rows of longer chunks fill tiles of their own.
constexpr int32_t kShareMaxRows = 64;

// Consecutive rows (of requests first_seq..end_seq-1) over keys [0, len) of table row
// `seq`, and their tiles, KV head after KV head, each with nsplit partials from slot
// `part` on.
struct SharedTile {
  int32_t row0, npos, part, nsplit;
};
struct SharedRun {
  int32_t seq, first_seq, end_seq, row0, rows;
  int64_t len;
  std::vector<SharedTile> tiles;
};

// How a step with shared prefixes is cut: tile positions, and the most keys of a
// prefill and of a decode item; tile 0 where it is not worth sharing.
struct SharedCut {
  int32_t tile = 0;
  int64_t prefill = 0, decode = 0, row_keys = 0;   // rows of at most row_keys own keys go to single waves
};

// Sharing pays where it can save a step about 100,000 keys (times KV heads) or more, those of
// every row of a group but one: below, the requests find the prefix in the caches, and the
// tiles' longer items and the join cost as much as they save. Measured, attention with its
// merge, decode rows, 2 KV heads: 8 requests of 2,048 shared keys (29,000 saved) 12.3 us against 11.6 apart; 16 of 4,096 (123,000)
// 16.8 against 15.3 to 17.0 against 18.6 with what else they hold; 32 of 4,096
// (254,000) 17.2 against 23.7; 64 of 8,192 with up to 4,000 of their own 38 against 92.
constexpr int64_t kShareMinSaved = 100000;

// Most own keys of a decode row that a single wave takes (a wave streams a key in about
// 42 ns, a workgroup in 8). Packed so, rows take a quarter or an eighth of the workgroups:
// 256 rows of 16 to 512 own keys and 384 tile items 77 -> 70 us; where workgroups are few,
// they only take longer (206 rows of 217 to 439 keys and 28 tiles 21.5 -> 25.5 us).
constexpr int64_t kRowKeys = 512;
static_assert(kRowKeys <= kRowMaxKeys, "a wave takes the row");

// Microseconds of a step with pieces of at most so many keys, fitted to 32,000 plans of 105
// steps, each timed over a hundred passes in a row (5 to 6 % rms; the choice made with it
// takes 4 % longer than the best of them on average, 1.3 times at worst): a fixed part; the
// time that the items take on the workgroup slots in launch order, and the one that the
// decode rows' keys take from memory (with a share of a slot's time for every decode item),
// which hide one another in part (the `power` mean of the two); then the merge, by its
// partials' bytes and the splits of a row. A tile's key takes `key` alone and `key_full` with
// every slot taken (for 16 positions 5 % above the fit, which timed full chips of them too
// short).
struct SharedCost {
  double fixed, item, key, key_full, decode_item, decode_key, row, row_key, tbs, tbs_many, decode_slot, power, mb, split;
};
constexpr SharedCost kShared16{7.05, 5.0, 0.0168, 0.0258, 4.9, 0.0088, 9.5, 0.0374, 21.4, 7.27, 4.1, 1.33, 0.295, 0.095};
constexpr SharedCost kShared32{7.74, 6.7, 0.0233, 0.0244, 5.4, 0.0100, 14.2, 0.0376, 9.35, 6.49, 5.0, 2.61, 0.297, 0.066};
double together(double slots_us, double memory_us, double power) {
  const double most = std::max(slots_us, memory_us), least = std::min(slots_us, memory_us);
  return most <= 0 ? 0 : most * std::pow(1 + std::pow(least / most, power), 1 / power);
}

// Items of one length: their keys, and how many (per KV head).
struct Lot {
  double keys, count;
};

// When the last of the lots ends (`keys`: an item's time) that `slots` workgroup slots take
// in order, each on the slots that are free first. Slots that are free at about the same
// time are one entry of `free`.
double last_end(const std::vector<Lot>& lots, double slots) {
  std::vector<Lot> free{{0, slots}};   // time, slots
  double end = 0;
  for (const Lot& lot : lots) {
    for (double left = lot.count; left > 1e-6;) {
      auto first = std::min_element(free.begin(), free.end(), [](const Lot& x, const Lot& y) { return x.keys < y.keys; });
      const double start = first->keys, n = std::min(first->count, left), t = start + lot.keys;
      first->count -= n;
      if (first->count < 1e-6) free.erase(first);
      auto same = std::find_if(free.begin(), free.end(), [&](const Lot& f) { return std::fabs(f.keys - t) < 0.2; });
      if (same == free.end()) free.push_back(Lot{t, n});
      else same->count += n;
      end = std::max(end, t);
      left -= n;
    }
  }
  return end;
}

struct Job {
  WorkItem item;
  double cost;
  int32_t piece;
};

// A job's place in its queue: longest first, in cost buckets of 256 keys; inside a
// bucket items of the same request and KV head stay together, so that neighbours share
// keys in one L2. Packed, so that the sort compares plain integers (a third of a
// plan's time).
struct Place {
  uint64_t cost_seq, head_pos, piece_job;
  bool operator<(const Place& o) const {
    if (cost_seq != o.cost_seq) return cost_seq < o.cost_seq;
    if (head_pos != o.head_pos) return head_pos < o.head_pos;
    return piece_job < o.piece_job;
  }
};
Place place_of(const Job& j, size_t job) {
  const uint64_t bucket = UINT32_MAX - uint64_t(int64_t(j.cost) >> 8);   // a cost is below 2^33
  return Place{bucket << 32 | uint32_t(j.item.seq), uint64_t(j.item.kvh) << 32 | (UINT32_MAX - uint32_t(j.item.pos0)),
               uint64_t(j.piece) << 32 | uint64_t(job)};
}

// What a step's items are cut from, by length. `own` is the first own key of every request.
struct Load {          // tiles' keys, runs' and chunks'
  double len = 0, rows = 0, tiles[2] = {0, 0};   // of kTilePosSmall and kTilePosLarge
};
struct Own {           // decode rows' keys, by whole blocks, which is all that a piece's length depends on
  int64_t blocks;
  double count = 0, behind = 0;   // rows, and those behind a shared prefix
};
struct StepLoads {
  std::vector<Load> tiles;
  std::vector<Own> decode;
  int64_t longest_run = 0, decode_keys = 0;
};

// Tiles come in at most kLoads steps of length (a mean each), so that an option of the choice
// costs the same for any number of requests (2,048 of 33 rows took 14 ms in lots of their own).
// Requests of several tiles count their middle one.
StepLoads loads_of(const ppas_seq* seqs, int32_t n_seqs, const std::vector<SharedRun>& runs,
                   const std::vector<int32_t>& own) {
  constexpr int64_t kLoads = 64;
  StepLoads r;
  std::vector<int64_t> each;   // twice a decode row's blocks, and one where there is a prefix
  auto chunk_len = [&](int32_t s) { return int64_t(seqs[s].cached_len) + (seqs[s].n_query + 1) / 2 - own[size_t(s)]; };
  for (const SharedRun& run : runs) r.longest_run = std::max(r.longest_run, run.len);
  int64_t longest = r.longest_run;
  for (int32_t s = 0; s < n_seqs; ++s) {
    if (seqs[s].n_query > 1) {
      longest = std::max(longest, chunk_len(s));
      continue;
    }
    const int64_t keys = int64_t(seqs[s].cached_len) + 1 - own[size_t(s)];
    r.decode_keys += keys;
    each.push_back(2 * ceil_div(keys, kDecodeBlock) + (own[size_t(s)] ? 1 : 0));
  }
  const int64_t step = std::max<int64_t>(kPrefillBlock, longest / kLoads + 1);
  std::vector<Load> by_len(size_t(longest / step) + 1);
  auto put = [&](int64_t rows, int64_t len) {
    Load& l = by_len[size_t(len / step)];
    l.len += double(len) * double(rows);
    l.rows += double(rows);
    l.tiles[0] += double(ceil_div(rows, kTilePosSmall));
    l.tiles[1] += double(ceil_div(rows, kTilePosLarge));
  };
  for (const SharedRun& run : runs) put(run.rows, run.len);
  for (int32_t s = 0; s < n_seqs; ++s)
    if (seqs[s].n_query > 1) put(seqs[s].n_query, chunk_len(s));
  for (Load& l : by_len)
    if (l.rows > 0) {
      l.len /= l.rows;
      r.tiles.push_back(l);
    }
  std::sort(each.begin(), each.end());
  for (const int64_t e : each) {
    if (r.decode.empty() || r.decode.back().blocks != e / 2) r.decode.push_back(Own{e / 2});
    r.decode.back().count += 1;
    r.decode.back().behind += double(e & 1);
  }
  return r;
}

void add_lot(std::vector<Lot>& lots, double keys, double count) {
  for (Lot& l : lots)
    if (std::fabs(l.keys - keys) < 1) {
      l.count += count;
      return;
    }
  lots.push_back(Lot{keys, count});
}
bool longer(const Lot& x, const Lot& y) { return x.keys > y.keys; }

// The decode rows in pieces of at most `most` keys, by length in steps of 128: those that a
// wave can take apart.
struct DecodePieces {
  int64_t most = 0;
  std::vector<Lot> items, rows;
  double n_items = 0, n_rows = 0, keys = 0, slots = 0, splits = 1;
};
DecodePieces decode_pieces(const StepLoads& loads, int64_t most) {
  DecodePieces d;
  d.most = most;
  d.keys = double(loads.decode_keys);
  for (const Own& o : loads.decode) {
    const int64_t keys = o.blocks * kDecodeBlock, n = ceil_div(keys, most);
    const double len = keys <= 64 * n ? 32 : 128.0 * double(ceil_div(keys, 128 * n)) - 64;
    if (n == 1 && keys <= kRowKeys) {
      add_lot(d.rows, len, o.count);
      d.n_rows += o.count;
    } else {
      add_lot(d.items, len, o.count * double(n));
      d.n_items += o.count * double(n);
    }
    d.slots += (n > 1 ? o.count : o.behind) * double(n) * kGroup;
    d.splits = std::max(d.splits, double(n));
  }
  std::sort(d.items.begin(), d.items.end(), longer);
  std::sort(d.rows.begin(), d.rows.end(), longer);
  return d;
}

// The tiles in pieces of at most `most` keys, or, in a plan apart, of about as many, where
// rows in one piece are written whole.
struct TilePieces {
  int32_t tile;
  int64_t most;
  std::vector<Lot> items;
  double n = 0, keys = 0, slots = 0, splits = 0;
};
TilePieces tile_pieces(const StepLoads& loads, int32_t tile, int64_t most, bool apart) {
  TilePieces t{tile, most, {}};
  for (const Load& l : loads.tiles) {
    const double n = std::max(1.0, apart ? std::floor(l.len / double(most) + 0.5) : std::ceil(l.len / double(most)));
    const double items = l.tiles[tile == kTilePosLarge] * n;
    add_lot(t.items, l.len / n, items);
    t.n += items;
    t.keys += items * l.len / n;
    if (!apart || n > 1) t.slots += l.rows * n * kGroup;
    if (apart) t.splits = std::max(t.splits, n);
  }
  if (!apart) t.splits = double(ceil_div(loads.longest_run, most));
  std::sort(t.items.begin(), t.items.end(), longer);
  return t;
}

// A way to cut a step, and its time by the model: `bound` with no slot idle, and time_of.
struct Option {
  const TilePieces* t;
  const DecodePieces* d;
  bool pack;                    // the decode rows of few keys go to single waves
  double bound, rest, memory;   // rest: what depends on neither the slots nor memory
};
const SharedCost& cost_of(const TilePieces& t) { return t.tile == kTilePosSmall ? kShared16 : kShared32; }
double waves_of(const TilePieces& t) { return t.tile == kTilePosSmall ? 4.0 : 8.0; }
double slots_of(const TilePieces& t, int num_cus) { return double(num_cus) * (t.tile == kTilePosSmall ? 2 : 1); }
double per_key(const TilePieces& t, int hkv, int num_cus) {
  const SharedCost& c = cost_of(t);
  return c.key + (c.key_full - c.key) * std::min(1.0, t.n * hkv / slots_of(t, num_cus));
}
Option option_of(const TilePieces& t, const DecodePieces& d, bool pack, int hkv, int num_cus) {
  const SharedCost& c = cost_of(t);
  const double key = per_key(t, hkv, num_cus), slots = slots_of(t, num_cus);
  double work = t.n * c.item + t.keys * key, n = t.n + d.n_items;
  for (const Lot& l : d.items) work += l.count * (c.decode_item + c.decode_key * l.keys);
  for (const Lot& l : d.rows)
    work += pack ? l.count / waves_of(t) * (c.row + c.row_key * l.keys) : l.count * (c.decode_item + c.decode_key * l.keys);
  n += pack ? d.n_rows / waves_of(t) : d.n_rows;
  const double memory = hkv * d.keys * 4.0 * kHeadDim / ((n * hkv <= num_cus ? c.tbs : c.tbs_many) * 1e6) +
                        hkv * (d.n_items + (pack ? 0 : d.n_rows)) * c.decode_slot / slots;
  const double rest = c.fixed + c.mb * hkv * (t.slots + d.slots) * (kHeadDim + 2) * 4e-6 + c.split * (t.splits + d.splits);
  const double one = t.items.empty() ? 0 : c.item + key * t.items[0].keys;
  return Option{&t, &d, pack, rest + together(std::max(work * hkv / slots, one), memory, c.power), rest, memory};
}
double time_of(const Option& o, int hkv, int num_cus) {
  const SharedCost& c = cost_of(*o.t);
  const double key = per_key(*o.t, hkv, num_cus);
  // lots in launch order, as their times: tiles and decode items, longest first, then the rows
  std::vector<Lot> lots;
  for (const Lot& l : o.t->items) lots.push_back(Lot{c.item + key * l.keys, l.count * hkv});
  for (const Lot& l : o.d->items) lots.push_back(Lot{c.decode_item + c.decode_key * l.keys, l.count * hkv});
  if (!o.pack)
    for (const Lot& l : o.d->rows) lots.push_back(Lot{c.decode_item + c.decode_key * l.keys, l.count * hkv});
  std::sort(lots.begin(), lots.end(), longer);
  if (o.pack)
    for (const Lot& l : o.d->rows) lots.push_back(Lot{c.row + c.row_key * l.keys, l.count * hkv / waves_of(*o.t)});
  return o.rest + together(last_end(lots, slots_of(*o.t, num_cus)), o.memory, c.power);
}

// How a step is cut without shared prefixes: the tile's positions, and the most keys of a
// piece (about as many, of a tile).
struct PlainCut {
  int32_t tile = 0;
  int64_t prefill = 0, decode = 0, prefill_keys = 0, decode_keys = 0;
};
PlainCut plain_cut(const ppas_seq* seqs, int32_t n_seqs, int hkv, int num_cus, const PlanOpts& opts) {
  PlainCut cut;
  // Total work, to size the key splits so that the launch has several
  // workgroups per compute unit: keys summed over prefill tiles (of either
  // size) and over decode rows.
  auto prefill_keys_for = [&](int32_t tile) {
    int64_t keys = 0;
    for (int32_t s = 0; s < n_seqs; ++s) {
      const ppas_seq& q = seqs[s];
      if (q.n_query == 1) continue;
      for (int32_t t0 = 0; t0 < q.n_query; t0 += tile)
        keys += int64_t(q.cached_len) + std::min(q.n_query, t0 + tile);
    }
    return keys * hkv;
  };
  int64_t large_tiles = 0;
  for (int32_t s = 0; s < n_seqs; ++s) {
    const ppas_seq& q = seqs[s];
    if (q.n_query == 1)
      cut.decode_keys += int64_t(q.cached_len + 1) * hkv;
    else
      large_tiles += ceil_div(q.n_query, kTilePosLarge) * hkv;
  }

  // Tile shape. The eight-wave kernel stages each K/V block once for 256 rows
  // instead of 128, which pays when the step's prefill alone fills the chip with
  // 32-position tiles (two per CU before any key split) and decode rows are a
  // small share of the work (a workgroup then holds a whole CU, so a prefill
  // tile no longer shares its CU with a decode item).
  cut.tile = opts.tile_pos;
  if (cut.tile != kTilePosSmall && cut.tile != kTilePosLarge) {
    const int64_t small_keys = prefill_keys_for(kTilePosSmall);
    const bool big = large_tiles >= int64_t(2) * num_cus;
    const bool few_decodes = double(cut.decode_keys) * 2.0 < kLargeTileDecodeShare * double(small_keys);
    cut.tile = (big && few_decodes) ? kTilePosLarge : kTilePosSmall;
  }
  cut.prefill_keys = prefill_keys_for(cut.tile);

  cut.prefill = opts.prefill_split;
  if (cut.prefill <= 0) {
    const int64_t target = int64_t(PPAS_PREFILL_ITEMS_PER_CU) * num_cus;
    cut.prefill = std::max<int64_t>(256, ceil_div(cut.prefill_keys, target));
  }
  cut.prefill = std::max<int64_t>(kPrefillBlock, ceil_div(cut.prefill, kPrefillBlock) * kPrefillBlock);
  cut.decode = opts.decode_split;
  if (cut.decode <= 0) {
    const int64_t target = int64_t(2) * num_cus;
    cut.decode = std::min<int64_t>(8192, std::max<int64_t>(512, ceil_div(cut.decode_keys, target)));
  }
  cut.decode = std::max<int64_t>(kDecodeBlock, ceil_div(cut.decode, kDecodeBlock) * kDecodeBlock);
  cut.decode = std::min<int64_t>(cut.decode, kDecodeMaxKeys);
  return cut;
}

// Whether requests first..end-1 need fewer tiles together than apart (or decode rows' streams,
// all but one of them): the rows of a chunk share its tiles' keys already, so that requests of 16,
// 32, 48 or 64 rows save nothing, and their partials are all that sharing them adds (64 of 64 rows
// behind 1,024 keys 79 us, apart 50; 128 behind 4,096 303, apart 247; two or eight of them as long
// either way).
bool saves_tiles(const ppas_seq* seqs, int32_t first, int32_t end) {
  int64_t apart = 0, chunk_rows = 0;
  for (int32_t s = first; s < end; ++s) {
    apart += ceil_div(seqs[s].n_query, kTilePosSmall);
    if (seqs[s].n_query > 1) chunk_rows += seqs[s].n_query;
  }
  return apart > std::max<int64_t>(1, ceil_div(chunk_rows, kTilePosSmall));
}

// `own` is the first own key of every request; opts' fields that are set stand.
SharedCut choose_shared(const ppas_seq* seqs, int32_t n_seqs, int hkv, int num_cus, const PlanOpts& opts,
                        const std::vector<SharedRun>& runs, const std::vector<int32_t>& own) {
  SharedCut best;
  int64_t saved = 0;
  for (const SharedRun& r : runs) saved += int64_t(r.rows - 1) * r.len * hkv;
  if (saved < kShareMinSaved && opts.prefill_split <= 0) return best;
  static constexpr int64_t kPrefill[] = {128, 256, 512, 768, 1024, 1280, 1536, 2048, 2816, 4224, 5632, 8448};
  static constexpr int64_t kDecode[] = {256, 512, 768, 1024, 1536, 2048, 2560, 4096};
  auto up = [](int64_t keys, int64_t block) { return std::max(block, ceil_div(keys, block) * block); };
  const StepLoads loads = loads_of(seqs, n_seqs, runs, own);

  std::vector<DecodePieces> decode;
  if (opts.decode_split > 0)
    decode.push_back(decode_pieces(loads, std::min<int64_t>(up(opts.decode_split, kDecodeBlock), kDecodeMaxKeys - kDecodeBlock)));
  else
    for (int64_t most : kDecode) {
      decode.push_back(decode_pieces(loads, most));
      if (decode.back().splits == 1) break;   // longer pieces are the same ones
    }
  std::vector<TilePieces> tiles;
  for (int32_t tile : {kTilePosSmall, kTilePosLarge}) {
    if (opts.tile_pos != 0 && opts.tile_pos != tile) continue;
    if (opts.prefill_split > 0)
      tiles.push_back(tile_pieces(loads, tile, up(opts.prefill_split, kPrefillBlock), false));
    else
      for (int64_t most : kPrefill) tiles.push_back(tile_pieces(loads, tile, most, false));
  }

  // With chunks in the groups, the plan apart by the same model: a few tiles saved may not be
  // worth the partials of every row (128 requests of 17 rows behind 512 keys 46 us, apart 32).
  double apart_us = std::numeric_limits<double>::infinity();
  const bool chunks = std::any_of(runs.begin(), runs.end(), [](const SharedRun& r) { return r.rows > r.end_seq - r.first_seq; });
  if (chunks && opts.prefill_split <= 0) {
    const PlainCut cut = plain_cut(seqs, n_seqs, hkv, num_cus, opts);
    const StepLoads all = loads_of(seqs, n_seqs, {}, std::vector<int32_t>(size_t(n_seqs), 0));
    const TilePieces t = tile_pieces(all, cut.tile, cut.prefill, true);
    const DecodePieces d = decode_pieces(all, cut.decode);
    apart_us = time_of(option_of(t, d, false, hkv, num_cus), hkv, num_cus);
  }

  // Every combination's lower bound; then, from the lowest on, the time with idle slots,
  // until no bound is below the best time.
  std::vector<Option> options;
  for (const TilePieces& t : tiles)
    for (const DecodePieces& d : decode)
      for (const bool pack : {false, true})
        if (!pack || d.n_rows > 0) options.push_back(option_of(t, d, pack, hkv, num_cus));
  std::sort(options.begin(), options.end(), [](const Option& x, const Option& y) { return x.bound < y.bound; });
  double best_us = 0;
  for (const Option& o : options) {
    if (best.tile != 0 && o.bound >= best_us) break;
    if (o.bound >= apart_us) break;
    const double us = time_of(o, hkv, num_cus);
    if (best.tile == 0 || us < best_us) {
      best_us = us;
      best.tile = o.t->tile;
      best.prefill = o.t->most;
      best.decode = o.d->most;
      best.row_keys = o.pack ? kRowKeys : 0;
    }
  }
  if (best_us >= apart_us) best.tile = 0;
  return best;
}

}  // namespace

void make_plan(const ppas_shape& shape, const ppas_seq* seqs, int32_t n_seqs, int num_cus, const PlanOpts& opts,
               Plan& plan, const ppas_prefix* prefixes, int32_t n_prefixes) {
  plan.items.clear();
  plan.rows.clear();
  plan.combine.clear();
  plan.combine_pos = 0;
  plan.part_slots = 0;
  const int hkv = shape.n_kv_heads;
  if (num_cus <= 0) num_cus = 256;

  // Shared prefixes: runs of consecutive rows whose first keys are attended by tiles
  // of all of them together, over whole 64-key blocks, so that their items need no
  // mask and own key ranges start on a block; the rest of the prefix is read by every
  // request for itself. own[s] is the first key of request s's own range.
  std::vector<int32_t> own(size_t(n_seqs), 0);
  std::vector<SharedRun> runs;
  for (int32_t k = 0; k < n_prefixes; ++k) {
    const ppas_prefix& p = prefixes[k];
    const int32_t len = p.len / kPrefillBlock * kPrefillBlock;
    if (len == 0) continue;
    const int32_t end = p.first_seq + p.n_seqs;
    for (int32_t s = p.first_seq; s < end;) {
      int32_t e = s;
      while (e < end && seqs[e].n_query <= kShareMaxRows) ++e;
      if (e - s > 1 && (opts.prefill_split > 0 || saves_tiles(seqs, s, e))) {
        const int32_t row0 = seqs[s].query_start;
        runs.push_back(SharedRun{p.first_seq, s, e, row0, seqs[e - 1].query_start + seqs[e - 1].n_query - row0, len, {}});
        for (int32_t i = s; i < e; ++i) own[size_t(i)] = len;
      }
      s = std::max(e, s + 1);
    }
  }

  SharedCut cut;
  if (!runs.empty()) {
    cut = choose_shared(seqs, n_seqs, hkv, num_cus, opts, runs, own);
    if (cut.tile == 0) {
      runs.clear();
      std::fill(own.begin(), own.end(), 0);
    }
  }

  PlainCut plain;
  if (!cut.tile) plain = plain_cut(seqs, n_seqs, hkv, num_cus, opts);
  const int32_t tile = cut.tile ? cut.tile : plain.tile;
  const int64_t ksp = cut.tile ? cut.prefill : plain.prefill, ksd = cut.tile ? cut.decode : plain.decode;
  const int64_t prefill_keys = plain.prefill_keys, decode_keys = plain.decode_keys;
  plan.tile_pos = tile;

  // Prefill tiles load the matrix cores and decode items the memory system. When
  // the decode work is comparable to the prefill work, the two kinds are
  // interleaved in the launch order (below); otherwise decode goes last.
  const double tile_cost = double(tile) / kTilePosSmall;   // per key, relative to a 16-position tile
  const bool interleave = 2.0 * double(decode_keys) >= kInterleaveRatio * tile_cost * double(prefill_keys);

  // Key ranges of one tile or decode row. Decode rows, and prefill tiles of
  // interleaved steps, take pieces of `split` keys from key 0 (the last one
  // ragged: the short pieces fill the gaps between long items). Other prefill
  // tiles take round(keys / split) even pieces, so a step's items come close to
  // a whole number per workgroup slot. Prefill boundaries are multiples of the
  // 64-key block at or before the tile's first position, so every row sees a
  // key in every piece.
  //
  // A step of decode rows only (and no split size requested) cuts each row's keys
  // into even pieces instead, about one item per CU over the whole step: every
  // workgroup then streams from its own CU and all of them finish together
  // (measured on 48 rows of 20k-30k keys: 190 us with ~one item per CU against
  // 205 us with about two per CU, ragged). A piece never exceeds the page-id
  // capacity of a decode item.
  //
  // Fewer, longer pieces in a step of a few rows would shorten the merge (11.7 us after
  // 5.4 us of attention for one row of 3,071 keys in 96 pieces per KV head), but cost
  // precision: probabilities are rounded to bf16 relative to the largest of their piece,
  // which is then exactly 1, so fewer pieces leave more of the large probabilities
  // rounded. Against 64 bits that row's error would go from 2.12e-3 to 2.31e-3 in ten
  // pieces, that of 500 keys left whole from 2.01e-3 to 2.25e-3.
  const bool decode_even = prefill_keys == 0 && decode_keys > 0 && opts.decode_split <= 0;
  // lo: the first key, a multiple of 64
  std::vector<int64_t> b;   // the latest bounds
  auto piece_bounds = [&](int64_t lo, int64_t hi, int64_t pos0, int kind) -> const std::vector<int64_t>& {
    b.assign(1, lo);
    const int64_t kend = hi - lo;
    if (cut.tile) {   // even pieces (the last one may have up to a block more than the others)
      const int64_t n = ceil_div(kend, kind == kKindDecode ? ksd : ksp);
      const int64_t unit = kind == kKindDecode ? kDecodeBlock : kPrefillBlock;
      const int64_t top = kind == kKindDecode ? hi : pos0 / kPrefillBlock * kPrefillBlock;
      for (int64_t k = 1; k < n; ++k) b.push_back(std::min(top, lo + kend * k / n / unit * unit));
    } else if (kind == kKindDecode && decode_even) {
      const int64_t n = std::max<int64_t>(ceil_div(kend, int64_t(kDecodeMaxKeys - kDecodeBlock)),
                                          (kend * num_cus + decode_keys / 2) / decode_keys);
      for (int64_t k = 1; k < n; ++k) b.push_back(lo + kend * k / n / kDecodeBlock * kDecodeBlock);
    } else if (kind == kKindDecode) {
      for (int64_t k = 1; k * ksd < kend; ++k) b.push_back(lo + k * ksd);
    } else if (interleave) {
      for (int64_t k = 1; lo + k * ksp <= pos0; ++k) b.push_back(lo + k * ksp);
    } else {
      const int64_t n = std::max<int64_t>(1, (kend + ksp / 2) / ksp);
      const int64_t top = pos0 / kPrefillBlock * kPrefillBlock;
      for (int64_t k = 1; k < n; ++k) b.push_back(std::min(top, lo + kend * k / n / kPrefillBlock * kPrefillBlock));
    }
    b.push_back(hi);
    b.erase(std::unique(b.begin(), b.end()), b.end());
    return b;
  };

  std::vector<Job> jobs;
  jobs.reserve(size_t(4) * size_t(num_cus));
  // One item per piece of `bounds`; the partials' first slot, or -1 where rows are written whole.
  auto add_items = [&](int32_t s, int32_t g, int32_t row0, int32_t pos0, int32_t npos, int kind,
                       const std::vector<int64_t>& bounds, bool partial) {
    const int64_t nsplit = int64_t(bounds.size()) - 1;
    int32_t part = -1;
    if (partial) {
      part = int32_t(plan.part_slots);
      plan.part_slots += nsplit * int64_t(npos) * kGroup;
    }
    for (int64_t k = 0; k < nsplit; ++k) {
      const int64_t lo = bounds[size_t(k)], hi = bounds[size_t(k) + 1];
      Job j;
      j.item = WorkItem{s, g, row0, pos0, npos | (kind << 16), int32_t(lo), int32_t(hi),
                        part < 0 ? -1 : int32_t(part + k * int64_t(npos) * kGroup)};
      // relative cost: a prefill key of a 16-position tile costs 128 rows of MFMA
      // work (twice that in a 32-position tile), a decode key ~512 bytes of HBM
      // traffic; one decode key is about two prefill keys of a 16-position tile.
      // With shared prefixes the queues are one, in nanoseconds / 8: half a decode row's
      // items are shorter than a tile's there, and have to fill in behind the longest.
      j.cost = double(hi - lo) * (kind == kKindDecode ? 2.0 : tile_cost);
      if (cut.tile) j.cost = (kind == kKindDecode ? 3000 + 12.0 * double(hi - lo) : 5000 + 20.0 * tile_cost * double(hi - lo)) / 8;
      j.piece = int32_t(k);
      jobs.push_back(j);
    }
    return part;
  };
  auto merge = [&](int32_t g, int32_t row0, int32_t npos, int32_t part, int32_t nsplit, int32_t stride,
                   const SharedTile* t) {
    plan.combine.push_back(CombineItem{row0, g, npos, nsplit, part, t ? t->part + (row0 - t->row0) * kGroup : 0,
                                       t ? t->nsplit : 0, stride | (t ? t->npos * kGroup << 16 : 0)});
    plan.combine_pos = std::max(plan.combine_pos, npos);
  };
  // Rows row0.. of request s with its own keys, and with the tiles of its run (no shared prefix: null).
  auto add_unit = [&](int32_t s, int32_t g, int32_t row0, int32_t pos0, int32_t npos, int kind,
                      const SharedRun* pre) {
    const int64_t kend = int64_t(pos0) + npos;        // keys own..kend-1 are visible to some row
    const std::vector<int64_t>& bounds = piece_bounds(own[size_t(s)], kend, pos0, kind);
    const int32_t nsplit = int32_t(bounds.size()) - 1;
    int32_t part = -1;
    if (cut.tile && kind == kKindDecode && nsplit == 1 && kend - own[size_t(s)] <= cut.row_keys) {
      if (pre) {
        part = int32_t(plan.part_slots);
        plan.part_slots += kGroup;
      }
      plan.rows.push_back(WorkItem{s, g, row0, pos0, 1 | (kKindDecode << 16), own[size_t(s)], int32_t(kend), part});
    } else {
      part = add_items(s, g, row0, pos0, npos, kind, bounds, nsplit > 1 || pre);
    }
    if (!pre) {
      if (nsplit > 1) merge(g, row0, npos, part, nsplit, npos * kGroup, nullptr);
      return;
    }
    const size_t per_head = pre->tiles.size() / size_t(hkv);
    for (int32_t lo = row0; lo < row0 + npos;) {
      const SharedTile& t = pre->tiles[size_t(g) * per_head + size_t((lo - pre->row0) / tile)];
      const int32_t hi = std::min(row0 + npos, t.row0 + t.npos);
      merge(g, lo, hi - lo, part + (lo - row0) * kGroup, nsplit, npos * kGroup, &t);
      lo = hi;
    }
  };
  // A run's tiles see every key of their pieces: their position is the first one behind the prefix.
  for (SharedRun& r : runs) {
    const std::vector<int64_t>& bounds = piece_bounds(0, r.len, r.len, kKindPrefill);
    for (int32_t g = 0; g < hkv; ++g)
      for (int32_t t0 = 0; t0 < r.rows; t0 += tile) {
        const int32_t npos = std::min(tile, r.rows - t0);
        const int32_t part = add_items(r.seq, g, r.row0 + t0, int32_t(r.len), npos, kKindPrefill, bounds, true);
        r.tiles.push_back(SharedTile{r.row0 + t0, npos, part, int32_t(bounds.size()) - 1});
      }
  }
  size_t run = 0;   // the first one that ends behind the request
  for (int32_t s = 0; s < n_seqs; ++s) {
    const ppas_seq& q = seqs[s];
    for (int32_t g = 0; g < hkv; ++g) {
      while (run < runs.size() && runs[run].end_seq <= s) ++run;
      const SharedRun* pre = own[size_t(s)] ? &runs[run] : nullptr;
      if (q.n_query == 1) {
        add_unit(s, g, q.query_start, q.cached_len, 1, kKindDecode, pre);
      } else {
        for (int32_t t0 = 0; t0 < q.n_query; t0 += tile)
          add_unit(s, g, q.query_start + t0, q.cached_len + t0, std::min(tile, q.n_query - t0), kKindPrefill, pre);
      }
    }
  }

  std::stable_sort(plan.rows.begin(), plan.rows.end(),
                   [](const WorkItem& x, const WorkItem& y) { return x.key_hi - x.key_lo > y.key_hi - y.key_lo; });
  // The two kinds' queues.
  std::vector<Place> pre, dec;
  double tot_p = 0, tot_d = 0;
  for (size_t i = 0; i < jobs.size(); ++i) {
    const bool decode = !cut.tile && (jobs[i].item.npos_kind >> 16) == kKindDecode;
    (decode ? dec : pre).push_back(place_of(jobs[i], i));
    (decode ? tot_d : tot_p) += jobs[i].cost;
  }
  std::sort(pre.begin(), pre.end());
  std::sort(dec.begin(), dec.end());
  // Interleaved steps merge the two queues so that both advance at the same
  // fraction of their total work and finish together (prefill tiles load the
  // matrix cores, decode items the memory system); otherwise decode goes last
  // and fills the tail of the prefill rounds.
  std::vector<uint32_t> order;
  order.reserve(jobs.size());
  size_t ip = 0, id = 0;
  double done_p = 0, done_d = 0;
  while (ip < pre.size() || id < dec.size()) {
    const bool take_p = id >= dec.size() ||
                        (ip < pre.size() && (!interleave || done_p * tot_d <= PPAS_INTERLEAVE_BIAS * done_d * tot_p));
    const uint32_t job = uint32_t(take_p ? pre[ip++].piece_job : dec[id++].piece_job);
    (take_p ? done_p : done_d) += jobs[job].cost;
    order.push_back(job);
  }

  // Workgroup b of a launch runs on XCD b % 8. Hand each XCD runs of 8
  // consecutive items of the sorted list, with runs dealt round-robin so every XCD
  // gets the same mix of long and short items: within each block of 64 launch
  // slots, slot 8v + x takes sorted item 8x + v.
  const size_t n = order.size();
  plan.items.resize(n);
  const size_t full = n / 64 * 64;
  for (size_t b = 0; b < full; ++b) {
    const size_t x = b % 8, k = b / 8;
    const size_t src = ((k / 8) * 8 + x) * 8 + (k % 8);
    plan.items[b] = jobs[order[src]].item;
  }
  for (size_t b = full; b < n; ++b) plan.items[b] = jobs[order[b]].item;

  plan.off_rows = align_up(n * sizeof(WorkItem), 256);
  plan.off_combine = align_up(plan.off_rows + plan.rows.size() * sizeof(WorkItem), 256);
  plan.list_bytes = plan.off_combine + plan.combine.size() * sizeof(CombineItem);
  plan.off_ml = 0;
  plan.off_acc = align_up(size_t(plan.part_slots) * 8, 256);
  plan.total = std::max<size_t>(256, align_up(plan.off_acc + size_t(plan.part_slots) * kHeadDim * 4, 256));
}

void make_append_items(const ppas_seq* seqs, int32_t n_seqs, std::vector<AppendItem>& items) {
  items.clear();
  for (int32_t s = 0; s < n_seqs; ++s) {
    const ppas_seq& q = seqs[s];
    const int32_t first = q.cached_len / kPage;
    const int32_t last = int32_t((int64_t(q.cached_len) + q.n_query - 1) / kPage);
    for (int32_t lp = first; lp <= last; ++lp)
      items.push_back(AppendItem{s, lp, q.cached_len, q.n_query, q.query_start, 0, 0, 0});
  }
}

}  // namespace ppas
