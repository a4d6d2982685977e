// The projection of 8-bit integers, whose kernels (but for the tiles of 128 x 128) are the bf16 projection's with 16x16x64
// integer MFMAs: rows of 128 features are 128 bytes as 64 bf16 features are, so stages,
// transfers, swizzles and schedule are the same, and one instruction takes as long. The
// int32 sums are exact, so no sum needs two levels and any split gives the same result;
// the epilogue turns them into values with their token's and channel's scale.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device.h"
#include "gateup_i8_mid.h"
#include "gateup_kernels.h"

namespace ppas {

namespace {

// How token rows go: the projection's choice, or the tiles of 128 x 128.
struct Way {
  GateupChoice c;
  bool mid = false;
  double cost = 0;
};

// Microseconds of the 128 x 128 tiles where they fit one round, else none; by the share of
// the compute units that they fill. Fitted to calls of 64 to 4,096 tokens and seven
// projections (7 %), weights from memory. They win from a few hundred tokens to about
// 2,000: 700 x 2,048 x 2,048 11.3 us against 13.2, 1,024 x 5,504 x 2,048 22.1 against 25.2,
// 512 x 4,096 x 4,096 19.1 against 24.0, 2,048 x 11,008 x 2,048 53.6 against 67.1; not on
// a full chip with a short reduction (1,500 x 2,048 x 2,560 17.3 against 16.1), nor where
// the others can split a long one (1,024 x 11,008 x 2,048 51.1 against 39.5).
bool mid_cost(int32_t T, int32_t H, int32_t N2, int cus, double* us) {
  const int64_t tiles = (int64_t(T) + 127) / 128 * ((int64_t(N2) + 127) / 128);
  if (tiles > cus) return false;
  const double full = double(tiles) / cus;
  *us = 5.5 + 4.0 * full * full + H / 128 * (0.33 + 0.17 * full);
  return true;
}

Way choose_way(int32_t T, const Int8Product& p, bool act, int max_splits, int cus) {
  Way r;
  r.c = gateup_choose(T, p.H / 2, p.N2, act, true, max_splits, cus, true);
  r.cost = r.c.cost;
  double us = 0;
  if (!act && r.c.kernel == GateupChoice::kTiles && mid_cost(T, p.H, p.N2, cus, &us) && us < r.cost) {
    r.mid = true;
    r.cost = us;
  }
  return r;
}

// One launch (two with splits) of token rows first .. first + T - 1.
hipError_t launch_rows_of(const Int8Product& p, int32_t first, int32_t T, const Way& way, bool act, void* part,
                          hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  const GateupChoice& c = way.c;
  GemmArgs a{};
  a.x = reinterpret_cast<const uint16_t*>(p.x + size_t(first) * p.H);
  a.w = reinterpret_cast<const uint16_t*>(p.w);
  a.y = p.y + size_t(first) * (act ? p.N2 / 2 : p.N2);
  a.sx = p.sx + first;
  a.sw = p.sw;
  a.part = static_cast<float*>(part);
  a.T = T;
  a.H = p.H / 2;
  a.N2 = p.N2;
  if (way.mid) return launch_gateup_i8_mid(a, stream, ev_start, ev_stop);
  const hipError_t e = launch_choice<Int8>(a, c, act, stream, ev_start, ev_stop);
  return e != hipSuccess || c.splits == 1 ? e : launch_reduce<Int8>(a, act, c.splits, stream, ev_stop);
}

// A call's launches: its token rows in one, or the last ones in another one.
struct Ways {
  Way first, last;
  int32_t last_rows = 0;
  bool general = false;
};

// The rows past the last whole 64 in a launch of their own, where they would make a
// round of tiles for themselves (the sums are the same): 2,056 tokens x 11,008 x 2,048,
// a chunk with eight decode rows, with the quantiser 73 us instead of 78 (65 with the
// tiles of 128 x 128).
Ways choose_ways(const Int8Product& p, bool act, bool aligned, int max_splits, int cus) {
  Ways r;
  // whole 128-byte stages of 16-byte aligned rows, and at least two of them (the scales'
  // transfer); anything else in the general kernel
  r.general = !aligned || p.H % (2 * kBK) != 0 || p.H <= 2 * kBK;
  if (r.general) return r;
  r.first = choose_way(p.T, p, act, max_splits, cus);
  r.general = r.first.c.kernel == GateupChoice::kGeneral;
  const int32_t tail = p.T % kTailBM, main = p.T - tail;
  if (r.first.c.kernel != GateupChoice::kTiles || tail == 0 || main == 0) return r;
  // both parts' partial sums fit where the whole call's do
  const Way m = choose_way(main, p, act, max_splits, cus), t = choose_way(tail, p, act, 1, cus);
  if (m.c.kernel != GateupChoice::kGeneral && t.c.kernel != GateupChoice::kGeneral && m.cost + t.cost < 0.97 * r.first.cost) {
    r.first = m;
    r.last = t;
    r.last_rows = tail;
  }
  return r;
}

}  // namespace

hipError_t launch_gateup_i8(const Int8Product& p, bool act, int max_splits, void* part, int cus, hipStream_t stream,
                            hipEvent_t ev_start, hipEvent_t ev_stop) {
  if (p.T <= 0) return hipSuccess;
  if (max_splits < 1 || (max_splits > 1 && !part) || (act && p.N2 % 2 != 0)) return hipErrorInvalidValue;
  const bool aligned = reinterpret_cast<uintptr_t>(p.x) % 16 == 0 && reinterpret_cast<uintptr_t>(p.w) % 16 == 0;
  const Ways r = choose_ways(p, act, aligned, max_splits, cus);
  if (r.general) return launch_gateup_i8_any(p, act, stream, ev_start, ev_stop);
  if (r.last_rows == 0) return launch_rows_of(p, 0, p.T, r.first, act, part, stream, ev_start, ev_stop);
  const int32_t main = p.T - r.last_rows;
  const hipError_t e = launch_rows_of(p, 0, main, r.first, act, part, stream, ev_start, nullptr);
  return e != hipSuccess ? e : launch_rows_of(p, main, r.last_rows, r.last, act, part, stream, nullptr, ev_stop);
}

void gateup_i8_choice(int32_t T, int32_t H, int32_t N2, bool act, bool aligned, int max_splits, int cus, int32_t* choice) {
  const Ways r = choose_ways(Int8Product{nullptr, nullptr, nullptr, nullptr, nullptr, T, H, N2}, act, aligned, max_splits, cus);
  std::fill(choice, choice + 16, 0);
  auto put = [&](int32_t* to, const Way& w, int32_t rows) {
    const GateupChoice& c = w.c;
    const int32_t v[8] = {rows, w.mid ? 3 : int32_t(c.kernel), w.mid ? 128 : c.rows, w.mid ? 0 : c.main_m, w.mid ? 0 : c.tail_m,
                          w.mid ? 0 : c.g, w.mid ? 0 : c.wr, w.mid ? 1 : c.splits};
    std::copy(v, v + 8, to);
  };
  if (r.general) {
    choice[0] = T;
    choice[1] = GateupChoice::kGeneral;
    choice[7] = 1;
    return;
  }
  put(choice, r.first, T - r.last_rows);
  if (r.last_rows > 0) put(choice + 8, r.last, r.last_rows);
}

}  // namespace ppas
