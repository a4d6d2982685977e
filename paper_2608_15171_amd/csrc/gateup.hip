// Fused gate-up projection of a decoder block's MLP on gfx950 (CDNA4):
//   Y[T][N2] = X[T][H] * W[N2][H]^T
// bf16 inputs, fp32 accumulation on 16x16x32 MFMAs, output rounded to bf16
// (nearest even). W stacks the gate rows over the up rows, so one launch
// computes both projections of a prefill chunk. Here: the choice of kernel and the
// bf16 calls; the kernels are in gateup_kernels.h.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "device.h"
#include "gateup_kernels.h"

namespace ppas {

namespace {

// How a call is tiled and split.
struct Shape {
  int bm = 0;               // main tiles of 256 or 128 rows; 64: small tiles only
  int splits = 1;
  int32_t main_m = 0, tail_m = 0, light = 0;
  int64_t items = 0;
  double cost = 0;
};

// Microseconds of one stage and, beside the stages, of one tile, by tile rows; of
// the reducing launch, for each split (its chain of loads), and of its partial sums'
// bytes; and the share by which a full chip slows every stage. Fitted to 520 timed
// calls (64 to 8,200 tokens, the decoder layer's four projections, every tile shape
// and split; 8 % rms), over which the choice made with them is 0.8 % slower than the
// best one on average. kWeightBytes, the rate that the weights come in no faster than,
// and kReduceSplit (more rows hide the chain) belong to the fit at rows_cost.
constexpr double kStage256 = 0.92, kStage128 = 0.66, kStage64 = 0.53;
constexpr double kTile256 = 5.3, kTile128 = 1.4, kTile64 = 0.4;
// 64-row tiles of 8-bit rows, in 128-feature stages (3,400 timed calls of 15 projections, 1 to
// 4,100 tokens; with kRowsInt the choice is 0.7 % slower than the best on average)
constexpr double kStage64Int = 0.48, kTile64Int = 1.5;
constexpr double kReduce = 4.25, kReduceSplit = 0.12, kPartBytes = 5.5e6, kLoaded = 0.186, kWeightBytes = 9.45e6;

constexpr int kRowsMaxT = 256;   // the few-row kernel measured up to here; from about 64 rows the tiles win on wide outputs
// 8-bit rows: measured up to here (154 calls of 200 to 1,500 tokens, where the model's choice
// is 1.3 % slower than the best on average; without the few-row kernel above 256 it was
// 19 %: 512 tokens x 4,096 x 512 15.7 us instead of 7.7)
constexpr int kRowsMaxTInt = 1536;

Shape shape_cost(int32_t T, int32_t H, int32_t N2, int grid_max, int bm, int splits, bool int_sums) {
  Shape s;
  s.bm = bm;
  s.splits = splits;
  const int64_t tiles_n = (N2 + kBN - 1) / kBN;
  s.main_m = bm == kTailBM ? 0 : T / bm;
  const int64_t rest = T - int64_t(s.main_m) * bm;
  s.tail_m = int32_t((rest + kTailBM - 1) / kTailBM);
  const int64_t nf = s.main_m * tiles_n * splits, ns = s.tail_m * tiles_n * splits;
  s.items = nf + ns;
  const double nk = double(H / kBK) / splits;
  const double cf = bm == 256 ? nk * kStage256 + kTile256 : nk * kStage128 + kTile128;
  const double cs = int_sums ? nk * kStage64Int + kTile64Int : nk * kStage64 + kTile64;
  s.light = std::max(0, int(cf / cs));
  const int64_t grid = std::min<int64_t>(s.items, grid_max);
  const int64_t rem = nf % grid, light = grid - rem;
  const int64_t in_light = std::min<int64_t>(ns, s.light * light);
  const int64_t extra = (ns - in_light + grid - 1) / grid;
  const double t_light = double(nf / grid) * cf + double((in_light + light - 1) / light + extra) * cs;
  const double t_heavy = rem ? double(nf / grid + 1) * cf + double(extra) * cs : 0;
  s.cost = std::max(std::max(t_light, t_heavy) * (1 + kLoaded * std::min(1.0, double(s.items) / grid_max)),
                    2.0 * N2 * H / kWeightBytes);
  if (splits > 1) s.cost += kReduce + (T <= kRowsMaxT ? kReduceSplit * splits : 0) + 2.0 * splits * double(T) * N2 * 4 / kPartBytes;
  return s;
}

// The few-row kernel's variants: weight-row tiles per workgroup and their rows.
// One eight-row tile doubles the workgroups where the columns are few.
struct RowsShape {
  int g, wr;
  bool with_act, without;
};
constexpr RowsShape kRowsShapes[] = {{1, 8, false, true}, {1, 16, false, true}, {2, 8, true, false},
                                     {2, 16, true, true}, {4, 16, true, true},  {6, 16, true, true}};

// Microseconds: the weights stream at 8 TB/s over the chip or 56 GB/s into one compute
// unit, X (from L2) at 99 GB/s, one after the other; every round of resident workgroups
// takes 2.8 us to fill; the rest is the launch and the final sums. Where variants come
// out alike, more workgroups of fewer weight-row tiles have more loads in flight: 8,192
// x 8,192 with one token 30.0 us in one tile against 32.9 in two. Fitted with
// kTilesBase, the launches of a call of the tile kernels, to 14,500 timed calls (60
// projections, 1 to 1,000 tokens, every variant, the weights from memory: none is read
// again before 640 MB of others; 15 % rms, the tiles 14 %). The choice is then 1.5 %
// slower than the best on average. Constants fitted to weights that a repeated call
// finds in the 256 MB cache made it 3.6 %, and some calls slower than one tile kernel
// for all sizes had been: 11,008 x 512 with 48 tokens 24.2 us where that one takes 22.3
// (now 18.9), 16,384 x 8,192 with 16 tokens 82.4 against 73.8 (now 65.2).
constexpr double kTilesBase = 4.64;
struct RowsCost {
  double base, cu, chip, x, result, fill, tile;   // microseconds, or bytes per microsecond
};
constexpr RowsCost kRowsBf16{2.9, 5.57e4, 8.0e6, 9.93e4, 0.02, 2.84, 0.01};
constexpr RowsCost kRowsInt{0.91, 12.9e4, 12.3e6, 9.04e4, 0.11, 2.18, 0.11};
double rows_cost(int32_t T, int32_t H, int32_t N2, int cus, const RowsShape& v, const RowsCost& k) {
  const int xt = rows_tokens(T) / 16;
  const double cols = double((int64_t(N2) + v.g * v.wr - 1) / (v.g * v.wr));
  const double mt = (T + 16 * xt - 1) / (16 * xt);
  const int slot = (v.g * v.wr + 16 * xt) * kRow;
  const int ring = 4 * slot * std::min(4, kSmem / 4 / slot);
  const int per_cu = std::max(1, kSmem / std::max(ring, 4 * v.g * xt * 1024));
  const double wgs = cols * mt, room = double(cus) * per_cu;
  const double rounds = wgs > room ? std::ceil(wgs / room) * per_cu : std::max(1.0, wgs / cus);
  const double w = 2.0 * v.g * v.wr * H, x = 2.0 * T / mt * H;
  const double cost = k.base + std::max(rounds * w / k.cu, mt * 2.0 * N2 * H / k.chip) + rounds * x / k.x +
                      k.result * v.g * xt + k.fill * std::ceil(wgs / room);
  return cost * (1 + k.tile * (v.g - 1));
}

}  // namespace

int64_t gateup_tiles(int32_t T, int32_t N2) {
  return (int64_t(T / 256) + (T % 256 + kTailBM - 1) / kTailBM) * ((N2 + kBN - 1) / kBN);
}

int gateup_splits(int32_t T, int32_t H, int32_t N2, int cus) {
  const int64_t tiles = gateup_tiles(T, N2);
  const int nk = H / kBK;
  if (tiles <= 0 || tiles >= cus) return 1;
  // about one workgroup per compute unit, each with at least four stages
  return int(std::max<int64_t>(1, std::min<int64_t>(cus / tiles, nk / 4)));
}

size_t gateup_workspace_bytes(int32_t T, int32_t N2, int splits) {
  return splits > 1 ? size_t(splits) * size_t(T) * size_t(N2) * sizeof(float) : 0;
}

GateupChoice gateup_choose(int32_t T, int32_t H, int32_t N2, bool act, bool aligned, int max_splits, int cus,
                           bool int_sums) {
  GateupChoice r;
  r.splits = max_splits;
  // The transfers need 16-byte aligned rows and 32-bit offsets within a unit.
  if (!aligned || int64_t(H) * 2 >= kMaxPitch) return r;
  // one workgroup per compute unit (a multiple of 8, so that each stays on one XCD's
  // share of the tiles)
  const int grid_max = std::max(8, cus / 8 * 8);
  // Narrow outputs (the K and V projections, whose results are cached) are summed in
  // 256-feature blocks added in order, where the hidden size is up to eight whole such
  // blocks: by blocks of four stages, or by a split into exactly these blocks. The
  // result then does not depend on the number of tokens beside it or on the workspace.
  // Other outputs, longer narrow ones among them, take the cheapest split: 2,056 x 4,096
  // x 512 takes 41.6 us unsplit, 24.0 us in three splits.
  // Integer sums are the same in any order, and bound by none of this.
  const bool narrow = !int_sums && !act && N2 <= 2 * kBN && H % (4 * kBK) == 0 && H <= 8 * 4 * kBK;
  // A choice of fewer splits than allowed makes no fp32 chain longer than the most
  // splits would (`longest` stages): 256-row tiles, which keep one chain, take them all,
  // and the others sum by blocks of four stages where eight would be longer.
  const int longest = (H / kBK + max_splits - 1) / max_splits;
  Shape best;
  for (int bm : {256, 128, 64}) {
    if (bm > kTailBM && T < bm) continue;   // no tile of that height
    for (int s = 1; s <= max_splits; ++s) {
      if (bm == 256 && s < max_splits && !int_sums) continue;
      if (narrow && ((s > 1 && s * 4 * kBK != H) || bm == 256)) continue;
      const Shape c = shape_cost(T, H, N2, grid_max, bm, s, int_sums);
      if (c.items > INT32_MAX / 2) continue;
      if (best.bm == 0 || c.cost < best.cost) best = c;
    }
  }
  if (best.bm == 0) return r;
  r.kernel = GateupChoice::kTiles;
  r.rows = best.bm;
  r.splits = best.splits;
  r.main_m = best.main_m;
  r.tail_m = best.tail_m;
  r.light = best.light;
  r.grid = int32_t(std::min<int64_t>(best.items, grid_max));
  r.block = narrow || longest < 8 ? 4 : 8;
  double cost = best.cost + kTilesBase;
  r.cost = cost;
  if (T > (int_sums ? kRowsMaxTInt : kRowsMaxT)) return r;
  for (const RowsShape& v : kRowsShapes) {
    if (!(act ? v.with_act : v.without) || N2 / (v.g * v.wr) >= (1 << 22) || (narrow && v.g > 1)) continue;
    const double c = rows_cost(T, H, N2, grid_max, v, int_sums ? kRowsInt : kRowsBf16);
    if (c < cost) {
      r.cost = cost = c;
      r.kernel = GateupChoice::kRows;
      r.rows = rows_tokens(T);
      r.splits = 1;
      r.g = v.g;
      r.wr = v.wr;
    }
  }
  return r;
}

hipError_t launch_gateup(const uint16_t* x, const uint16_t* w, uint16_t* y, int32_t T, int32_t H, int32_t N2,
                         bool act, int max_splits, float* part, int cus, hipStream_t stream, hipEvent_t ev_start,
                         hipEvent_t ev_stop) {
  if (T <= 0) return hipSuccess;
  if (max_splits < 1 || max_splits > H / kBK || (max_splits > 1 && !part) || (act && N2 % 2 != 0))
    return hipErrorInvalidValue;
  const bool aligned = reinterpret_cast<uintptr_t>(x) % 16 == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0;
  const GateupChoice c = gateup_choose(T, H, N2, act, aligned, max_splits, cus, false);
  GemmArgs a{};
  a.x = x;
  a.w = w;
  a.y = y;
  a.part = part;
  a.T = T;
  a.H = H;
  a.N2 = N2;
  const hipError_t e = c.kernel == GateupChoice::kGeneral
                           ? launch_gateup_any(x, w, y, T, H, N2, act, c.splits, part, cus, stream, ev_start,
                                               c.splits > 1 ? nullptr : ev_stop)
                           : launch_choice<Bf16>(a, c, act, stream, ev_start, ev_stop);
  return e != hipSuccess || c.splits == 1 ? e : launch_reduce<Bf16>(a, act, c.splits, stream, ev_stop);
}

}  // namespace ppas
