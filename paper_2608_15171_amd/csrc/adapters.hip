// Low-rank adapters of many requests beside a shared projection.
//
// Row t with adapter a gets, on top of the projection's y[t],
//   s_a (x[t] A_a^T) B_a^T,  A_a [r][H], B_a [N][r],
// rounded once with the sum to bf16; with the activation silu(g) u of the sum's halves is
// rounded instead. Rows of one adapter lie anywhere in a step: a small kernel sorts their
// numbers by adapter once per step (a stable counting sort), and tiles of up to 16 or 64
// rows of one adapter are what the two products work on:
//   v = x A^T, fp32 (bf16 matrix instructions, x and A straight from memory in operand
//     order), split over hidden where tiles are few;
//   out = y + (s v) B^T: s v is taken as three bf16 numbers, each the rounding of what the
//     ones before leave, so that it keeps its 24 bits where B's product needs bf16 operands
//     (the further instructions cost next to nothing beside the rows' bytes).
//
// What bounds them: x for the first, y in and out for the second at many rows (a rank of
// 16 is 64 operations per element of y); at few rows the adapters' weights, and at one the
// two launches. Measured: 16,384 rows of rank 64 from 2,048 features onto 22,016 308-311 us, 4.9
// TB/s (the second product 293-308, a copy of as many bytes 288); 2,056 of rank 32 with the
// activation 50.5 (136 MB in 43-46: waves wait for their rows 65 % of the time, and of 1,131
// workgroups a compute unit holds four, so that a tenth of them start when others end); 64
// decode rows with 24 adapters 13.4, one row 8.2 behind its order's 3.6. Orders of 16,384
// rows take 29 us where they lie in runs of one adapter, up to 374 where 1,024 adapters mix.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "adapters.h"
#include "gateup_device.h"
#include "grid.h"

namespace ppas {
namespace {

// ---------------------------------------------------------------------------
// The order: a stable counting sort by one workgroup, whose waves take consecutive
// stretches of the rows. Counts by wave and adapter, their sums, then every row's place.
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;

__device__ __forceinline__ int group_of(int32_t adapter, int n) { return adapter >= 0 && adapter < n ? adapter : n; }

// Lanes of the wave with the same group as this one.
__device__ __forceinline__ uint64_t same_group(int group, bool valid) {
  uint64_t left = __ballot(valid), mine = 0;
  while (left) {
    const int first = int(__ffsll((unsigned long long)left)) - 1;
    const uint64_t b = __ballot(valid && group == __builtin_amdgcn_readlane(group, first));
    if ((b >> (threadIdx.x & 63)) & 1) mine = b;
    left &= ~b;
  }
  return mine;
}

__device__ __forceinline__ int wave_prefix(int v) {   // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

__global__ __launch_bounds__(kSortThreads) void adapter_rows_kernel(const int32_t* row_adapter, AdapterOrder o,
                                                                    AdapterHeader* head, AdapterTile* tiles16,
                                                                    AdapterTile* tiles64, int32_t* order) {
  __shared__ int32_t count[kSortWaves][kAdaptersMax + 1];   // then the next place of each
  __shared__ int32_t first[kAdaptersMax + 2], first16[kAdaptersMax + 2], first64[kAdaptersMax + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid / 64, groups = o.n + 1;
  for (int i = tid; i < kSortWaves * groups; i += kSortThreads) count[i / groups][i % groups] = 0;
  __syncthreads();
  const int32_t per = (o.T + kSortThreads - 1) / kSortThreads * 64;   // rows of a wave, whole steps
  const int64_t lo = int64_t(wave) * per, hi = min(lo + per, int64_t(o.T));
  // a step's groups and their lanes; a wave's first step keeps them for its rows' places
  struct Step {
    int g;
    uint64_t same;
    bool valid;
  };
  auto look = [&](int64_t t) {
    Step s;
    s.valid = t + lane < hi;
    s.g = s.valid ? group_of(row_adapter[t + lane], o.n) : 0;
    s.same = same_group(s.g, s.valid);
    return s;
  };
  const Step kept = look(lo);
  for (int64_t t = lo; t < hi; t += 64) {
    const Step s = t == lo ? kept : look(t);
    // the group's first lane counts for all
    if (s.valid && lane == int(__ffsll((unsigned long long)s.same)) - 1) count[wave][s.g] += int(__popcll(s.same));
  }
  __syncthreads();
  for (int g = tid; g < groups; g += kSortThreads) {
    int sum = 0;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = count[w][g];
      count[w][g] = sum;
      sum += c;
    }
    first[g] = sum;
  }
  __syncthreads();
  if (wave == 0) {
    int at = 0, at16 = 0, at64 = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
      const int g = g0 + lane, c = g < groups ? first[g] : 0;
      const int n = wave_prefix(c), n16 = wave_prefix((c + 15) / 16), n64 = wave_prefix((c + 63) / 64);
      if (g < groups) {
        first[g] = at + n - c;
        first16[g] = at16 + n16 - (c + 15) / 16;
        first64[g] = at64 + n64 - (c + 63) / 64;
      }
      at += __shfl(n, 63);
      at16 += __shfl(n16, 63);
      at64 += __shfl(n64, 63);
    }
    if (lane == 0) {
      first[groups] = at;
      first16[groups] = at16;
      first64[groups] = at64;
      *head = AdapterHeader{at16, at64, 0, 0};
    }
  }
  __syncthreads();
  for (int64_t t = lo; t < hi; t += 64) {
    const Step s = t == lo ? kept : look(t);
    if (!s.valid) continue;
    const int before = int(__popcll(s.same & ((uint64_t(1) << lane) - 1)));
    const int base = count[wave][s.g];
    // (inside the order also if someone changes the rows' adapters meanwhile)
    order[min(first[s.g] + base + before, o.T - 1)] = int32_t(t + lane);
    // behind every lane's read: a wave's accesses to LDS are in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (before == 0) count[wave][s.g] = base + int(__popcll(s.same));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  __syncthreads();   // the order is read below
  auto list = [&](AdapterTile* tiles, const int32_t* starts, int height) {
    for (int i = tid; i < starts[groups]; i += kSortThreads) {
      int g = 0;   // the last group that starts at or before tile i
      for (int d = 1024; d >= 1; d >>= 1)
        if (g + d < groups && starts[g + d] <= i) g += d;
      const int at = first[g] + (i - starts[g]) * height, n = min(height, first[g + 1] - at);
      const int32_t row = order[at], last = order[at + n - 1];
      tiles[i] = AdapterTile{g < o.n ? g : -1, at, n, last - row == n - 1 ? row : -1};
    }
  };
  list(tiles16, first16, 16);
  list(tiles64, first64, 64);
}

// ---------------------------------------------------------------------------
// The products
// ---------------------------------------------------------------------------
struct AdapterArgs {
  AdapterCall c;
  const AdapterHeader* head;
  const AdapterTile* tiles;
  const int32_t* order;
  int64_t slots;              // of the tile list
  int32_t splits, per;        // of hidden: per features each, a multiple of 256
  int32_t parts;              // of a tile that are workgroups of their own in the first product
  int32_t blocks, block;      // of the outputs: `block` columns each
  bool in_place;
};

// The tile of a workgroup. What it says is checked against the call: an order that was
// made for another one reads and writes nothing past the call's rows.
__device__ __forceinline__ bool tile_of(const AdapterArgs& a, int64_t i, int height, AdapterTile& t) {
  const int64_t n = height == 16 ? a.head->tiles16 : a.head->tiles64;   // both asked for at once
  t = a.tiles[min(i, a.slots - 1)];
  return i < min(n, a.slots) && t.adapter >= -1 && t.adapter < a.c.adapters && t.count >= 1 && t.count <= height &&
         t.first >= 0 && t.first <= a.c.T - t.count && t.row >= -1 && t.row <= a.c.T - t.count;
}
__device__ __forceinline__ int32_t row_of(const AdapterArgs& a, const AdapterTile& t, int local) {
  const int at = min(local, t.count - 1);   // rows past the tile's are its last one again
  return min(max(t.row >= 0 ? t.row + at : a.order[t.first + at], 0), a.c.T - 1);
}

// Sixteen bytes from any element on: global memory needs no alignment, and rows of odd lengths
// and strides are as fast as others but for the lines that they cross (5,933
// rows onto 3,247 columns, rank 32, 56 us, element by element 92; 6,181 onto 9,235, rank 114, 206 and 469).
typedef u32x4 AnyVec __attribute__((aligned(2)));

// Eight elements of a row of n, from element k on: zeros past its end. kVec: n is a multiple of 8.
template <bool kVec>
__device__ __forceinline__ u32x4 eight(const uint16_t* row, int64_t k, int64_t n) {
  u32x4 v = {0, 0, 0, 0};
  if (kVec ? k < n : k + 8 <= n) {
    v = *reinterpret_cast<const AnyVec*>(row + k);
  } else if (!kVec && k < n) {
    uint32_t one[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) one[e] = row[min(k + e, n - 1)];   // all at once
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e < n) v[e / 2] |= one[e] << (16 * (e % 2));
  }
  return v;
}

// LDS that the lanes of one wave exchange: in order as it is, but not for the compiler.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Both products bring their operands as 16-byte pieces of whole 128-byte lines, eight lanes
// to a row, and turn them into operand order in LDS, as they turn the share into the order
// of y's memory. Straight in the order of the matrix instructions, 64 bytes of a row at a
// time, 16,384 rows of rank 64 onto 22,016 columns took 754 us where this takes 310.

// v = x A^T. A workgroup takes a tile of 16 MF rows (half of one of 64), 16 RF ranks and a
// split of hidden; its waves take 64 features of every 256 and add up through LDS. Each wave
// for itself, without a barrier on the way; whole tiles of 64 rows leave a compute unit one
// workgroup (16,384 rows of rank 64: 21 us either way, 700 rows of 11,008: 9.4 against 8.2).
constexpr int kDownPitch = 72;   // elements of a row of 64 in LDS: 16 rows' reads spread over the banks

template <int MF, int RF, bool kVec>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterArgs a) {
  constexpr int F = MF * RF, kBatch = F < 8 ? F : 8, kRows = 16 * (MF + RF), kLoads = kRows / 8;
  constexpr int kStage = 4 * kRows * kDownPitch * 2, kSums = 4 * kBatch * 64 * 16;
  __shared__ __attribute__((aligned(16))) char smem[kStage > kSums ? kStage : kSums];
  const int64_t block = block_of();
  AdapterTile t;
  // a tile of the list is `parts` of the workgroup's rows
  const int64_t which = block / a.splits;
  if (!tile_of(a, which / a.parts, 16 * MF * a.parts, t) || t.adapter < 0) return;
  const int skip = int(which % a.parts) * 16 * MF;
  if (skip >= t.count) return;
  t.first += skip;
  t.count = min(t.count - skip, 16 * MF);
  if (t.row >= 0) t.row += skip;
  const int split = int(block % a.splits);
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, col = lane & 15, g = lane >> 4;
  const int64_t H = a.c.hidden;
  uint16_t* stage = reinterpret_cast<uint16_t*>(smem) + wave * kRows * kDownPitch;
  // the lane's rows: the tile's of x, then the adapter's of A; those past either's end are zeros
  const int piece = 8 * (lane % 8);
  const uint16_t* src[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int row = 8 * j + lane / 8, rank = row - 16 * MF;
    if (j < 2 * MF) src[j] = row < t.count ? a.c.x + row_of(a, t, row) * a.c.x_stride + piece : nullptr;
    else src[j] = rank < a.c.rank ? a.c.a + (int64_t(t.adapter) * a.c.rank + rank) * H + piece : nullptr;
  }
  f32x4 acc[MF][RF];
#pragma unroll
  for (int m = 0; m < MF; ++m)
#pragma unroll
    for (int r = 0; r < RF; ++r) acc[m][r] = Bf16::zero();
  const int64_t k1 = min(H, (int64_t(split) + 1) * a.per);
  u32x4 raw[kLoads];
  auto bring = [&](int64_t k) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      raw[j] = u32x4{0, 0, 0, 0};
      if (src[j]) raw[j] = eight<kVec>(src[j], k, H - piece);
    }
  };
  int64_t k = int64_t(split) * a.per + 64 * wave;
  if (k < k1) bring(k);
  for (; k < k1; k += 256) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      *reinterpret_cast<u32x4*>(stage + (8 * j + lane / 8) * kDownPitch + piece) = raw[j];
    wave_fence();
    if (k + 256 < k1) bring(k + 256);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 fx[MF], fw[RF];
      const uint16_t* at = stage + col * kDownPitch + 32 * h + 8 * g;
#pragma unroll
      for (int m = 0; m < MF; ++m) fx[m] = *reinterpret_cast<const u32x4*>(at + 16 * m * kDownPitch);
#pragma unroll
      for (int r = 0; r < RF; ++r) fw[r] = *reinterpret_cast<const u32x4*>(at + 16 * (MF + r) * kDownPitch);
#pragma unroll
      for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int r = 0; r < RF; ++r) acc[m][r] = Bf16::mma(fw[r], fx[m], acc[m][r]);
    }
    wave_fence();
  }
  f32x4* sums = reinterpret_cast<f32x4*>(smem);   // [4][kBatch][64]
  float* part = a.c.part + (int64_t(split) * a.c.T + t.first) * (16 * RF);
#pragma unroll
  for (int f0 = 0; f0 < F; f0 += kBatch) {
    __syncthreads();
#pragma unroll
    for (int f = 0; f < kBatch; ++f) sums[(wave * kBatch + f) * 64 + lane] = acc[(f0 + f) / RF][(f0 + f) % RF];
    __syncthreads();
    for (int f = wave; f < kBatch; f += 4) {
      f32x4 s = sums[f * 64 + lane];
#pragma unroll
      for (int i = 1; i < 4; ++i) s += sums[(i * kBatch + f) * 64 + lane];
      const int row = 16 * ((f0 + f) / RF) + col;
      if (row < t.count)
        *reinterpret_cast<f32x4*>(part + int64_t(row) * (16 * RF) + 16 * ((f0 + f) % RF) + 4 * g) = s;
    }
  }
}

// Three bf16 numbers whose sum is a float: its rounding, that of the rest, and the last
// eight bits (0 and 0 where the first is not finite). Two alone leave 2^-17 of it, which
// changes the rounding of one result in some thousands against the sum in fp32.
__device__ __forceinline__ void thirds(const float (&v)[8], u32x4 (&p)[3]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    float rest[2] = {v[2 * w], v[2 * w + 1]};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      p[i][w] = pack_bf16x2(rest[0], rest[1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float top = __uint_as_float(e ? p[i][w] & 0xffff0000u : p[i][w] << 16);
        rest[e] = fabsf(top) < __builtin_inff() ? rest[e] - top : 0.f;
      }
    }
  }
}

// g / (1 + e^-g) by t = e^-|g|, whose denominator is within [1, 2]: a reciprocal of one unit
// in the last place instead of a division's eleven instructions. t's exponent is split into a
// whole number and the rest, which is taken with log2 e in two parts (Cody and Waite): as one
// fp32 number it is off by up to 2^-18 at |g| = 80, which were 29 units of 2^-24 in results.
// Past 150, t is 0 either way.
__device__ __forceinline__ float silu(float g) {
  const float a = fminf(fabsf(g), 150.f), n = rintf(a * -1.44269504f);
  const float f = fmaf(a, -1.9259629911266175e-8f, fmaf(a, -1.44269502162933349609375f, -n));
  const float t = ldexpf(__builtin_amdgcn_exp2f(f), int(n));
  const float r = g * __builtin_amdgcn_rcpf(1.f + t);
  return g < 0.f ? r * t : r;
}

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Columns n .. n + 7 of a row, and those of an output (elements past `lim`: zeros, and not
// stored).
__device__ __forceinline__ u32x4 row_load(const uint16_t* row, int n, int lim) {
  if (n + 8 <= lim) return __builtin_nontemporal_load(reinterpret_cast<const AnyVec*>(row + n));
  u32x4 v = {0, 0, 0, 0};   // one by one: the end of a row is not worth the registers of eight loads
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (n + e < lim) v[e / 2] |= uint32_t(row[n + e]) << (16 * (e % 2));
  return v;
}
__device__ __forceinline__ void row_store(uint16_t* row, int n, int lim, u32x4 p) {
  if (n + 8 <= lim) {
    __builtin_nontemporal_store(p, reinterpret_cast<AnyVec*>(row + n));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (n + e < lim) row[n + e] = uint16_t(p[e / 2] >> (16 * (e % 2)));
  }
}

// out = y + (s v) B^T. A workgroup takes a tile and a block of columns; a wave 16 rows and 64
// columns at a time: of a tile of 64 rows each wave its own rows and all the same columns,
// whose rows of B they share in LDS (kWide; of up to 32 ranks two steps in turn, with one
// barrier each); of a tile of 16 each wave its own columns and B. The share goes through LDS into the order of
// memory, 128 bytes of a row to eight lanes. With the activation a step is 64 gate columns
// and the up columns of the same features. Up to rank 16 (RS = 0) one instruction takes two
// of the three numbers of s v against the same B; else RS of 32 ranks each take B once for three.
// Loads come back in the order in which they were asked for: the first step's B and y before
// the share's sums, then a step's y and its B behind the results of the step before.
constexpr int kSharePitch = 68;   // floats of a row of 64 in LDS

// A barrier that waits for this wave's LDS accesses, but not for its loads and stores.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
  bare_barrier();
}

// Waves of a SIMD that the compiler has to leave registers for: one more than it does by itself
// where the three numbers' 24 or 48 registers would cost a wave (16,384 rows of rank 64 319 us
// without, 308 with; 8,192 of rank 128 onto 22,016 columns 268 and 252). Nothing spills.
constexpr int up_waves(bool wide, int RS, bool vec, bool act) {
  return wide && vec && !act ? (RS == 2 ? 5 : RS == 4 ? 4 : 1) : 1;
}

template <bool kWide, int RS, bool kVec, bool kAct>
__global__ __launch_bounds__(256, up_waves(kWide, RS, kVec, kAct)) void adapter_up_kernel(AdapterArgs a) {
  constexpr int S = RS ? RS : 1, kParts = RS ? 3 : 2, kHalves = kAct ? 2 : 1;
  constexpr int kChunks = RS ? 4 * RS : 2;      // of eight ranks, in a row of B
  constexpr int kPitch = 8 * kChunks + 8;       // elements of such a row in LDS
  // shared B of more ranks leaves too few workgroups with two buffers (us with two and one: 2,023
  // rows, rank 128 with the activation 99 and 70, 64 81 and 66; 16,384 of rank 64 318 and 310)
  constexpr bool kTwice = RS < 2;
  constexpr int kBufs = kWide ? (kTwice ? 2 : 1) : 4, kStep = kWide ? 64 : 256;
  constexpr int kThreads = kWide ? 256 : 64, kItems = kHalves * 64 * kChunks;
  constexpr int kLoads = (kItems + kThreads - 1) / kThreads;
  // a wave's own B is in registers before its share takes its place
  constexpr bool kOver = !kWide && !kAct;
  constexpr int kB = kHalves * 64 * kPitch, kShare = 16 * kSharePitch * 2;
  constexpr int kBPitch = kOver && kB < kShare ? kShare : kB;   // of a buffer of B
  __shared__ __attribute__((aligned(16))) uint16_t b_stage[kBufs][kBPitch];
  __shared__ __attribute__((aligned(16))) float share_stage[kOver ? 1 : 4][kOver ? 4 : 16 * kSharePitch];
  const int64_t block = block_of();
  AdapterTile t;
  if (!tile_of(a, block / a.blocks, kWide ? 64 : 16, t)) return;
  if (t.adapter < 0 && a.in_place) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, col = lane & 15, g = lane >> 4;
  const int R = a.c.rank, half = a.c.n_out / 2, lim = kAct ? half : a.c.n_out;
  const int first = int(block % a.blocks) * a.block, n1 = min(first + a.block, lim);
  const int n0 = kWide ? first : first + 64 * wave;
  const int wave_row = kWide ? 16 * wave : 0, count = t.count - wave_row;   // of this wave, maybe none
  float* ss = kOver ? reinterpret_cast<float*>(b_stage[wave]) : share_stage[kOver ? 0 : wave];
  // the lane's two rows and eight columns
  const int sub = lane / 8, at = 8 * (lane % 8);
  int32_t rows[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) rows[i] = row_of(a, t, wave_row + 8 * i + sub);
  const uint16_t* b = t.adapter < 0 ? nullptr : a.c.b + int64_t(t.adapter) * a.c.n_out * R;
  const int item0 = kWide ? int(threadIdx.x) : lane;
  u32x4 raw[kLoads];
  auto bring = [&](int n) {   // B of the step's columns
    if (!b) return;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = item0 + j * kThreads, c = n + i / kChunks % 64, up = kAct && i >= kItems / 2 ? half : 0;
      raw[j] = u32x4{0, 0, 0, 0};
      if (i < kItems && c < lim) raw[j] = eight<kVec>(b + int64_t(c + up) * R, 8 * (i % kChunks), R);
    }
  };
  auto stage = [&](int buf) {
    if (!b) return;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = item0 + j * kThreads;
      if (i < kItems) *reinterpret_cast<u32x4*>(&b_stage[buf][i / kChunks * kPitch + 8 * (i % kChunks)]) = raw[j];
    }
  };
  u32x4 old[2][kHalves];
  auto fetch = [&](int i, int n) {
    if (8 * i + sub >= count || n + at >= lim) return;
    const uint16_t* y = a.c.y + rows[i] * a.c.y_stride;
    old[i][0] = row_load(y, n + at, lim);
    if (kAct) old[i][kHalves - 1] = row_load(y + half, n + at, lim);
  };
  if (n0 < n1) bring(n0);
#pragma unroll
  for (int i = 0; i < 2; ++i) fetch(i, n0);
  u32x4 v[S][kParts];
  if (b) {
    const float scale = a.c.scale ? a.c.scale[t.adapter] : 1.f;
    constexpr int kPart = RS ? 32 * RS : 16;
    // several splits' loads at once (no difference measured at 323 rows of 5,504, rank 128: 23.4
    // us, and one split after the other as long)
    constexpr int kAtOnce = S == 1 ? 8 : S == 2 ? 4 : 2;
    const float* p0 = a.c.part + (int64_t(t.first) + min(wave_row + col, t.count - 1)) * kPart;
    const int64_t next = int64_t(a.c.T) * kPart;
    f32x4 sum[S][2] = {};
    for (int i0 = 0; i0 < a.splits; i0 += kAtOnce) {
      f32x4 some[kAtOnce][S][2];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            some[i][s][h] = *reinterpret_cast<const f32x4*>(p0 + min(i0 + i, a.splits - 1) * next +
                                                            (RS ? 32 * s + 8 * g : 8 * (g & 1)) + 4 * h);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (i0 + i >= a.splits) break;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int h = 0; h < 2; ++h) sum[s][h] += some[i][s][h];
      }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int r0 = RS ? 32 * s + 8 * g : 8 * (g & 1);
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = r0 + e < R ? scale * sum[s][e / 4][e % 4] : 0.f;
      u32x4 p[3];
      thirds(f, p);
      if (RS) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) v[s][i] = p[i];
      } else {
        v[s][0] = g < 2 ? p[0] : p[1];
        v[s][1] = g < 2 ? p[2] : u32x4{0, 0, 0, 0};
      }
    }
  }
  int buf = kWide ? 0 : wave;
  if (kWide) {
    stage(0);
    if (n0 + kStep < n1) bring(n0 + kStep);
    lds_barrier();
  }
  for (int n = n0; n < n1; n += kStep) {
    if (!kWide) {
      stage(buf);
      wave_fence();
      if (n + kStep < n1) bring(n + kStep);
    }
    if (count > 0) {
      float f[kHalves][2][8];
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        if (b) {
          f32x4 acc[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[q] = Bf16::zero();
#pragma unroll
          for (int s = 0; s < S; ++s)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const u32x4 fb = *reinterpret_cast<const u32x4*>(
                  &b_stage[buf][(64 * h + 16 * q + col) * kPitch + (RS ? 32 * s + 8 * g : 8 * (g & 1))]);
#pragma unroll
              for (int i = 0; i < kParts; ++i) acc[q] = Bf16::mma(fb, v[s][i], acc[q]);
            }
          wave_fence();
#pragma unroll
          for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4*>(ss + col * kSharePitch + 16 * q + 4 * g) = acc[q];
          wave_fence();
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 8; e += 4) {
            f32x4 d = {};
            if (b) d = *reinterpret_cast<const f32x4*>(ss + (8 * i + sub) * kSharePitch + at + e);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t w = old[i][h][(e + j) / 2];
              f[h][i][e + j] = (j % 2 ? hi_f(w) : lo_f(w)) + d[j];
            }
          }
        wave_fence();
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u32x4 done = old[i][0];   // a row of no adapter is copied bit for bit
        if (kAct || b) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            float x0 = f[0][i][2 * w], x1 = f[0][i][2 * w + 1];
            if (kAct) {
              x0 = silu(x0) * f[kHalves - 1][i][2 * w];
              x1 = silu(x1) * f[kHalves - 1][i][2 * w + 1];
            }
            done[w] = pack_bf16x2(x0, x1);
          }
        }
        if (8 * i + sub < count) row_store(a.c.out + rows[i] * a.c.out_stride, n + at, n1, done);
        if (n + kStep < n1) fetch(i, n + kStep);
      }
    }
    if (kWide && b) {
      if (kTwice) buf ^= 1;
      else lds_barrier();
      if (n + kStep < n1) stage(buf);
      if (n + 2 * kStep < n1) bring(n + 2 * kStep);
      lds_barrier();
    }
  }
}

// Rows per tile: 64 where an adapter has 32 or more on average, by the adapters that the set
// holds: the host does not know which of them a step uses. Few in use of a large set go by 16
// rows where 64 would do (16,384 rows of rank 64 on one adapter of 1,024 442 us, of four 310).
int tile_height(int32_t T, int32_t adapters) { return T / adapters >= 32 ? 64 : 16; }

// Frags of 16 ranks that the first product computes: 1, 2, 4 or 8.
int rank_frags(int32_t rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8; }

template <int MF, int RF>
void launch_down(const AdapterArgs& a, bool vec, dim3 grid, hipStream_t stream, hipEvent_t ev_start) {
  if (vec)
    hipExtLaunchKernelGGL((adapter_down_kernel<MF, RF, true>), grid, dim3(256), 0, stream, ev_start, nullptr, 0, a);
  else
    hipExtLaunchKernelGGL((adapter_down_kernel<MF, RF, false>), grid, dim3(256), 0, stream, ev_start, nullptr, 0, a);
}

template <bool kWide, int RS, bool kAct>
void launch_up(const AdapterArgs& a, bool vec, dim3 grid, hipStream_t stream, hipEvent_t ev_stop) {
  if (vec)
    hipExtLaunchKernelGGL((adapter_up_kernel<kWide, RS, true, kAct>), grid, dim3(256), 0, stream, nullptr, ev_stop, 0, a);
  else
    hipExtLaunchKernelGGL((adapter_up_kernel<kWide, RS, false, kAct>), grid, dim3(256), 0, stream, nullptr, ev_stop, 0, a);
}

template <bool kWide>
void launch_both(AdapterArgs& a, bool act, bool down_vec, bool up_vec, hipStream_t stream, hipEvent_t ev_start,
                 hipEvent_t ev_stop) {
  constexpr int MF = kWide ? 2 : 1;   // rows of the first product's workgroups, in 16: tiles of 64 as two of them
  a.parts = kWide ? 4 / MF : 1;
  const dim3 down = grid_of(a.slots * a.parts * a.splits), up = grid_of(a.slots * a.blocks);
  switch (rank_frags(a.c.rank)) {
    case 1: launch_down<MF, 1>(a, down_vec, down, stream, ev_start); break;
    case 2: launch_down<MF, 2>(a, down_vec, down, stream, ev_start); break;
    case 4: launch_down<MF, 4>(a, down_vec, down, stream, ev_start); break;
    default: launch_down<MF, 8>(a, down_vec, down, stream, ev_start);
  }
  switch (rank_frags(a.c.rank) + (act ? 16 : 0)) {
    case 1: launch_up<kWide, 0, false>(a, up_vec, up, stream, ev_stop); break;
    case 2: launch_up<kWide, 1, false>(a, up_vec, up, stream, ev_stop); break;
    case 4: launch_up<kWide, 2, false>(a, up_vec, up, stream, ev_stop); break;
    case 8: launch_up<kWide, 4, false>(a, up_vec, up, stream, ev_stop); break;
    case 17: launch_up<kWide, 0, true>(a, up_vec, up, stream, ev_stop); break;
    case 18: launch_up<kWide, 1, true>(a, up_vec, up, stream, ev_stop); break;
    case 20: launch_up<kWide, 2, true>(a, up_vec, up, stream, ev_stop); break;
    default: launch_up<kWide, 4, true>(a, up_vec, up, stream, ev_stop);
  }
}

}  // namespace

hipError_t launch_adapter_rows(const int32_t* row_adapter, AdapterOrder o, void* rows, hipStream_t stream,
                               hipEvent_t ev_start, hipEvent_t ev_stop) {
  if (o.T <= 0) return hipSuccess;
  if (o.n < 1 || o.n > kAdaptersMax) return hipErrorInvalidValue;
  auto* head = static_cast<AdapterHeader*>(rows);
  auto* tiles16 = reinterpret_cast<AdapterTile*>(head + 1);
  auto* tiles64 = tiles16 + o.slots16();
  hipExtLaunchKernelGGL(adapter_rows_kernel, dim3(1), dim3(kSortThreads), 0, stream, ev_start, ev_stop, 0, row_adapter,
                        o, head, tiles16, tiles64, reinterpret_cast<int32_t*>(tiles64 + o.slots64()));
  return hipGetLastError();
}

// About two workgroups per compute unit, each of 512 features at least, eight splits at most:
// every workgroup of the second product adds them up (155 rows of 11,008, rank 64: 17.8 us with
// up to 8, 19.9 with 16, 22.4 with 24; 700 of rank 8 15.2, 17.2, 19.0; 2,056 of 2,048 features,
// rank 32, 50.1 with 4, 53.9 with 8).
int adapter_splits(int32_t T, int32_t hidden, int32_t adapters, int cus) {
  const int64_t tiles = AdapterOrder{T, adapters}.slots(tile_height(T, adapters));
  const int64_t most = std::min<int64_t>(8, (int64_t(hidden) + 511) / 512);
  return int(std::max<int64_t>(1, std::min<int64_t>(most, 2 * int64_t(cus) / tiles)));
}

size_t adapter_workspace_bytes(int32_t T, int32_t rank, int splits) {
  return size_t(splits) * size_t(T) * size_t(16 * rank_frags(rank)) * sizeof(float);
}

hipError_t launch_adapters(const AdapterCall& c, bool act, int cus, hipStream_t stream, hipEvent_t ev_start,
                           hipEvent_t ev_stop) {
  if (c.T <= 0) return hipSuccess;
  if (c.rank < 1 || c.rank > kAdapterMaxRank || c.adapters < 1 || c.adapters > kAdaptersMax || c.splits < 1)
    return hipErrorInvalidValue;
  const AdapterOrder o{c.T, c.adapters};
  const int height = tile_height(c.T, c.adapters);
  AdapterArgs a;
  a.c = c;
  a.head = static_cast<const AdapterHeader*>(c.rows);
  const auto* tiles16 = reinterpret_cast<const AdapterTile*>(a.head + 1);
  const auto* tiles64 = tiles16 + o.slots16();
  a.tiles = height == 16 ? tiles16 : tiles64;
  a.order = reinterpret_cast<const int32_t*>(tiles64 + o.slots64());
  a.slots = o.slots(height);
  a.splits = c.splits;
  a.per = int32_t(((int64_t(c.hidden) + a.splits - 1) / a.splits + 255) / 256 * 256);
  // blocks of columns: whole steps, about four workgroups per compute unit where that leaves
  // as many, up to 512 columns (256 of a small rank, whose B and share cost a start less):
  // when the rest was not yet what it is, 2,056 rows with the activation took 71 us a step of
  // 64 at a time, 53 at 512, 76 at 1,024; 16,384 of rank 64 439, 315 and 336; 56 decode rows
  // 17.4 at 256, 13.7 at 512
  const int32_t cols = act ? c.n_out / 2 : c.n_out, step = height == 16 ? 256 : 64;
  const int64_t each = int64_t(cols) * a.slots / (4 * int64_t(cus)) / step * step;
  // more where the start reads more than four such steps' rows of partial sums, but one
  // workgroup per compute unit (2,023 rows of 11,008 features onto 2,048 columns, rank 64: 41.3 and 36.0)
  const int64_t start = int64_t(a.splits) * 16 * rank_frags(c.rank) / 4;
  const int64_t least = std::min<int64_t>(start, int64_t(cols) * a.slots / cus) / step * step;
  a.block = int32_t(std::min<int64_t>(std::max<int64_t>({step, each, least}), height == 64 && c.rank <= 16 ? 256 : 512));
  a.blocks = int32_t((int64_t(cols) + a.block - 1) / a.block);
  a.in_place = !act && c.y == c.out && c.y_stride == c.out_stride;
  const bool down_vec = c.hidden % 8 == 0, up_vec = c.rank % 8 == 0;
  if (height == 16) launch_both<false>(a, act, down_vec, up_vec, stream, ev_start, ev_stop);
  else launch_both<true>(a, act, down_vec, up_vec, stream, ev_start, ev_stop);
  return hipGetLastError();
}

}  // namespace ppas
