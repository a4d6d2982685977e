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
//   out = y + (s v) B^T: s v is taken as two bf16 numbers, its rounding and the rest, so
//     that it keeps 16 bits where B's product needs bf16 operands (2^-17 of v; the second
//     instruction costs nothing beside the rows' bytes).
//
// What bounds them: x for the first, y in and out for the second at many rows (a rank of
// 16 is 64 operations per element of y); at few rows the adapters' weights, and at one the
// two launches.
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
  for (int64_t t = lo; t < hi; t += 64) {
    const bool valid = t + lane < hi;
    const int g = valid ? group_of(row_adapter[t + lane], o.n) : 0;
    const uint64_t same = same_group(g, valid);
    // the group's first lane counts for all
    if (valid && lane == int(__ffsll((unsigned long long)same)) - 1) count[wave][g] += int(__popcll(same));
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
  auto list = [&](AdapterTile* tiles, const int32_t* starts, int height) {
    for (int i = tid; i < starts[groups]; i += kSortThreads) {
      int g = 0;   // the last group that starts at or before tile i
      for (int d = 1024; d >= 1; d >>= 1)
        if (g + d < groups && starts[g + d] <= i) g += d;
      const int at = first[g] + (i - starts[g]) * height;
      tiles[i] = AdapterTile{g < o.n ? g : -1, at, min(height, first[g + 1] - at), 0};
    }
  };
  list(tiles16, first16, 16);
  list(tiles64, first64, 64);
  for (int64_t t = lo; t < hi; t += 64) {
    const bool valid = t + lane < hi;
    const int g = valid ? group_of(row_adapter[t + lane], o.n) : 0;
    const uint64_t same = same_group(g, valid);
    if (!valid) continue;
    const int before = int(__popcll(same & ((uint64_t(1) << lane) - 1)));
    const int base = count[wave][g];
    order[first[g] + base + before] = int32_t(t + lane);
    // behind every lane's read: a wave's accesses to LDS are in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (before == 0) count[wave][g] = base + int(__popcll(same));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
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
  int32_t blocks, block;      // of the outputs: `block` columns each
  bool rows_vec;              // y and out by 16 bytes
  bool in_place;
};

// The tile of a workgroup. What it says is checked against the call: an order that was
// made for another one reads and writes nothing past the call's rows.
__device__ __forceinline__ bool tile_of(const AdapterArgs& a, int64_t i, int height, AdapterTile& t) {
  const int64_t n = height == 16 ? a.head->tiles16 : a.head->tiles64;
  if (i >= min(n, a.slots)) return false;
  t = a.tiles[i];
  return t.adapter >= -1 && t.adapter < a.c.adapters && t.count >= 1 && t.count <= height && t.first >= 0 &&
         t.first <= a.c.T - t.count;
}
__device__ __forceinline__ int32_t row_of(const AdapterArgs& a, const AdapterTile& t, int local) {
  const int32_t r = a.order[t.first + min(local, t.count - 1)];   // rows past the tile's are its last one again
  return min(max(r, 0), a.c.T - 1);
}

// Eight elements of a row of n, from element k on: zeros past its end.
template <bool kVec>
__device__ __forceinline__ u32x4 eight(const uint16_t* row, int64_t k, int64_t n) {
  u32x4 v = {0, 0, 0, 0};
  if (kVec) {
    if (k < n) v = *reinterpret_cast<const u32x4*>(row + k);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k + e < n) v[e / 2] |= uint32_t(row[k + e]) << (16 * (e % 2));
  }
  return v;
}

// v = x A^T. A workgroup takes a tile of 16 MF rows, 16 RF ranks and a split of hidden; its
// waves take 64 features of every 256 and add up through LDS.
template <int MF, int RF, bool kVec>
__global__ __launch_bounds__(256) void adapter_down_kernel(AdapterArgs a) {
  constexpr int F = MF * RF, kBatch = F < 8 ? F : 8;
  __shared__ f32x4 sums[4][kBatch][64];
  const int64_t block = block_of();
  AdapterTile t;
  if (!tile_of(a, block / a.splits, 16 * MF, t) || t.adapter < 0) return;
  const int split = int(block % a.splits);
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, col = lane & 15, g = lane >> 4;
  const int64_t H = a.c.hidden;
  const uint16_t *x[MF], *w[RF];
#pragma unroll
  for (int m = 0; m < MF; ++m) x[m] = a.c.x + row_of(a, t, 16 * m + col) * a.c.x_stride;
#pragma unroll
  for (int r = 0; r < RF; ++r)
    w[r] = a.c.a + (int64_t(t.adapter) * a.c.rank + min(16 * r + col, a.c.rank - 1)) * H;
  f32x4 acc[MF][RF];
#pragma unroll
  for (int m = 0; m < MF; ++m)
#pragma unroll
    for (int r = 0; r < RF; ++r) acc[m][r] = Bf16::zero();
  const int64_t k1 = min(H, (int64_t(split) + 1) * a.per);
  for (int64_t k = int64_t(split) * a.per + 64 * wave; k < k1; k += 256) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t at = k + 32 * h + 8 * g;
      u32x4 fx[MF], fw[RF];
#pragma unroll
      for (int m = 0; m < MF; ++m) fx[m] = eight<kVec>(x[m], at, H);
#pragma unroll
      for (int r = 0; r < RF; ++r) fw[r] = eight<kVec>(w[r], at, H);
#pragma unroll
      for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int r = 0; r < RF; ++r) acc[m][r] = Bf16::mma(fw[r], fx[m], acc[m][r]);
    }
  }
  float* part = a.c.part + (int64_t(split) * a.c.T + t.first) * (16 * RF);
#pragma unroll
  for (int f0 = 0; f0 < F; f0 += kBatch) {
    if (f0) __syncthreads();
#pragma unroll
    for (int f = 0; f < kBatch; ++f) sums[wave][f][lane] = acc[(f0 + f) / RF][(f0 + f) % RF];
    __syncthreads();
    for (int f = wave; f < kBatch; f += 4) {
      f32x4 s = sums[0][f][lane];
#pragma unroll
      for (int i = 1; i < 4; ++i) s += sums[i][f][lane];
      const int row = 16 * ((f0 + f) / RF) + col;
      if (row < t.count)
        *reinterpret_cast<f32x4*>(part + int64_t(row) * (16 * RF) + 16 * ((f0 + f) % RF) + 4 * g) = s;
    }
  }
}

// Two bf16 numbers that are a float but for 2^-17 of it: its rounding, and that of the rest
// (0 where the first is not finite).
__device__ __forceinline__ void halves(const float (&v)[8], u32x4& hi, u32x4& lo) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    hi[w] = pack_bf16x2(v[2 * w], v[2 * w + 1]);
    float rest[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float top = __uint_as_float(e ? hi[w] & 0xffff0000u : hi[w] << 16);
      rest[e] = fabsf(top) < __builtin_inff() ? v[2 * w + e] - top : 0.f;
    }
    lo[w] = pack_bf16x2(rest[0], rest[1]);
  }
}

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Columns n .. n + 7 of a row, and those of an output (elements past `lim`: zeros, and not
// stored).
__device__ __forceinline__ u32x4 row_load(const uint16_t* row, int n, int lim, bool vec) {
  if (vec && n + 8 <= lim) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + n));
  return eight<false>(row, n, lim);
}
__device__ __forceinline__ void row_store(uint16_t* row, int n, int lim, bool vec, u32x4 p) {
  if (vec && n + 8 <= lim) {
    __builtin_nontemporal_store(p, reinterpret_cast<u32x4*>(row + n));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (n + e < lim) row[n + e] = uint16_t(p[e / 2] >> (16 * (e % 2)));
  }
}

// out = y + (s v) B^T. A workgroup takes a tile of 16 MF rows and a block of columns; a wave
// 32 kPairs columns at a time (kAct: half of them gate, half up of the same features). The
// rows of B go to the matrix instructions in an order that leaves a lane with eight columns
// of one row, 16 bytes of y. Up to rank 16 (RS = 0) one instruction takes both numbers of
// s v against the same B; else RS of 32 ranks each take B once for two.
template <int MF, int RS, bool kVec, bool kAct>
__global__ __launch_bounds__(256) void adapter_up_kernel(AdapterArgs a) {
  constexpr int S = RS ? RS : 1, kParts = RS ? 2 : 1;
  constexpr int kPairs = MF * S >= 16 && !kAct ? 1 : 2;
  constexpr int kStep = kAct ? 16 * kPairs : 32 * kPairs;   // columns of out
  const int64_t block = block_of();
  AdapterTile t;
  if (!tile_of(a, block / a.blocks, 16 * MF, t)) return;
  if (t.adapter < 0 && a.in_place) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, col = lane & 15, g = lane >> 4;
  const int R = a.c.rank, half = a.c.n_out / 2, lim = kAct ? half : a.c.n_out;
  const int n0 = int(block % a.blocks) * a.block, n1 = min(n0 + a.block, lim);
  const uint16_t* y[MF];
  uint16_t* out[MF];
#pragma unroll
  for (int m = 0; m < MF; ++m) {
    const int64_t row = row_of(a, t, 16 * m + col);
    y[m] = a.c.y + row * a.c.y_stride;
    out[m] = a.c.out + row * a.c.out_stride;
  }
  u32x4 v[MF][S][kParts];
  const uint16_t* b = nullptr;
  if (t.adapter >= 0) {
    b = a.c.b + int64_t(t.adapter) * a.c.n_out * R;
    const float scale = a.c.scale ? a.c.scale[t.adapter] : 1.f;
    constexpr int kPitch = RS ? 32 * RS : 16;
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int r0 = RS ? 32 * s + 8 * g : 8 * (g & 1);
        const float* p = a.c.part + (int64_t(t.first) + min(16 * m + col, t.count - 1)) * kPitch + r0;
        f32x4 sum[2] = {};
        for (int i = 0; i < a.splits; ++i) {
#pragma unroll
          for (int h = 0; h < 2; ++h) sum[h] += *reinterpret_cast<const f32x4*>(p + int64_t(i) * a.c.T * kPitch + 4 * h);
        }
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = r0 + e < R ? scale * sum[e / 4][e % 4] : 0.f;
        u32x4 hi, lo;
        halves(f, hi, lo);
        if (RS) {
          v[m][s][0] = hi;
          v[m][s][kParts - 1] = lo;
        } else {
          v[m][s][0] = g < 2 ? hi : lo;
        }
      }
  }
  // the column of frag q of a pair that this lane brings: lane group c / 4 gets eight of them
  const int brings = 8 * (col >> 2) + (col & 3);
  for (int n = n0 + wave * kStep; n < n1; n += 4 * kStep) {
    u32x4 old[MF][kPairs];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
      for (int p = 0; p < kPairs; ++p) {
        // with the activation a pair is the gate columns, the next the up columns of the same features
        const int at = n + (kAct ? 32 * (p / 2) : 32 * p) + 8 * g;
        const uint16_t* row = kAct && p % 2 ? y[m] + half : y[m];
        old[m][p] = row_load(row, at, lim, a.rows_vec);
      }
    f32x4 acc[MF][kPairs][2];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
      for (int p = 0; p < kPairs; ++p) acc[m][p][0] = acc[m][p][1] = Bf16::zero();
    if (t.adapter >= 0) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int r0 = RS ? 32 * s + 8 * g : 8 * (g & 1);
        u32x4 fb[kPairs][2];
#pragma unroll
        for (int p = 0; p < kPairs; ++p)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int c = min(n + (kAct ? 32 * (p / 2) : 32 * p) + brings + 4 * q, lim - 1);
            fb[p][q] = eight<kVec>(b + int64_t(kAct && p % 2 ? c + half : c) * R, r0, R);
          }
#pragma unroll
        for (int m = 0; m < MF; ++m)
#pragma unroll
          for (int p = 0; p < kPairs; ++p)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int i = 0; i < kParts; ++i) acc[m][p][q] = Bf16::mma(fb[p][q], v[m][s][i], acc[m][p][q]);
      }
    }
#pragma unroll
    for (int m = 0; m < MF; ++m) {
      if (16 * m + col >= t.count) continue;
#pragma unroll
      for (int p = 0; p < kPairs; p += kAct ? 2 : 1) {
        const int at = n + (kAct ? 32 * (p / 2) : 32 * p) + 8 * g;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t w = old[m][p][e / 2];
          f[e] = (e % 2 ? hi_f(w) : lo_f(w)) + acc[m][p][e / 4][e % 4];
          if (kAct) {
            const uint32_t u = old[m][p + 1 < kPairs ? p + 1 : p][e / 2];
            f[e] = silu_f32(f[e]) * ((e % 2 ? hi_f(u) : lo_f(u)) + acc[m][p + 1 < kPairs ? p + 1 : p][e / 4][e % 4]);
          }
        }
        u32x4 v8 = old[m][p];   // a row of no adapter is copied bit for bit
        if (kAct || t.adapter >= 0) {
#pragma unroll
          for (int w = 0; w < 4; ++w) v8[w] = pack_bf16x2(f[2 * w], f[2 * w + 1]);
        }
        row_store(out[m], at, n1, a.rows_vec, v8);
      }
    }
  }
}

bool on16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Rows per tile: 64 where an adapter has 32 or more on average.
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

template <int MF, int RS, bool kAct>
void launch_up(const AdapterArgs& a, bool vec, dim3 grid, hipStream_t stream, hipEvent_t ev_stop) {
  if (vec)
    hipExtLaunchKernelGGL((adapter_up_kernel<MF, RS, true, kAct>), grid, dim3(256), 0, stream, nullptr, ev_stop, 0, a);
  else
    hipExtLaunchKernelGGL((adapter_up_kernel<MF, RS, false, kAct>), grid, dim3(256), 0, stream, nullptr, ev_stop, 0, a);
}

template <int MF>
void launch_both(AdapterArgs& a, bool act, bool down_vec, bool up_vec, hipStream_t stream, hipEvent_t ev_start,
                 hipEvent_t ev_stop) {
  const dim3 down = grid_of(a.slots * a.splits), up = grid_of(a.slots * a.blocks);
  switch (rank_frags(a.c.rank)) {
    case 1: launch_down<MF, 1>(a, down_vec, down, stream, ev_start); break;
    case 2: launch_down<MF, 2>(a, down_vec, down, stream, ev_start); break;
    case 4: launch_down<MF, 4>(a, down_vec, down, stream, ev_start); break;
    default: launch_down<MF, 8>(a, down_vec, down, stream, ev_start);
  }
  switch (rank_frags(a.c.rank) + (act ? 16 : 0)) {
    case 1: launch_up<MF, 0, false>(a, up_vec, up, stream, ev_stop); break;
    case 2: launch_up<MF, 1, false>(a, up_vec, up, stream, ev_stop); break;
    case 4: launch_up<MF, 2, false>(a, up_vec, up, stream, ev_stop); break;
    case 8: launch_up<MF, 4, false>(a, up_vec, up, stream, ev_stop); break;
    case 17: launch_up<MF, 0, true>(a, up_vec, up, stream, ev_stop); break;
    case 18: launch_up<MF, 1, true>(a, up_vec, up, stream, ev_stop); break;
    case 20: launch_up<MF, 2, true>(a, up_vec, up, stream, ev_stop); break;
    default: launch_up<MF, 4, true>(a, up_vec, up, stream, ev_stop);
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

// About two workgroups per compute unit, each of 256 features at least.
int adapter_splits(int32_t T, int32_t hidden, int32_t adapters, int cus) {
  const int64_t tiles = AdapterOrder{T, adapters}.slots(tile_height(T, adapters));
  const int64_t most = std::min<int64_t>(16, (int64_t(hidden) + 255) / 256);
  return int(std::max<int64_t>(1, std::min<int64_t>(most, 2 * int64_t(cus) / tiles)));
}

size_t adapter_workspace_bytes(int32_t T, int32_t hidden, int32_t rank, int32_t adapters, int cus) {
  return size_t(adapter_splits(T, hidden, adapters, cus)) * size_t(T) * size_t(16 * rank_frags(rank)) * sizeof(float);
}

hipError_t launch_adapters(const AdapterCall& c, bool act, int cus, hipStream_t stream, hipEvent_t ev_start,
                           hipEvent_t ev_stop) {
  if (c.T <= 0) return hipSuccess;
  if (c.rank < 1 || c.rank > kAdapterMaxRank || c.adapters < 1 || c.adapters > kAdaptersMax) return hipErrorInvalidValue;
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
  a.splits = adapter_splits(c.T, c.hidden, c.adapters, cus);
  a.per = int32_t(((int64_t(c.hidden) + a.splits - 1) / a.splits + 255) / 256 * 256);
  // blocks of columns: about eight workgroups per compute unit, 256 columns at least
  const int32_t cols = act ? c.n_out / 2 : c.n_out;
  const int64_t want = std::max<int64_t>(1, 8 * int64_t(cus) / a.slots);
  a.block = int32_t(std::max<int64_t>(256, ((int64_t(cols) + want - 1) / want + 255) / 256 * 256));
  a.blocks = int32_t((int64_t(cols) + a.block - 1) / a.block);
  a.rows_vec = on16(c.y) && on16(c.out) && c.y_stride % 8 == 0 && c.out_stride % 8 == 0 && (!act || cols % 8 == 0);
  a.in_place = !act && c.y == c.out && c.y_stride == c.out_stride;
  const bool down_vec = on16(c.x) && on16(c.a) && c.x_stride % 8 == 0 && c.hidden % 8 == 0;
  const bool up_vec = on16(c.b) && c.rank % 8 == 0;
  if (height == 16) launch_both<1>(a, act, down_vec, up_vec, stream, ev_start, ev_stop);
  else launch_both<4>(a, act, down_vec, up_vec, stream, ev_start, ev_stop);
  return hipGetLastError();
}

}  // namespace ppas
