// Rotary positions of rows of heads, and of a step's rows on their way into the
// paged cache.
//
// Pair j of a head, at position p, turns by t = p w_j (w_j: the frequency table
// that the host makes, with its scaling for long contexts), and both results are
// multiplied by a magnitude m:
//   a' = m (a cos t - b sin t),  b' = m (b cos t + a sin t).
// A pair is (j, j + R/2) in the half layout and (2j, 2j + 1) in the interleaved
// one; features from R on are copied, whatever they hold. The transposed turn
// (gradients; for m = 1 the inverse) takes -t.
//
// Angles are reduced in fp64 (whole turns removed: fp32 would lose 1e-2 radians at
// 100,000 positions), cos and sin are taken in fp32, the turn is fp32 and rounded
// once to bf16 nearest-even.
//
// What bounds them: memory, at 4 bytes per feature. A workgroup takes a few rows
// (or a page's slots), computes their cos/sin once into LDS for all heads, and
// has its first loads in flight meanwhile. A task is a group of pairs whose
// features are read and written by one thread only, so that the turn may be done
// in place: two 16-byte runs of eight pairs in the half layout, one run of four
// pairs in the interleaved one, and a single pair where the sizes or the
// alignment allow no 16-byte runs.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "grid.h"
#include "rope.h"

namespace ppas {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

enum Mode : int { kHalf = 0, kInterleaved = 1, kPair = 2 };

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
// Every byte is used once, so loads and stores ask the caches not to keep it: 16,384
// rows of 18 heads from memory take 27.6 us with both, 31.5 with the loads alone, 37.7
// with neither (a copy of as many bytes 29.7).
__device__ __forceinline__ u32x4 load16(const uint16_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}
__device__ __forceinline__ void store16(uint16_t* p, u32x4 v) {
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ float turn_a(float a, float b, float2 c) { return fmaf(a, c.x, -(b * c.y)); }
__device__ __forceinline__ float turn_b(float a, float b, float2 c) { return fmaf(b, c.x, a * c.y); }

// cos and sin of a position's turn of one pair, times the magnitude.
__device__ __forceinline__ float2 cos_sin(double position, double turns, float magnitude, bool transposed) {
  const double t = position * turns;
  const float ang = float((t - rint(t)) * (2.0 * M_PI));   // in [-pi, pi]
  float sn, cn;
  sincosf(ang, &sn, &cn);
  return make_float2(cn * magnitude, (transposed ? -sn : sn) * magnitude);
}

// A head as tasks ("units"). `half` is the layout in kPair mode.
struct Head {
  int dim, pairs;
  bool half;
};

template <int kMode>
__device__ __forceinline__ int first_feature(const Head& h, int u) {
  if (kMode == kHalf) return u < h.pairs / 8 ? 8 * u : h.pairs + 8 * u;   // copies: 2 pairs + 8 (u - pairs / 8)
  if (kMode == kInterleaved) return 8 * u;
  return u < h.pairs && h.half ? u : 2 * u;
}
// the second run of a rotated unit (kInterleaved: none)
template <int kMode>
__device__ __forceinline__ int second_feature(const Head& h, int u) {
  if (kMode == kHalf) return h.pairs + 8 * u;
  return u < h.pairs && h.half ? u + h.pairs : 2 * u + 1;
}

struct Unit {
  u32x4 x, y;
};

template <int kMode>
__device__ __forceinline__ Unit fetch(const uint16_t* src, const Head& h, int u) {
  Unit r;
  if (kMode == kPair) {
    r.x[0] = src[first_feature<kMode>(h, u)];
    r.y[0] = src[second_feature<kMode>(h, u)];
  } else {
    r.x = load16(src + first_feature<kMode>(h, u));
    if (kMode == kHalf) {
      if (u < h.pairs / 8) r.y = load16(src + second_feature<kMode>(h, u));
    }
  }
  return r;
}

// Turns a unit and stores it; dst(f) is the address of feature f (eight features
// from a multiple of 8 on follow each other).
template <int kMode, typename Dst>
__device__ __forceinline__ void put(Unit r, const Head& h, int u, const float2* cs, Dst dst) {
  if (kMode == kPair) {
    uint16_t *p = dst(first_feature<kMode>(h, u)), *q = dst(second_feature<kMode>(h, u));
    if (u < h.pairs) {
      const float a = lo_f(r.x[0]), b = lo_f(r.y[0]);
      const uint32_t v = pack2(turn_a(a, b, cs[u]), turn_b(a, b, cs[u]));
      r.x[0] = v & 0xffffu;
      r.y[0] = v >> 16;
    }
    *p = uint16_t(r.x[0]);
    *q = uint16_t(r.y[0]);
    return;
  }
  if (kMode == kHalf) {
    if (u < h.pairs / 8) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2 c0 = cs[8 * u + 2 * w], c1 = cs[8 * u + 2 * w + 1];
        const float x0 = lo_f(r.x[w]), x1 = hi_f(r.x[w]), y0 = lo_f(r.y[w]), y1 = hi_f(r.y[w]);
        r.x[w] = pack2(turn_a(x0, y0, c0), turn_a(x1, y1, c1));
        r.y[w] = pack2(turn_b(x0, y0, c0), turn_b(x1, y1, c1));
      }
      store16(dst(second_feature<kMode>(h, u)), r.y);
    }
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int j = 4 * u + w;
      if (j < h.pairs) {
        const float2 c = cs[j];
        const float a = lo_f(r.x[w]), b = hi_f(r.x[w]);
        r.x[w] = pack2(turn_a(a, b, c), turn_b(a, b, c));
      }
    }
  }
  store16(dst(first_feature<kMode>(h, u)), r.x);
}

// Units of a head; where nothing is copied (in place), those that turn.
template <int kMode>
__device__ __forceinline__ int units_of(const Head& h, bool copies) {
  if (kMode == kHalf) return h.pairs / 8 + (copies ? (h.dim - 2 * h.pairs) / 8 : 0);
  if (kMode == kInterleaved) return copies ? h.dim / 8 : (2 * h.pairs + 7) / 8;
  return copies ? h.dim / 2 : h.pairs;
}

constexpr int kThreads = 256;
constexpr int kAhead = 4;   // units a thread has in flight

// Every (row, head, unit) of n_rows rows; a thread keeps its unit and steps through the
// heads without a division (two per task were a third of the kernel's instructions).
// `ready` is called once, behind the first loads, and makes the table cs[row][pair].
template <int kMode, typename Src, typename Dst, typename Ready>
__device__ __forceinline__ void turn_rows(int n_rows, int heads, const Head& h, bool copies, const float2* cs, Src src,
                                          Dst dst, Ready ready) {
  const int units = units_of<kMode>(h, copies), step = kThreads / units;   // at most 128 units
  const int unit = int(threadIdx.x) % units, start = int(threadIdx.x) / units;
  const int step_row = step / heads, step_head = step % heads;
  // threads past the last whole head have no rows
  int row = start < step ? start / heads : n_rows, head = start % heads;
  bool first = true;
  while (first || row < n_rows) {
    Unit r[kAhead];
    int rows[kAhead], at_head[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      rows[i] = row;
      at_head[i] = head;
      if (row < n_rows) r[i] = fetch<kMode>(src(row, head), h, unit);
      row += step_row;
      head += step_head;
      if (head >= heads) {
        head -= heads;
        ++row;
      }
    }
    if (first) {
      ready();
      __syncthreads();
      first = false;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (rows[i] >= n_rows) continue;
      uint16_t* base = dst(rows[i], at_head[i]);
      put<kMode>(r[i], h, unit, cs + rows[i] * h.pairs, [&](int f) { return base + f; });
    }
  }
}

// ---------------------------------------------------------------------------
// Rows at given positions
// ---------------------------------------------------------------------------
constexpr int kMaxRows = 16;   // rows of a workgroup

struct RowsArgs {
  RopeRows r;
  RopeTable t;
  int32_t per;   // rows of a workgroup
};

template <int kMode>
__global__ __launch_bounds__(kThreads) void rope_rows_kernel(RowsArgs a) {
  __shared__ float2 cs[kMaxRows * kRopeMaxPairs];
  const int64_t row0 = block_of() * a.per;
  if (row0 >= a.r.rows) return;
  const int n = int(min(int64_t(a.per), a.r.rows - row0));
  const Head h{a.r.head_dim, a.t.pairs, a.t.layout == PPAS_ROPE_HALF};
  turn_rows<kMode>(
      n, a.r.heads, h, a.r.x != a.r.y, cs,
      [&](int row, int head) { return a.r.x + (row0 + row) * a.r.x_stride + int64_t(head) * a.r.head_dim; },
      [&](int row, int head) { return a.r.y + (row0 + row) * a.r.y_stride + int64_t(head) * a.r.head_dim; },
      [&]() {
        for (int e = threadIdx.x; e < n * h.pairs; e += kThreads) {
          const int row = e / h.pairs, j = e % h.pairs;
          cs[e] = cos_sin(double(a.r.positions[row0 + row]), a.t.turns[j], a.t.magnitude, a.r.transposed);
        }
      });
}

// ---------------------------------------------------------------------------
// A step's rows on their way into the pages. Workgroup (item, y) of a (request,
// touched page): for y = 0 the keys and values of its slots, so that a page's stores
// are whole runs (256 bytes of a key chunk's 16 slots, 32 of a value feature's), else
// the queries of slots 4 (y - 1) .. + 3. Each is one batch of loads, all in flight
// while its cos/sin are computed.
//
// Steps of few requests bring their descriptors in the kernel's arguments: the page
// list in host memory costs every workgroup a read over the bus before its first load
// (16,384 rows: 5 of 40 us).
// ---------------------------------------------------------------------------
constexpr int kSlots = 4;                     // query slots of a workgroup
constexpr int kParts = kPage / kSlots + 1;    // workgroups of a page
static_assert(int64_t(kAppendMaxItems) * kThreads < int64_t(1) << 32, "one grid dimension");
static_assert(kThreads == 2 * kHeadDim && kThreads == 16 * kPage, "one value task and one 16-byte run per thread");

struct AppendArgs {
  RopeAppend r;
  bool v_aligned;   // rows of v start on 16 bytes
  int32_t layout, pairs;
  float magnitude;
  double turns[kHeadDim / 2];
  AppendDesc desc[kAppendInline];
};

// The descriptors are sorted by their first item: item i is of the last one at or before it.
__device__ __forceinline__ AppendItem inline_item(const AppendArgs& a, int item) {
  const int lane = threadIdx.x & 63;
  const bool before = lane < a.r.n_desc && a.desc[lane].first_item <= item;
  const int s = int(__popcll(__ballot(before))) - 1;
  const AppendDesc d = a.desc[__builtin_amdgcn_readfirstlane(s)];
  return AppendItem{s, d.cached_len / kPage + item - d.first_item, d.cached_len, d.n_query, d.query_start, 0, 0, 0};
}

template <int kMode>
__global__ __launch_bounds__(kThreads) void rope_qkv_append_kernel(AppendArgs a) {
  __shared__ float2 cs[kPage * kHeadDim / 2];
  const RopeAppend& r = a.r;
  const AppendItem it = r.n_desc > 0 ? inline_item(a, blockIdx.x) : r.items[blockIdx.x];
  const int tid = threadIdx.x, part = blockIdx.y;
  const int pos_lo = it.lpage * kPage;   // position of slot 0
  int slot_lo = max(it.cached_len - pos_lo, 0), slot_hi = min(it.cached_len + it.n_query - pos_lo, kPage);
  if (part > 0) {
    slot_lo = max(slot_lo, (part - 1) * kSlots);
    slot_hi = min(slot_hi, part * kSlots);
    if (slot_lo >= slot_hi) return;
  }
  const int n = slot_hi - slot_lo;
  const int64_t row0 = int64_t(it.query_start) + (pos_lo + slot_lo - it.cached_len);   // the first slot's row
  const Head h{kHeadDim, a.pairs, a.layout == PPAS_ROPE_HALF};
  auto table = [&]() {
    for (int e = tid; e < n * h.pairs; e += kThreads) {
      const int row = e / h.pairs, j = e % h.pairs;
      cs[e] = cos_sin(double(pos_lo + slot_lo + row), a.turns[j], a.magnitude, false);
    }
  };
  if (part > 0) {
    turn_rows<kMode>(
        n, r.hq, h, r.q != r.q_out, cs,
        [&](int row, int head) { return r.q + (row0 + row) * r.q_stride + head * kHeadDim; },
        [&](int row, int head) { return r.q_out + ((row0 + row) * r.hq + head) * kHeadDim; }, table);
    return;
  }

  const int32_t page = r.bt[int64_t(it.seq) * r.bt_stride + it.lpage];
  // Keys: task (head, unit, slot), slot fastest; a thread's first ones are fetched ahead.
  const int units = units_of<kMode>(h, true), k_tasks = r.hkv * units * n;
  Unit key[2];
  auto fetch_key = [&](int t) {
    return fetch<kMode>(r.k + (row0 + t % n) * r.k_stride + t / (n * units) * kHeadDim, h, (t / n) % units);
  };
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (tid + i * kThreads < k_tasks) key[i] = fetch_key(tid + i * kThreads);
  // Values, transposed through LDS a head at a time: rows in by 16 bytes (or one element),
  // then per task (feature, eight slots) one 16-byte store where all eight are new.
  __shared__ __attribute__((aligned(16))) uint16_t rows[kPage][kHeadDim + 8];
  u32x4 v = {};
  auto fetch_value = [&](int g) {
    if (a.v_aligned && tid < n * 16) v = load16(r.v + (row0 + tid / 16) * r.v_stride + g * kHeadDim + 8 * (tid % 16));
  };
  fetch_value(0);
  table();
  __syncthreads();
  auto put_key = [&](const Unit& x, int t) {
    const int s = t % n, u = (t / n) % units, g = t / (n * units);
    uint16_t* dst = r.k_pages + (int64_t(page) * r.hkv + g) * kPage * kHeadDim + (slot_lo + s) * 8;
    put<kMode>(x, h, u, cs + s * h.pairs, [&](int f) { return dst + (f >> 3) * (kPage * 8) + (f & 7); });
  };
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (tid + i * kThreads < k_tasks) put_key(key[i], tid + i * kThreads);
  for (int t = tid + 2 * kThreads; t < k_tasks; t += kThreads) put_key(fetch_key(t), t);

  for (int g = 0; g < r.hkv; ++g) {
    if (a.v_aligned) {
      if (tid < n * 16) *reinterpret_cast<u32x4*>(&rows[slot_lo + tid / 16][8 * (tid % 16)]) = v;
    } else {
      const uint16_t* src = r.v + row0 * r.v_stride + g * kHeadDim;
      for (int t = tid; t < n * kHeadDim; t += kThreads)
        rows[slot_lo + t / kHeadDim][t % kHeadDim] = src[t / kHeadDim * r.v_stride + t % kHeadDim];
    }
    __syncthreads();
    if (g + 1 < r.hkv) fetch_value(g + 1);
    const int d = tid / 2, s0 = 8 * (tid & 1), lo = max(slot_lo - s0, 0), hi = min(slot_hi - s0, 8);
    uint16_t* dst = r.v_pages + (int64_t(page) * r.hkv + g) * kPage * kHeadDim + d * kPage + s0;
    if (hi - lo == 8) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = uint32_t(rows[s0 + 2 * e][d]) | (uint32_t(rows[s0 + 2 * e + 1][d]) << 16);
      store16(dst, w);
    } else {
      for (int e = lo; e < hi; ++e) dst[e] = rows[s0 + e][d];
    }
    __syncthreads();
  }
}

// 16-byte runs need every run's start on 16 bytes: bases, row strides, heads, and in
// the half layout the second half.
Mode mode_of(const RopeTable& t, int32_t head_dim, bool aligned) {
  if (!aligned || head_dim % 8 != 0) return kPair;
  if (t.layout == PPAS_ROPE_INTERLEAVED) return kInterleaved;
  return t.pairs % 8 == 0 ? kHalf : kPair;
}

bool on16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

hipError_t launch_rope_rows(const RopeRows& r, const RopeTable& t, hipStream_t stream, hipEvent_t ev_start,
                            hipEvent_t ev_stop) {
  if (r.rows <= 0) return hipSuccess;
  RowsArgs a;
  a.r = r;
  a.t = t;
  // one batch of loads per thread, but at least about four workgroups per compute unit
  const int64_t units = int64_t(r.heads) * std::max(1, t.layout == PPAS_ROPE_HALF ? t.pairs / 8 : r.head_dim / 8);
  a.per = int32_t(std::max<int64_t>(1, std::min<int64_t>({kMaxRows, r.rows / 1024, kThreads * kAhead / units})));
  const dim3 grid = grid_of((int64_t(r.rows) + a.per - 1) / a.per);
  const bool aligned = on16(r.x) && on16(r.y) && r.x_stride % 8 == 0 && r.y_stride % 8 == 0;
  switch (mode_of(t, r.head_dim, aligned)) {
    case kHalf: hipExtLaunchKernelGGL(rope_rows_kernel<kHalf>, grid, dim3(kThreads), 0, stream, ev_start, ev_stop, 0, a); break;
    case kInterleaved:
      hipExtLaunchKernelGGL(rope_rows_kernel<kInterleaved>, grid, dim3(kThreads), 0, stream, ev_start, ev_stop, 0, a);
      break;
    default: hipExtLaunchKernelGGL(rope_rows_kernel<kPair>, grid, dim3(kThreads), 0, stream, ev_start, ev_stop, 0, a);
  }
  return hipGetLastError();
}

hipError_t launch_rope_qkv_append(const RopeAppend& r, const RopeTable& t, hipStream_t stream, hipEvent_t ev_start,
                                  hipEvent_t ev_stop) {
  if (r.n_items <= 0) return hipSuccess;
  if (t.pairs > kHeadDim / 2 || r.n_desc > kAppendInline || r.n_items > kAppendMaxItems) return hipErrorInvalidValue;
  AppendArgs a;
  a.r = r;
  a.layout = t.layout;
  a.pairs = t.pairs;
  a.magnitude = t.magnitude;
  std::copy(t.turns, t.turns + t.pairs, a.turns);
  std::copy(r.desc, r.desc + r.n_desc, a.desc);
  a.v_aligned = on16(r.v) && r.v_stride % 8 == 0;
  const dim3 grid{unsigned(r.n_items), kParts};
  const bool aligned = on16(r.q) && on16(r.k) && on16(r.q_out) && r.q_stride % 8 == 0 && r.k_stride % 8 == 0;
  switch (mode_of(t, kHeadDim, aligned)) {
    case kHalf:
      hipExtLaunchKernelGGL(rope_qkv_append_kernel<kHalf>, grid, dim3(kThreads), 0, stream, ev_start, ev_stop, 0, a);
      break;
    case kInterleaved:
      hipExtLaunchKernelGGL(rope_qkv_append_kernel<kInterleaved>, grid, dim3(kThreads), 0, stream, ev_start, ev_stop, 0, a);
      break;
    default:
      hipExtLaunchKernelGGL(rope_qkv_append_kernel<kPair>, grid, dim3(kThreads), 0, stream, ev_start, ev_stop, 0, a);
  }
  return hipGetLastError();
}

}  // namespace ppas
