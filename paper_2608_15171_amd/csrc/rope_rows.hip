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
    r.x = *reinterpret_cast<const u32x4*>(src + first_feature<kMode>(h, u));
    if (kMode == kHalf) {
      if (u < h.pairs / 8) r.y = *reinterpret_cast<const u32x4*>(src + second_feature<kMode>(h, u));
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
      *reinterpret_cast<u32x4*>(dst(second_feature<kMode>(h, u))) = r.y;
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
  *reinterpret_cast<u32x4*>(dst(first_feature<kMode>(h, u))) = r.x;
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

// Every (row, head, unit) of n_rows rows, units fastest: `ready` is called once,
// behind the first loads, and makes the table cs[row][pair].
template <int kMode, typename Src, typename Dst, typename Ready>
__device__ __forceinline__ void turn_rows(int n_rows, int heads, const Head& h, bool copies, const float2* cs, Src src,
                                          Dst dst, Ready ready) {
  const int units = units_of<kMode>(h, copies);
  const int tasks = n_rows * heads * units;
  bool first = true;
  for (int t0 = threadIdx.x; first || t0 < tasks; t0 += kThreads * kAhead) {
    Unit r[kAhead];
    int row[kAhead], head[kAhead], unit[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int t = t0 + i * kThreads;
      unit[i] = t % units;
      const int rest = t / units;
      head[i] = rest % heads;
      row[i] = rest / heads;
      if (t < tasks) r[i] = fetch<kMode>(src(row[i], head[i]), h, unit[i]);
    }
    if (first) {
      ready();
      __syncthreads();
      first = false;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (t0 + i * kThreads >= tasks) continue;
      uint16_t* base = dst(row[i], head[i]);
      put<kMode>(r[i], h, unit[i], cs + row[i] * h.pairs, [&](int f) { return base + f; });
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
  const int row0 = blockIdx.x * a.per, n = min(a.per, a.r.rows - row0);
  const Head h{a.r.head_dim, a.t.pairs, a.t.layout == PPAS_ROPE_HALF};
  turn_rows<kMode>(
      n, a.r.heads, h, a.r.x != a.r.y, cs,
      [&](int row, int head) { return a.r.x + int64_t(row0 + row) * a.r.x_stride + int64_t(head) * a.r.head_dim; },
      [&](int row, int head) { return a.r.y + int64_t(row0 + row) * a.r.y_stride + int64_t(head) * a.r.head_dim; },
      [&]() {
        for (int e = threadIdx.x; e < n * h.pairs; e += kThreads) {
          const int row = e / h.pairs, j = e % h.pairs;
          cs[e] = cos_sin(double(a.r.positions[row0 + row]), a.t.turns[j], a.t.magnitude, a.r.transposed);
        }
      });
}

// ---------------------------------------------------------------------------
// A step's rows on their way into the pages: one workgroup per (request, touched
// page), as in the append that takes packed rows.
// ---------------------------------------------------------------------------
struct AppendArgs {
  RopeAppend r;
  RopeTable t;
};

template <int kMode>
__global__ __launch_bounds__(kThreads) void rope_qkv_append_kernel(AppendArgs a) {
  __shared__ float2 cs[kPage * kHeadDim / 2];
  const RopeAppend& r = a.r;
  const AppendItem it = r.items[blockIdx.x];
  const int tid = threadIdx.x;
  const int pos_lo = it.lpage * kPage;   // position of slot 0
  const int slot_lo = max(it.cached_len - pos_lo, 0), slot_hi = min(it.cached_len + it.n_query - pos_lo, kPage);
  const int n = slot_hi - slot_lo;
  const int64_t row0 = int64_t(it.query_start) + (pos_lo + slot_lo - it.cached_len);   // the first slot's row
  const int32_t page = r.bt[int64_t(it.seq) * r.bt_stride + it.lpage];
  const Head h{kHeadDim, a.t.pairs, a.t.layout == PPAS_ROPE_HALF};

  turn_rows<kMode>(
      n, r.hq, h, r.q != r.q_out, cs,
      [&](int row, int head) { return r.q + (row0 + row) * r.q_stride + head * kHeadDim; },
      [&](int row, int head) { return r.q_out + ((row0 + row) * r.hq + head) * kHeadDim; },
      [&]() {
        for (int e = tid; e < n * h.pairs; e += kThreads) {
          const int row = e / h.pairs, j = e % h.pairs;
          cs[e] = cos_sin(double(pos_lo + slot_lo + row), a.t.turns[j], a.t.magnitude, false);
        }
      });

  // Keys: task (head, unit, slot), slot fastest, so that the stores of a chunk are one run.
  const int units = units_of<kMode>(h, true);
  for (int t = tid; t < r.hkv * units * n; t += kThreads) {
    const int s = t % n, u = (t / n) % units, g = t / (n * units);
    const Unit x = fetch<kMode>(r.k + (row0 + s) * r.k_stride + g * kHeadDim, h, u);
    uint16_t* dst = r.k_pages + (int64_t(page) * r.hkv + g) * kPage * kHeadDim + (slot_lo + s) * 8;
    put<kMode>(x, h, u, cs + s * h.pairs, [&](int f) { return dst + (f >> 3) * (kPage * 8) + (f & 7); });
  }

  // Values: task (head, feature, eight slots), whole 16-byte stores where all eight are new.
  for (int t = tid; t < r.hkv * kHeadDim * 2; t += kThreads) {
    const int g = t / (2 * kHeadDim), d = (t >> 1) % kHeadDim, s0 = 8 * (t & 1);
    if (s0 >= slot_hi || s0 + 8 <= slot_lo) continue;
    uint16_t* dst = r.v_pages + (int64_t(page) * r.hkv + g) * kPage * kHeadDim + d * kPage + s0;
    const uint16_t* src = r.v + (row0 - slot_lo + s0) * r.v_stride + g * kHeadDim + d;
    const int lo = max(slot_lo - s0, 0), hi = min(slot_hi - s0, 8);
    uint16_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e >= lo && e < hi ? src[e * r.v_stride] : uint16_t(0);
    if (hi - lo == 8) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = uint32_t(v[2 * e]) | (uint32_t(v[2 * e + 1]) << 16);
      *reinterpret_cast<u32x4*>(dst) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e >= lo && e < hi) dst[e] = v[e];
    }
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
  // about four workgroups per compute unit, then more rows each
  a.per = std::min<int32_t>(kMaxRows, std::max<int32_t>(1, r.rows / 1024));
  const dim3 grid(unsigned((int64_t(r.rows) + a.per - 1) / a.per));
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
  AppendArgs a;
  a.r = r;
  a.t = t;
  const dim3 grid{unsigned(r.n_items)};
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
