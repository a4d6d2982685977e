// What the kernels that turn heads by their positions share (device code), and the host's part of their launches.
#pragma once

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

// Units of a head; where nothing is copied (in place), those that turn.
template <int kMode>
__device__ __forceinline__ int units_of(const Head& h, bool copies) {
  if (kMode == kHalf) return h.pairs / 8 + (copies ? (h.dim - 2 * h.pairs) / 8 : 0);
  if (kMode == kInterleaved) return copies ? h.dim / 8 : (2 * h.pairs + 7) / 8;
  return copies ? h.dim / 2 : h.pairs;
}

constexpr int kThreads = 256;
constexpr int kAhead = 4;   // units a thread has in flight

// ---------------------------------------------------------------------------
// A step's rows on their way into the pages
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

// 16-byte runs need every run's start on 16 bytes: bases, row strides, heads, and in
// the half layout the second half.
Mode mode_of(const RopeTable& t, int32_t head_dim, bool aligned) {
  if (!aligned || head_dim % 8 != 0) return kPair;
  if (t.layout == PPAS_ROPE_INTERLEAVED) return kInterleaved;
  return t.pairs % 8 == 0 ? kHalf : kPair;
}

bool on16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// The kernel's arguments of a step's rows.
AppendArgs append_args(const RopeAppend& r, const RopeTable& t) {
  AppendArgs a;
  a.r = r;
  a.layout = t.layout;
  a.pairs = t.pairs;
  a.magnitude = t.magnitude;
  std::copy(t.turns, t.turns + t.pairs, a.turns);
  std::copy(r.desc, r.desc + r.n_desc, a.desc);
  a.v_aligned = on16(r.v) && r.v_stride % 8 == 0;
  return a;
}

}  // namespace
}  // namespace ppas
