// Norms of heads, and their turn by positions in the same pass: rows of heads, and a
// step's query and key rows on their way into the paged cache.
//
// A head x of D features becomes
//   z = (x - mu) / sqrt(var + eps) * (offset + w),  var = mean (x - mu)^2,
// mu its mean in the centred form and 0 otherwise, w its weights; then the turn of
// rope_rows.hip over the first R features of z. Statistics, norm and turn are fp32, the
// result is rounded once to bf16 nearest-even.
//
// What bounds it: memory, at 4 bytes per feature, as the turn alone. A head's features are
// held by a group of 1 to 64 lanes of one wave, each with the pairs that it turns: its
// loads are all in flight before the first sum, the sums go over the group by lane
// exchanges, and every feature is read and written by one lane only, so that rows may be
// done in place. 16,384 rows of a step (16 query and 2 KV heads of 128) take 37.3 us, 4.5 TB/s
// with the vector units busy 48 % (without norms 33; a copy of as many bytes 33); one row of
// each of 64 requests 4.6 us on the device.
//
// A sum of squares that passes fp32 (features from 1e18 on) is taken again of features
// times 2^-70, so that every finite head has its finite norm; a head with an infinity or
// a NaN gives what the formula gives in IEEE arithmetic.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "grid.h"
#include "rope_device.h"

namespace ppas {
namespace {

// Units that a lane holds, and their features.
template <int kMode>
constexpr int kUnits = kMode == kPair ? 2 : 1;
template <int kMode>
constexpr int kValues = kMode == kHalf ? 16 : kMode == kInterleaved ? 8 : 4;

template <int kCtrl>
__device__ __forceinline__ float from_lane(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, true));
}
// The sum over a group of lanes (a power of two of them, the same in all). The exchanges are
// within quads, their pairs, 16 lanes (mirrored: the lanes of one half hold the same sum by
// then), and across.
__device__ __forceinline__ float group_sum(float s, int lanes) {
  if (lanes > 1) s += from_lane<0xb1>(s);
  if (lanes > 2) s += from_lane<0x4e>(s);
  if (lanes > 4) s += from_lane<0x141>(s);
  if (lanes > 8) s += from_lane<0x140>(s);
  if (lanes > 16) s += __shfl_xor(s, 16);
  if (lanes > 32) s += __shfl_xor(s, 32);
  return s;
}

// What a lane of a group does: unit (and unit + lanes, of pairs) of every head it meets.
struct Lane {
  int lanes, unit, units;
};
template <int kMode>
__device__ __forceinline__ Lane lane_of(const Head& h) {
  Lane l;
  l.units = units_of<kMode>(h, true);
  const int per = (l.units + kUnits<kMode> - 1) / kUnits<kMode>;   // at most 64
  l.lanes = per <= 1 ? 1 : 1 << (32 - __clz(per - 1));
  l.unit = int(threadIdx.x) & (l.lanes - 1);
  return l;
}

// The lane's features of a head as loaded (zeros where it has none), and whether the unit
// turns.
template <int kMode>
struct Raw {
  Unit u[kUnits<kMode>];
};
template <int kMode>
__device__ __forceinline__ bool has_second(const Head& h, int u) {
  return kMode == kPair || (kMode == kHalf && u < h.pairs / 8);
}
template <int kMode>
__device__ __forceinline__ Raw<kMode> fetch_raw(const uint16_t* src, const Head& h, const Lane& l) {
  Raw<kMode> r;
#pragma unroll
  for (int i = 0; i < kUnits<kMode>; ++i) {
    r.u[i].x = r.u[i].y = u32x4{0, 0, 0, 0};
    if (l.unit + i * l.lanes < l.units) {
      const Unit v = fetch<kMode>(src, h, l.unit + i * l.lanes);
      if (kMode == kPair) {
        r.u[i].x[0] = v.x[0];
        r.u[i].y[0] = v.y[0];
      } else {
        r.u[i].x = v.x;
        if (has_second<kMode>(h, l.unit)) r.u[i].y = v.y;
      }
    }
  }
  return r;
}
template <int kMode>
__device__ __forceinline__ void values_of(const Raw<kMode>& r, float (&f)[kValues<kMode>]) {
  if (kMode == kPair) {
#pragma unroll
    for (int i = 0; i < kUnits<kMode>; ++i) {
      f[2 * i] = lo_f(r.u[i].x[0]);
      f[2 * i + 1] = lo_f(r.u[i].y[0]);
    }
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[2 * w] = lo_f(r.u[0].x[w]);
      f[2 * w + 1] = hi_f(r.u[0].x[w]);
      if (kMode == kHalf) {
        f[8 + 2 * w] = lo_f(r.u[0].y[w]);
        f[9 + 2 * w] = hi_f(r.u[0].y[w]);
      }
    }
  }
}

// The lane's weights of a head, through the caches.
template <int kMode>
__device__ __forceinline__ Raw<kMode> fetch_weights(const uint16_t* w, const Head& h, const Lane& l) {
  Raw<kMode> r;
#pragma unroll
  for (int i = 0; i < kUnits<kMode>; ++i) {
    const int u = l.unit + i * l.lanes;
    r.u[i].x = r.u[i].y = u32x4{0, 0, 0, 0};
    if (u >= l.units) continue;
    const uint16_t* p = w + first_feature<kMode>(h, u);
    if (kMode == kPair) {
      r.u[i].x[0] = *p;
      r.u[i].y[0] = w[second_feature<kMode>(h, u)];
    } else {
      r.u[i].x = *reinterpret_cast<const u32x4*>(p);
      if (has_second<kMode>(h, u)) r.u[i].y = *reinterpret_cast<const u32x4*>(w + second_feature<kMode>(h, u));
    }
  }
  return r;
}

// The norm of a head's features, in f.
template <int kMode>
__device__ __forceinline__ void normalise(const Raw<kMode>& r, const Head& h, const Lane& l, const HeadNorm& norm,
                                          const Raw<kMode>& w, float (&f)[kValues<kMode>]) {
  constexpr int n = kValues<kMode>;
  const float per = 1.f / float(h.dim);
  // the values that are features: sums of differences leave the others out
  auto mine = [&](int i) {
    if (kMode == kPair) return l.unit + (i >> 1) * l.lanes < l.units;
    return l.unit < l.units && (i < 8 || has_second<kMode>(h, l.unit));
  };
  auto squares = [&](float scale) {
    values_of<kMode>(r, f);
    if (scale != 1.f) {
#pragma unroll
      for (int i = 0; i < n; ++i) f[i] *= scale;
    }
    if (norm.center) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < n; ++i) s += f[i];
      // A true division, and what its rounding leaves of the sum: features that are near one
      // another have an exact sum, and then as good as exact differences (equal ones zeros, of
      // any number; with the sum times a rounded 1 / D, up to 1 for 112 features).
      const float sum = group_sum(s, l.lanes), mu = sum / float(h.dim);
      const float rest = fmaf(-mu, float(h.dim), sum) * per;
#pragma unroll
      for (int i = 0; i < n; ++i) f[i] = mine(i) ? (f[i] - mu) - rest : 0.f;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < n; ++i) s = fmaf(f[i], f[i], s);
    return group_sum(s, l.lanes) * per;
  };
  float var = squares(1.f), eps = norm.eps;
  if (!(var < __builtin_inff())) {   // the same in the whole group
    constexpr float kDown = 0x1p-70f;
    var = squares(kDown);
    eps = fmaxf(eps * kDown * kDown, 0x1p-126f);   // equal features have no variance
  }
  const float to_one = rsqrtf(var + eps);
#pragma unroll
  for (int i = 0; i < n; ++i) f[i] *= to_one;
  if (norm.weight) {
    float g[n];
    values_of<kMode>(w, g);
#pragma unroll
    for (int i = 0; i < n; ++i) f[i] *= g[i] + norm.offset;
  }
}

// Turns the lane's pairs by cs[pair] and stores its features at dst.
template <int kMode, bool kStream>
__device__ __forceinline__ void turn_and_store(float (&f)[kValues<kMode>], const Head& h, const Lane& l,
                                               const float2* cs, uint16_t* dst) {
  auto store = [&](uint16_t* p, u32x4 v) {
    if (kStream) store16(p, v);
    else *reinterpret_cast<u32x4*>(p) = v;
  };
  auto turn = [](float& a, float& b, float2 c) {
    const float x = a;
    a = turn_a(x, b, c);
    b = turn_b(x, b, c);
  };
  if (kMode == kPair) {
#pragma unroll
    for (int i = 0; i < kUnits<kMode>; ++i) {
      const int u = l.unit + i * l.lanes;
      if (u >= l.units) continue;
      if (u < h.pairs) turn(f[2 * i], f[2 * i + 1], cs[u]);
      const uint32_t v = pack2(f[2 * i], f[2 * i + 1]);
      dst[first_feature<kMode>(h, u)] = uint16_t(v);
      dst[second_feature<kMode>(h, u)] = uint16_t(v >> 16);
    }
    return;
  }
  if (l.unit >= l.units) return;
  if (kMode == kHalf) {
    if (has_second<kMode>(h, l.unit)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn(f[i], f[(8 + i) % kValues<kMode>], cs[8 * l.unit + i]);
      u32x4 y;
#pragma unroll
      for (int w = 0; w < 4; ++w) y[w] = pack2(f[(8 + 2 * w) % kValues<kMode>], f[(9 + 2 * w) % kValues<kMode>]);
      store(dst + second_feature<kMode>(h, l.unit), y);
    }
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (4 * l.unit + w < h.pairs)
        turn(f[(2 * w) % kValues<kMode>], f[(2 * w + 1) % kValues<kMode>], cs[4 * l.unit + w]);
  }
  u32x4 x;
#pragma unroll
  for (int w = 0; w < 4; ++w) x[w] = pack2(f[(2 * w) % kValues<kMode>], f[(2 * w + 1) % kValues<kMode>]);
  store(dst + first_feature<kMode>(h, l.unit), x);
}

// Every head of n_rows rows: a group of lanes steps through (row, head). `ready` is called
// once, behind the first loads, and makes the table cs[row][pair].
template <int kMode, bool kStream, int kBatch, typename Src, typename Dst, typename Ready>
__device__ __forceinline__ void norm_rows(int n_rows, int heads, const Head& h, const HeadNorm& norm, int first_head,
                                          const float2* cs, Src src, Dst dst, Ready ready) {
  const Lane l = lane_of<kMode>(h);
  const int step = kThreads / l.lanes, start = int(threadIdx.x) / l.lanes;
  const int step_row = step / heads, step_head = step % heads;
  int row = start / heads, head = start % heads;
  // weights of all heads are brought once, those of each where they are used, behind the
  // store of the head before (16,384 rows of 18 heads 33.0 and 33.9 us, interleaved 33.4 and
  // 34.6; without weights 32.5, the turn alone 29.7 and 32.6)
  const bool by_head = norm.weight && norm.head_stride != 0;
  Raw<kMode> w;
  if (norm.weight && !by_head) w = fetch_weights<kMode>(norm.weight, h, l);
  bool first = true;
  while (first || row < n_rows) {
    Raw<kMode> r[kBatch];
    int rows[kBatch], at_head[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      rows[i] = row;
      at_head[i] = head;
      if (row < n_rows) r[i] = fetch_raw<kMode>(src(row, head), h, l);
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
    for (int i = 0; i < kBatch; ++i) {
      if (rows[i] >= n_rows) continue;   // whole groups
      if (by_head) w = fetch_weights<kMode>(norm.weight + (first_head + at_head[i]) * norm.head_stride, h, l);
      float f[kValues<kMode>];
      normalise<kMode>(r[i], h, l, norm, w, f);
      turn_and_store<kMode, kStream>(f, h, l, cs + rows[i] * h.pairs, dst(rows[i], at_head[i]));
    }
  }
}

// ---------------------------------------------------------------------------
// Rows at given positions
// ---------------------------------------------------------------------------
constexpr int kMaxRows = 16;   // rows of a workgroup

struct NormRowsArgs {
  RopeRows r;
  HeadNorm norm;
  RopeTable t;
  int32_t per;   // rows of a workgroup
};

template <int kMode>
__global__ __launch_bounds__(kThreads) void norm_rope_rows_kernel(NormRowsArgs a) {
  __shared__ float2 cs[kMaxRows * kRopeMaxPairs];
  const int64_t row0 = block_of() * a.per;
  if (row0 >= a.r.rows) return;
  const int n = int(min(int64_t(a.per), a.r.rows - row0));
  const Head h{a.r.head_dim, a.t.pairs, a.t.layout == PPAS_ROPE_HALF};
  norm_rows<kMode, true, kAhead>(
      n, a.r.heads, h, a.norm, 0, cs,
      [&](int row, int head) { return a.r.x + (row0 + row) * a.r.x_stride + int64_t(head) * a.r.head_dim; },
      [&](int row, int head) { return a.r.y + (row0 + row) * a.r.y_stride + int64_t(head) * a.r.head_dim; },
      [&]() {
        for (int e = threadIdx.x; e < n * h.pairs; e += kThreads) {
          const int row = e / h.pairs, j = e % h.pairs;
          cs[e] = cos_sin(double(a.r.positions[row0 + row]), a.t.turns[j], a.t.magnitude, false);
        }
      });
}

// ---------------------------------------------------------------------------
// A step's rows on their way into the pages, in the workgroups of rope_qkv_append_kernel:
// for y = 0 the keys and for y = 1 the values of a page's new slots, else the queries of
// four of them. (One workgroup for keys and values was the last to end: 16,384 rows 41.5 us.)
// Keys pass through LDS, two heads at a time: their norm needs a head's lanes side by side,
// the page's layout (16 slots of each chunk of eight features) the slots.
// ---------------------------------------------------------------------------
// The values of a page's new slots, transposed through LDS a head at a time: rows in by 16
// bytes (or one element), then per task (feature, eight slots) one 16-byte store where all
// eight are new. `v` is this thread's part of the first head (fetch_value).
struct PageSlots {
  int64_t row0;          // the first slot's row
  int32_t page, slot_lo, slot_hi;
};
__device__ __forceinline__ u32x4 fetch_value(const AppendArgs& a, const PageSlots& p, int g) {
  const int t = threadIdx.x, n = p.slot_hi - p.slot_lo;
  u32x4 v = {};
  if (a.v_aligned && t < n * 16) v = load16(a.r.v + (p.row0 + t / 16) * a.r.v_stride + g * kHeadDim + 8 * (t % 16));
  return v;
}
__device__ __forceinline__ void put_values(const AppendArgs& a, const PageSlots& p, u32x4 v,
                                           uint16_t (*rows)[kHeadDim + 8]) {
  const RopeAppend& r = a.r;
  const int tid = threadIdx.x, n = p.slot_hi - p.slot_lo;
  for (int g = 0; g < r.hkv; ++g) {
    if (a.v_aligned) {
      if (tid < n * 16) *reinterpret_cast<u32x4*>(&rows[p.slot_lo + tid / 16][8 * (tid % 16)]) = v;
    } else {
      const uint16_t* src = r.v + p.row0 * r.v_stride + g * kHeadDim;
      for (int t = tid; t < n * kHeadDim; t += kThreads)
        rows[p.slot_lo + t / kHeadDim][t % kHeadDim] = src[t / kHeadDim * r.v_stride + t % kHeadDim];
    }
    __syncthreads();
    if (g + 1 < r.hkv) v = fetch_value(a, p, g + 1);
    const int d = tid / 2, s0 = 8 * (tid & 1), lo = max(p.slot_lo - s0, 0), hi = min(p.slot_hi - s0, 8);
    uint16_t* dst = r.v_pages + (int64_t(p.page) * r.hkv + g) * kPage * kHeadDim + d * kPage + s0;
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

constexpr int kKeyHeads = 2;
constexpr int kWrites = 1;                    // the part that writes values; 0 writes keys
constexpr int kNormParts = kParts + kWrites;   // workgroups of a page

struct NormAppendArgs {
  AppendArgs a;
  HeadNorm q, k;
};

template <int kMode>
__global__ __launch_bounds__(kThreads) void norm_rope_qkv_append_kernel(NormAppendArgs args) {
  __shared__ float2 cs[kPage * kHeadDim / 2];
  const AppendArgs& a = args.a;
  const RopeAppend& r = a.r;
  const AppendItem it = r.n_desc > 0 ? inline_item(a, blockIdx.x) : r.items[blockIdx.x];
  const int tid = threadIdx.x, part = blockIdx.y;
  const int pos_lo = it.lpage * kPage;   // position of slot 0
  int slot_lo = max(it.cached_len - pos_lo, 0), slot_hi = min(it.cached_len + it.n_query - pos_lo, kPage);
  if (part > kWrites) {
    slot_lo = max(slot_lo, (part - kWrites - 1) * kSlots);
    slot_hi = min(slot_hi, (part - kWrites) * kSlots);
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
  if (part > kWrites) {
    norm_rows<kMode, true, 2>(
        n, r.hq, h, args.q, 0, cs,
        [&](int row, int head) { return r.q + (row0 + row) * r.q_stride + head * kHeadDim; },
        [&](int row, int head) { return r.q_out + ((row0 + row) * r.hq + head) * kHeadDim; }, table);
    return;
  }

  __shared__ __attribute__((aligned(16))) uint16_t keys[kKeyHeads][kPage][kHeadDim + 8];
  const int32_t page = r.bt[int64_t(it.seq) * r.bt_stride + it.lpage];
  if (part == kWrites) {
    const PageSlots slots{row0, page, slot_lo, slot_hi};
    put_values(a, slots, fetch_value(a, slots, 0), keys[0]);
    return;
  }
  for (int g0 = 0; g0 < r.hkv; g0 += kKeyHeads) {
    const int heads = min(kKeyHeads, r.hkv - g0);
    norm_rows<kMode, false, 2>(
        n, heads, h, args.k, g0, cs,
        [&](int row, int head) { return r.k + (row0 + row) * r.k_stride + (g0 + head) * kHeadDim; },
        [&](int row, int head) { return &keys[head][slot_lo + row][0]; }, [&]() {
          if (g0 == 0) table();
        });
    __syncthreads();
    // task (head, chunk, slot): a wave stores four chunks' runs of 16 slots
    for (int t = tid; t < heads * 16 * kPage; t += kThreads) {
      const int s = t % kPage, c = t / kPage % 16, g = t / (16 * kPage);
      if (s >= slot_lo && s < slot_hi)
        store16(r.k_pages + ((int64_t(page) * r.hkv + g0 + g) * 16 + c) * (kPage * 8) + s * 8,
                *reinterpret_cast<const u32x4*>(&keys[g][s][8 * c]));
    }
    __syncthreads();
  }
}

// 16-byte runs of the weights too.
bool weights_aligned(const HeadNorm& n) { return on16(n.weight) && n.head_stride % 8 == 0; }

}  // namespace

hipError_t launch_norm_rope_rows(const RopeRows& r, const HeadNorm& norm, const RopeTable& t, hipStream_t stream,
                                 hipEvent_t ev_start, hipEvent_t ev_stop) {
  if (r.rows <= 0) return hipSuccess;
  NormRowsArgs a;
  a.r = r;
  a.norm = norm;
  a.t = t;
  // one batch of loads per thread, but at least about four workgroups per compute unit
  const int64_t lanes = int64_t(r.heads) * std::max(1, t.layout == PPAS_ROPE_HALF ? t.pairs / 8 : r.head_dim / 8);
  a.per = int32_t(std::max<int64_t>(1, std::min<int64_t>({kMaxRows, r.rows / 1024, kThreads * kAhead / lanes})));
  const dim3 grid = grid_of((int64_t(r.rows) + a.per - 1) / a.per), block(kThreads);
  const bool aligned =
      on16(r.x) && on16(r.y) && r.x_stride % 8 == 0 && r.y_stride % 8 == 0 && weights_aligned(norm);
  switch (mode_of(t, r.head_dim, aligned)) {
    case kHalf: hipExtLaunchKernelGGL(norm_rope_rows_kernel<kHalf>, grid, block, 0, stream, ev_start, ev_stop, 0, a); break;
    case kInterleaved:
      hipExtLaunchKernelGGL(norm_rope_rows_kernel<kInterleaved>, grid, block, 0, stream, ev_start, ev_stop, 0, a);
      break;
    default: hipExtLaunchKernelGGL(norm_rope_rows_kernel<kPair>, grid, block, 0, stream, ev_start, ev_stop, 0, a);
  }
  return hipGetLastError();
}

hipError_t launch_norm_rope_qkv_append(const RopeAppend& r, const HeadNorm& q_norm, const HeadNorm& k_norm,
                                       const RopeTable& t, hipStream_t stream, hipEvent_t ev_start,
                                       hipEvent_t ev_stop) {
  if (r.n_items <= 0) return hipSuccess;
  if (t.pairs > kHeadDim / 2 || r.n_desc > kAppendInline || r.n_items > kAppendMaxItems) return hipErrorInvalidValue;
  const NormAppendArgs a{append_args(r, t), q_norm, k_norm};
  const dim3 grid{unsigned(r.n_items), kNormParts}, block(kThreads);
  const bool aligned = on16(r.q) && on16(r.k) && on16(r.q_out) && r.q_stride % 8 == 0 && r.k_stride % 8 == 0 &&
                       weights_aligned(q_norm) && weights_aligned(k_norm);
  switch (mode_of(t, kHeadDim, aligned)) {
    case kHalf:
      hipExtLaunchKernelGGL(norm_rope_qkv_append_kernel<kHalf>, grid, block, 0, stream, ev_start, ev_stop, 0, a);
      break;
    case kInterleaved:
      hipExtLaunchKernelGGL(norm_rope_qkv_append_kernel<kInterleaved>, grid, block, 0, stream, ev_start, ev_stop, 0, a);
      break;
    default:
      hipExtLaunchKernelGGL(norm_rope_qkv_append_kernel<kPair>, grid, block, 0, stream, ev_start, ev_stop, 0, a);
  }
  return hipGetLastError();
}

}  // namespace ppas
