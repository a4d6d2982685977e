// Log probabilities of given tokens, their ranks, the rows' entropy and the top
// alternatives, from logit rows in one pass.
//
// With l_i = scale x_i over the V tokens of a row, M a reference near the largest x, and
//   S = sum 2^(t_i), U = sum 2^(t_i) t_i,  t_i = (x_i - M) scale log2 e:
//   log p_i = scale (x_i - M) - ln S,  entropy = ln S - ln 2 U / S.
// Every lane keeps S and U of its logits relative to a reference of its own, which it
// moves when a logit comes whose t is more than 2 (U would lose digits against ln S
// otherwise), and the lanes' sums are brought to the largest reference at the
// end. Sums are fp32, of a few vectors at a time; logits more than 150 below the reference
// count as probability 0 (2^-150 is below fp32's least), so that masked tokens, whether
// -inf or the type's lowest value, add nothing.
//
// The top k (largest first, equal logits by lower token) come from the same pass. Every lane
// notes its largest logit and the vector that has it first; a search over the bits of the
// workgroup's notes gives a bound that k logits reach and few more do, and what reaches it is
// ordered by counting. Notes are ordered as the logits are (value, then vector), so that rows
// of equal logits end in as few candidates as others. Two kernels:
//   parts of a row that its workgroup's registers hold (up to 16,384 bf16 logits): all loads
//   at once, and the candidates are still there;
//   longer ones, two vectors ahead: notes for each quarter, and the quarters whose note
//   reaches the bound are read once more.
// Parts of a row meet in a second launch.
//
// What bounds it: reading the logits, and for bf16 as much the vector unit: an unpacking, an
// fma, an exponential (four slots), a sum, an fma, two maxima and a comparison per logit are
// about 10 slots, 2 bytes (2,048 rows of 131,072 bf16 logits with 5 alternatives: 99 us,
// 5.4 TB/s; a read of as many bytes 76). Few rows are a chain of small steps: a row takes a
// workgroup 12,500 cycles, of which the loads 2,700, the sums 3,100, the bound 2,100 and the
// order of its candidates 3,700, and 8,000 the launch that joins 16 of them (one row 10.4 us
// on the device, 48 of 100,003 13.5, 64 fp32 ones 17.3).
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device.h"
#include "grid.h"
#include "logprobs.h"

namespace ppas {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kAhead = 2;        // vectors that a lane has in flight
constexpr int kHeld = 8;         // vectors that a lane holds of a short part
constexpr float kNone = -3.402823466e38f;   // a reference below every logit
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T>
struct Type;
template <>
struct Type<uint16_t> {   // bf16
  static constexpr int kW = 8;
  static __device__ __forceinline__ float one(uint16_t v) { return __uint_as_float(uint32_t(v) << 16); }
  static __device__ __forceinline__ void unpack(u32x4 v, float (&x)[8]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      x[2 * w] = __uint_as_float(v[w] << 16);
      x[2 * w + 1] = __uint_as_float(v[w] & 0xffff0000u);
    }
  }
  static constexpr uint32_t kMasked = 0xff80ff80u;   // -inf
};
template <>
struct Type<float> {
  static constexpr int kW = 4;
  static __device__ __forceinline__ float one(float v) { return v; }
  static __device__ __forceinline__ void unpack(u32x4 v, float (&x)[4]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) x[w] = __uint_as_float(v[w]);
  }
  static constexpr uint32_t kMasked = 0xff800000u;
};

// Keys that order logits: larger values first, then lower tokens. 0 is below every key.
__device__ __forceinline__ uint64_t key_of(float x, int32_t id) {
  const uint32_t b = __float_as_uint(x + 0.f);   // -0 is 0
  const uint32_t o = b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
  return (uint64_t(o) << 32) | uint32_t(~id);
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t o = uint32_t(key >> 32);
  return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int32_t id_of(uint64_t key) { return int32_t(~uint32_t(key)); }

__device__ __forceinline__ uint64_t lanes_below() { return (uint64_t(1) << (threadIdx.x & 63)) - 1; }
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ float from_lane(float x, float other) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(x), kCtrl, kRows, 0xf, false));
}
__device__ __forceinline__ float last_lane(float v) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
// Over a wave, by lane exchanges: within quads, their pairs, rows of 16 (mirrored), and
// from a row's last lane to the next rows. The same in every lane.
template <typename Op>
__device__ __forceinline__ float over_wave(float v, float none, Op op) {
  v = op(v, from_lane<0xb1>(v, none));
  v = op(v, from_lane<0x4e>(v, none));
  v = op(v, from_lane<0x141>(v, none));
  v = op(v, from_lane<0x140>(v, none));
  v = op(v, from_lane<0x142, 0xa>(v, none));
  v = op(v, from_lane<0x143, 0xc>(v, none));
  return last_lane(v);
}
__device__ __forceinline__ float wave_max(float v) {
  return over_wave(v, -__builtin_inff(), [](float x, float y) { return fmaxf(x, y); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return over_wave(v, 0.f, [](float x, float y) { return x + y; });
}

// ---------------------------------------------------------------------------
// The sums
// ---------------------------------------------------------------------------
// With r = fp32(ref c), t = x c - r is one fma and rounds once; it is `off` = ref c - r above
// (x - ref) c. References whose r is past 2^16 (off could pass 2^-8 there, or r fp32's range)
// have none, and take the difference first.
struct Sums {
  float ref = kNone, S = 0.f, U = 0.f;
  float r = __builtin_nanf(""), off = 0.f;

  // To the sums relative to another reference, at or above this one: with its own r, or plainly.
  __device__ __forceinline__ void move(float to, float c, bool plain) {
    const float was = off;
    r = to * c;
    const bool has = fabsf(r) < 65536.f && !plain;
    off = has ? fmaf(to, c, -r) : 0.f;
    r = has ? r : __builtin_nanf("");
    const float d = fmaf(ref - to, c, off - was), f = __builtin_amdgcn_exp2f(d);
    U = f == 0.f ? 0.f : f * (U + S * d);
    S *= f;
    ref = to;
  }
};

template <int W>
__device__ __forceinline__ float tree(const float (&v)[W]) {
  float s[W / 2];
#pragma unroll
  for (int i = 0; i < W / 2; ++i) s[i] = v[2 * i] + v[2 * i + 1];
#pragma unroll
  for (int n = W / 4; n >= 1; n >>= 1)
#pragma unroll
    for (int i = 0; i < n; ++i) s[i] += s[i + n];
  return s[0];
}

// A batch of N vectors; top is the largest of its logits. Where a t is -infinity (masked
// logits, or differences past fp32) its term comes out NaN, and the batch is taken again
// with such terms as 0; `masked` says that the last one was, and the next goes there at once.
template <int N, int W>
__device__ __forceinline__ void add(Sums& a, bool& masked, const float (&x)[N][W], float top, float c) {
  float s = 0.f, u = 0.f;
  if (__any(!(fmaf(top, c, -a.r) <= 2.f)) && (top - a.ref) * c > 2.f) a.move(top, c, false);
  if (!masked && !__any(!(a.r == a.r))) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float e[W], v = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float t = fmaf(x[j][i], c, -a.r);
        e[i] = __builtin_amdgcn_exp2f(t);
        v = fmaf(e[i], t, v);
      }
      s += tree<W>(e);
      u += v;
    }
    masked = __any(!(fabsf(u) < __builtin_inff()));
    if (!masked) {
      a.S += s;
      a.U += u;
      return;
    }
    s = u = 0.f;
  }
  bool some = false;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float e[W], v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float t = fmaf(x[j][i] - a.ref, c, a.off);
      const bool none = t < -150.f;   // as good as 0
      some = some || none;
      e[i] = none ? 0.f : __builtin_amdgcn_exp2f(t);
      v = none ? v : fmaf(e[i], t, v);
    }
    s += tree<W>(e);
    u += v;
  }
  masked = __any(some);
  a.S += s;
  a.U += u;
}

// ---------------------------------------------------------------------------
// A wave's list of candidates
// ---------------------------------------------------------------------------
constexpr int kCap = 640, kShare = kCap / 64;
static_assert(kCap >= kLogprobsMaxTop + 64 * 8, "the kept ones and a whole vector of every lane");

// LDS that the lanes of one wave exchange: in order as it is, but not for the compiler.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// A lane's largest logit and the first vector that has it (-infinity: none).
struct Note {
  float x = -__builtin_inff();
  int32_t v = 0;
};
__device__ __forceinline__ uint64_t key_of(const Note& n) { return n.x > -__builtin_inff() ? key_of(n.x, n.v) : 0; }

// A bound that k to `enough` of a wave's keys reach (N of each lane; 0: fewer than k are not
// 0), bit by bit from the top: of the value while it leaves too many, then of the numbers
// below `past`.
template <int N>
__device__ __forceinline__ uint64_t bound_of(const uint64_t (&key)[N], int k, int enough, int32_t past) {
  const int bits = 32 - __builtin_clz(uint32_t(max(past, 1)));
  uint32_t hi = 0, lo = ~uint32_t(0) << bits;
  int n = INT32_MAX;
  for (uint32_t bit = 1u << 31; bit && n > enough; bit >>= 1) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) c += int(__popcll(__ballot(uint32_t(key[i] >> 32) >= (hi | bit))));
    if (c >= k) {
      hi |= bit;
      n = c;
    }
  }
  if (hi == 0) return 0;
  if (n <= enough) return uint64_t(hi) << 32;
  for (uint32_t bit = 1u << (bits - 1); bit && n > enough; bit >>= 1) {
    const uint64_t some = (uint64_t(hi) << 32) | lo | bit;
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) c += int(__popcll(__ballot(key[i] >= some)));
    if (c >= k) {
      lo |= bit;
      n = c;
    }
  }
  return (uint64_t(hi) << 32) | lo;
}
// Whether a logit of a vector reaches it: above its value, or equal and of a vector up to its one.
struct Bound {
  float x = -__builtin_inff();
  uint32_t end = 0;   // vectors below it
  __device__ __forceinline__ explicit Bound(uint64_t key) {
    if (key) {
      const uint32_t lo = uint32_t(key);
      x = value_of(key);
      end = lo ? 0u - lo : 0xffffffffu;
    }
  }
  __device__ __forceinline__ bool reached(float y, int32_t v) const { return y > x || (y == x && uint32_t(v) < end); }
};

// How many of n keys in LDS are above one; eight reads at a time.
__device__ __forceinline__ int before_of(const uint64_t* keys, int n, uint64_t key) {
  int before = 0;
  for (int j = 0; j < n; j += 8) {
    uint64_t some[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) some[i] = keys[min(j + i, n - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) before += j + i < n && some[i] > key;
  }
  return before;
}

// The candidates that a wave finds, in LDS.
struct List {
  uint64_t* buf;   // kCap keys
  int count, k;
  float bound;     // logits below it are not among the first k

  // All but the k largest are dropped, one by one from the top.
  __device__ __forceinline__ void exact() {
    const int lane = threadIdx.x & 63;
    uint64_t mine[kShare], last = ~uint64_t(0);
#pragma unroll
    for (int j = 0; j < kShare; ++j) mine[j] = lane + 64 * j < count ? buf[lane + 64 * j] : 0;
    const int n = min(count, k);
    for (int r = 0; r < n; ++r) {
      uint64_t best = 0;
#pragma unroll
      for (int j = 0; j < kShare; ++j) best = mine[j] < last && mine[j] > best ? mine[j] : best;
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)best, d);
        best = o > best ? o : best;
      }
      last = best;
      if (lane == 0) buf[r] = best;
    }
    count = n;
    if (n == k) bound = fmaxf(bound, value_of(last));
    wave_fence();
  }

  // The logits of the lanes' vectors for which hit(e) holds.
  template <int W, typename Hit>
  __device__ __forceinline__ void push(const float (&x)[W], int32_t id0, Hit hit) {
    if (count > kCap - 64 * W) exact();
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const bool h = hit(e);
      const uint64_t b = __ballot(h);
      if (!b) continue;
      if (h) buf[count + int(__popcll(b & lanes_below()))] = key_of(x[e], id0 + e);
      count += int(__popcll(b));
    }
    wave_fence();
  }
};

// ---------------------------------------------------------------------------
// A row, or one of its splits
// ---------------------------------------------------------------------------
struct RowStats {   // of a split
  float ref, S, U;
  int32_t above;    // logits before the given token
};

struct Args {
  LogprobRows r;
  float c;                 // scale log2 e
  int32_t splits, per;     // per: vectors of a split (0: an equal share)
  RowStats* stats;         // [rows][splits], with more than one
  uint64_t* keys;          // [rows][splits][top]
};

// The largest float below x: what is above it is at or above x.
__device__ __forceinline__ float below(float x) {
  const uint32_t b = __float_as_uint(x);
  return __uint_as_float((b << 1) == 0 ? 0x80000001u : b >> 31 ? b + 1 : b - 1);
}

template <int N>
struct Size {
  static constexpr int value = N;
};

struct Given {       // the row's token
  float x;           // its logit
  int32_t id;        // -1: none
};

// One row's results from its sums.
__device__ __forceinline__ bool has_distribution(const RowStats& s) { return s.S > 0.f && s.S < __builtin_inff(); }
// scale (x - ref); a difference of finite logits past fp32 is taken of their halves.
__device__ __forceinline__ float over_ref(const Args& a, float x, float ref) {
  const float d = x - ref;
  return fabsf(d) < __builtin_inff() ? a.r.scale * d : 2.f * a.r.scale * (0.5f * x - 0.5f * ref);
}
__device__ __forceinline__ void write_row(const Args& a, int64_t row, const RowStats& s, const Given& g) {
  const bool ok = has_distribution(s);
  const float nan = __builtin_nanf(""), ln = logf(s.S);
  if (a.r.entropy) a.r.entropy[row] = ok ? fmaxf(ln - kLn2 * (s.U / s.S), 0.f) : nan;
  if (a.r.logprob) a.r.logprob[row] = ok && g.id >= 0 ? over_ref(a, g.x, s.ref) - ln : nan;
  if (a.r.rank) a.r.rank[row] = ok && g.id >= 0 && g.x > -__builtin_inff() ? s.above : -1;
}
// Place i of its top alternatives (key 0: none); ln: of s.S.
__device__ __forceinline__ void write_top(const Args& a, int64_t row, const RowStats& s, float ln, int i, uint64_t key) {
  const bool ok = has_distribution(s);
  const int64_t at = row * a.r.top + i;
  if (a.r.top_ids) a.r.top_ids[at] = ok && key ? id_of(key) : -1;
  if (a.r.top_logprobs)
    a.r.top_logprobs[at] = !ok ? __builtin_nanf("") : key ? over_ref(a, value_of(key), s.ref) - ln : -__builtin_inff();
}

// Loads that are known to be from global memory: those that might be from LDS are waited for
// all at once.
template <typename T>
__device__ __forceinline__ T from_global(const T* p) {
  typedef const __attribute__((address_space(1))) T* Global;
  return *(Global)(reinterpret_cast<uintptr_t>(p));
}

template <typename T>
__device__ __forceinline__ Given given_token(const Args& a, int64_t row) {
  Given g{0.f, -1};
  if (a.r.tokens) {
    const int32_t t = from_global(a.r.tokens + row);
    if (t >= 0 && t < a.r.vocab) {
      g.id = t;
      g.x = Type<T>::one(from_global(static_cast<const T*>(a.r.logits) + row * a.r.stride + t));
    }
  }
  return g;
}

// n keys in LDS to their places among the first `top`, put(place, key), and 0 to those that
// are left over. Up to 64 by all waves, each against its part of them.
template <typename Put>
__device__ __forceinline__ void order_keys(const uint64_t* keys, int n, int top, int (*counts)[64], Put put) {
  if (n <= 64) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const uint64_t key = lane < n ? keys[lane] : 0;
    int before = 0;
    for (int j = wave; j < n; j += 8 * kWaves) {
      uint64_t some[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) some[i] = keys[min(j + i * kWaves, n - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) before += j + i * kWaves < n && some[i] > key;
    }
    counts[wave][lane] = before;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) before += counts[w][lane];
    if (lane >= n) before = lane;   // fewer than asked for
    if (before < top) put(before, key);
    return;
  }
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t key = keys[i];
    const int before = before_of(keys, n, key);
    if (before < top) put(before, key);
  }
}

// A workgroup's part of a row in vectors of W logits on 16 bytes: vector v holds tokens
// v W - shift .. + W - 1, the row's whole ones are v0 .. v1 - 1, the part's lo .. hi - 1.
template <typename T>
struct Part {
  static constexpr int W = Type<T>::kW;
  int64_t row;
  int split, shift;
  const T *x0, *base;
  int32_t v1, lo, hi;
  bool head, tail;   // it has the row's broken vector before, or behind, the whole ones

  __device__ __forceinline__ Part(const Args& a, int64_t block) {
    row = block / a.splits;
    split = int(block % a.splits);
    x0 = static_cast<const T*>(a.r.logits) + row * a.r.stride;
    shift = int(reinterpret_cast<uintptr_t>(x0) / sizeof(T) % W);
    base = x0 - shift;
    const int32_t v0 = shift ? 1 : 0;
    v1 = (shift + a.r.vocab) / W;
    const int32_t whole = max(v1 - v0, 0), per = a.per ? a.per : (whole + a.splits - 1) / a.splits;
    lo = v0 + min(split * per, whole);
    hi = v0 + min((split + 1) * per, whole);
    head = split == 0 && shift != 0;
    tail = split == a.splits - 1 && (shift + a.r.vocab) % W != 0 && (shift == 0 || v1 > 0);
  }
  // the pass asks the caches not to keep it: 2,048 rows of 131,072 bf16 logits 97 us against 90
  __device__ __forceinline__ u32x4 stream(int32_t v) const {
    typedef const __attribute__((address_space(1))) u32x4* Global;
    return __builtin_nontemporal_load((Global)(reinterpret_cast<uintptr_t>(base + int64_t(v) * W)));
  }
  __device__ __forceinline__ u32x4 load(int32_t v) const {
    return from_global(reinterpret_cast<const u32x4*>(base + int64_t(v) * W));
  }
  // Its broken vectors, in lanes 0 and 1 of a wave (what they lack, and the other lanes', is masked).
  __device__ __forceinline__ int32_t edge_vector() const { return (threadIdx.x & 63) == 0 ? 0 : v1; }
  __device__ __forceinline__ u32x4 edge(int32_t vocab) const {
    const int lane = threadIdx.x & 63;
    const bool has = lane == 0 ? head : lane == 1 && tail;
    uint32_t one[W];
#pragma unroll
    for (int e = 0; e < W; ++e) {   // all asked for at once, where there is none another of the row
      const int32_t id = min(max(edge_vector() * W - shift + e, 0), vocab - 1);
      if constexpr (sizeof(T) == 2) one[e] = from_global(x0 + id);
      else one[e] = __float_as_uint(from_global(x0 + id));
    }
    u32x4 v;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const int32_t id = edge_vector() * W - shift + e;
      constexpr uint32_t none = sizeof(T) == 2 ? Type<T>::kMasked & 0xffffu : Type<T>::kMasked;
      const uint32_t x = has && id >= 0 && id < vocab ? one[e] : none;
      if constexpr (sizeof(T) == 2) v[e / 2] = e % 2 ? v[e / 2] | (x << 16) : x;
      else v[e] = x;
    }
    return v;
  }
};

// The largest of a vector's logits.
template <int W>
__device__ __forceinline__ float largest(const float (&x)[W]) {
  float t = -__builtin_inff();
#pragma unroll
  for (int e = 0; e < W; e += 2) t = fmaxf(fmaxf(t, x[e]), x[e + 1]);
  return t;
}

// How many logits of a wave's vectors (at: each lane's) come before the given token.
template <int W>
__device__ __forceinline__ int count_above(const float (&x)[W], int32_t at, const Given& g, float not_below,
                                           int32_t given_at, int shift) {
  const float past = at < given_at ? not_below : g.x;
  int above = 0;
#pragma unroll
  for (int e = 0; e < W; ++e) above += int(__popcll(__ballot(x[e] > past)));
  if (__any(at == given_at)) {
#pragma unroll
    for (int e = 0; e < W; ++e)
      above += int(__popcll(__ballot(at == given_at && x[e] == g.x && at * W - shift + e < g.id)));
  }
  return above;
}

// The workgroup's sums from its waves' (a barrier).
__device__ __forceinline__ RowStats workgroup_sums(Sums& sums, int above, RowStats* parts, float c) {
  const float ref = wave_max(sums.ref);
  sums.move(ref, c, true);
  RowStats s{ref, wave_sum(sums.S), wave_sum(sums.U), above};
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x / 64] = s;
  __syncthreads();
  float to = parts[0].ref;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) to = fmaxf(to, parts[w].ref);
  s = RowStats{to, 0.f, 0.f, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    Sums one{parts[w].ref, parts[w].S, parts[w].U};
    one.move(to, c, true);
    s.S += one.S;
    s.U += one.U;
    s.above += parts[w].above;
  }
  return s;
}

// The bound of the workgroup's notes, by each of its waves.
__device__ __forceinline__ uint64_t row_bound(const uint64_t* notes, int k, int32_t past) {
  const int lane = threadIdx.x & 63;
  uint64_t key[kWaves];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) key[w] = notes[64 * w + lane];
  return bound_of(key, k, k + k / 4 + 4, past);
}

// The first of the waves' candidates in order, to the workspace or the results.
__device__ __forceinline__ void write_first(const Args& a, int64_t block, int64_t row, const RowStats& s,
                                            const List& list, const uint64_t* lists, int* counts) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  if (lane == 0) counts[wave] = list.count;
  __syncthreads();
  uint64_t* out = a.splits > 1 ? a.keys + block * a.r.top : nullptr;
  const float ln = logf(s.S);
  auto put = [&](int i, uint64_t key) {
    if (out) out[i] = key;
    else write_top(a, row, s, ln, i, key);
  };
  int n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) n += counts[w];
  if (n <= 64) {   // a wave, a key for each lane
    if (wave != 0) return;
    uint64_t key = 0;
    int from = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (lane >= from && lane < from + counts[w]) key = lists[w * kCap + lane - from];
      from += counts[w];
    }
    const int hi32 = int(key >> 32), lo32 = int(key);
    int before = 0;
    for (int j = 0; j < n; ++j) {
      const uint64_t other = (uint64_t(uint32_t(__builtin_amdgcn_readlane(hi32, j))) << 32) |
                             uint32_t(__builtin_amdgcn_readlane(lo32, j));
      before += other > key;
    }
    if (lane < n && before < a.r.top) put(before, key);
    if (lane >= n && lane < a.r.top) put(lane, 0);   // fewer than asked for
    return;
  }
  for (int i = lane; i < list.count; i += 64) {
    const uint64_t key = list.buf[i];
    int before = 0;
    for (int w = 0; w < kWaves; ++w) before += before_of(lists + w * kCap, counts[w], key);
    if (before < a.r.top) put(before, key);
  }
}

constexpr int kVectors = 512, kKeys = 1024;   // of a workgroup that may be candidates
static_assert(2 * kVectors + kKeys <= kWaves * kCap, "both in the lists' place");

// A part of at most N vectors for each lane, which hold them until its candidates are found:
// all loads at once, one reference and one bound.
template <typename T, bool kTop, int N>
__global__ __launch_bounds__(kThreads, 4) void logprob_held_kernel(Args a) {
  constexpr int W = Type<T>::kW;
  __shared__ __attribute__((aligned(16))) uint64_t lists[kTop ? kWaves * kCap : 1];
  __shared__ uint64_t notes[kTop ? kThreads : 1];
  __shared__ int32_t at[kTop ? kVectors : 1];
  __shared__ RowStats parts[kWaves];
  __shared__ int places[kTop ? kWaves : 1][64], counts[kWaves], n_vectors, n_keys;
  const int64_t block = block_of();
  if (block / a.splits >= a.r.rows) return;
  const Part<T> p(a, block);
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int32_t token = a.r.tokens ? from_global(a.r.tokens + p.row) : -1;
  u32x4 raw[N];
  if (p.hi > p.lo) {   // past the end its last one, masked below
#pragma unroll
    for (int j = 0; j < N; ++j) raw[j] = p.stream(min(p.lo + int(threadIdx.x) + j * kThreads, p.hi - 1));
  }
  const bool edges = wave == 0 && (p.head || p.tail);
  u32x4 edge[1];
  if (edges) edge[0] = p.edge(a.r.vocab);
  Given g{0.f, -1};
  if (token >= 0 && token < a.r.vocab) g = Given{Type<T>::one(from_global(p.x0 + token)), token};
  const int32_t given_at = g.id >= 0 ? (g.id + p.shift) / W : -1;
  const float not_below = below(g.x);
  if (kTop && threadIdx.x == 0) n_vectors = n_keys = 0;
  Sums sums;
  int above = 0;
  float tops[N], top = -__builtin_inff();
  Note best;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int32_t v = p.lo + int(threadIdx.x) + j * kThreads;
#pragma unroll
    for (int w = 0; w < 4; ++w) raw[j][w] = v < p.hi ? raw[j][w] : Type<T>::kMasked;
    float x[W];
    Type<T>::unpack(raw[j], x);
    tops[j] = largest(x);
    if (kTop && tops[j] > best.x) best = Note{tops[j], v};
    top = fmaxf(top, tops[j]);
  }
  constexpr int kPair = N < 2 ? N : 2;
  bool masked = false;
#pragma unroll
  for (int j0 = 0; j0 < N; j0 += kPair) {
    if (p.lo + j0 * kThreads >= p.hi) break;
    float x[kPair][W];
#pragma unroll
    for (int j = 0; j < kPair; ++j) {
      // unpacked again: kept from above, they are 64 registers more
#pragma unroll
      for (int w = 0; w < 4; ++w) asm volatile("" : "+v"(raw[j0 + j][w]));
      Type<T>::unpack(raw[j0 + j], x[j]);
    }
    add<kPair, W>(sums, masked, x, top, a.c);
    if (a.r.rank) {
#pragma unroll
      for (int j = 0; j < kPair; ++j)
        if (__any(tops[j0 + j] > not_below))
          above += count_above(x[j], p.lo + int(threadIdx.x) + (j0 + j) * kThreads, g, not_below, given_at, p.shift);
    }
  }
  float edge_top = -__builtin_inff();
  if (edges) {
    float x[1][W];
    Type<T>::unpack(edge[0], x[0]);
    edge_top = largest(x[0]);
    masked = true;
    add<1, W>(sums, masked, x, edge_top, a.c);
    if (a.r.rank && __any(edge_top > not_below))
      above += count_above(x[0], p.edge_vector(), g, not_below, given_at, p.shift);
  }
  if (kTop) notes[threadIdx.x] = key_of(best);
  const RowStats s = workgroup_sums(sums, above, parts, a.c);
  if (threadIdx.x == 0) {
    if (a.splits > 1) a.stats[block] = s;
    else write_row(a, p.row, s, g);
  }
  if (!kTop) return;
  // the vectors that reach the bound, then their logits, go to LDS
  const Bound bound(row_bound(notes, a.r.top, p.v1));
  auto reaches = [&](float x, int32_t v) { return bound.reached(x, v); };
  u32x4* vectors = reinterpret_cast<u32x4*>(lists);
  uint64_t* keys = lists + 2 * kVectors;
  uint64_t in[N + 1];
  int found = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    in[j] = __ballot(reaches(tops[j], p.lo + int(threadIdx.x) + j * kThreads));
    found += int(__popcll(in[j]));
  }
  in[N] = __ballot(edges && reaches(edge_top, p.edge_vector()));
  found += int(__popcll(in[N]));
  if (found) {
    int n = 0;
    if (lane == 0) n = atomicAdd(&n_vectors, found);
    n = __builtin_amdgcn_readfirstlane(n);
#pragma unroll
    for (int j = 0; j <= N; ++j) {
      const int to = n + int(__popcll(in[j] & lanes_below()));
      if ((in[j] >> lane & 1) && to < kVectors) {
        vectors[to] = j < N ? raw[j < N ? j : 0] : edge[0];
        at[to] = j < N ? p.lo + int(threadIdx.x) + j * kThreads : p.edge_vector();
      }
      n += int(__popcll(in[j]));
    }
  }
  __syncthreads();
  const int nv = n_vectors;
  if (nv <= kVectors) {
    for (int i = threadIdx.x; i < nv * W; i += kThreads) {
      const int32_t v = at[i / W];
      const float x = Type<T>::one(reinterpret_cast<const T*>(lists)[i]);
      if (!reaches(x, v)) continue;
      const int n = atomicAdd(&n_keys, 1);
      if (n < kKeys) keys[n] = key_of(x, v * W - p.shift + i % W);
    }
    __syncthreads();
    const int n = n_keys;
    if (n <= kKeys) {
      uint64_t* out = a.splits > 1 ? a.keys + block * a.r.top : nullptr;
      const float ln = logf(s.S);
      auto put = [&](int i, uint64_t key) {
        if (out) out[i] = key;
        else write_top(a, p.row, s, ln, i, key);
      };
      order_keys(keys, n, a.r.top, places, put);
      return;
    }
    __syncthreads();
  }
  // more than there is room for (many equal logits): each wave its own, the best of them kept
  List list{lists + wave * kCap, 0, a.r.top, bound.x};
  auto push = [&](const u32x4& raw_v, float top, int32_t v) {
    if (!__any(reaches(top, v))) return;
    float x[W];
    Type<T>::unpack(raw_v, x);
    list.push<W>(x, v * W - p.shift, [&](int e) { return x[e] >= list.bound && reaches(x[e], v); });
  };
#pragma unroll
  for (int j = 0; j < N; ++j) push(raw[j], tops[j], p.lo + int(threadIdx.x) + j * kThreads);
  if (edges) push(edge[0], edge_top, p.edge_vector());
  write_first(a, block, p.row, s, list, lists, counts);
}

constexpr int kQuarters = 4;

template <typename T, bool kTop>
__global__ __launch_bounds__(kThreads) void logprob_kernel(Args a) {
  constexpr int W = Type<T>::kW, kBatch = kAhead * kThreads;
  __shared__ uint64_t lists[kTop ? kWaves * kCap : 1];
  __shared__ uint64_t notes[kTop ? kQuarters * kThreads : 1];
  __shared__ uint16_t pairs[kTop ? kQuarters * kThreads : 1];
  __shared__ RowStats parts[kWaves];
  __shared__ int counts[kWaves], n_pairs;
  const int64_t block = block_of();
  if (block / a.splits >= a.r.rows) return;
  const Part<T> p(a, block);
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, shift = p.shift;
  const int64_t row = p.row;
  const int32_t lo = p.lo, hi = p.hi;
  // batches of kAhead vectors for each lane; the last one is broken
  const int32_t batches = (hi - lo) / kBatch, quarter = batches / kQuarters + 1;
  u32x4 next[kAhead];
  auto load_some = [&](int32_t v) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      next[j][0] = next[j][1] = next[j][2] = next[j][3] = Type<T>::kMasked;
      if (v + j * kThreads < hi) next[j] = p.load(v + j * kThreads);
    }
  };
  if (batches > 0) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) next[j] = p.stream(lo + j * kThreads + int(threadIdx.x));
  } else {
    load_some(lo + int(threadIdx.x));
  }

  const Given g = given_token<T>(a, row);
  const int32_t given_at = g.id >= 0 ? (g.id + shift) / W : -1;
  const float not_below = below(g.x);
  if (kTop && threadIdx.x == 0) n_pairs = 0;
  Sums sums;
  bool masked = false;
  int above = 0;
  Note best, note;   // of the lane, and of its quarter

  // N vectors of the lane, v and each kThreads behind the other; their largest logit
  auto stats = [&](const auto& raw, int32_t v, auto size) {
    constexpr int N = decltype(size)::value;
    float x[N][W], top = -__builtin_inff();
#pragma unroll
    for (int j = 0; j < N; ++j) {
      Type<T>::unpack(raw[j], x[j]);
      const float t = largest(x[j]);
      top = fmaxf(top, t);
      if (kTop && N > 1) {
        const bool more = t > note.x;
        note.x = more ? t : note.x;
        note.v = more ? v + j * kThreads : note.v;
      }
    }
    add<N, W>(sums, masked, x, top, a.c);
    if (a.r.rank && __any(top > not_below)) {
#pragma unroll
      for (int j = 0; j < N; ++j) above += count_above(x[j], v + j * kThreads, g, not_below, given_at, shift);
    }
    return top;
  };
  auto end_quarter = [&](int q) {
    if (!kTop) return;
    notes[q * kThreads + threadIdx.x] = key_of(note);
    if (note.x > best.x) best = note;
    note = Note{};
  };

  int q = 0;
  int32_t left = quarter;   // batches of the quarter
  for (int32_t i = 0; i < batches; ++i) {
    const int32_t v = lo + i * kBatch + int(threadIdx.x);
    u32x4 raw[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) raw[j] = next[j];
    // behind the last batch it is asked for again: loads under a condition would all be waited for
    const int32_t ahead = i + 1 < batches ? v + kBatch : v;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) next[j] = p.stream(ahead + j * kThreads);
    stats(raw, v, Size<kAhead>{});
    if (kTop && --left == 0) {
      end_quarter(q++);
      left = quarter;
    }
  }
  if (int32_t v = lo + batches * kBatch + int(threadIdx.x); v - lane < hi) {   // whole waves
    if (batches > 0) load_some(v);
    stats(next, v, Size<kAhead>{});
  }
  if (kTop)
    for (; q < kQuarters; ++q) end_quarter(q);
  u32x4 edge[1];
  const int32_t edge_v = p.edge_vector();
  float edge_top = -__builtin_inff();
  if (wave == 0 && (p.head || p.tail)) {
    edge[0] = p.edge(a.r.vocab);
    edge_top = stats(edge, edge_v, Size<1>{});
  }

  if (kTop) lists[threadIdx.x] = key_of(best);
  const RowStats s = workgroup_sums(sums, above, parts, a.c);
  if (threadIdx.x == 0) {
    if (a.splits > 1) a.stats[block] = s;
    else write_row(a, row, s, g);
  }
  if (!kTop) return;
  const uint64_t key_bound = row_bound(lists, a.r.top, p.v1);
  const Bound bound(key_bound);
  for (int i = 0; i < kQuarters; ++i) {
    const uint64_t key = notes[i * kThreads + threadIdx.x];
    const bool in = key != 0 && key >= key_bound;
    const uint64_t b = __ballot(in);
    if (!b) continue;
    int at = 0;
    if (lane == 0) at = atomicAdd(&n_pairs, int(__popcll(b)));
    at = __builtin_amdgcn_readfirstlane(at);
    if (in) pairs[at + int(__popcll(b & lanes_below()))] = uint16_t(i * kThreads + threadIdx.x);
  }
  __syncthreads();
  // their vectors: logits that the bound's vector has come in it or before it
  List list{lists + wave * kCap, 0, a.r.top, bound.x};
  const int32_t each = quarter * kAhead;   // vectors of a quarter
  auto find = [&](const u32x4& raw, int32_t v, bool in) {
    float x[W];
    Type<T>::unpack(raw, x);
    bool some = false;
#pragma unroll
    for (int e = 0; e < W; ++e) some = some || x[e] >= list.bound;
    if (__any(in && some))
      list.push<W>(x, v * W - shift, [&](int e) {
        return in && x[e] >= list.bound && bound.reached(x[e], v);
      });
  };
  const uint32_t items = uint32_t(n_pairs) * uint32_t(each);   // below 2^28: 1,024 of at most 2^18
  for (uint32_t i = 64 * wave; i < items; i += 2 * kThreads) {
    u32x4 raw[2];
    int32_t at[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t item = min(i + j * kThreads + lane, items - 1);   // past the end the last one, not taken
      const uint32_t nth = item / uint32_t(each), n = item - nth * uint32_t(each);
      const uint32_t pair = pairs[nth], batch = pair / kThreads * quarter + n / kAhead;
      at[j] = lo + int32_t((batch * kAhead + n % kAhead) * kThreads + pair % kThreads);
      // a quarter's last vectors may lie past the split
      if (at[j] >= hi || i + j * kThreads + lane >= items) at[j] = -1;
      raw[j] = p.load(at[j] < 0 ? lo : at[j]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (i + j * kThreads < items) find(raw[j], at[j], at[j] >= 0);
  }
  if (wave == 0 && __any(bound.reached(edge_top, edge_v))) {
    float x[W];
    Type<T>::unpack(edge[0], x);
    list.push<W>(x, edge_v * W - shift, [&](int e) { return x[e] >= list.bound && bound.reached(x[e], edge_v); });
  }
  write_first(a, block, row, s, list, lists, counts);
}

// The splits of a row. As in a split, a bound that enough keys reach, of the first (or, of
// few splits, later) places of their lists, leaves few, and one of their own fewer, to be
// ordered by counting; where the first leaves many (ascending logits: all the best in one split), a wave takes them one by one,
// each lane the next of a split's (tokens ascend with the splits, so that the first of equal
// lanes is next). The last wave joins the sums meanwhile.
constexpr int kFew = 512;

template <typename T>
__global__ __launch_bounds__(kThreads) void logprob_merge_kernel(Args a) {
  __shared__ uint64_t keys[kLogprobsMaxSplits * kLogprobsMaxTop];
  __shared__ uint64_t few[kFew];
  __shared__ RowStats total;
  __shared__ float total_ln;
  __shared__ int places[kWaves][64], n_few, n_fewer;
  const int64_t row = block_of();
  if (row >= a.r.rows) return;
  constexpr int kRest = kThreads - 64;
  const int tid = threadIdx.x, lane = tid & 63, top = a.r.top, n = a.splits * top;
  RowStats s{kNone, 0.f, 0.f, 0};
  Given g{0.f, -1};
  if (tid >= kRest) {
    if (lane < a.splits) s = a.stats[row * a.splits + lane];
    g = given_token<T>(a, row);
  } else {
    const uint64_t* from = a.keys + row * n;
#pragma unroll 4
    for (int i = tid; i < n; i += kRest) keys[i] = from_global(from + i);
    if (tid == 0) n_few = n_fewer = 0;
  }
  __syncthreads();
  if (tid >= kRest) {
    Sums sums{s.ref, s.S, s.U};
    const float ref = wave_max(s.ref);
    sums.move(ref, a.c, true);
    int above = s.above;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) above += __shfl_xor(above, d);
    s = RowStats{ref, wave_sum(sums.S), wave_sum(sums.U), above};
    if (lane == 0) {
      total = s;
      total_ln = logf(s.S);
      write_row(a, row, s, g);
    }
  } else if (top > 0) {
    // `lists` of the places 0 .. place hold top keys or more
    const int place = (top - 1) / a.splits, lists = (top + place) / (place + 1);
    const uint64_t head[1] = {lane < a.splits ? keys[lane * top + place] : 0};
    uint64_t bound = 1;
    if (lists < a.splits) bound = max(bound_of(head, lists, lists + (a.splits - lists) / 4, a.r.vocab), bound);
    else if (n > kFew) bound = max(bound_of(head, lists, 0, a.r.vocab), bound);   // the least of the heads
    for (int i = tid; i < n; i += kRest) {
      const uint64_t key = keys[i];
      if (key < bound) continue;
      const int at = atomicAdd(&n_few, 1);
      if (at < kFew) few[at] = key;
    }
  }
  if (top == 0) return;
  __syncthreads();
  const int m = n_few;
  auto put = [&](int i, uint64_t key) { write_top(a, row, total, total_ln, i, key); };
  if (m <= 64) {
    order_keys(few, m, top, places, put);
    return;
  }
  if (m <= kFew) {   // a bound of their own first (58 rows of 75,816 tokens with
    // 30 alternatives 17.0 us, without 28)
    uint64_t some[kFew / 64];
#pragma unroll
    for (int i = 0; i < kFew / 64; ++i) some[i] = lane + 64 * i < m ? few[lane + 64 * i] : 0;
    const uint64_t bound = bound_of(some, top, min(top + top / 4 + 4, 64), a.r.vocab);
#pragma unroll
    for (int i = 0; i < kFew / 64; ++i)
      if (tid == lane + 64 * (i % kWaves) && some[i] >= max(bound, uint64_t(1))) keys[atomicAdd(&n_fewer, 1)] = some[i];
    __syncthreads();
    order_keys(keys, n_fewer, top, places, put);
    return;
  }
  if (tid >= 64) return;
  int next = 0;
  uint64_t key = tid < a.splits ? keys[tid * top] : 0, mine = 0;
  for (int i = 0; i < top; ++i) {
    const float v = key ? value_of(key) : -__builtin_inff(), best = wave_max(v);
    const uint64_t b = __ballot(key != 0 && v == best);
    if (!b) break;
    const int winner = int(__ffsll((unsigned long long)b)) - 1;
    const uint64_t won = __shfl((unsigned long long)key, winner);
    if (tid == i) mine = won;
    if (tid == winner) key = ++next < top ? keys[tid * top + next] : 0;
  }
  if (tid < top) write_top(a, row, total, total_ln, tid, mine);
}

}  // namespace

// Parts that lanes hold: a row of up to eight vectors a lane in one workgroup (500 bf16 rows of
// 16,000 tokens with 20 alternatives 11.7 us, in two of four vectors 15.1), others with four
// vectors a lane or more (a row of 131,072 12.0 us with one or two, 11.6 with four, 12.8 with
// eight; 48 rows of 100,003 14.4, 14.3, 13.9, 16.3) in up to about four workgroups per compute
// unit (128 rows of 131,072 19.8 us in 4, 22.4 in 6, 20.9 read past; 200 of 100,000 22.9, 27.3;
// 551 of 24,522, two parts of which would be more than that, 24.0 and, read past, 14.8).
// Longer ones are read past: three workgroups per compute unit, of 8,192 tokens or more (300 rows
// 28.0 us with three or four, 33.9 with two).
LogprobSplit logprob_split(int32_t rows, int32_t vocab, bool f32, int cus) {
  const int64_t vectors = int64_t(vocab) / (f32 ? 4 : 8), row = (vectors + kThreads - 1) / kThreads;   // of a lane
  const int64_t lanes = int64_t(4) * cus * kThreads, fair = (vectors * rows + lanes - 1) / lanes;
  const int64_t held = row <= kHeld ? std::max<int64_t>(1, row) : std::max<int64_t>(4, fair);
  const int64_t parts = std::max<int64_t>(1, (row + held - 1) / held);
  if (held <= kHeld && parts <= kLogprobsMaxSplits && (parts == 1 || parts * rows <= int64_t(4) * cus))
    return {int(parts), int(held)};
  const int64_t most = std::min<int64_t>(kLogprobsMaxSplits, ((int64_t(vocab) + 7) / 8 + 1023) / 1024);
  return {int(std::max<int64_t>(1, std::min(most, int64_t(3) * cus / std::max(rows, 1)))), 0};
}

size_t logprob_workspace_bytes(int32_t rows, int32_t top, int splits) {
  return splits <= 1 ? 0 : size_t(rows) * size_t(splits) * (sizeof(RowStats) + size_t(top) * sizeof(uint64_t));
}

namespace {

template <typename T, bool kTop>
void launch_rows(const Args& a, int held, dim3 grid, hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  const dim3 block(kThreads);
  if (held == 0) hipExtLaunchKernelGGL((logprob_kernel<T, kTop>), grid, block, 0, stream, ev_start, ev_stop, 0, a);
  else if (held <= 2)
    hipExtLaunchKernelGGL((logprob_held_kernel<T, kTop, 2>), grid, block, 0, stream, ev_start, ev_stop, 0, a);
  else if (held <= 4)
    hipExtLaunchKernelGGL((logprob_held_kernel<T, kTop, 4>), grid, block, 0, stream, ev_start, ev_stop, 0, a);
  else
    hipExtLaunchKernelGGL((logprob_held_kernel<T, kTop, kHeld>), grid, block, 0, stream, ev_start, ev_stop, 0, a);
}

}  // namespace

hipError_t launch_logprobs(const LogprobRows& r, LogprobSplit split, void* workspace, hipStream_t stream,
                           hipEvent_t ev_start, hipEvent_t ev_stop) {
  if (r.rows <= 0) return hipSuccess;
  const int splits = split.splits;
  if (r.top > kLogprobsMaxTop || splits > kLogprobsMaxSplits || split.held > kHeld) return hipErrorInvalidValue;
  Args a;
  a.r = r;
  a.c = r.scale * kLog2e;
  a.splits = splits;
  a.per = split.held * kThreads;
  a.stats = static_cast<RowStats*>(workspace);
  a.keys = reinterpret_cast<uint64_t*>(a.stats + (splits > 1 ? int64_t(r.rows) * splits : 0));
  const dim3 grid = grid_of(int64_t(r.rows) * splits), block(kThreads);
  hipEvent_t main_stop = splits > 1 ? nullptr : ev_stop;
  if (r.f32) {
    if (r.top) launch_rows<float, true>(a, split.held, grid, stream, ev_start, main_stop);
    else launch_rows<float, false>(a, split.held, grid, stream, ev_start, main_stop);
  } else {
    if (r.top) launch_rows<uint16_t, true>(a, split.held, grid, stream, ev_start, main_stop);
    else launch_rows<uint16_t, false>(a, split.held, grid, stream, ev_start, main_stop);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits <= 1) return e;
  if (r.f32)
    hipExtLaunchKernelGGL(logprob_merge_kernel<float>, grid_of(r.rows), block, 0, stream, nullptr, ev_stop, 0, a);
  else
    hipExtLaunchKernelGGL(logprob_merge_kernel<uint16_t>, grid_of(r.rows), block, 0, stream, nullptr, ev_stop, 0, a);
  return hipGetLastError();
}

}  // namespace ppas
