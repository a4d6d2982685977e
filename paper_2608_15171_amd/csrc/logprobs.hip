// Log probabilities of given tokens, their ranks, the rows' entropy and the top
// alternatives, from logit rows in one pass.
//
// With l_i = scale x_i over the V tokens of a row, M a reference near the largest x, and
//   S = sum 2^(t_i), U = sum 2^(t_i) t_i,  t_i = (x_i - M) scale log2 e:
//   log p_i = scale (x_i - M) - ln S,  entropy = ln S - ln 2 U / S.
// Every lane keeps S and U of its logits relative to a reference of its own, which it
// moves when a logit comes whose t is more than 2 (U would lose digits against ln S
// otherwise), and the lanes' sums are brought to the largest reference at the
// end. Sums are fp32, of eight logits at a time; logits more than 150 below the reference
// count as probability 0 (2^-150 is below fp32's least), so that masked tokens, whether
// -inf or the type's lowest value, add nothing.
//
// The top k (largest first, equal logits by lower token) are found in the same pass: each
// wave keeps a list in LDS of the logits above a bound that at least k of its logits
// reach. The bound starts as the k-th largest of the first 64 vectors' maxima; when the
// list fills, each lane takes the largest of its share of it, and the k-th largest of those
// becomes the bound. A vector whose maximum does not pass the bound costs one comparison.
// Lists of the waves, then of the workgroups of a row, are merged at the end.
//
// What bounds it: reading the logits, and for bf16 as much the vector unit: an unpacking,
// an fma, an exponential (four slots), a sum, an fma, two maxima and a comparison per
// logit are about 10 slots, 2 bytes.
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
constexpr int kAhead = 4;        // vectors that a lane has in flight
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
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_min(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = fminf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
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

// A batch of N vectors; top and low are the largest and the smallest of its logits.
template <int N, int W>
__device__ __forceinline__ void add(Sums& a, const float (&x)[N][W], float top, float low, float c) {
  const float t_top = fmaf(top, c, -a.r), t_low = fmaf(low, c, -a.r);
  // NaNs among numbers pass here and reach the sums; infinities and lone NaNs do not
  if (!__any(!(t_top <= 2.f) || !(t_low >= -150.f))) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float e[W], u = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float t = fmaf(x[j][i], c, -a.r);
        e[i] = __builtin_amdgcn_exp2f(t);
        u = fmaf(e[i], t, u);
      }
      a.S += tree<W>(e);
      a.U += u;
    }
  } else {
    if ((top - a.ref) * c > 2.f) a.move(top, c, false);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float e[W], u = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float t = fmaf(x[j][i] - a.ref, c, a.off);
        const bool none = t < -150.f;
        e[i] = none ? 0.f : __builtin_amdgcn_exp2f(t);
        u = none ? u : fmaf(e[i], t, u);
      }
      a.S += tree<W>(e);
      a.U += u;
    }
  }
}

// ---------------------------------------------------------------------------
// A wave's list of candidates
// ---------------------------------------------------------------------------
constexpr int kCap = 640, kShare = kCap / 64;
static_assert(kCap >= kLogprobsMaxTop + 64 * 8, "the kept ones and a whole vector of every lane");

// LDS that the lanes of one wave exchange: in order as it is, but not for the compiler.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// The k-th largest of the lanes' values (k <= 64; equal ones counted each).
__device__ __forceinline__ float kth_value(float v, int k) {
  int above = 0;
#pragma unroll 16
  for (int j = 0; j < 64; ++j) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), j)) > v;
  return wave_min(above < k ? v : __builtin_inff());
}

struct List {
  uint64_t* buf;   // LDS, kCap keys
  int count, k;
  float bound;     // logits that do not pass it are not among the first k

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

  // Keeps the keys whose logits are at or above v.
  __device__ __forceinline__ void keep(float v) {
    const int lane = threadIdx.x & 63;
    uint64_t mine[kShare];
#pragma unroll
    for (int j = 0; j < kShare; ++j) mine[j] = lane + 64 * j < count ? buf[lane + 64 * j] : 0;
    int n = 0;
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
      const bool kept = mine[j] != 0 && value_of(mine[j]) >= v;
      const uint64_t b = __ballot(kept);
      if (kept) buf[n + int(__popcll(b & lanes_below()))] = mine[j];
      n += int(__popcll(b));
    }
    count = n;
    wave_fence();
  }

  // Keeps what reaches a bound that at least k keys of the list reach.
  __device__ __forceinline__ void tighten() {
    const int lane = threadIdx.x & 63;
    uint64_t best = 0;
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
      const uint64_t key = lane + 64 * j < count ? buf[lane + 64 * j] : 0;
      best = key > best ? key : best;
    }
    bound = fmaxf(bound, kth_value(best ? value_of(best) : -__builtin_inff(), k));
    keep(bound);
  }

  template <int W>
  __device__ __forceinline__ void room() {
    if (count > kCap - 64 * W) {
      tighten();
      if (count > kCap - 64 * W) exact();
    }
  }

  // The logits of the lanes' vectors for which hit(e) holds.
  template <int W, typename Hit>
  __device__ __forceinline__ void push(const float (&x)[W], int32_t id0, Hit hit) {
    room<W>();
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const bool h = hit(e);
      const uint64_t b = __ballot(h);
      if (h) buf[count + int(__popcll(b & lanes_below()))] = key_of(x[e], id0 + e);
      count += int(__popcll(b));
    }
    wave_fence();
  }

  // The first vectors of the wave: the k-th largest of the lanes' maxima is a bound, equal
  // ones counted from the first lane (their tokens ascend). Whether the lane's is among them.
  __device__ __forceinline__ bool begin(float top) {
    bound = kth_value(top, k);
    const bool equal = top == bound;
    const int want = k - int(__popcll(__ballot(top > bound)));
    return top > bound || (equal && int(__popcll(__ballot(equal) & lanes_below())) < want);
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
  int32_t splits;
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
__device__ __forceinline__ void write_row(const Args& a, int64_t row, const RowStats& s, const Given& g) {
  const bool ok = has_distribution(s);
  const float nan = __builtin_nanf(""), ln = logf(s.S);
  if (a.r.entropy) a.r.entropy[row] = ok ? fmaxf(ln - kLn2 * (s.U / s.S), 0.f) : nan;
  if (a.r.logprob) a.r.logprob[row] = ok && g.id >= 0 ? a.r.scale * (g.x - s.ref) - ln : nan;
  if (a.r.rank) a.r.rank[row] = ok && g.id >= 0 && g.x > -__builtin_inff() ? s.above : -1;
}
// Place i of its top alternatives (key 0: none).
__device__ __forceinline__ void write_top(const Args& a, int64_t row, const RowStats& s, int i, uint64_t key) {
  const bool ok = has_distribution(s);
  const int64_t at = row * a.r.top + i;
  if (a.r.top_ids) a.r.top_ids[at] = ok && key ? id_of(key) : -1;
  if (a.r.top_logprobs)
    a.r.top_logprobs[at] = !ok ? __builtin_nanf("") : key ? a.r.scale * (value_of(key) - s.ref) - logf(s.S) : -__builtin_inff();
}

template <typename T>
__device__ __forceinline__ Given given_token(const Args& a, int64_t row) {
  Given g{0.f, -1};
  if (a.r.tokens) {
    const int32_t t = a.r.tokens[row];
    if (t >= 0 && t < a.r.vocab) {
      g.id = t;
      g.x = Type<T>::one(static_cast<const T*>(a.r.logits)[row * a.r.stride + t]);
    }
  }
  return g;
}

template <typename T, bool kTop>
__global__ __launch_bounds__(kThreads) void logprob_kernel(Args a) {
  constexpr int W = Type<T>::kW;
  __shared__ uint64_t lists[kTop ? kWaves * kCap : 1];
  __shared__ RowStats parts[kWaves];
  __shared__ float bounds[kWaves];
  __shared__ int counts[kWaves];
  const int64_t block = block_of();
  const int64_t row = block / a.splits;
  if (row >= a.r.rows) return;
  const int split = int(block % a.splits);
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const T* x0 = static_cast<const T*>(a.r.logits) + row * a.r.stride;
  // vectors of W logits on 16 bytes; vector v holds tokens v W - shift .. + W - 1, the
  // whole ones are v0 .. v1 - 1
  const int shift = int(reinterpret_cast<uintptr_t>(x0) / sizeof(T) % W);
  const T* base = x0 - shift;
  const int32_t v0 = shift ? 1 : 0, v1 = (shift + a.r.vocab) / W;
  const int32_t whole = max(v1 - v0, 0);
  const int32_t per = (whole + a.splits - 1) / a.splits;
  const int32_t lo = v0 + min(split * per, whole), hi = v0 + min((split + 1) * per, whole);
  auto load = [&](int32_t v) {
    u32x4 r;
    r[0] = r[1] = r[2] = r[3] = Type<T>::kMasked;
    if (v < hi) r = *reinterpret_cast<const u32x4*>(base + int64_t(v) * W);
    return r;
  };
  u32x4 next[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) next[j] = load(lo + j * kThreads + int(threadIdx.x));

  const Given g = given_token<T>(a, row);
  const int32_t given_at = g.id >= 0 ? (g.id + shift) / W : -1;
  const float not_below = below(g.x);
  Sums sums;
  List list;
  list.buf = lists + (kTop ? wave * kCap : 0);
  list.count = 0;
  list.k = a.r.top;
  list.bound = -__builtin_inff();
  int above = 0;

  // N vectors of the lane, v and each kThreads behind the other
  auto stats = [&](const auto& raw, int32_t v, auto size) {
    constexpr int N = decltype(size)::value;
    float x[N][W], top = -__builtin_inff(), low = __builtin_inff();
#pragma unroll
    for (int j = 0; j < N; ++j) {
      Type<T>::unpack(raw[j], x[j]);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        top = fmaxf(top, x[j][e]);
        low = fminf(low, x[j][e]);
      }
    }
    add<N, W>(sums, x, top, low, a.c);
    if (a.r.rank) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int32_t at = v + j * kThreads;
        const float past = at < given_at ? not_below : g.x;
#pragma unroll
        for (int e = 0; e < W; ++e) above += int(__popcll(__ballot(x[j][e] > past)));
        if (__any(at == given_at)) {
#pragma unroll
          for (int e = 0; e < W; ++e)
            above += int(__popcll(__ballot(at == given_at && x[j][e] == g.x && at * W - shift + e < g.id)));
        }
      }
    }
    return top;
  };

  bool first = true;
  for (int32_t v = lo + int(threadIdx.x); v - lane < hi; v += kAhead * kThreads) {   // whole waves
    u32x4 raw[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) raw[j] = next[j];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) next[j] = load(v + (kAhead + j) * kThreads);
    const float top = stats(raw, v, Size<kAhead>{});
    if (kTop && __any(first || top > list.bound)) {
#pragma unroll 1
      for (int j = 0; j < kAhead; ++j) {
        u32x4 r = raw[0];
#pragma unroll
        for (int i = 1; i < kAhead; ++i) r = j == i ? raw[i] : r;
        float x[W];
        Type<T>::unpack(r, x);
        float best = x[0];
#pragma unroll
        for (int e = 1; e < W; ++e) best = fmaxf(best, x[e]);
        const int32_t id0 = (v + j * kThreads) * W - shift;
        bool taken = best > list.bound;
        bool equal = false;
        if (first) {
          taken = list.begin(best);
          equal = true;
          first = false;
        }
        if (__any(taken))
          list.push<W>(x, id0, [&](int e) {
            return taken && x[e] > -__builtin_inff() && (equal ? x[e] >= list.bound : x[e] > list.bound);
          });
      }
    }
  }
  // the row's broken vectors, before and behind the whole ones, by lanes 0 and 1 of a wave.
  // Tokens before those seen already may come: logits equal to the bound count
  const bool head = split == 0 && shift != 0, tail = split == a.splits - 1 && (shift == 0 || v1 > 0);
  if (wave == 0 && (head || tail)) {
    u32x4 r[1];
    r[0][0] = r[0][1] = r[0][2] = r[0][3] = Type<T>::kMasked;
    const int32_t v = lane == 0 ? 0 : v1;
    if (lane == 0 ? head : lane == 1 && tail) {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const int32_t id = v * W - shift + e;
        if (id >= 0 && id < a.r.vocab) {
          if constexpr (sizeof(T) == 2) {
            const uint32_t b = x0[id];
            r[0][e / 2] = e % 2 ? (r[0][e / 2] & 0xffffu) | (b << 16) : (r[0][e / 2] & 0xffff0000u) | b;
          } else {
            r[0][e] = __float_as_uint(x0[id]);
          }
        }
      }
    }
    const float top = stats(r, v, Size<1>{});
    if (kTop && __any(top >= list.bound && top > -__builtin_inff())) {
      float x[W];
      Type<T>::unpack(r[0], x);
      list.push<W>(x, v * W - shift, [&](int e) { return x[e] >= list.bound && x[e] > -__builtin_inff(); });
    }
  }

  // the wave's sums, then the workgroup's
  const float ref = wave_max(sums.ref);
  sums.move(ref, a.c, true);
  RowStats s{ref, wave_sum(sums.S), wave_sum(sums.U), above};
  if (kTop) {
    if (list.count > list.k) list.tighten();
    if (lane == 0) bounds[wave] = list.bound;
  }
  if (lane == 0) parts[wave] = s;
  __syncthreads();
  float to = parts[0].ref;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) to = fmaxf(to, parts[w].ref);
  s = RowStats{to, 0.f, 0.f, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    Sums one{parts[w].ref, parts[w].S, parts[w].U};
    one.move(to, a.c, true);
    s.S += one.S;
    s.U += one.U;
    s.above += parts[w].above;
  }
  if (threadIdx.x == 0) {
    if (a.splits > 1) a.stats[block] = s;
    else write_row(a, row, s, g);
  }
  if (!kTop) return;
  // any wave's bound holds for the row; what reaches it is ordered by counting
  float bound = bounds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) bound = fmaxf(bound, bounds[w]);
  list.keep(bound);
  if (lane == 0) counts[wave] = list.count;
  __syncthreads();
  uint64_t* out = a.splits > 1 ? a.keys + block * a.r.top : nullptr;
  auto put = [&](int i, uint64_t key) {
    if (out) out[i] = key;
    else write_top(a, row, s, i, key);
  };
  int n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) n += counts[w];
  for (int i = lane; i < list.count; i += 64) {
    const uint64_t key = list.buf[i];
    int before = 0;
    for (int w = 0; w < kWaves; ++w)
      for (int j = 0; j < counts[w]; ++j) before += lists[w * kCap + j] > key;
    if (before < a.r.top) put(before, key);
  }
  for (int i = n + int(threadIdx.x); i < a.r.top; i += kThreads) put(i, 0);
}

// The splits of a row: a wave, each lane with a split and its ordered keys (tokens ascend
// with the splits, so that the first of equal lanes is next).
template <typename T>
__global__ __launch_bounds__(64) void logprob_merge_kernel(Args a) {
  const int64_t row = block_of();
  if (row >= a.r.rows) return;
  const int lane = threadIdx.x;
  RowStats s{kNone, 0.f, 0.f, 0};
  const int64_t at = row * a.splits + lane;
  if (lane < a.splits) s = a.stats[at];
  Sums sums{s.ref, s.S, s.U};
  const float ref = wave_max(s.ref);
  sums.move(ref, a.c, true);
  int above = s.above;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) above += __shfl_xor(above, d);
  s = RowStats{ref, wave_sum(sums.S), wave_sum(sums.U), above};
  const Given g = given_token<T>(a, row);
  if (lane == 0) write_row(a, row, s, g);
  const uint64_t* keys = a.keys + at * a.r.top;
  int next = 0;
  uint64_t key = lane < a.splits && a.r.top > 0 ? keys[0] : 0;
  uint64_t mine = 0;
  for (int i = 0; i < a.r.top; ++i) {
    const float v = key ? value_of(key) : -__builtin_inff();
    const float m = wave_max(v);
    const uint64_t b = __ballot(key != 0 && v == m);
    if (!b) break;
    const int from = int(__ffsll((unsigned long long)b)) - 1;
    const uint64_t won = __shfl((unsigned long long)key, from);
    if (lane == i) mine = won;
    if (lane == from) key = ++next < a.r.top ? keys[next] : 0;
  }
  if (lane < a.r.top) write_top(a, row, s, lane, mine);
}

}  // namespace

// Splits of a row: about four workgroups per compute unit, each of 256 vectors at least.
int logprob_splits(int32_t rows, int32_t vocab, int cus) {
  const int64_t vectors = (int64_t(vocab) + 7) / 8;
  const int64_t most = std::min<int64_t>(kLogprobsMaxSplits, (vectors + kThreads - 1) / kThreads);
  return int(std::max<int64_t>(1, std::min(most, int64_t(4) * cus / std::max(rows, 1))));
}

size_t logprob_workspace_bytes(int32_t rows, int32_t top, int splits) {
  return splits <= 1 ? 0 : size_t(rows) * size_t(splits) * (sizeof(RowStats) + size_t(top) * sizeof(uint64_t));
}

hipError_t launch_logprobs(const LogprobRows& r, int splits, void* workspace, hipStream_t stream, hipEvent_t ev_start,
                           hipEvent_t ev_stop) {
  if (r.rows <= 0) return hipSuccess;
  if (r.top > kLogprobsMaxTop || splits > kLogprobsMaxSplits) return hipErrorInvalidValue;
  Args a;
  a.r = r;
  a.c = r.scale * kLog2e;
  a.splits = splits;
  a.stats = static_cast<RowStats*>(workspace);
  a.keys = reinterpret_cast<uint64_t*>(a.stats + (splits > 1 ? int64_t(r.rows) * splits : 0));
  const dim3 grid = grid_of(int64_t(r.rows) * splits), block(kThreads);
  hipEvent_t main_stop = splits > 1 ? nullptr : ev_stop;
  if (r.f32) {
    if (r.top) hipExtLaunchKernelGGL((logprob_kernel<float, true>), grid, block, 0, stream, ev_start, main_stop, 0, a);
    else hipExtLaunchKernelGGL((logprob_kernel<float, false>), grid, block, 0, stream, ev_start, main_stop, 0, a);
  } else {
    if (r.top) hipExtLaunchKernelGGL((logprob_kernel<uint16_t, true>), grid, block, 0, stream, ev_start, main_stop, 0, a);
    else hipExtLaunchKernelGGL((logprob_kernel<uint16_t, false>), grid, block, 0, stream, ev_start, main_stop, 0, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits <= 1) return e;
  if (r.f32)
    hipExtLaunchKernelGGL(logprob_merge_kernel<float>, grid_of(r.rows), dim3(64), 0, stream, nullptr, ev_stop, 0, a);
  else
    hipExtLaunchKernelGGL(logprob_merge_kernel<uint16_t>, grid_of(r.rows), dim3(64), 0, stream, nullptr, ev_stop, 0, a);
  return hipGetLastError();
}

}  // namespace ppas
