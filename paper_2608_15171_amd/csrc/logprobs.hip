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
// The top k (largest first, equal logits by lower token) come from the same pass and a few
// vectors read again. In the pass every lane notes the largest logit of each quarter of its
// vectors, and the vector that has it first. Then the k-th best of each wave's lanes is a
// bound that k logits reach, the best such bound of the waves holds for the row, and only
// the quarters whose note reaches it, k of them and some more, can hold logits that do: they
// are read once more, by all lanes, and what reaches the bound is ordered by counting. Notes
// are ordered as the logits are (value, then vector), so that rows of equal logits end in as
// few candidates as others.
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
constexpr int kAhead = 2;        // vectors that a lane has in flight
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
__device__ __forceinline__ float wave_min(float v) {
  return over_wave(v, __builtin_inff(), [](float x, float y) { return fminf(x, y); });
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

// The k-th largest of the lanes' values (k <= 64; equal ones counted each): a few by taking
// the largest away, more by counting for each lane (12 instructions for each of the k
// against 200).
__device__ __forceinline__ float kth_value(float v, int k) {
  if (k <= 16) {
    float m = wave_max(v);
    for (int i = 1; i < k; ++i) {
      const uint64_t b = __ballot(v == m);
      if (!b) return -__builtin_inff();   // NaNs only
      if (int(threadIdx.x & 63) == int(__ffsll((unsigned long long)b)) - 1) v = -__builtin_inff();
      m = wave_max(v);
    }
    return m;
  }
  int above = 0;
#pragma unroll 16
  for (int j = 0; j < 64; ++j) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), j)) > v;
  return wave_min(above < k ? v : __builtin_inff());
}

// A lane's largest logit and the first vector that has it (-infinity: none).
struct Note {
  float x = -__builtin_inff();
  int32_t v = 0;
};
__device__ __forceinline__ uint64_t key_of(const Note& n) { return n.x > -__builtin_inff() ? key_of(n.x, n.v) : 0; }

// The key of the k-th best note of the lanes, 0 where fewer have one.
__device__ __forceinline__ uint64_t kth_note(const Note& n, int k) {
  const float x = kth_value(n.x, k);
  if (!(x > -__builtin_inff())) return 0;
  uint64_t equal = __ballot(n.x == x);
  // of equal ones as many as are left, from the first vector on
  int left = k - int(__popcll(__ballot(n.x > x)));
  if (int(__popcll(equal)) > left) {
    int32_t v = -1;
    bool in = n.x == x;
    for (; left > 0; --left) {
      v = in ? n.v : INT32_MAX;
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) v = min(v, __shfl_xor(v, d));
      in = in && n.v != v;
    }
    return key_of(x, v);
  }
  int32_t v = 0;
  for (; equal; equal &= equal - 1)
    v = max(v, int32_t(__builtin_amdgcn_readlane(n.v, int(__ffsll((unsigned long long)equal)) - 1)));
  return key_of(x, v);
}

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
// Place i of its top alternatives (key 0: none).
__device__ __forceinline__ void write_top(const Args& a, int64_t row, const RowStats& s, int i, uint64_t key) {
  const bool ok = has_distribution(s);
  const int64_t at = row * a.r.top + i;
  if (a.r.top_ids) a.r.top_ids[at] = ok && key ? id_of(key) : -1;
  if (a.r.top_logprobs)
    a.r.top_logprobs[at] = !ok ? __builtin_nanf("") : key ? over_ref(a, value_of(key), s.ref) - logf(s.S) : -__builtin_inff();
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

constexpr int kQuarters = 4;

template <typename T, bool kTop>
__global__ __launch_bounds__(kThreads) void logprob_kernel(Args a) {
  constexpr int W = Type<T>::kW, kBatch = kAhead * kThreads;
  __shared__ uint64_t lists[kTop ? kWaves * kCap : 1];
  __shared__ uint64_t notes[kTop ? kQuarters * kThreads : 1];
  __shared__ uint16_t pairs[kTop ? kQuarters * kThreads : 1];
  __shared__ RowStats parts[kWaves];
  __shared__ uint64_t bounds[kWaves];
  __shared__ int counts[kWaves], n_pairs, n_best;
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
  // batches of kAhead vectors for each lane; the last one is broken
  const int32_t batches = (hi - lo) / kBatch, quarter = batches / kQuarters + 1;
  // the pass asks the caches not to keep it: 2,048 rows of 131,072 bf16 logits 97 us against 90
  auto stream = [&](int32_t v) {
    typedef const __attribute__((address_space(1))) u32x4* Global;
    return __builtin_nontemporal_load((Global)(reinterpret_cast<uintptr_t>(base + int64_t(v) * W)));
  };
  auto load = [&](int32_t v) { return from_global(reinterpret_cast<const u32x4*>(base + int64_t(v) * W)); };
  u32x4 next[kAhead];
  auto load_some = [&](int32_t v) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      next[j][0] = next[j][1] = next[j][2] = next[j][3] = Type<T>::kMasked;
      if (v + j * kThreads < hi) next[j] = load(v + j * kThreads);
    }
  };
  if (batches > 0) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) next[j] = stream(lo + j * kThreads + int(threadIdx.x));
  } else {
    load_some(lo + int(threadIdx.x));
  }

  const Given g = given_token<T>(a, row);
  const int32_t given_at = g.id >= 0 ? (g.id + shift) / W : -1;
  const float not_below = below(g.x);
  if (kTop && threadIdx.x == 0) n_pairs = n_best = 0;
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
      float t = -__builtin_inff();
#pragma unroll
      for (int e = 0; e < W; e += 2) t = fmaxf(fmaxf(t, x[j][e]), x[j][e + 1]);
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
    for (int j = 0; j < kAhead; ++j) next[j] = stream(ahead + j * kThreads);
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
  // the row's broken vectors, before and behind the whole ones, by lanes 0 and 1 of a wave
  const bool head = split == 0 && shift != 0, tail = split == a.splits - 1 && (shift == 0 || v1 > 0);
  u32x4 edge[1];
  edge[0][0] = edge[0][1] = edge[0][2] = edge[0][3] = Type<T>::kMasked;
  const int32_t edge_v = lane == 0 ? 0 : v1;
  float edge_top = -__builtin_inff();
  if (wave == 0 && (head || tail)) {
    if (lane == 0 ? head : lane == 1 && tail) {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const int32_t id = edge_v * W - shift + e;
        if (id >= 0 && id < a.r.vocab) {
          if constexpr (sizeof(T) == 2) {
            const uint32_t b = from_global(x0 + id);
            edge[0][e / 2] = e % 2 ? (edge[0][e / 2] & 0xffffu) | (b << 16) : (edge[0][e / 2] & 0xffff0000u) | b;
          } else {
            edge[0][e] = __float_as_uint(from_global(x0 + id));
          }
        }
      }
    }
    edge_top = stats(edge, edge_v, Size<1>{});
  }

  // the wave's sums, then the workgroup's
  const float ref = wave_max(sums.ref);
  sums.move(ref, a.c, true);
  RowStats s{ref, wave_sum(sums.S), wave_sum(sums.U), above};
  if (kTop) {
    const uint64_t bound = kth_note(best, a.r.top);
    if (lane == 0) bounds[wave] = bound;
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
  // Any wave's bound holds for the row, and so does the k-th best of the lanes that reach the
  // best of them (each wave's alone is about the 3 k-th of the row's).
  uint64_t bound = bounds[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) bound = max(bound, bounds[w]);
  if (bound) {
    const uint64_t mine = key_of(best);
    if (mine >= bound) lists[atomicAdd(&n_best, 1)] = mine;
    __syncthreads();
    const int n = n_best;
    if (int(threadIdx.x) < n) {
      const uint64_t key = lists[threadIdx.x];
      if (before_of(lists, n, key) == a.r.top - 1) bounds[0] = key;
    }
    __syncthreads();
    bound = bounds[0];
  }
  for (int i = 0; i < kQuarters; ++i) {
    const uint64_t key = notes[i * kThreads + threadIdx.x];
    const bool in = key != 0 && key >= bound;
    const uint64_t b = __ballot(in);
    if (!b) continue;
    int at = 0;
    if (lane == 0) at = atomicAdd(&n_pairs, int(__popcll(b)));
    at = __builtin_amdgcn_readfirstlane(at);
    if (in) pairs[at + int(__popcll(b & lanes_below()))] = uint16_t(i * kThreads + threadIdx.x);
  }
  __syncthreads();
  // their vectors: logits that the bound's vector has come in it or before it
  const float bound_x = bound ? value_of(bound) : -__builtin_inff();
  const int32_t bound_v = bound ? id_of(bound) : INT32_MAX;
  List list{lists + wave * kCap, 0, a.r.top, bound_x};
  const int32_t each = quarter * kAhead;   // vectors of a quarter
  auto find = [&](const u32x4& raw, int32_t v, bool in) {
    float x[W];
    Type<T>::unpack(raw, x);
    bool some = false;
#pragma unroll
    for (int e = 0; e < W; ++e) some = some || x[e] >= list.bound;
    if (__any(in && some))
      list.push<W>(x, v * W - shift, [&](int e) {
        return in && x[e] >= list.bound && x[e] > -__builtin_inff() && (x[e] > bound_x || v <= bound_v);
      });
  };
  const uint32_t items = uint32_t(n_pairs) * uint32_t(each);   // below 2^28: 1,024 of at most 2^18
  for (uint32_t i = 64 * wave; i < items; i += 2 * kThreads) {
    u32x4 raw[2];
    int32_t at[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t item = min(i + j * kThreads + lane, items - 1);   // past the end the last one, not taken
      const uint32_t p = item / uint32_t(each), n = item - p * uint32_t(each);
      const uint32_t pair = pairs[p], batch = pair / kThreads * quarter + n / kAhead;
      at[j] = lo + int32_t((batch * kAhead + n % kAhead) * kThreads + pair % kThreads);
      // a quarter's last vectors may lie past the split
      if (at[j] >= hi || i + j * kThreads + lane >= items) at[j] = -1;
      raw[j] = load(at[j] < 0 ? lo : at[j]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (i + j * kThreads < items) find(raw[j], at[j], at[j] >= 0);
  }
  if (wave == 0 && __any(edge_top >= bound_x && edge_top > -__builtin_inff())) {
    // before or behind all others, so that the bound's vector does not count
    float x[W];
    Type<T>::unpack(edge[0], x);
    list.push<W>(x, edge_v * W - shift, [&](int e) { return x[e] >= bound_x && x[e] > -__builtin_inff(); });
  }
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

// The splits of a row. As in a split, a bound that enough keys reach, of the first (or, of
// few splits, later) places of their lists, leaves few to be ordered by counting; where it
// leaves many (ascending logits: all the best in one split), a wave takes them one by one,
// each lane the next of a split's (tokens ascend with the splits, so that the first of equal
// lanes is next).
constexpr int kFew = 512;

template <typename T>
__global__ __launch_bounds__(kThreads) void logprob_merge_kernel(Args a) {
  __shared__ uint64_t keys[kLogprobsMaxSplits * kLogprobsMaxTop];
  __shared__ uint64_t heads[kLogprobsMaxSplits], few[kFew], bound;
  __shared__ RowStats total;
  __shared__ int n_few;
  const int64_t row = block_of();
  if (row >= a.r.rows) return;
  const int tid = threadIdx.x, top = a.r.top, n = a.splits * top;
  const uint64_t* from = a.keys + row * n;
  constexpr int kAtOnce = kLogprobsMaxSplits * kLogprobsMaxTop / kThreads;
#pragma unroll
  for (int j = 0; j < kAtOnce; ++j)
    if (tid + j * kThreads < n) keys[tid + j * kThreads] = from_global(from + tid + j * kThreads);
  if (tid == 0) {
    n_few = 0;
    bound = 0;
  }
  if (tid < 64) {
    RowStats s{kNone, 0.f, 0.f, 0};
    if (tid < a.splits) s = a.stats[row * a.splits + tid];
    const Given g = given_token<T>(a, row);
    Sums sums{s.ref, s.S, s.U};
    const float ref = wave_max(s.ref);
    sums.move(ref, a.c, true);
    int above = s.above;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) above += __shfl_xor(above, d);
    s = RowStats{ref, wave_sum(sums.S), wave_sum(sums.U), above};
    if (tid == 0) {
      total = s;
      write_row(a, row, s, g);
    }
  }
  if (top == 0) return;
  __syncthreads();
  // `lists` of the places 0 .. place hold top keys or more
  const int place = (top - 1) / a.splits, lists = (top + place) / (place + 1);
  if (tid < a.splits) heads[tid] = keys[tid * top + place];
  __syncthreads();
  if (tid < a.splits && heads[tid] != 0 && before_of(heads, a.splits, heads[tid]) == lists - 1) bound = heads[tid];
  __syncthreads();
  for (int i = tid; i < n; i += kThreads) {
    const uint64_t key = keys[i];
    if (key == 0 || key < bound) continue;
    const int at = atomicAdd(&n_few, 1);
    if (at < kFew) few[at] = key;
  }
  __syncthreads();
  const int m = n_few;
  if (m <= kFew) {
    for (int i = tid; i < m; i += kThreads) {
      const int before = before_of(few, m, few[i]);
      if (before < top) write_top(a, row, total, before, few[i]);
    }
    for (int i = m + tid; i < top; i += kThreads) write_top(a, row, total, i, 0);
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
  if (tid < top) write_top(a, row, total, tid, mine);
}

}  // namespace

// Splits of a row: about three workgroups per compute unit (64 fp32 rows of 131,072 tokens with
// 20 alternatives 21.4 us with two, 22.6 with three, 23.5 with four; 128 bf16 rows with 5 19.6,
// 20.1, 19.1; 300 33.9, 29.3, 28.9), each of 8,192 tokens at least (8 rows 17.4 us, of 2,048
// tokens 19.9).
int logprob_splits(int32_t rows, int32_t vocab, int cus) {
  const int64_t vectors = (int64_t(vocab) + 7) / 8;
  const int64_t most = std::min<int64_t>(kLogprobsMaxSplits, (vectors + 1023) / 1024);
  return int(std::max<int64_t>(1, std::min(most, int64_t(3) * cus / std::max(rows, 1))));
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
    hipExtLaunchKernelGGL(logprob_merge_kernel<float>, grid_of(r.rows), block, 0, stream, nullptr, ev_stop, 0, a);
  else
    hipExtLaunchKernelGGL(logprob_merge_kernel<uint16_t>, grid_of(r.rows), block, 0, stream, nullptr, ev_stop, 0, a);
  return hipGetLastError();
}

}  // namespace ppas
