// 8-bit integers with scales: the quantiser of token or weight rows, and the
// product's kernel for any hidden size and alignment (the others are the bf16
// projection's kernels with another matrix instruction).
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device.h"
#include "gateup_device.h"
#include "grid.h"

namespace ppas {
namespace {

// ---------------------------------------------------------------------------
// Quantiser: scale = max|x| / 127 and q = 127 x / max|x| to the nearest integer,
// ties to even, for every row.
//
// Without a division per element: t = x r with r = fp32(127 / max) is within 2^-23 of
// the true quotient, relative. The quotient of two bf16 values times 127 is either
// exactly half-way between integers, or at least 1.5e-5 away from it, relative
// (254 mx - (2k + 1) ma 2^d is a nonzero integer, mx and ma below 256, 2^d the ratio of
// their binades). t rounded to 18 significant bits (2^-18 relative) is therefore the
// half-way point itself in the first case and on its own side of it in the second, so
// that its nearest even integer is that of the true quotient.
// Rows whose maximum is below 2^-110 (the scale and r would leave fp32's normal range)
// count as zero: scale 0. A row with an infinity or NaN gets a NaN scale and zeros, so
// that it cannot pass for a number in any product.
//
// Bound by memory: 16,384 rows of 2,048 take 19 us, 5.3 TB/s (a large copy 5.2); 24 rows
// take 2 us, mostly the launch.
// ---------------------------------------------------------------------------
constexpr uint32_t kTiny = (127 - 110) << 7;   // bf16 bits of 2^-110
constexpr uint32_t kInf = 0x7f80;

__device__ __forceinline__ int quantise(float x, float r) {
  const uint32_t t = (__float_as_uint(x * r) + 0x20u) & ~0x3fu;
  return int(rintf(__uint_as_float(t)));
}
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// |x| as bf16 bits: ordered like the values, infinities and NaN above all
__device__ __forceinline__ uint32_t max_bits(uint32_t m, uint32_t w) {
  return max(m, max(w & 0x7fffu, (w >> 16) & 0x7fffu));
}
__device__ __forceinline__ bool usable(uint32_t m) { return m >= kTiny && m < kInf; }
__device__ __forceinline__ float ratio_of(uint32_t m) { return usable(m) ? 127.f / __uint_as_float(m << 16) : 0.f; }
__device__ __forceinline__ float scale_of(uint32_t m) {
  return usable(m) ? __uint_as_float(m << 16) / 127.f : m >= kInf ? __builtin_nanf("") : 0.f;
}

struct QuantArgs {
  const uint16_t* x;
  int64_t x_stride;
  int8_t* xq;
  float* scale;
  int32_t T, H;
};

// The maximum over the `kThreads` threads of a row.
template <int kThreads>
__device__ __forceinline__ uint32_t row_max(uint32_t m) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = max(m, uint32_t(__shfl_xor(int(m), d)));
  if (kThreads > 64) {
    __shared__ uint32_t wave[kThreads / 64];
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x / 64] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) m = max(m, wave[w]);
  }
  return m;
}

// Rows in registers: kRow threads per row, kC eight-feature chunks each (16-byte loads,
// 8-byte stores), read once. Rows past 8,192 features take 512 threads: 2,056 rows of
// 11,008 13.8 us (4.9 TB/s), with 256 threads of twice the chunks 14.2; 16,384 rows 91.8
// against 95.3.
template <int kRow, int kC>
__global__ __launch_bounds__(kRow > 256 ? kRow : 256) void quant_i8_kernel(QuantArgs a) {
  static_assert(kRow == 64 || kRow == 256 || kRow == 512, "a wave or a workgroup per row");
  constexpr int kRows = kRow > 256 ? 1 : 256 / kRow;   // of a workgroup
  const int t = threadIdx.x % kRow;
  const int64_t row = block_of() * kRows + threadIdx.x / kRow;
  if (row >= a.T) return;   // whole waves, or the workgroup
  const int chunks = a.H / 8;
  const uint16_t* x = a.x + row * a.x_stride;
  u32x4 v[kC];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kC; ++i) {
    const int c = t + i * kRow;
    v[i] = c < chunks ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x + 8 * c)) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < kC; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) m = max_bits(m, v[i][w]);
  m = row_max<kRow>(m);
  const float r = ratio_of(m);
  const bool ok = usable(m);
  int8_t* out = a.xq + row * a.H;
#pragma unroll
  for (int i = 0; i < kC; ++i) {
    const int c = t + i * kRow;
    if (c >= chunks) continue;
    u32x2 q = {0, 0};
    if (ok) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t p = (uint32_t(quantise(lo_f(v[i][w]), r)) & 0xffu) | ((uint32_t(quantise(hi_f(v[i][w]), r)) & 0xffu) << 8);
        q[w >> 1] |= p << (16 * (w & 1));
      }
    }
    *reinterpret_cast<u32x2*>(out + 8 * c) = q;
  }
  if (t == 0) a.scale[row] = scale_of(m);
}

// Any length and alignment: a workgroup reads its row twice, element by element.
__global__ __launch_bounds__(256) void quant_i8_any_kernel(QuantArgs a) {
  const int64_t row = block_of();
  if (row >= a.T) return;
  const uint16_t* x = a.x + row * a.x_stride;
  const uint32_t H = a.H;
  uint32_t m = 0;
  for (uint32_t i = threadIdx.x; i < H; i += 256) m = max(m, uint32_t(x[i]) & 0x7fffu);
  m = row_max<256>(m);
  const float r = ratio_of(m);
  const bool ok = usable(m);
  int8_t* out = a.xq + row * a.H;
  for (uint32_t i = threadIdx.x; i < H; i += 256) out[i] = ok ? int8_t(quantise(lo_f(x[i]), r)) : int8_t(0);
  if (threadIdx.x == 0) a.scale[row] = scale_of(m);
}

// ---------------------------------------------------------------------------
// The product for any hidden size and alignment: 64 token rows x 64 weight rows (with
// the activation 32 gate and 32 up rows) per workgroup, 64 features at a time through
// LDS, zeros past the edges. Bytes that are not on 16 come one by one, which bounds it;
// sizes of whole 128-feature stages on 16 bytes do not come here.
// ---------------------------------------------------------------------------
constexpr int kAny = 64, kAnyPitch = 80;   // bytes of a row in LDS: 16 rows' reads spread over the banks

template <bool kAct>
__global__ __launch_bounds__(256) void gateup_i8_any_kernel(Int8Product a) {
  __shared__ __attribute__((aligned(16))) char xs[kAny * kAnyPitch], ws[kAny * kAnyPitch];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int I = a.N2 / 2;
  const int ncols = kAct ? I : a.N2;
  constexpr int kCols = kAct ? kAny / 2 : kAny;
  const int tiles_n = (ncols + kCols - 1) / kCols;
  const uint32_t tile = uint32_t(block_of());   // at most 2^31 tiles
  if (tile >= uint32_t(tiles_n) * ((uint32_t(a.T) + kAny - 1) / kAny)) return;
  const int m0 = int(tile / tiles_n) * kAny, n0 = int(tile % tiles_n) * kCols;
  // thread t brings 16 bytes of row t / 4
  const int lr = tid / 4, lc = 16 * (tid % 4);
  const int xrow = m0 + lr;
  const int wcol = kAct ? n0 + lr % 32 : n0 + lr;
  const int64_t wrow = kAct && lr >= 32 ? int64_t(I) + wcol : wcol;
  const int8_t* xp = a.x + int64_t(xrow) * a.H;
  const int8_t* wp = a.w + wrow * a.H;
  auto bring = [&](const int8_t* p, bool valid, int k) {
    u32x4 v = {0, 0, 0, 0};
    if (!valid) return v;
    if (k + 16 <= a.H && reinterpret_cast<uintptr_t>(p + k) % 16 == 0) return *reinterpret_cast<const u32x4*>(p + k);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (k + e < a.H) v[e >> 2] |= uint32_t(uint8_t(p[k + e])) << (8 * (e & 3));
    return v;
  };
  // wave w: token rows 16 w .. + 15, all 64 weight rows
  i32x4 acc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = Int8::zero();
  for (int k = 0; k < a.H; k += 64) {
    const u32x4 vx = bring(xp, xrow < a.T, k + lc), vw = bring(wp, wcol < ncols, k + lc);
    __syncthreads();
    *reinterpret_cast<u32x4*>(xs + lr * kAnyPitch + lc) = vx;
    *reinterpret_cast<u32x4*>(ws + lr * kAnyPitch + lc) = vw;
    __syncthreads();
    const int at = (lane & 15) * kAnyPitch + 16 * (lane >> 4);
    const u32x4 fx = lds16(xs + 16 * w * kAnyPitch + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = Int8::mma(lds16(ws + 16 * i * kAnyPitch + at), fx, acc[i]);
  }
  const int m = m0 + 16 * w + (lane & 15);
  if (m >= a.T) return;
  const float sm = a.sx[m];
  uint16_t* row = a.y + int64_t(m) * ncols;
#pragma unroll
  for (int i = 0; i < (kAct ? 2 : 4); ++i) {
    const int n = n0 + 16 * i + 4 * (lane >> 4);
    const f32x4 sg = scales4(a.sw, n, ncols) * sm;
    f32x4 su = {};
    if (kAct) su = scales4(a.sw + I, n, I) * sm;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = as_value(acc[i][e], sg[e]);
      if (kAct) v = silu_f32(v) * as_value(acc[(i + 2) & 3][e], su[e]);
      if (n + e < ncols) row[n + e] = uint16_t(pack_bf16x2(v, 0.f) & 0xffff);
    }
  }
}

}  // namespace

hipError_t launch_quant_i8(const uint16_t* x, int64_t x_stride, int8_t* xq, float* scale, int32_t T, int32_t H,
                           hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  if (T <= 0) return hipSuccess;
  const QuantArgs a{x, x_stride, xq, scale, T, H};
  const bool vec = H % 8 == 0 && x_stride % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0 &&
                   reinterpret_cast<uintptr_t>(xq) % 8 == 0;
  const dim3 block(256), rows = grid_of(T), waves = grid_of((int64_t(T) + 3) / 4);
  const int chunks = H / 8;
  if (!vec || chunks > 4 * 512)
    hipExtLaunchKernelGGL(quant_i8_any_kernel, rows, block, 0, stream, ev_start, ev_stop, 0, a);
  // a wave per row where there are rows enough to fill the chip and they fit its registers
  else if (T >= 1024 && chunks <= 4 * 64)
    hipExtLaunchKernelGGL((quant_i8_kernel<64, 4>), waves, block, 0, stream, ev_start, ev_stop, 0, a);
  else if (chunks <= 256)
    hipExtLaunchKernelGGL((quant_i8_kernel<256, 1>), rows, block, 0, stream, ev_start, ev_stop, 0, a);
  else if (chunks <= 4 * 256)
    hipExtLaunchKernelGGL((quant_i8_kernel<256, 4>), rows, block, 0, stream, ev_start, ev_stop, 0, a);
  else if (chunks <= 3 * 512)
    hipExtLaunchKernelGGL((quant_i8_kernel<512, 3>), rows, dim3(512), 0, stream, ev_start, ev_stop, 0, a);
  else
    hipExtLaunchKernelGGL((quant_i8_kernel<512, 4>), rows, dim3(512), 0, stream, ev_start, ev_stop, 0, a);
  return hipGetLastError();
}

int64_t gateup_i8_any_tiles(int32_t T, int32_t N2, bool act) {
  const int64_t cols = act ? N2 / 2 : N2, per = act ? kAny / 2 : kAny;
  return (cols + per - 1) / per * ((int64_t(T) + kAny - 1) / kAny);
}

hipError_t launch_gateup_i8_any(const Int8Product& p, bool act, hipStream_t stream, hipEvent_t ev_start,
                                hipEvent_t ev_stop) {
  const int64_t tiles = gateup_i8_any_tiles(p.T, p.N2, act);
  if (tiles > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid = grid_of(tiles);
  if (act)
    hipExtLaunchKernelGGL(gateup_i8_any_kernel<true>, grid, dim3(256), 0, stream, ev_start, ev_stop, 0, p);
  else
    hipExtLaunchKernelGGL(gateup_i8_any_kernel<false>, grid, dim3(256), 0, stream, ev_start, ev_stop, 0, p);
  return hipGetLastError();
}

}  // namespace ppas
