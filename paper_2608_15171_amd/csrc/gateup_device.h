// What the projection's kernels share (device code).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ppas {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ u32x4 lds16(const char* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// silu(g) = g / (1 + e^-g) in fp32 (e^-g through the hardware base-2 exponential;
// +inf for large negative g, which gives -0).
__device__ __forceinline__ float silu_f32(float g) {
  return g / (1.f + __builtin_amdgcn_exp2f(-g * 1.4426950408889634f));
}

// The products' element types: 16 operand bytes of a lane are eight bf16 or sixteen
// 8-bit integers, and one matrix instruction takes 64 bytes of a row in either case,
// so that everything but the instruction and the epilogue is the same.
struct Bf16 {
  using Acc = f32x4;
  static constexpr bool kInt = false;
  static __device__ __forceinline__ Acc zero() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ Acc mma(u32x4 w, u32x4 x, Acc c) {
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(x), c, 0, 0, 0);
#else
    return c;
#endif
  }
};
// Sums of 8-bit products are exact in int32 (at most 131,071 features), whatever their order.
struct Int8 {
  using Acc = i32x4;
  static constexpr bool kInt = true;
  static __device__ __forceinline__ Acc zero() { return i32x4{0, 0, 0, 0}; }
  static __device__ __forceinline__ Acc mma(u32x4 w, u32x4 x, Acc c) {
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, x), c, 0, 0, 0);
#else
    return c;
#endif
  }
};

// Scales of the columns n .. n + 3 (0 from `lim` on).
__device__ __forceinline__ f32x4 scales4(const float* s, int n, int lim) {
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = n + e < lim ? s[n + e] : 0.f;
  return v;
}
// A sum as a value: the sum itself, or an integer sum times its token's and its
// column's scale (the scales' product is rounded to fp32 first, then the integer,
// then their product: three roundings of 2^-24).
__device__ __forceinline__ float as_value(float sum, float) { return sum; }
__device__ __forceinline__ float as_value(int32_t sum, float scale) { return float(sum) * scale; }

// Wait until at most N of this wave's transfers (and stores) are in flight
// (vmcnt: bits 3:0 and 15:14 of the s_waitcnt immediate; they complete in order).
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

// Workgroup barrier without a memory fence (the fence of __syncthreads would wait
// for every transfer in flight). The LDS data it guards is written only by the
// transfers, whose completion each wave waits for explicitly before it; the empty
// asm keeps the compiler from moving memory accesses across it.
__device__ __forceinline__ void bare_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// Partial sums (fp32, or int32 of 8-bit products): columns n .. n + 3 of a token row,
// valid below `lim`.
template <typename T, typename Acc>
__device__ __forceinline__ void store_part(T* row, int n, int lim, bool vec, Acc v) {
  if (n + 4 <= lim && vec) {
    *reinterpret_cast<Acc*>(row + n) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < lim) row[n + e] = v[e];
  }
}

}  // namespace
}  // namespace ppas
