// Launches of more workgroups than one grid dimension takes (2^32 threads): workgroup
// numbers over two dimensions, the last ones past the end.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace ppas {

constexpr int32_t kMaxGridX = 1 << 22;   // of up to 512 threads

inline dim3 grid_of(int64_t blocks) {
  const int64_t x = std::min<int64_t>(blocks, kMaxGridX);
  return dim3(unsigned(x), unsigned((blocks + x - 1) / x));
}
__device__ __forceinline__ int64_t block_of() { return int64_t(blockIdx.y) * gridDim.x + blockIdx.x; }

}  // namespace ppas
