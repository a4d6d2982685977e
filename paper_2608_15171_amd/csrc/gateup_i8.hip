// The projection of 8-bit integers, whose kernels are the bf16 projection's with 16x16x64
// integer MFMAs: rows of 128 features are 128 bytes as 64 bf16 features are, so stages,
// transfers, swizzles and schedule are the same, and one instruction takes as long. The
// int32 sums are exact, so no sum needs two levels and any split gives the same result;
// the epilogue turns them into values with their token's and channel's scale.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device.h"
#include "gateup_kernels.h"

namespace ppas {

hipError_t launch_gateup_i8(const Int8Product& p, bool act, int max_splits, void* part, int cus, hipStream_t stream,
                            hipEvent_t ev_start, hipEvent_t ev_stop) {
  if (p.T <= 0) return hipSuccess;
  if (max_splits < 1 || (max_splits > 1 && !part) || (act && p.N2 % 2 != 0)) return hipErrorInvalidValue;
  // whole 128-byte stages of 16-byte aligned rows, and at least two of them (the scales'
  // transfer); anything else in the general kernel
  const bool aligned = p.H % (2 * kBK) == 0 && p.H > 2 * kBK && reinterpret_cast<uintptr_t>(p.x) % 16 == 0 &&
                       reinterpret_cast<uintptr_t>(p.w) % 16 == 0;
  GateupChoice c;
  if (aligned) c = gateup_choose(p.T, p.H / 2, p.N2, act, true, std::min(max_splits, p.H / (2 * kBK)), cus, true);
  if (c.kernel == GateupChoice::kGeneral) return launch_gateup_i8_any(p, act, stream, ev_start, ev_stop);
  GemmArgs a{};
  a.x = reinterpret_cast<const uint16_t*>(p.x);
  a.w = reinterpret_cast<const uint16_t*>(p.w);
  a.y = p.y;
  a.sx = p.sx;
  a.sw = p.sw;
  a.part = static_cast<float*>(part);
  a.T = p.T;
  a.H = p.H / 2;
  a.N2 = p.N2;
  const hipError_t e = launch_choice<Int8>(a, c, act, stream, ev_start, ev_stop);
  return e != hipSuccess || c.splits == 1 ? e : launch_reduce<Int8>(a, act, c.splits, stream, ev_stop);
}

}  // namespace ppas
