// The 8-bit product of a few hundred to a few thousand tokens: tiles of 128 token rows x
// 128 weight rows.
//
// What bounds tiles of this size is the way from L2 to LDS: the projection's 64 x 256
// tiles bring 40 KB per 128-feature stage, these 32 KB for as many products, and a full
// chip brings 16 to 17 TB/s with either (2,048 tokens x 11,008 x 2,048 54 us against 45).
// A ring of five stages, and reads waited for a slot later, change nothing. For LDS not to
// bound them next, the halves of the workgroup take alternate stages instead of parts of
// the tile, as integer sums are exact in any order: four waves of 64 x 64 read 64 KB per
// stage where eight waves of 32 x 64 read 96, and while one half reads its stage, the
// other one's MFMAs run on the same SIMDs. The halves' sums meet in LDS at the end.
//
// Slot t of the loop: one half reads stage t into registers, the other multiplies stage
// t - 1, and all waves issue the transfers of stage t + kMidRing - 1 into the ring buffer
// that stage t - 1 was read from in the slot before. A barrier ends the slot, when stage
// t + 1 has landed.
#pragma once

#include "gateup_kernels.h"

namespace ppas {
namespace {

constexpr int kMid = 128;                       // token rows and weight rows of a tile
constexpr int kMidStage = 2 * kMid * kRow;      // 32 KB
constexpr int kMidRing = 4;

// by value (a choice between elements of an array would put it into memory)
__device__ __forceinline__ i32x4 pick(bool first, i32x4 x, i32x4 y) {
  i32x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = first ? x[e] : y[e];
  return r;
}

__global__ __launch_bounds__(kThreads, 1) void gateup_i8_mid_kernel(GemmArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
  __shared__ __attribute__((aligned(1024))) char smem[kMidRing * kMidStage];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = w >> 2, wm = (w >> 1) & 1, wn = w & 1;
  // the tile, in the order of item_at
  const int tiles_m = (a.T + kMid - 1) / kMid, ntiles = tiles_m * a.tiles_n;
  const int per_xcd = ntiles / 8, u = blockIdx.x;
  const int v = u < 8 * per_xcd ? (u % 8) * per_xcd + u / 8 : u;
  const int first_m = v / (kGroupM * a.tiles_n) * kGroupM, gm = min(kGroupM, tiles_m - first_m);
  const int in_grp = v - first_m * a.tiles_n;
  const int m0 = (first_m + in_grp % gm) * kMid, n0 = in_grp / gm * kMid;

  // Transfers, as the tile kernels': eight rows each, row R's chunk c at c ^ (R / 2) % 8.
  // Wave w brings rows 16 w .. + 15 of both operands.
  Rows rx, rw;
  rx.set(a.x, m0, a.T, kMid, a.H);
  rw.set(a.w, n0, a.N2, kMid, a.H);
  uint32_t off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (2 * w + i) * 8 + lane / 8;
    off[i] = uint32_t(r) * (uint32_t(a.H) * 2) + 16 * ((lane & 7) ^ ((r >> 1) & 7));
  }
  const int nk = a.H / kBK;
  // Transfer i < 4 of stage t; past the end the last stage's again, for nobody.
  auto issue = [&](int t, int i) {
    char* at = smem + t % kMidRing * kMidStage + (i >> 1) * kMid * kRow + (2 * w + (i & 1)) * 1024;
    transfer(i < 2 ? rx : rw, at, off[i & 1], uint32_t(min(t, nk - 1)) * kRow);
  };

  int ax[2], aw[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r = lane & 15;
    const int o = r * kRow + 16 * ((4 * j + (lane >> 4)) ^ ((r >> 1) & 7));
    ax[j] = wm * 64 * kRow + o;
    aw[j] = (kMid + wn * 64) * kRow + o;
  }
  u32x4 fx[4][2], fw[4][2];
  i32x4 acc[4][4];   // [weight-row tile][token-row tile]
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = Int8::zero();
  auto read = [&](int t) {
    const char* at = smem + t % kMidRing * kMidStage;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        fx[i][j] = lds16(at + ax[j] + 16 * i * kRow);
        fw[i][j] = lds16(at + aw[j] + 16 * i * kRow);
      }
  };
  // a slot of each kind; t: its number
  auto end_slot = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // the stage is read before its buffer may be refilled
    wait_vmcnt<4 * (kMidRing - 2)>();
    bare_barrier();
  };
  auto read_slot = [&](int t) {
    if (t < nk) read(t);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 4; ++i) issue(t + kMidRing - 1, i);
    end_slot();
  };
  auto mma_slot = [&](int t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int n = 2 * (i & 1); n < 2 * (i & 1) + 2; ++n)
#pragma unroll
        for (int m = 0; m < 4; ++m) acc[n][m] = Int8::mma(fw[n][i >> 1], fx[m][i >> 1], acc[n][m]);
      __builtin_amdgcn_sched_barrier(0);
      issue(t + kMidRing - 1, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    end_slot();
  };

#pragma unroll
  for (int t = 0; t < kMidRing - 1; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) issue(t, i);
  wait_vmcnt<4 * (kMidRing - 2)>();
  bare_barrier();
  // slots 0 .. nk: half h reads in slots h, h + 2, .. and multiplies in the ones after
  // them (it has nothing to read in slot nk)
  if (half == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) issue(kMidRing - 1, i);
    end_slot();
  }
  for (int t = half; t <= nk; t += 2) {
    read_slot(t);
    if (t < nk) mma_slot(t + 1);
  }
  wait_vmcnt<0>();   // no transfer lands in what follows
  __syncthreads();

  // Half h keeps weight-row tiles 2 h and 2 h + 1 of its waves, and takes the other half's
  // sums of them. Element r of [n][m] is token row 16 m + L % 16, column 16 n + 4 (L / 16) + r.
  char* give = smem + w * 8192;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const i32x4 s = pick(half, acc[n][m], acc[n + 2][m]);
      *reinterpret_cast<i32x4*>(give + (4 * n + m) * 1024 + 16 * lane) = s;
    }
  __syncthreads();
  const char* take = smem + (w ^ 4) * 8192;
  char* eb = smem + 64 * 1024 + w * 4096;
  const int m1 = m0 + 64 * wm, n1 = n0 + 64 * wn + 32 * half;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int row = 16 * m + (lane & 15);
    const float sm = m1 + row < a.T ? a.sx[m1 + row] : 0.f;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int col = 16 * n + 4 * (lane >> 4);
      const i32x4 s = pick(half, acc[n + 2][m], acc[n][m]) + *reinterpret_cast<const i32x4*>(take + (4 * n + m) * 1024 + 16 * lane);
      const f32x4 sc = scales4(a.sw, n1 + col, a.N2) * sm;
      Staged<32, 64>::put(eb, row, col, as_value(s[0], sc[0]), as_value(s[1], sc[1]), as_value(s[2], sc[2]),
                          as_value(s[3], sc[3]));
    }
  }
  __syncthreads();
  Staged<32, 64>::out(eb, lane, a.y, m1, n1, a.T, a.N2);
#endif
}

// a.tiles_n is set here; at most one round of tiles is asked for.
hipError_t launch_gateup_i8_mid(GemmArgs a, hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop) {
  a.tiles_n = (a.N2 + kMid - 1) / kMid;
  const int64_t tiles = (int64_t(a.T) + kMid - 1) / kMid * a.tiles_n;
  hipExtLaunchKernelGGL(gateup_i8_mid_kernel, dim3(unsigned(tiles)), dim3(kThreads), 0, stream, ev_start, ev_stop, 0, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace ppas
