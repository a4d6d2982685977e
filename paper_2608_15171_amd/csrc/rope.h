// Rotary positions: the host's frequency table and the launchers of the kernels that use it.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "plan.h"
#include "ppas.h"

namespace ppas {

constexpr int kRopeMaxPairs = 128;   // rows of up to 256 features per head

// What the kernels take of a ppas_rope: turns (of 2 pi) per position of every pair.
struct RopeTable {
  int32_t layout = 0;
  int32_t pairs = 0;
  float magnitude = 1.f;
  double turns[kRopeMaxPairs];   // `pairs` of them
};

constexpr int32_t kAppendMaxItems = (1 << 24) - 1;   // pages of a step's append

// Radians per position of every pair (kRopeMaxPairs doubles), and the table made of them;
// PPAS_EINVAL for a field out of range (host only).
ppas_status rope_frequencies(const ppas_rope* rope, int32_t head_dim, double* w);
ppas_status rope_table(const ppas_rope* rope, int32_t head_dim, RopeTable& table);

// Rows of heads turned by their positions; x == y is allowed.
struct RopeRows {
  const uint16_t* x;
  uint16_t* y;
  int64_t x_stride, y_stride;   // elements between rows; heads follow each other
  const int32_t* positions;
  int32_t rows, heads, head_dim;
  bool transposed;
};
hipError_t launch_rope_rows(const RopeRows& r, const RopeTable& t, hipStream_t stream, hipEvent_t ev_start,
                            hipEvent_t ev_stop);

// A step's rows: q rotated to q_out, k rotated and v copied into the pages.
struct RopeAppend {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;
  uint16_t* q_out;
  uint16_t* k_pages;
  uint16_t* v_pages;
  const AppendItem* items = nullptr;
  const AppendDesc* desc;       // n_desc of them (host memory) in place of the items, or none
  const int32_t* bt;
  int32_t n_items, n_desc, bt_stride, hq, hkv;
};
hipError_t launch_rope_qkv_append(const RopeAppend& r, const RopeTable& t, hipStream_t stream, hipEvent_t ev_start,
                                  hipEvent_t ev_stop);

}  // namespace ppas
