// Low-rank adapters beside a projection: the order of a step's rows by adapter, and the launchers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace ppas {

constexpr int kAdaptersMax = 1024, kAdapterMaxRank = 128;

// Rows of one adapter (-1: of none): places first .. first + count - 1 of the order, at
// most 16 or 64 of them. `row` is the first one where they follow each other, -1 otherwise:
// a decode row's number then comes with its tile, and a chunk's.
struct AdapterTile {
  int32_t adapter, first, count, row;
};
static_assert(sizeof(AdapterTile) == 16, "read as one vector");

// A step's rows sorted by adapter, stably, those without one last, as it lies in the
// caller's buffer: the header, tiles of up to 16 rows, tiles of up to 64, the order.
struct AdapterHeader {
  int32_t tiles16, tiles64, pad0, pad1;
};
struct AdapterOrder {
  int32_t T, n;
  int64_t slots16() const { return slots(16); }
  int64_t slots64() const { return slots(64); }
  int64_t slots(int height) const {   // each adapter's last tile may be broken
    const int64_t groups = n + 1 < T ? n + 1 : T;
    return (int64_t(T) - groups) / height + groups;
  }
  size_t bytes() const {
    return sizeof(AdapterHeader) + size_t(slots16() + slots64()) * sizeof(AdapterTile) + size_t(T) * sizeof(int32_t);
  }
};
hipError_t launch_adapter_rows(const int32_t* row_adapter, AdapterOrder o, void* rows, hipStream_t stream,
                               hipEvent_t ev_start, hipEvent_t ev_stop);

// out[t] = y[t] + scale[a] (x[t] A[a]^T) B[a]^T, a the adapter of row t; with act the gated
// activation of its two halves.
struct AdapterCall {
  const uint16_t *a, *b;
  const float* scale;   // or nullptr: ones
  const uint16_t *x, *y;
  uint16_t* out;
  int64_t x_stride, y_stride, out_stride;   // elements
  int32_t T, hidden, n_out, rank, adapters;
  const void* rows;
  float* part;          // the rows' products with A: [splits][T][rank, padded]
  int32_t splits;       // of hidden: up to adapter_splits
};
// Splits that are the fastest, and the workspace of so many.
int adapter_splits(int32_t T, int32_t hidden, int32_t adapters, int cus);
size_t adapter_workspace_bytes(int32_t T, int32_t rank, int splits);
hipError_t launch_adapters(const AdapterCall& c, bool act, int cus, hipStream_t stream, hipEvent_t ev_start,
                           hipEvent_t ev_stop);

}  // namespace ppas
