// Log probabilities of logit rows: the launcher of their kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace ppas {

constexpr int kLogprobsMaxTop = 64, kLogprobsMaxSplits = 64;

// What ppas_logprobs takes; any output may be nullptr.
struct LogprobRows {
  const void* logits;   // bf16, or fp32 where f32
  int64_t stride;       // elements between rows
  const int32_t* tokens;
  float* logprob;
  int32_t* rank;
  float* entropy;
  int32_t* top_ids;
  float* top_logprobs;
  float scale;
  int32_t rows, vocab, top;
  bool f32;
};
// Workgroups of a row on a device with `cus` compute units, the workspace that they share
// their results in (none for one), and the launch. `held`: 16-byte vectors that each of their
// lanes keeps (0: they read past parts of any length, and the few that matter again).
struct LogprobSplit {
  int splits, held;
};
LogprobSplit logprob_split(int32_t rows, int32_t vocab, bool f32, int cus);
size_t logprob_workspace_bytes(int32_t rows, int32_t top, int splits);
hipError_t launch_logprobs(const LogprobRows& r, LogprobSplit split, void* workspace, hipStream_t stream,
                           hipEvent_t ev_start, hipEvent_t ev_stop);

}  // namespace ppas
