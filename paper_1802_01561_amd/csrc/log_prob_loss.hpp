// Host-side declarations of the V-trace losses from log-probabilities.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "launch.hpp"

namespace vtrace {

// A tile's steps are addressed with 31-bit byte offsets.
constexpr int64_t kLogProbMaxLanes = int64_t(1) << 22;

struct LogProbArgs {
  // T, B, the inputs and outputs that a loss call shares, and the workspace's counter
  // and loss partials; its logits are not used.
  StepArgs step;
  const float* target;     // [T,B] log pi(a_t|x_t)
  const float* behaviour;  // [T,B] log mu(a_t|x_t)
  const float* entropy;    // [T,B] or null
  const int32_t* lengths;  // [B] or null
  float* d_log_probs;      // [T,B]
  float* d_entropy;        // [T,B] or null
  // Long unrolls are split along time: each chunk's composite of the recursion.
  int64_t chunks, chunk_tiles;
  double* composites;  // [chunks, B, 2]
  unsigned int* counters;
};

size_t log_prob_workspace_bytes(int64_t T, int64_t B);
void attach_log_prob_workspace(LogProbArgs* a, void* ws);
hipError_t launch_log_prob_loss(const LogProbArgs& a, hipStream_t s);

}  // namespace vtrace
