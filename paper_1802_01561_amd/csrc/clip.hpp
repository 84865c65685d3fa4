// Host-side declarations of the global gradient norm and clipping.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace vtrace {

constexpr int64_t kClipMostTensors = 1 << 16;
// Of one gradient: its chunks are a launch's workgroups.
constexpr int64_t kClipMostElements = int64_t(1) << 36;
constexpr int kClipMostBlocks = 2048;

// One gradient of a call.
struct ClipItem {
  const void* in;
  void* out;  // null: the norm alone
  int64_t size;
  bool bf16;
};

size_t clip_workspace_bytes();
// items: count gradients, none empty.  Enqueues the norm, and the scaling where `scale`.
hipError_t launch_clip(const ClipItem* items, int64_t count, bool scale, float max_norm, float* norm, void* ws,
                       hipStream_t s);

}  // namespace vtrace
