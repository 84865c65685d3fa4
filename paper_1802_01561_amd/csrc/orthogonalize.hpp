// Host-side declarations of updates made orthogonal by Newton-Schulz products.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <vector>

namespace vtrace {

constexpr int64_t kOrthoMostMatrices = 1 << 16;
constexpr int64_t kOrthoMostSize = 1 << 16;  // rows or columns
constexpr int kOrthoMostSteps = 64;

// One matrix of a call, rows x columns, neither 0.
struct OrthoItem {
  const void* in;
  void* out;
  int64_t rows, columns;
  float scale;
  bool bf16;
};

// One step's X <- a X + (b X X^T + c (X X^T)^2) X.
struct OrthoStep {
  float a, b, c;
};

// What singular values in [0, 1] become in these steps: within the range of the float16 operands?
bool ortho_steps_ok(const OrthoStep* steps, int count);

// The bytes for a call's matrices (their pointers are not used).
size_t ortho_workspace_bytes(const OrthoItem* items, int64_t count);
hipError_t launch_orthogonalize(const OrthoItem* items, int64_t count, const OrthoStep* steps, int step_count, float epsilon,
                                void* ws, hipStream_t s);

}  // namespace vtrace
