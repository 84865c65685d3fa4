// What the Newton-Schulz kernels share: a launch's matrices, their pieces of the workspace, and
// operands of products.
#pragma once

#include "contraction.hpp"
#include "orthogonalize.hpp"

namespace vtrace {

// The operands' scales: X 2^12, A and B 2^13.
constexpr float kScaleX = 4096.0f, kScaleA = 8192.0f;

// A matrix of a launch.  Its pieces lie one after the other from `base` on (pieces_of).
struct Entry {
  const void* in;
  void* out;
  char* base;
  int32_t r, c;    // r <= c
  int32_t pr, pc;  // rounded up to 64: pitches
  float scale;
  int32_t transposed;
  int32_t first_partial, partials;
  int32_t first_block;  // of the kernel that scales: 64 x 64 each
  int32_t first_tile[3];
};

// As many as 4 KB of arguments hold.
struct Table {
  static constexpr int kMost = 44;
  Entry at[kMost];
  double* partials;
  int count;
  int total_partials, total_blocks, total_tiles[3];
  int size[3];  // of the tiles of A, B and X
  float epsilon;
  bool small;  // the small matrices' kernels, which keep X^T as well
};
static_assert(sizeof(Table) <= 4000, "kernel arguments");

struct Pieces {
  float* x;           // [r, pc] X, of float32 matrices
  uint16_t* low;      // [r, pc] of bfloat16 ones what the operand leaves of X
  uint16_t* from[2];  // [r, pc] X as an operand: high and (float32 matrices) low parts
  uint16_t* to[2];    // [r, pc] the same behind this step
  uint16_t* a[2];     // [r, pr] A without its diagonal
  uint16_t* b[2];     // B without its diagonal
  float* d;           // [r] A's diagonal
  float* e;           // [r] B's
};
__host__ __device__ inline int64_t round_up(int64_t n, int64_t k) { return (n + k - 1) / k * k; }
template <bool kPair>
__host__ __device__ inline int64_t piece_bytes(int64_t r, int64_t pr, int64_t pc) {
  constexpr int kParts = kPair ? 2 : 1;
  return r * pc * (2 * kParts + 2 * 2 * kParts) + r * pr * 2 * 2 * kParts + 2 * round_up(r * 4, 256);
}
// Behind them, for the small matrices' kernels: X^T as an operand, before and after a step.
template <bool kPair>
__host__ __device__ inline int64_t transposed_bytes(int64_t c, int64_t pr) {
  return c * pr * 2 * 2 * (kPair ? 2 : 1);
}
namespace {

template <bool kPair>
__device__ __forceinline__ Pieces pieces_of(const Entry& t, int turn) {
  constexpr int kParts = kPair ? 2 : 1;
  Pieces p;
  char* at = t.base;
  const int64_t x = static_cast<int64_t>(t.r) * t.pc * 2, a = static_cast<int64_t>(t.r) * t.pr * 2;
  p.x = reinterpret_cast<float*>(at);
  p.low = reinterpret_cast<uint16_t*>(at);
  at += x * kParts;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    p.from[k] = reinterpret_cast<uint16_t*>(at + (turn * kParts + (kPair ? k : 0)) * x);
    p.to[k] = reinterpret_cast<uint16_t*>(at + ((turn ^ 1) * kParts + (kPair ? k : 0)) * x);
    p.a[k] = reinterpret_cast<uint16_t*>(at + 2 * kParts * x + (kPair ? k : 0) * a);
    p.b[k] = reinterpret_cast<uint16_t*>(at + 2 * kParts * x + (kParts + (kPair ? k : 0)) * a);
  }
  at += 2 * kParts * (x + a);
  p.d = reinterpret_cast<float*>(at);
  p.e = reinterpret_cast<float*>(at + round_up(static_cast<int64_t>(t.r) * 4, 256));
  return p;
}

struct TransposedPieces {
  uint16_t* from[2];  // [c, pr]: high and low parts
  uint16_t* to[2];
};
template <bool kPair>
__device__ __forceinline__ TransposedPieces transposed_of(const Entry& t, int turn) {
  constexpr int kParts = kPair ? 2 : 1;
  char* const at = t.base + piece_bytes<kPair>(t.r, t.pr, t.pc);
  const int64_t plane = static_cast<int64_t>(t.c) * t.pr * 2;
  TransposedPieces p;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    p.from[k] = reinterpret_cast<uint16_t*>(at + (turn * kParts + (kPair ? k : 0)) * plane);
    p.to[k] = reinterpret_cast<uint16_t*>(at + ((turn ^ 1) * kParts + (kPair ? k : 0)) * plane);
  }
  return p;
}

// The last entry whose first number is not above `id`.
template <typename First>
__device__ __forceinline__ int entry_of(const Table& t, int id, First first) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (first(t.at[mid]) <= id) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ uint16_t half_bits(float x) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x)); }
__device__ __forceinline__ float half_value(uint16_t bits) { return static_cast<float>(__builtin_bit_cast(_Float16, bits)); }

// Two values as operands: float16, and what that leaves of them (twice half a step of
// float16: 22 bits together).
__device__ __forceinline__ unsigned high2(float x, float y) {
  return half_bits(x) | static_cast<unsigned>(half_bits(y)) << 16;
}
__device__ __forceinline__ float high_of(unsigned pair, int i) { return half_value(static_cast<uint16_t>(pair >> (16 * i))); }
__device__ __forceinline__ unsigned low2(float x, float y, unsigned high) {
  return high2(x - high_of(high, 0), y - high_of(high, 1));
}
// Four.
__device__ __forceinline__ v2u high4(const float (&y)[4]) { return {high2(y[0], y[1]), high2(y[2], y[3])}; }
__device__ __forceinline__ v2u low4(const float (&y)[4], v2u high) { return {low2(y[0], y[1], high[0]), low2(y[2], y[3], high[1])}; }

// Tile `id` of a lower triangle: rows 0, 1 1, 2 2 2, ...
__device__ __forceinline__ TileAt triangle_at(int id) {
  int row = static_cast<int>((sqrtf(8.0f * static_cast<float>(id) + 1.0f) - 1.0f) * 0.5f);
  while (row * (row + 1) / 2 > id) --row;
  while ((row + 1) * (row + 2) / 2 <= id) ++row;
  return {row, id - row * (row + 1) / 2};
}

// Four consecutive elements of a row of the result, as many as it has.
template <typename Out>
__device__ __forceinline__ void store_result(Out* p, const float (&y)[4], int left, bool vectors) {
  if (vectors && left >= 4) {
    if constexpr (sizeof(Out) == 4) {
      *reinterpret_cast<f32x4*>(p) = f32x4{y[0], y[1], y[2], y[3]};
    } else {
      v2u w;
      w[0] = pack_bf16x2(y[0], y[1]);
      w[1] = pack_bf16x2(y[2], y[3]);
      *reinterpret_cast<v2u*>(p) = w;
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (q >= left) continue;
    if constexpr (sizeof(Out) == 4) p[q] = y[q];
    else p[q] = to_bf16(y[q]);
  }
}

}  // namespace

// The launches of one translation unit each, of one step: A (square false) or B (true), and X.
// `pair`: float32 matrices.
hipError_t launch_ortho_tiles_symmetric(const Table& t, bool square, bool pair, int size, int turn, const OrthoStep& p,
                                        hipStream_t s);
// `left`: steps that follow.
hipError_t launch_ortho_tiles_update(const Table& t, bool pair, int left, int size, int turn, const OrthoStep& p, hipStream_t s);
hipError_t launch_ortho_small(const Table& t, int kind, bool pair, bool last, int turn, const OrthoStep& p, hipStream_t s);

}  // namespace vtrace
