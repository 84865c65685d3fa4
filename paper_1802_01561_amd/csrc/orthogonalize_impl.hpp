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

// What the tiles kernels' workgroups take one after the other: tiles, of which those from begin[s] to
// end[s] are split along k into pieces[s] (X's are not: their kernel took 1.4 to 2.8 times as long, with
// no tile split).
struct Units {
  static constexpr int kSplits = 2;
  int total;
  int begin[kSplits], end[kSplits], pieces[kSplits];
};
// Of float32 matrices' A and B in tiles of 256 none is: a tile of two matrices in two parts has no
// registers left for the sums of other pieces.
template <bool kPair, int kSize, int kKind>
constexpr bool kWhole = kPair && kSize == kTile && kKind == 1;
struct Unit {
  int tile, piece, pieces;
  int slot;     // of the piece's sums
  int counter;  // of the tile's pieces that are there
};
__host__ __device__ inline Unit unit_at(const Units& u, int id) {
  int tile = id, slot = 0, counter = 0;
  for (int s = 0; s < Units::kSplits; ++s) {
    if (tile < u.begin[s]) break;
    const int n = u.end[s] - u.begin[s], inside = tile - u.begin[s];
    if (inside < n * u.pieces[s]) {
      const int of = inside / u.pieces[s];
      return {u.begin[s] + of, inside - of * u.pieces[s], u.pieces[s], slot + inside, counter + of};
    }
    tile -= n * (u.pieces[s] - 1);
    slot += n * u.pieces[s];
    counter += n;
  }
  return {tile, 0, 1, 0, 0};
}

// As many as 4 KB of arguments hold.
struct Table {
  static constexpr int kMost = 38;
  Entry at[kMost];
  double* partials;
  char* sums;          // of the tiles' pieces
  unsigned* counters;  // zero between launches
  Units units[3];      // of X: its tiles
  int count;           // matrices of the tiles' kernels
  int few;             // behind them, those of few rows
  bool few_later;      // their results with the others' first A
  int few_chunks, few_block, few_blocks;
  int total_partials, total_blocks, total_tiles[3];
  int size[3];  // of the tiles of A, B and X
  float epsilon;
  bool twos;   // the first two steps at once
  bool small;  // the small matrices' kernels, which keep X^T as well
};

// A symmetric matrix C = of_m M + of_n N + of_mn M N from those numbered m and n, which commute; or
// (A) from X.
struct Product {
  int out, m, n;
  float of_m, of_n, of_mn;
};
// The steps of the matrices of few rows.
struct FewSteps {
  OrthoStep at[kOrthoMostSteps];
  int count;
};
static_assert(sizeof(Table) + sizeof(Product) + sizeof(FewSteps) + 16 <= 4096, "kernel arguments");
// What a product is of: X and X^T, one matrix, or two.
enum { kOfX = 0, kOfOne = 1, kOfTwo = 2 };

constexpr int kSymmetric = 3;

struct Pieces {
  float* x;           // [r, pc] X, of float32 matrices
  uint16_t* low;      // [r, pc] of bfloat16 ones what the operand leaves of X
  uint16_t* from[2];  // [r, pc] X as an operand: high and (float32 matrices) low parts
  uint16_t* to[2];    // [r, pc] the same behind this step
  // Symmetric matrices (A, B and what is made of them): [r, pr] without the diagonal, and that, [r].
  uint16_t* sym[kSymmetric][2];
  float* diagonal[kSymmetric];
};
__host__ __device__ inline int64_t round_up(int64_t n, int64_t k) { return (n + k - 1) / k * k; }
template <bool kPair>
__host__ __device__ inline int64_t piece_bytes(int64_t r, int64_t pr, int64_t pc) {
  constexpr int kParts = kPair ? 2 : 1;
  return r * pc * (2 * kParts + 2 * 2 * kParts) + kSymmetric * (r * pr * 2 * kParts + round_up(r * 4, 256));
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
  }
  at += 2 * kParts * x;
#pragma unroll
  for (int m = 0; m < kSymmetric; ++m) {
#pragma unroll
    for (int k = 0; k < 2; ++k) p.sym[m][k] = reinterpret_cast<uint16_t*>(at + (m * kParts + (kPair ? k : 0)) * a);
    p.diagonal[m] = reinterpret_cast<float*>(at + kSymmetric * kParts * a + m * round_up(static_cast<int64_t>(t.r) * 4, 256));
  }
  return p;
}
// One of them, whichever it is (an index into an array in registers would put it into memory).
template <bool kPair>
__device__ __forceinline__ uint16_t* symmetric_of(const Entry& t, const Pieces& p, int m, int k) {
  return p.sym[0][k] + static_cast<int64_t>(m) * t.r * t.pr * (kPair ? 2 : 1);
}
__device__ __forceinline__ float* diagonal_of(const Entry& t, const Pieces& p, int m) {
  return p.diagonal[0] + m * (round_up(static_cast<int64_t>(t.r) * 4, 256) / 4);
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

// The last entry (of those from `from` on, `count` of them) whose first number is not above `id`.
template <typename First>
__device__ __forceinline__ int entry_of(const Table& t, int id, First first, int from, int count) {
  int lo = from, hi = from + count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (first(t.at[mid]) <= id) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
template <typename First>
__device__ __forceinline__ int entry_of(const Table& t, int id, First first) {
  return entry_of(t, id, first, 0, t.count);
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

// bfloat16 matrices: X as what its operand leaves of it beside the operand, times 2^11, at most half a
// step of the operand: float16 without leaving its range up to 2^15, nor its digits where the
// operand itself is below float16's (norms below epsilon).
constexpr float kScaleLeft = 2048.0f;
__device__ __forceinline__ v2u left4(const float (&y)[4], v2u high) {
  float left[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) left[q] = (y[q] - high_of(high[q / 2], q % 2)) * kScaleLeft;
  return high4(left);
}
__device__ __forceinline__ float whole_of(v2u high, v2u left, int q) {
  return fmaf(high_of(left[q / 2], q % 2), 1.0f / kScaleLeft, high_of(high[q / 2], q % 2));
}

// An element of a product beside the diagonal, and on it, from its factors' elements there (on the
// diagonal: dm, dn) and the sum of O O'.
template <int kOf>
__device__ __forceinline__ float product_off(const Product& f, float m, float n, float dm_i, float dn_j, float oo) {
  if constexpr (kOf == kOfOne) return fmaf(m, fmaf(f.of_mn, dm_i + dn_j, f.of_m), f.of_mn * oo);
  else return fmaf(m, fmaf(f.of_mn, dn_j, f.of_m), fmaf(n, fmaf(f.of_mn, dm_i, f.of_n), f.of_mn * oo));
}
template <int kOf>
__device__ __forceinline__ float product_diagonal(const Product& f, float dm, float dn, float oo) {
  const float linear = kOf == kOfOne ? f.of_m * dm : fmaf(f.of_m, dm, f.of_n * dn);
  return linear + f.of_mn * fmaf(dm, dn, oo);
}

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
// Eight: `vectors` where they are whole ones of 16 bytes.
template <typename Out>
__device__ __forceinline__ void store_results(Out* p, const float (&y)[2][4], int left, bool vectors) {
  if constexpr (sizeof(Out) == 2) {
    if (vectors && left >= 8) {
      *reinterpret_cast<v4u*>(p) = v4u{pack_bf16x2(y[0][0], y[0][1]), pack_bf16x2(y[0][2], y[0][3]), pack_bf16x2(y[1][0], y[1][1]),
                                       pack_bf16x2(y[1][2], y[1][3])};
      return;
    }
  }
  store_result(p, y[0], left, vectors);
  store_result(p + 4, y[1], left - 4, vectors);
}

}  // namespace

// The launches of one translation unit each: a symmetric matrix, or X <- of_x X + C X with the
// symmetric matrix numbered `by`.  `pair`: float32 matrices.
struct Update {
  int by;
  float of_x;
  bool last;
};
hipError_t launch_ortho_tiles_symmetric(const Table& t, int of, bool pair, int turn, const Product& p, hipStream_t s);
hipError_t launch_ortho_tiles_update(const Table& t, bool pair, int turn, const Update& u, hipStream_t s);
// `few`: of A from X, with the results of the matrices of few rows.
hipError_t launch_ortho_small_symmetric(const Table& t, int of, bool pair, int turn, const Product& p, const FewSteps* few, hipStream_t s);
hipError_t launch_ortho_small_update(const Table& t, bool pair, int turn, const Update& u, hipStream_t s);

}  // namespace vtrace
