// The contraction at the heart of the vocabulary layer's kernels: 256 x 256 tiles
// on the matrix cores (gfx950, wave64).
//
// All three products of the layer are C[m, n] = sum_k A(m, k) B(n, k) with bfloat16
// operands and float32 accumulation:
//   logits    m: token, n: step, k: hidden unit   (both operands have k innermost)
//   d_weight  m: hidden unit, n: token, k: step   (both have k outermost)
//   d_hidden  m: hidden unit, n: step, k: token   (A outermost, B innermost)
// A workgroup of eight waves computes a 256 x 256 tile in steps of 64 along k; wave
// (wm, wn) = (wave % 2, wave / 2) holds a 128 x 64 piece in registers, as 8 x 4 tiles
// of a 16x16x32 MFMA.  The next step's operands are copied from memory straight into
// the other half of LDS while this one's are multiplied.
//
// LDS.  A direct copy writes a wave's 64 16-byte vectors to consecutive addresses, so
// the order of a tile in LDS is set by which vectors the lanes ask for.
//   k innermost ("along"): rows of 64 k, 128 bytes; vector c of row r lies in slot
//   c ^ f(r).  A fragment is one 16-byte read.
//   k outermost ("across"): 64 rows (one for each k) of 256, 512 bytes; the 32-byte
//   piece p of row k lies at p ^ f(k).  A fragment is two transposing reads: each gives
//   lane (s, g) column s of four of its rows.
// With f(r) = bits 0, 1 and 3 of r the 64 lanes of each kind of read fall on all banks
// evenly.
#pragma once

#include "device_common.hpp"
#include "vocab.hpp"
#include "wave_ops.hpp"

namespace vtrace {
namespace {

constexpr int kTile = 256;
constexpr int kTileK = 64;
constexpr int kGemmThreads = 512;
constexpr int kOperandBytes = kTile * kTileK * 2;
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kGemmLds = 2 * kStageBytes;
constexpr int kWaveM = 128, kWaveN = 64;
constexpr int kMT = kWaveM / 16, kNT = kWaveN / 16;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t Rsrc;
typedef __attribute__((address_space(3))) void LdsVoid;

constexpr int kRawBufferFlags = 0x00020000;      // raw buffer, 32-bit elements, no swizzle
constexpr uint32_t kOutOfRange = 0x80000000u;    // at or beyond the end of every descriptor: reads 0
constexpr int64_t kMostRecords = 0x7fffffff;
constexpr float kLog2eF = 1.44269504088896340736f;

__device__ __forceinline__ Rsrc make_rsrc(const void* base, int64_t left) {
  const int64_t n = left < 0 ? 0 : (left < kMostRecords ? left : kMostRecords);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, static_cast<int>(n), kRawBufferFlags);
}

// 16 bytes a lane, straight into LDS: a wave's 64 vectors one after the other.
__device__ __forceinline__ void copy_to_lds(Rsrc r, char* lds, uint32_t offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsVoid*)lds, 16, offset, 0, 0, 0);
}

__device__ __forceinline__ int swizzle_of(int r) { return (r & 3) | ((r >> 1) & 4); }

// Copies one operand's tiles of kRows x 64 to LDS (by kWaves waves), step after step along k.  `base` and
// `left` (bytes to the array's end) move with the steps; vectors outside the operand
// are asked for beyond the end and arrive as zeros.
template <int kRows = kTile, int kWaves = kGemmThreads / kWave>
struct Loader {
  static constexpr int kCopyRows = 8 * kWaves;            // "along": of one copy by all threads
  static constexpr int kCopies = kRows / kCopyRows;       // of a thread and step
  static constexpr int kCopyBytes = 1024 * kWaves;
  const char* base;
  int64_t left;
  int64_t step;       // bytes per step of 64 k
  uint32_t off[kCopies];
  // "along" only: the lane's first k of a step, and where k ends.
  int lane_k, k, k_end;
  // After `first` steps the operand starts again at `again` (the low parts of G).
  int done, first;
  const char* again;
  int64_t again_left;

  __device__ __forceinline__ void start(const void* p, int64_t bytes) {
    base = static_cast<const char*>(p);
    left = bytes;
    done = 0;
    first = -1;
    k = 0;
  }
  __device__ __forceinline__ void restart_after(int steps, const void* p, int64_t bytes) {
    first = steps;
    again = static_cast<const char*>(p);
    again_left = bytes;
  }

  // k innermost: row_offset(r) is row r's byte offset from `p`, or kOutOfRange.
  template <typename F>
  __device__ __forceinline__ void along(const void* p, int64_t bytes, int ks, int wave, int lane, F row_offset) {
    start(p, bytes);
    step = kTileK * 2;
    k_end = ks;
    const int r0 = wave * 8 + lane / 8;
    const int c = (lane % 8) ^ swizzle_of(r0);
    lane_k = c * 8;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const uint32_t o = row_offset(i * kCopyRows + r0);
      off[i] = o == kOutOfRange ? o : o + c * 16;
    }
  }
  // k outermost: rows of `pitch` elements, the tile's columns from `p`, `width` of them in the array.
  __device__ __forceinline__ void across(const void* p, int64_t bytes, int64_t pitch, int64_t width, int wave,
                                         int lane) {
    static_assert(kRows == kTile && kWaves == 8, "rows of 512 bytes in LDS, 16 a copy");
    start(p, bytes);
    step = kTileK * 2 * pitch;
    k_end = 0x7fffffff;
    lane_k = 0;
    const int r0 = wave * 2 + lane / 32;
    const int slot = lane % 32;
    const int c = (((slot >> 1) ^ swizzle_of(r0)) << 1) | (slot & 1);
#pragma unroll
    for (int i = 0; i < kCopies; ++i)
      off[i] = c * 8 < width ? static_cast<uint32_t>((i * 16 + r0) * pitch * 2) + c * 16 : kOutOfRange;
  }
  __device__ __forceinline__ void copy(char* lds, int wave) {
    if (done == first) {
      base = again;
      left = again_left;
      k = 0;
    }
    const Rsrc r = make_rsrc(base, left);
    // The last step of an operand whose k is no multiple of 64 ends inside a row.
    const bool cut = k + kTileK > k_end && k + lane_k >= k_end;
#pragma unroll
    for (int i = 0; i < kCopies; ++i)
      copy_to_lds(r, lds + i * kCopyBytes + wave * 1024, cut ? kOutOfRange : off[i]);
    base += step;
    left -= step;
    k += kTileK;
    ++done;
  }
};

// Where a lane reads its fragments of an operand: byte offsets in the operand's half
// of a stage.  kTransposed: "across".  kPaired ("along"): tiles 2p and 2p + 1 together
// give lane group g the rows 32p + 8g .. 32p + 8g + 7 in its accumulators, four of each
// (so that eight consecutive results are one 16-byte store).
template <bool kTransposed, bool kPaired, int kTiles>
struct Reader {
  int at[kTransposed ? kTiles : 2];

  __device__ __forceinline__ void start(int first_row, int s, int g) {
    if constexpr (kTransposed) {
      const int k = 8 * g + s / 4;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
        at[t] = k * (kTile * 2) + (((first_row / 16 + t) ^ swizzle_of(k)) * 32) + (s % 4) * 8;
    } else {
      const int r = first_row + (kPaired ? 8 * (s / 4) + s % 4 : s);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) at[kk] = r * 128 + (((kk * 4 + g) ^ swizzle_of(r)) * 16);
    }
  }
  __device__ __forceinline__ bf16x8 read(const char* lds, int tile, int kk) const {
    if constexpr (kTransposed) {
      typedef __attribute__((address_space(3))) s16x4* LdsVec;
      const char* p = lds + at[tile] + kk * (32 * kTile * 2);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVec)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVec)(p + 4 * kTile * 2));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int row = kPaired ? 32 * (tile / 2) + 4 * (tile % 2) : 16 * tile;
      return *reinterpret_cast<const bf16x8*>(lds + at[kk] + row * 128);
    }
  }
};

// vmcnt(0) and lgkmcnt(0): the copies into LDS have arrived and this wave's reads are done.
constexpr int kWaitAll = 0x0070;

__device__ __forceinline__ void stage_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(kWaitAll);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// acc += A B over `steps` steps of 64 k.  kSteps of the two stages: a wave passes the
// barrier when its own copies into this stage have arrived and its reads of the other
// are done, so after the barrier this stage is whole and the other free.
template <bool kAAcross, bool kBAcross>
__device__ __forceinline__ void contract(Loader<>& la, Loader<>& lb, int steps, char* lds, int wave, int lane,
                                         f32x4 (&acc)[kMT][kNT]) {
  const int s = lane % 16, g = lane / 16;
  Reader<kAAcross, !kAAcross, kMT> ra;
  Reader<kBAcross, false, kNT> rb;
  ra.start((wave % 2) * kWaveM, s, g);
  rb.start((wave / 2) * kWaveN, s, g);
  if (steps > 0) {
    la.copy(lds, wave);
    lb.copy(lds + kOperandBytes, wave);
  }
  for (int it = 0; it < steps; ++it) {
    char* cur = lds + (it & 1) * kStageBytes;
    char* next = lds + ((it & 1) ^ 1) * kStageBytes;
    stage_barrier();
    if (it + 1 < steps) {
      la.copy(next, wave);
      lb.copy(next + kOperandBytes, wave);
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      bf16x8 a[kMT], b[kNT];
#pragma unroll
      for (int m = 0; m < kMT; ++m) a[m] = ra.read(cur, m, kk);
#pragma unroll
      for (int n = 0; n < kNT; ++n) b[n] = rb.read(cur + kOperandBytes, n, kk);
#pragma unroll
      for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int n = 0; n < kNT; ++n)
          acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[m], b[n], acc[m][n], 0, 0, 0);
    }
  }
}

// Sums (or maxima) over the four lane groups, the same in all of them.
template <typename Op>
__device__ __forceinline__ float over_groups(float x, Op op) {
  const v2u p = __builtin_bit_cast(
      v2u, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = op(__uint_as_float(p.x), __uint_as_float(p.y));
  const v2u q = __builtin_bit_cast(
      v2u, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return op(__uint_as_float(q.x), __uint_as_float(q.y));
}
__device__ __forceinline__ float group_max(float x) {
  return over_groups(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float group_sum(float x) {
  return over_groups(x, [](float a, float b) { return a + b; });
}

// Where a token's logit starts: its bias.  Behind the vocabulary's end, and for a bias
// so low that the logit's scaling could overflow, the token is ruled out.  (Without a bias
// the buffer is empty and reads 0.)
constexpr float kRuledOut = -1e37f;
__device__ __forceinline__ float start_of_logit(const VocabArgs& a, int64_t v) {
  const Rsrc bias = make_rsrc(a.bias, a.bias ? a.V * 4 : 0);
  const float b = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(bias, static_cast<uint32_t>(v) * 4, 0, 0));
  return v >= a.V || b < kRuledOut ? -INFINITY : b;
}
// A token ruled out adds p log p = 0, not 0 * -inf.
constexpr float kLeastLog = -1e30f;

// A workgroup's tile: `wide` x `deep` tiles, the id numbered so that workgroups that
// run together on one XCD share operands in its L2 (groups of 8 tiles along `wide`,
// then along `deep`).
struct TileAt {
  int64_t wide, deep;
};
__device__ __forceinline__ TileAt tile_at(int64_t id, int64_t wide, int64_t deep) {
  constexpr int64_t kGroup = 8;
  const int64_t per = kGroup * deep;
  const int64_t grp = id / per, in = id % per;
  const int64_t first = grp * kGroup;
  const int64_t n = wide - first < kGroup ? wide - first : kGroup;
  return {first + in % n, in / n};
}

}  // namespace
}  // namespace vtrace
