// The contraction at the heart of the vocabulary layer's kernels: 256 x 256 tiles
// on the matrix cores (gfx950, wave64).
//
// All three products of the layer are C[m, n] = sum_k A(m, k) B(n, k) with bfloat16
// operands and float32 accumulation:
//   logits    m: token, n: step, k: hidden unit   (both operands have k innermost)
//   d_weight  m: hidden unit, n: token, k: step   (both have k outermost)
//   d_hidden  m: hidden unit, n: step, k: token   (A outermost, B innermost)
// A workgroup of four waves computes a 256 x 256 tile in steps of 64 along k; wave
// (wm, wn) = (wave % 2, wave / 2) holds a 128 x 128 piece in registers, as 8 x 8 tiles
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
constexpr int kGemmThreads = 256;
constexpr int kOperandBytes = kTile * kTileK * 2;
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kGemmLds = 2 * kStageBytes;
constexpr int kWaveM = 128, kWaveN = 128;
constexpr int kMT = kWaveM / 16, kNT = kWaveN / 16;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t Rsrc;
typedef __attribute__((address_space(3))) void LdsVoid;

constexpr int kRawBufferFlags = 0x00020000;      // raw buffer, 32-bit elements, no swizzle
constexpr uint32_t kOutOfRange = 0x80000000u;    // at or beyond the end of every descriptor: reads 0
constexpr float kLog2eF = 1.44269504088896340736f;

// A descriptor of `left` bytes from base on (none if negative), held in scalar registers:
// every wave of a workgroup forms the same one.
__device__ __forceinline__ Rsrc make_rsrc(const void* base, int64_t left) {
  const int beyond = static_cast<int>(left >> 31);  // 32-bit comparisons stay on the scalar unit
  const int n = beyond == 0 ? static_cast<int>(left) : beyond < 0 ? 0 : 0x7fffffff;
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(static_cast<uint64_t>(hi) << 32 | lo), 0,
                                           __builtin_amdgcn_readfirstlane(n), kRawBufferFlags);
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
  bool cut;
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
    static_assert(kRows == kTile, "rows of 512 bytes in LDS");
    start(p, bytes);
    step = kTileK * 2 * pitch;
    k_end = 0x7fffffff;
    lane_k = 0;
    const int slot = lane % 32;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r = i * 2 * kWaves + wave * 2 + lane / 32;
      const int c = (((slot >> 1) ^ swizzle_of(r)) << 1) | (slot & 1);
      off[i] = c * 8 < width ? static_cast<uint32_t>(r * pitch * 2) + c * 16 : kOutOfRange;
    }
  }
  // One step's copies: the descriptor, then each of them.  Behind the last step they may go
  // on with `more` false: nothing is read, zeros arrive.
  __device__ __forceinline__ Rsrc begin(bool more = true) {
    if (done == first) {
      base = again;
      left = again_left;
      k = 0;
    }
    const Rsrc r = make_rsrc(base, more ? left : 0);
    // The last step of an operand whose k is no multiple of 64 ends inside a row.
    cut = k + kTileK > k_end && k + lane_k >= k_end;
    base += step;
    left -= step;
    k += kTileK;
    ++done;
    return r;
  }
  __device__ __forceinline__ void copy(Rsrc r, char* lds, int wave, int i) const {
    copy_to_lds(r, lds + i * kCopyBytes + wave * 1024, cut ? kOutOfRange : off[i]);
  }
  __device__ __forceinline__ void copy(char* lds, int wave) {
    const Rsrc r = begin();
#pragma unroll
    for (int i = 0; i < kCopies; ++i) copy(r, lds, wave, i);
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

// c += a b.  As an instruction of our own so that the accumulators stay in the accumulation
// registers: the compiler's allocation moves them to and fro (three moves an MFMA).  It knows
// nothing of its latency: see settle().
__device__ __forceinline__ void mfma(f32x4& c, bf16x8 a, bf16x8 b) {
  asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// What a wave does between two barriers: it multiplies the second half of a step (a1, b1)
// and reads the first half of the next from `from`, multiplies that and reads the second,
// while its copies of the step after go to `to`.  The two stages do not overlap, and
// __restrict says so: the compiler otherwise waits for every copy in flight before a read.
template <bool kAAcross, bool kBAcross>
struct Contraction {
  Reader<kAAcross, !kAAcross, kMT> ra;
  Reader<kBAcross, false, kNT> rb;
  bf16x8 a0[kMT], b0[kNT], a1[kMT], b1[kNT];

  // Two of a half's 16 fragments.
  __device__ __forceinline__ void read(const char* from, int kk, int i, bf16x8 (&a)[kMT], bf16x8 (&b)[kNT]) {
    if (i < kNT / 2) {
      b[2 * i] = rb.read(from + kOperandBytes, 2 * i, kk);
      b[2 * i + 1] = rb.read(from + kOperandBytes, 2 * i + 1, kk);
    } else {
      a[2 * i - kNT] = ra.read(from, 2 * i - kNT, kk);
      a[2 * i - kNT + 1] = ra.read(from, 2 * i - kNT + 1, kk);
    }
  }
  template <bool kFirst>
  __device__ __forceinline__ void step(char* __restrict to, const char* __restrict from, Loader<>& la, Loader<>& lb,
                                       bool more, int wave, f32x4 (&acc)[kMT][kNT]) {
    const Rsrc da = la.begin(more), db = lb.begin(more);
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      read(from, 0, m, a0, b0);
      la.copy(da, to, wave, m);
      lb.copy(db, to + kOperandBytes, wave, m);
      if constexpr (!kFirst) {
#pragma unroll
        for (int n = 0; n < kNT; ++n) mfma(acc[m][n], a1[m], b1[n]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      read(from, 1, m, a1, b1);
#pragma unroll
      for (int n = 0; n < kNT; ++n) mfma(acc[m][n], a0[m], b0[n]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// acc += A B over `steps` steps of 64 k.  A step's two halves of 32 k take turns in
// registers: while one is multiplied the other is read.  A wave passes the barrier when it
// has read all of a step and its copies of the next have arrived, so behind it the next
// stage is whole and this one free.
template <bool kAAcross, bool kBAcross>
__device__ __forceinline__ void contract(Loader<>& la, Loader<>& lb, int steps, char* lds, int wave, int lane,
                                         f32x4 (&acc)[kMT][kNT]) {
  if (steps <= 0) return;
  Contraction<kAAcross, kBAcross> c;
  c.ra.start((wave % 2) * kWaveM, lane % 16, lane / 16);
  c.rb.start((wave / 2) * kWaveN, lane % 16, lane / 16);
  la.copy(lds, wave);
  lb.copy(lds + kOperandBytes, wave);
  stage_barrier();
  c.template step<true>(lds + kStageBytes, lds, la, lb, 1 < steps, wave, acc);
  for (int it = 1; it < steps; ++it) {
    stage_barrier();
    c.template step<false>(lds + ((it + 1) & 1) * kStageBytes, lds + (it & 1) * kStageBytes, la, lb, it + 1 < steps, wave,
                           acc);
  }
#pragma unroll
  for (int m = 0; m < kMT; ++m)
#pragma unroll
    for (int n = 0; n < kNT; ++n) mfma(acc[m][n], c.a1[m], c.b1[n]);
  // The last copies (of nothing) have ended, and the last products are written.
  __builtin_amdgcn_s_waitcnt(kWaitAll);
  asm volatile("s_nop 15\n\ts_nop 15"
               : "+a"(acc[7][0]), "+a"(acc[7][1]), "+a"(acc[7][2]), "+a"(acc[7][3]), "+a"(acc[7][4]), "+a"(acc[7][5]),
                 "+a"(acc[7][6]), "+a"(acc[7][7]));
  __builtin_amdgcn_sched_barrier(0);
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
