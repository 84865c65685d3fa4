// The contraction at the heart of the vocabulary layer's kernels: 256 x 256 tiles (where
// there are few of those, 128 x 128) on the matrix cores (gfx950, wave64).
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
//
// Bound by the matrix cores: a step of 64 k takes 1.56 us on all CUs, 1.375 PFLOP/s (large
// products of the vendor's library 1.45 to 1.49).  A tile costs 7 to 14 us more: filling and
// draining the pipeline, and its stores, which all CUs make at about the same time (without
// those of G its kernel takes 836 us instead of 914, without its exponentials 914).  Waiting
// at the next tile's start for the copies alone and not for the stores behind them, stores
// past the caches, whole 256-byte rows by way of LDS, and row pitches off the powers of two
// changed nothing.
#pragma once

#include "device_common.hpp"
#include "vocab.hpp"
#include "wave_ops.hpp"

namespace vtrace {
namespace {

constexpr int kTile = 256, kSmallTile = 128;
constexpr int kTileK = 64;
constexpr int kGemmThreads = 256;
// Of a tile of kSize x kSize: an operand's bytes of a step, and two steps of both.
constexpr int operand_bytes(int size) { return size * kTileK * 2; }
constexpr int tile_lds(int size) { return 4 * operand_bytes(size); }

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// A wave's quarter of a tile.
template <int kSize>
using Accumulators = f32x4[kSize / 32][kSize / 32];
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

// Copies one operand's tiles of kRows x 64 to LDS (by kWaves waves), step after step along k.
// A lane's places in a tile are fixed once, along() or across(); aim() points the tile at an
// array, `base` and `left` (bytes to its end) moving with the steps.  Rows behind the array's
// end arrive as zeros.  Columns behind a row's end hold what comes next in memory: they are
// columns of the result that nobody stores.
template <int kRows = kTile, int kWaves = kGemmThreads / kWave>
struct Loader {
  static constexpr int kCopyRows = 8 * kWaves;            // "along": of one copy by all threads
  static constexpr int kCopies = kRows / kCopyRows;       // of a thread and step
  static constexpr int kCopyBytes = 1024 * kWaves;
  int64_t step;       // bytes per step of 64 k
  uint32_t off[kCopies];
  int lane_k;         // "along": the lane's first k of a step
  const char* base;
  int64_t left;
  int k, k_end;       // "along": where the step begins, and where k ends
  uint32_t cut;       // kOutOfRange, to be added to an offset, where this lane's k lie behind k_end
  // After `first` steps the operand starts again at `again` (the low parts of G).
  int done, first;
  const char* again;
  int64_t again_left;

  // k innermost, rows of `pitch` elements; rows from `rows` on are not read.
  __device__ __forceinline__ void along(int64_t pitch, int rows, int wave, int lane) {
    step = kTileK * 2;
    const int r0 = wave * 8 + lane / 8;
    const int c = (lane % 8) ^ swizzle_of(r0);
    lane_k = c * 8;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r = i * kCopyRows + r0;
      off[i] = r < rows ? static_cast<uint32_t>(r * pitch * 2) + c * 16 : kOutOfRange;
    }
  }
  // k outermost, rows of `pitch` elements.
  __device__ __forceinline__ void across(int64_t pitch, int wave, int lane) {
    constexpr int kSlots = kRows / 8, kWaveRows = kWave / kSlots;
    step = kTileK * 2 * pitch;
    lane_k = 0;
    const int slot = lane % kSlots;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r = (i * kWaves + wave) * kWaveRows + lane / kSlots;
      const int c = (((slot >> 1) ^ swizzle_of(r)) << 1) | (slot & 1);
      off[i] = static_cast<uint32_t>(r * pitch * 2) + c * 16;
    }
  }
  __device__ __forceinline__ void aim(const void* p, int64_t bytes, int ks = 0x7fffffff) {
    base = static_cast<const char*>(p);
    left = bytes;
    k = 0;
    k_end = ks;
    done = 0;
    first = -1;
  }
  __device__ __forceinline__ void restart_after(int steps, const void* p, int64_t bytes) {
    first = steps;
    again = static_cast<const char*>(p);
    again_left = bytes;
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
    cut = k + kTileK > k_end && k + lane_k >= k_end ? kOutOfRange : 0u;
    base += step;
    left -= step;
    k += kTileK;
    ++done;
    return r;
  }
  __device__ __forceinline__ void copy(Rsrc r, char* lds, int wave, int i) const {
    copy_to_lds(r, lds + i * kCopyBytes + wave * 1024, off[i] | cut);
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
template <bool kTransposed, bool kPaired, int kTiles, int kRows = kTile>
struct Reader {
  int at[kTransposed ? kTiles : 2];

  __device__ __forceinline__ void start(int first_row, int s, int g) {
    if constexpr (kTransposed) {
      const int k = 8 * g + s / 4;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
        at[t] = k * (kRows * 2) + (((first_row / 16 + t) ^ swizzle_of(k)) * 32) + (s % 4) * 8;
    } else {
      const int r = first_row + (kPaired ? 8 * (s / 4) + s % 4 : s);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) at[kk] = r * 128 + (((kk * 4 + g) ^ swizzle_of(r)) * 16);
    }
  }
  __device__ __forceinline__ bf16x8 read(const char* lds, int tile, int kk) const {
    if constexpr (kTransposed) {
      typedef __attribute__((address_space(3))) s16x4* LdsVec;
      const char* p = lds + at[tile] + kk * (32 * kRows * 2);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVec)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVec)(p + 4 * kRows * 2));
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
// nothing of its latency: contract() waits for the last.
__device__ __forceinline__ void mfma(f32x4& c, bf16x8 a, bf16x8 b) {
  asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// An accumulator's element, read where it is used: by itself the compiler moves all of a
// tile's into vector registers at once, which do not hold them.
__device__ __forceinline__ float element(const f32x4& c, int i) {
  float x;
  asm("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c[i]));
  return x;
}

// What a wave does between two barriers: it multiplies the second half of a step (a1, b1)
// and reads the first half of the next from `from`, multiplies that and reads the second,
// while its copies of the step after go to `to`.  The two stages do not overlap, and
// __restrict says so: the compiler otherwise waits for every copy in flight before a read.
//
// The copies are spread over the first half: four at a time instead of two cost 4%, as
// the path into LDS takes one 16-byte vector a lane at a time.  With both operands "along" a
// quarter of them goes with the second half (kSpread: logits of 6200 steps, H = 4096, V =
// 131072 5.42 -> 5.23 ms); d_weight, both "across", took 2% longer so.
template <bool kAAcross, bool kBAcross, int kSize>
struct Contraction {
  static constexpr int kMT = kSize / 32, kNT = kSize / 32, kOperandBytes = operand_bytes(kSize);
  static constexpr bool kSpread = !kAAcross && !kBAcross;
  Reader<kAAcross, !kAAcross, kMT, kSize> ra;
  Reader<kBAcross, false, kNT, kSize> rb;
  bf16x8 a0[kMT], b0[kNT], a1[kMT], b1[kNT];

  // Two of a half's fragments.
  __device__ __forceinline__ void read(const char* from, int kk, int i, bf16x8 (&a)[kMT], bf16x8 (&b)[kNT]) {
    if (i < kNT / 2) {
      b[2 * i] = rb.read(from + kOperandBytes, 2 * i, kk);
      b[2 * i + 1] = rb.read(from + kOperandBytes, 2 * i + 1, kk);
    } else {
      a[2 * i - kNT] = ra.read(from, 2 * i - kNT, kk);
      a[2 * i - kNT + 1] = ra.read(from, 2 * i - kNT + 1, kk);
    }
  }
  __device__ __forceinline__ void step(char* __restrict to, const char* __restrict from, Loader<kSize>& la,
                                       Loader<kSize>& lb, bool more, int wave, Accumulators<kSize>& acc) {
    const Rsrc da = la.begin(more), db = lb.begin(more);
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      read(from, 0, m, a0, b0);
      la.copy(da, to, wave, m);
      if constexpr (!kSpread) lb.copy(db, to + kOperandBytes, wave, m);
      else if (m % 2 == 0) lb.copy(db, to + kOperandBytes, wave, m / 2);
#pragma unroll
      for (int n = 0; n < kNT; ++n) mfma(acc[m][n], a1[m], b1[n]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      read(from, 1, m, a1, b1);
      if (kSpread && m < kMT / 2) lb.copy(db, to + kOperandBytes, wave, kMT / 2 + m);
#pragma unroll
      for (int n = 0; n < kNT; ++n) mfma(acc[m][n], a0[m], b0[n]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// A tile's contraction: where its operands start, and how many steps of 64 k it has (at
// least one; 0: there is no tile).
template <int kSize>
struct Job {
  Loader<kSize> a, b;
  int steps = 0;

  __device__ __forceinline__ void copy(char* stage, int wave) {
    a.copy(stage, wave);
    b.copy(stage + operand_bytes(kSize), wave);
  }
};

// acc += A B over the job's steps.  A step's two halves of 32 k take turns in registers:
// while one is multiplied the other is read.  A wave passes the barrier when it has read
// all of a step and its copies of the next have arrived, so behind it the next stage is
// whole and this one free.
//
// The first step's copies are under way when this is called (to stage `parity`).  With the
// last step's products go the copies of the next tile's first: next() makes `job` that
// tile's, and what follows the contraction hides their latency.
template <bool kAAcross, bool kBAcross, int kSize, typename Next>
__device__ __forceinline__ void contract(Job<kSize>& job, char* lds, int& parity, int wave, int lane,
                                         Accumulators<kSize>& acc, Next next) {
  constexpr int kMT = kSize / 32, kNT = kSize / 32, kStage = 2 * operand_bytes(kSize);
  const int steps = job.steps;
  Contraction<kAAcross, kBAcross, kSize> c;
  c.ra.start((wave % 2) * (kSize / 2), lane % 16, lane / 16);
  c.rb.start((wave / 2) * (kSize / 2), lane % 16, lane / 16);
  // The first step finds no second half before it: zeros (64 products, against a branch
  // around each of them).
#pragma unroll
  for (int i = 0; i < kMT; ++i) c.a1[i] = bf16x8{};
#pragma unroll
  for (int i = 0; i < kNT; ++i) c.b1[i] = bf16x8{};
  int it = 0;
  do {
    stage_barrier();
    bool more = true;
    if (it + 1 == steps) {
      next();
      more = job.steps > 0;
    }
    c.step(lds + (parity ^ 1) * kStage, lds + parity * kStage, job.a, job.b, more, wave, acc);
    parity ^= 1;
  } while (++it < steps);
#pragma unroll
  for (int m = 0; m < kMT; ++m)
#pragma unroll
    for (int n = 0; n < kNT; ++n) mfma(acc[m][n], c.a1[m], c.b1[n]);
  // The last products are written.
#pragma unroll
  for (int n = 0; n < kNT; ++n) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[kMT - 1][n]));
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
// so low that the logit's scaling could overflow, the token is ruled out.  (A buffer without
// a bias is empty and reads 0.)
constexpr float kRuledOut = -1e37f;
template <bool kBias = true>
__device__ __forceinline__ float start_of_logit(const VocabArgs& a, int64_t v) {
  if constexpr (!kBias) return v >= a.V ? -INFINITY : 0.0f;
  const Rsrc bias = make_rsrc(a.bias, a.bias ? a.V * 4 : 0);
  const float b = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(bias, static_cast<uint32_t>(v) * 4, 0, 0));
  return v >= a.V || b < kRuledOut ? -INFINITY : b;
}
// A token ruled out adds p log p = 0, not 0 * -inf.
constexpr float kLeastLog = -1e30f;

constexpr int kCus = 256;

// Workgroups of a launch over tiles of kSize: as many as fit the CUs at a time (a tile of
// 256 fills a CU's LDS, one of 128 leaves room for another), each with every so many'th.
__host__ __device__ constexpr int resident_tiles(int size) { return size == kTile ? kCus : 2 * kCus; }
__host__ __device__ inline int64_t tiles_of(int64_t n, int size) { return (n + size - 1) / size; }
inline unsigned workgroups_of(int64_t tiles, int size) {
  return static_cast<unsigned>(tiles < resident_tiles(size) ? tiles : resident_tiles(size));
}
// us of a round of them over `steps` steps of 64 k.  640 steps, H = 256, V = 32768: logits 40
// us in two rounds of 256, 32 in three of 128; d_weight (float32) 47 in one half empty, 29 in a
// small one.  3200 steps, H = 1024: 261 in seven, 303 in thirteen small ones.
__host__ __device__ inline double round_cost(int size, int64_t steps) {
  return size == kTile ? 1.56 * static_cast<double>(steps) + 13.0 : 1.2 * static_cast<double>(steps) + 6.0;
}

// The tiles of this workgroup, one after the other.  Those that are worked on at a time are
// consecutive numbers, and those of one XCD are too.
struct Tiles {
  int total, at;

  __device__ __forceinline__ explicit Tiles(int64_t n) : total(static_cast<int>(n)) {
    at = static_cast<int>(xcd_tile(blockIdx.x, gridDim.x));
  }
  __device__ __forceinline__ bool any() const { return at < total; }
  __device__ __forceinline__ void next() { at += gridDim.x; }
};

// Tile number `id` of `wide` x `deep`: consecutive numbers share operands in an XCD's L2
// (8 tiles along `wide`, then along `deep`).
struct TileAt {
  int wide, deep;
};
__device__ __forceinline__ TileAt tile_at(int id, int wide, int deep) {
  constexpr int kGroup = 8;
  const unsigned per = kGroup * deep;
  const unsigned grp = static_cast<unsigned>(id) / per, in = static_cast<unsigned>(id) % per;
  const int first = grp * kGroup;
  const unsigned n = wide - first < kGroup ? wide - first : kGroup;
  return {first + static_cast<int>(in % n), static_cast<int>(in / n)};
}
}  // namespace
}  // namespace vtrace
