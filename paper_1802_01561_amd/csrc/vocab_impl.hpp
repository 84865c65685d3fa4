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
// A step of 64 k takes 1.56 us on all CUs, 1.375 PFLOP/s (large products of the vendor's
// library 1.45 to 1.49), with the matrix units busy 54 to 64% of it.  What bounds it are the
// copies, 64 KB a CU and step, 10.5 TB/s from the L2s with 80% hits: without them a timing copy
// took 22 to 28% less, without the reads of LDS too 35 to 41%.  A tile costs 7 to 14 us more:
// filling and draining the pipeline, and its stores, which all CUs make at about the same time
// (a timing copy without those of G took 9% less, one without its exponentials as long).  Waiting
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

// The same but for the last kYounger vector memory operations (they complete in order).
constexpr int wait_but(int younger) { return (younger & 15) | (younger >> 4) << 14 | kWaitAll; }

template <int kYounger = 0>
__device__ __forceinline__ void stage_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(wait_but(kYounger));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// c += a b.  As an instruction of our own so that the accumulators stay in the accumulation
// registers: the compiler's allocation moves them to and fro (three moves an MFMA).  It knows
// nothing of its latency: Contraction::end waits for the last.
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

// What a wave does between two barriers.  Of a step's two halves of 32 k one is multiplied
// while the other is read to registers, and copies go out among the products: the path into
// LDS takes a 16-byte vector of four lanes at a time, and copies in a bunch hold up the wave
// (all of a step's within the first quarter, the first half: 11.2, 10.3 ms of the largest
// gradient).  What is read and what is copied to do not overlap, and __restrict says so: the
// compiler otherwise waits for every copy in flight before a read.
template <bool kAAcross, bool kBAcross, int kSize>
struct Contraction {
  static constexpr int kMT = kSize / 32, kNT = kSize / 32, kOperandBytes = operand_bytes(kSize);
  Reader<kAAcross, !kAAcross, kMT, kSize> ra;
  Reader<kBAcross, false, kNT, kSize> rb;
  bf16x8 a0[kMT], b0[kNT], a1[kMT], b1[kNT];

  // The first half finds none before it: zeros (64 products, against a branch around each).
  __device__ __forceinline__ void start(int wave, int lane) {
    ra.start((wave % 2) * (kSize / 2), lane % 16, lane / 16);
    rb.start((wave / 2) * (kSize / 2), lane % 16, lane / 16);
#pragma unroll
    for (int i = 0; i < kMT; ++i) a1[i] = bf16x8{};
#pragma unroll
    for (int i = 0; i < kNT; ++i) b1[i] = bf16x8{};
  }
  // The last half, and the time until the last products are written.
  __device__ __forceinline__ void end(Accumulators<kSize>& acc) {
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
      for (int n = 0; n < kNT; ++n) mfma(acc[m][n], a1[m], b1[n]);
#pragma unroll
    for (int n = 0; n < kNT; ++n) asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[kMT - 1][n]));
    __builtin_amdgcn_sched_barrier(0);
  }

  // Two of a half's fragments.
  __device__ __forceinline__ void read(const char* from_a, const char* from_b, int kk, int i, bf16x8 (&a)[kMT],
                                       bf16x8 (&b)[kNT]) {
    if (i < kNT / 2) {
      b[2 * i] = rb.read(from_b, 2 * i, kk);
      b[2 * i + 1] = rb.read(from_b, 2 * i + 1, kk);
    } else {
      a[2 * i - kNT] = ra.read(from_a, 2 * i - kNT, kk);
      a[2 * i - kNT + 1] = ra.read(from_a, 2 * i - kNT + 1, kk);
    }
  }
  // Both halves of a step: the second half of the step before (a1, b1) and the first of this
  // one are multiplied, both of this one read from `from`, and the next step copied to `to`.
  // Operands "along": 12 copies with the first half, 4 with the second, which have less time to
  // arrive (logits of 6200 steps, H = 4096, V = 131072 5.23 ms; 16 and 0 5.42, 10 and 6 5.40).
  // "Across" all with the first half (d_weight of the largest gradient 2% faster so).
  __device__ __forceinline__ void step(char* __restrict to, const char* __restrict from, Loader<kSize>& la,
                                       Loader<kSize>& lb, bool more, int wave, Accumulators<kSize>& acc) {
    const Rsrc da = la.begin(more), db = lb.begin(more);
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      read(from, from + kOperandBytes, 0, m, a0, b0);
      la.copy(da, to, wave, m);
      if constexpr (kBAcross) lb.copy(db, to + kOperandBytes, wave, m);
      else if (m % 2 == 0) lb.copy(db, to + kOperandBytes, wave, m / 2);
#pragma unroll
      for (int n = 0; n < kNT; ++n) mfma(acc[m][n], a1[m], b1[n]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      read(from, from + kOperandBytes, 1, m, a1, b1);
      if (!kBAcross && m < kMT / 2) lb.copy(db, to + kOperandBytes, wave, kMT / 2 + m);
#pragma unroll
      for (int n = 0; n < kNT; ++n) mfma(acc[m][n], a0[m], b0[n]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // The same for half a step, kk: the other half in registers (a, b) is multiplied, this one
  // read to (na, nb), and a whole step of one operand copied, or (kHalves) two halves.
  template <bool kHalves>
  __device__ __forceinline__ void half(char* __restrict to, char* __restrict then_to, const char* __restrict from_a,
                                       const char* __restrict from_b, const Loader<kSize>& load, Rsrc d, Rsrc then_d,
                                       int kk, int wave, const bf16x8 (&a)[kMT], const bf16x8 (&b)[kNT],
                                       bf16x8 (&na)[kMT], bf16x8 (&nb)[kNT], Accumulators<kSize>& acc) {
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      read(from_a, from_b, kk, m, na, nb);
      if (!kHalves || m < kMT / 2) load.copy(d, to, wave, m);
      else load.copy(then_d, then_to, wave, m - kMT / 2);
#pragma unroll
      for (int n = 0; n < kNT; ++n) mfma(acc[m][n], a[m], b[n]);
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

// acc += A B over the job's steps, both operands "along" or both "across".  A wave passes the barrier when it
// has read all of a step and its copies of the next have arrived, so behind it the next stage
// is whole and this one free.
//
// The first step's copies are under way when this is called (to stage `parity`).  With the
// last step's products go the copies of the next tile's first: next() makes `job` that
// tile's, and what follows the contraction hides their latency.
template <bool kAcross, int kSize, typename Next>
__device__ __forceinline__ void contract(Job<kSize>& job, char* lds, int& parity, int wave, int lane,
                                         Accumulators<kSize>& acc, Next next) {
  constexpr int kStage = 2 * operand_bytes(kSize);
  const int steps = job.steps;
  Contraction<kAcross, kAcross, kSize> c;
  c.start(wave, lane);
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
  c.end(acc);
}

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

// One operand's copies, tile after tile of this workgroup and ahead of the products: `left`
// steps (or halves) of its tile are still to come.
template <int kSize>
struct Feed {
  Loader<kSize> load;
  Tiles tiles;
  int left = 0;

  __device__ __forceinline__ explicit Feed(const Tiles& t) : tiles(t) {}
  // The next one's descriptor; start() aims the loader at a tile and returns its steps.  Behind
  // the last tile nothing is read, and zeros arrive.
  template <typename Start>
  __device__ __forceinline__ Rsrc begin(Start start) {
    if (left == 0) {
      left = 0x7fffffff;
      load.aim(nullptr, 0);
      if (tiles.any()) left = start(*this);
      tiles.next();
    }
    --left;
    return load.begin();
  }
};

// acc += A B over `steps` steps, A "across", so that its halves of a step are apart in LDS, and
// B "along".  The copies are spread evenly over the products: while the first half of step i is
// read, those of B's step i + 1 go out, and while the second is, those of A's second half of step
// i + 1 and first of i + 2 (to where halves were read just before).  Each has half a step of
// products or more to arrive, and a wave waits for no younger ones.
//   LDS: two steps of A, then two of B.  In flight when a tile begins: A's first half, B's first
// step, A's next two halves.
//   Against one barrier a step, as in contract(): d_hidden of 843 ragged steps, H = 1000, V =
// 50021 (two products for float32, 98 steps a tile) 203 -> 172 us, where H is a power of two the
// same.  (d_weight, both operands "across": so 222 -> 213 us there, but 203 -> 215 for 3200 steps,
// H = 1024, V = 32768 and 1% longer for the largest gradient.)
template <int kSize, typename StartA, typename StartB>
__device__ __forceinline__ void contract_halves(int steps, Feed<kSize>& feed_a, Feed<kSize>& feed_b, char* lds,
                                                int& parity, int wave, int lane, Accumulators<kSize>& acc,
                                                StartA start_a, StartB start_b) {
  constexpr int kBytes = operand_bytes(kSize), kCopies = kSize / 32;
  Contraction<true, false, kSize> c;
  c.start(wave, lane);
  int it = 0;
  do {
    char* const a = lds + parity * kBytes;
    char* const b = a + 2 * kBytes;
    char* const next_a = lds + (parity ^ 1) * kBytes;
    char* const next_b = next_a + 2 * kBytes;
    stage_barrier<kCopies>();
    const Rsrc d = feed_b.begin(start_b);
    c.template half<false>(next_b, next_b, a, b, feed_b.load, d, d, 0, wave, c.a1, c.b1, c.a0, c.b0, acc);
    stage_barrier<kCopies + kCopies / 2>();
    const Rsrc d1 = feed_a.begin(start_a), d2 = feed_a.begin(start_a);
    c.template half<true>(next_a + kBytes / 2, a, a, b, feed_a.load, d1, d2, 1, wave, c.a0, c.b0, c.a1, c.b1, acc);
    parity ^= 1;
  } while (++it < steps);
  c.end(acc);
}
// What is in flight when the first tile begins.
template <int kSize, typename StartA, typename StartB>
__device__ __forceinline__ void start_halves(Feed<kSize>& feed_a, Feed<kSize>& feed_b, char* lds, int wave,
                                             StartA start_a, StartB start_b) {
  constexpr int kBytes = operand_bytes(kSize), kCopies = kSize / 32;
  for (int h = 0; h < 3; ++h) {
    const Rsrc a = feed_a.begin(start_a);
#pragma unroll
    for (int i = 0; i < kCopies / 2; ++i) feed_a.load.copy(a, lds + h * (kBytes / 2), wave, i);
    if (h == 0) {
      const Rsrc b = feed_b.begin(start_b);
#pragma unroll
      for (int i = 0; i < kCopies; ++i) feed_b.load.copy(b, lds + 2 * kBytes, wave, i);
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
// so low that the logit's scaling could overflow, the token is ruled out.  (A buffer without
// a bias is empty and reads 0.)
constexpr float kRuledOut = -1e37f;
__device__ __forceinline__ float start_of_logit(const VocabArgs& a, int64_t v) {
  const Rsrc bias = make_rsrc(a.bias, a.bias ? a.V * 4 : 0);
  const float b = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(bias, static_cast<uint32_t>(v) * 4, 0, 0));
  return v >= a.V || b < kRuledOut ? -INFINITY : b;
}
// A token ruled out adds p log p = 0, not 0 * -inf.
constexpr float kLeastLog = -1e30f;
// A logit's exponent about another one, in log2 units.  The difference comes first: scaled
// each for itself, logits near 1e10 (a finite mask's) round to hundreds of units off, and
// 2^hundreds overflows.
__device__ __forceinline__ float log2_ratio(float z, float about) { return (z - about) * kLog2eF; }

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
