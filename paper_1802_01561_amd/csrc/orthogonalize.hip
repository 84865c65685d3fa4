// Matrices made nearly orthogonal by Newton-Schulz products: with X = G / max(|G|, epsilon),
// |G| the Frobenius norm, and `steps` times
//   A = X X^T,   B = b A + c A A,   X <- a X + B X,
// which takes every singular value s of X to a s + b s^3 + c s^5 and leaves the singular
// vectors.  X is kept with at most as many rows (r) as columns (c): a taller matrix is
// transposed when it is read, and back when the result is written.
//
// Numerics.  X is kept in float32, and the products' operands are float16, of fixed powers of
// two: singular values stay within a small range (the entry point checks the coefficients), so
// that bfloat16's exponents are not needed and float16's three more bits are had for
// nothing (bfloat16 operands: results 1.3e-2 to 3e-2 off, in relation to their norm).  The
// diagonals of A and B are far larger than the rest where the rows are nearly orthogonal; they
// are kept out of the operands, in float32:
//   with A = D + O:  B = b (D + O) + c (D D + D O + O D + O O),   B X = diag(B) X + offdiag(B) X,
// where only O O and offdiag(B) X are products on the matrix cores (with the diagonals in the
// operands 1.7e-3 to 2.8e-3 off, without 2e-4 to 7e-4, and one rounding to bfloat16 is 1.7e-3).
// Float32 matrices have operands in two parts, high + low, and three products for each: 5e-7
// to 3e-6 off, from the float32 sums (a library's float32 products 2e-6 to 7e-5: small singular
// values grow by 3.44 a step, and rounding errors beside the largest with them).
//
// A and B are symmetric: their tiles on and below the diagonal are computed, and stored twice.
#include "contraction.hpp"
#include "orthogonalize.hpp"

#include <algorithm>
#include <cmath>

namespace vtrace {
namespace {

// The operands' scales: X 2^12, A and B 2^13.
constexpr float kScaleX = 4096.0f, kScaleA = 8192.0f;
// A's and B's entries beside the diagonal are at most half the range of their eigenvalues.
constexpr double kMostSingular = 3.5, kMostRange = 12.0;

constexpr int kNormThreads = 256;
constexpr int64_t kNormChunk = 16384;  // least elements of a partial sum, a multiple of 8 vectors a thread
constexpr int64_t kMostPartials = 256;

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
  float epsilon;
};
static_assert(sizeof(Table) <= 4000, "kernel arguments");

struct Pieces {
  float* x;           // [r, pc] X
  uint16_t* from[2];  // [r, pc] X as an operand: high and low parts
  uint16_t* to[2];    // [r, pc] the same behind this step
  uint16_t* a[2];     // [r, pr] A without its diagonal
  uint16_t* b[2];     // B without its diagonal
  float* d;           // [r] A's diagonal
  float* e;           // [r] B's
};
__host__ __device__ inline int64_t round_up(int64_t n, int64_t k) { return (n + k - 1) / k * k; }
template <bool kPair>
__host__ __device__ inline int64_t piece_bytes(int64_t r, int64_t pr, int64_t pc) {
  return r * pc * (4 + 2 * 2 * (kPair ? 2 : 1)) + r * pr * 2 * 2 * (kPair ? 2 : 1) + 2 * round_up(r * 4, 256);
}
template <bool kPair>
__device__ __forceinline__ Pieces pieces_of(const Entry& t, int turn) {
  constexpr int kParts = kPair ? 2 : 1;
  Pieces p;
  char* at = t.base;
  const int64_t x = static_cast<int64_t>(t.r) * t.pc, a = static_cast<int64_t>(t.r) * t.pr;
  p.x = reinterpret_cast<float*>(at);
  at += x * 4;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    p.from[k] = reinterpret_cast<uint16_t*>(at + (turn * kParts + (kPair ? k : 0)) * x * 2);
    p.to[k] = reinterpret_cast<uint16_t*>(at + ((turn ^ 1) * kParts + (kPair ? k : 0)) * x * 2);
  }
  at += 2 * kParts * x * 2;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    p.a[k] = reinterpret_cast<uint16_t*>(at);
    if (k < kParts) at += a * 2;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    p.b[k] = reinterpret_cast<uint16_t*>(at);
    if (k < kParts) at += a * 2;
  }
  p.d = reinterpret_cast<float*>(at);
  p.e = reinterpret_cast<float*>(at + round_up(static_cast<int64_t>(t.r) * 4, 256));
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

// ---- |G|, and X = G / |G|. ----

__host__ __device__ inline int64_t norm_chunk(int64_t elements) {
  const int64_t least = (elements + kMostPartials - 1) / kMostPartials;
  return least <= kNormChunk ? kNormChunk : round_up(least, kNormChunk);
}

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double s_sum[kNormThreads / kWave];
  x = wave_sum(x);
  if (threadIdx.x % kWave == 0) s_sum[threadIdx.x / kWave] = x;
  __syncthreads();
  x = s_sum[0];
#pragma unroll
  for (int w = 1; w < kNormThreads / kWave; ++w) x += s_sum[w];
  return x;
}

template <typename In>
__global__ __launch_bounds__(kNormThreads) void ortho_norm_kernel(Table t) {
  constexpr int kPer = 16 / sizeof(In);
  const Entry& g = t.at[entry_of(t, blockIdx.x, [](const Entry& e) { return e.first_partial; })];
  const int64_t elements = static_cast<int64_t>(g.r) * g.c, chunk = norm_chunk(elements);
  const int64_t from = (blockIdx.x - g.first_partial) * chunk, to = from + chunk < elements ? from + chunk : elements;
  const In* const in = static_cast<const In*>(g.in);
  double sum[2] = {0.0, 0.0};
  auto add = [&](int k, float x) {
    const double d = x;
    sum[k] = fma(d, d, sum[k]);
  };
  int64_t vectors = 0;
  if (reinterpret_cast<uintptr_t>(in) % 16 == 0) {
    vectors = (to - from) / kPer;
    const v4u* const vec = reinterpret_cast<const v4u*>(in + from);
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < vectors; i += kNormThreads) {
      const v4u w = vec[i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(In) == 4) {
          add(k % 2, __uint_as_float(w[k]));
        } else {
          add(0, __uint_as_float(w[k] << 16));
          add(1, __uint_as_float(w[k] & 0xffff0000u));
        }
      }
    }
  }
  for (int64_t i = from + vectors * kPer + threadIdx.x; i < to; i += kNormThreads) add(0, logit_to_float(in[i]));
  const double all = block_sum(sum[0] + sum[1]);
  if (threadIdx.x == 0) t.partials[blockIdx.x] = all;
}

__device__ __forceinline__ uint16_t half_bits(float x) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x)); }
__device__ __forceinline__ float half_value(uint16_t bits) { return static_cast<float>(__builtin_bit_cast(_Float16, bits)); }

// Four consecutive values as operands: float16, and (kPair) what that leaves of them.
template <bool kPair>
__device__ __forceinline__ void split4(const float (&y)[4], v2u* high, v2u* low) {
  uint16_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = half_bits(y[i]);
    l[i] = kPair ? half_bits(y[i] - half_value(h[i])) : 0;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    (*high)[i] = h[2 * i] | static_cast<unsigned>(h[2 * i + 1]) << 16;
    (*low)[i] = l[2 * i] | static_cast<unsigned>(l[2 * i + 1]) << 16;
  }
}

constexpr int kScaleTile = 64;
template <typename In, bool kPair>
__global__ __launch_bounds__(kNormThreads) void ortho_scale_kernel(Table t) {
  __shared__ float s_tile[kScaleTile][kScaleTile + 1];
  const Entry& g = t.at[entry_of(t, blockIdx.x, [](const Entry& e) { return e.first_block; })];
  const double squares = block_sum(static_cast<int>(threadIdx.x) < g.partials ? t.partials[g.first_partial + threadIdx.x] : 0.0);
  const double norm = sqrt(squares), least = t.epsilon;
  const double factor = 1.0 / (norm < least ? least : norm);  // a NaN norm stays
  const int wide = g.pc / kScaleTile, block = blockIdx.x - g.first_block;
  const int i0 = block / wide * kScaleTile, j0 = block % wide * kScaleTile;
  const In* const in = static_cast<const In*>(g.in);
  constexpr int kPerPass = kNormThreads / kScaleTile;
  // Along the rows of the matrix as it is given.
  const int y0 = g.transposed ? j0 : i0, x0 = g.transposed ? i0 : j0;
  const int rows = g.transposed ? g.c : g.r, columns = g.transposed ? g.r : g.c;
  const int x = x0 + threadIdx.x % kScaleTile;
#pragma unroll 4
  for (int k = threadIdx.x / kScaleTile; k < kScaleTile; k += kPerPass) {
    const int y = y0 + k;
    float v = 0.0f;
    if (y < rows && x < columns)
      v = static_cast<float>(static_cast<double>(logit_to_float(in[static_cast<int64_t>(y) * columns + x])) * factor);
    if (g.transposed) s_tile[threadIdx.x % kScaleTile][k] = v;
    else s_tile[k][threadIdx.x % kScaleTile] = v;
  }
  __syncthreads();
  const Pieces p = pieces_of<kPair>(g, 1);
  const int j = 4 * (threadIdx.x % (kScaleTile / 4));
  for (int k = threadIdx.x / (kScaleTile / 4); k < kScaleTile; k += kNormThreads / (kScaleTile / 4)) {
    if (i0 + k >= g.r) break;
    const int64_t at = static_cast<int64_t>(i0 + k) * g.pc + j0 + j;
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = s_tile[k][j + q];
    *reinterpret_cast<f32x4*>(p.x + at) = f32x4{v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] *= kScaleX;
    v2u high, low;
    split4<kPair>(v, &high, &low);
    *reinterpret_cast<v2u*>(p.to[0] + at) = high;
    if constexpr (kPair) *reinterpret_cast<v2u*>(p.to[1] + at) = low;
  }
}

// ---- The products. ----

template <bool kPair, int kSize>
using OrthoLoader = std::conditional_t<kPair, PartsLoader<kSize>, Loader<kSize>>;

// Tile `id` of a lower triangle: rows 0, 1 1, 2 2 2, ...
__device__ __forceinline__ TileAt triangle_at(int id) {
  int row = static_cast<int>((sqrtf(8.0f * static_cast<float>(id) + 1.0f) - 1.0f) * 0.5f);
  while (row * (row + 1) / 2 > id) --row;
  while ((row + 1) * (row + 2) / 2 <= id) ++row;
  return {row, id - row * (row + 1) / 2};
}

// A tile's entry and its place: (row, column) in tiles.
struct Place {
  int entry;
  int i, j;
};

// A (kSquare false, from X) or B (true, from A): the tiles (i, j), j <= i, of a symmetric
// product M M^T, M's rows "along" for both operands.  A lane of the MFMA layout holds columns
// j + 8 g + 32 (m / 2) + 4 (m % 2) + 0..3 of row i + 16 n + s.
template <bool kSquare, bool kPair, int kSize>
__global__ __launch_bounds__(kGemmThreads, kSize == kTile ? 1 : 2) void ortho_symmetric_kernel(Table t, int turn, float b, float c) {
  constexpr int kMT = kSize / 32, kNT = kSize / 32, kKind = kSquare ? 1 : 0;
  __shared__ __align__(1024) char lds[tile_lds(kSize)];
  Tiles tiles(t.total_tiles[kKind]);
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;

  Job<kSize, OrthoLoader<kPair, kSize>> job;
  Place at = {};
  auto start = [&] {
    job.steps = 0;
    if (!tiles.any()) return;
    at.entry = entry_of(t, tiles.at, [](const Entry& e) { return e.first_tile[kKind]; });
    const Entry& e = t.at[at.entry];
    const TileAt tile = triangle_at(tiles.at - e.first_tile[kKind]);
    at.i = tile.wide;
    at.j = tile.deep;
    const Pieces p = pieces_of<kPair>(e, turn);
    const int64_t pitch = kSquare ? e.pr : e.pc;
    const uint16_t* const high = kSquare ? p.a[0] : p.from[0];
    const uint16_t* const low = kSquare ? p.a[1] : p.from[1];
    const int64_t ia = static_cast<int64_t>(at.j) * kSize, ib = static_cast<int64_t>(at.i) * kSize;
    const int64_t left_a = (e.r - ia) * pitch * 2, left_b = (e.r - ib) * pitch * 2;
    const int once = static_cast<int>(pitch / kTileK);
    job.a.along(pitch, kSize, wave, lane);
    job.b.along(pitch, kSize, wave, lane);
    if constexpr (kPair) {
      job.a.aim(low + ia * pitch, left_a);
      job.a.parts(once, high + ia * pitch, high + ia * pitch, left_a);
      job.b.aim(high + ib * pitch, left_b);
      job.b.parts(once, low + ib * pitch, high + ib * pitch, left_b);
      job.steps = 3 * once;
    } else {
      job.a.aim(high + ia * pitch, left_a);
      job.b.aim(high + ib * pitch, left_b);
      job.steps = once;
    }
  };
  int parity = 0;
  start();
  if (job.steps > 0) job.copy(lds, wave);
  while (tiles.any()) {
    const Place here = at;
    Accumulators<kSize> acc = {};
    contract<false, false, true>(job, lds, parity, wave, lane, acc, [&] {
      tiles.next();
      start();
    });
    const Entry& e = t.at[here.entry];
    const Pieces p = pieces_of<kPair>(e, turn);
    const int i0 = here.i * kSize + (wave / 2) * (kSize / 2), j0 = here.j * kSize + (wave % 2) * (kSize / 2) + 8 * g;
    const bool mirrored = here.i != here.j;
    uint16_t* const high = kSquare ? p.b[0] : p.a[0];
    uint16_t* const low = kSquare ? p.b[1] : p.a[1];
    float* const diagonal = kSquare ? p.e : p.d;
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      const int i = i0 + 16 * n + s;
      const bool row = i < e.r;
      float di = 0.0f;
      if constexpr (kSquare) di = row ? p.d[i] : 0.0f;
#pragma unroll
      for (int m = 0; m < kMT; ++m) {
        const int j = j0 + 32 * (m / 2) + 4 * (m % 2);
        const int64_t to = static_cast<int64_t>(i) * e.pr + j;
        float y[4];
        if constexpr (kSquare) {
          v2u ah = {}, al = {};
          if (row && j < e.pr) {
            ah = *reinterpret_cast<const v2u*>(p.a[0] + to);
            if constexpr (kPair) al = *reinterpret_cast<const v2u*>(p.a[1] + to);
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float oo = element(acc[m][n], q) * (1.0f / (kScaleA * kScaleA));
            const int shift = 16 * (q % 2);
            float o = half_value(static_cast<uint16_t>(ah[q / 2] >> shift));
            if constexpr (kPair) o += half_value(static_cast<uint16_t>(al[q / 2] >> shift));
            const float dj = j + q < e.r ? p.d[j + q] : 0.0f;
            y[q] = fmaf(o * (1.0f / kScaleA), fmaf(c, di + dj, b), c * oo);
            if (i == j + q && row) diagonal[i] = fmaf(b, di, c * fmaf(di, di, oo));
          }
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            y[q] = element(acc[m][n], q) * (1.0f / (kScaleX * kScaleX));
            if (i == j + q && row) diagonal[i] = y[q];
          }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = i == j + q ? 0.0f : y[q] * kScaleA;
        v2u h, l;
        split4<kPair>(y, &h, &l);
        if (row && j < e.pr) {
          *reinterpret_cast<v2u*>(high + to) = h;
          if constexpr (kPair) *reinterpret_cast<v2u*>(low + to) = l;
        }
        if (mirrored && i < e.pr) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (j + q >= e.r) continue;
            const int64_t back = static_cast<int64_t>(j + q) * e.pr + i;
            high[back] = static_cast<uint16_t>(h[q / 2] >> (16 * (q % 2)));
            if constexpr (kPair) low[back] = static_cast<uint16_t>(l[q / 2] >> (16 * (q % 2)));
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy into LDS outlives the workgroup
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

// X <- a X + B X, or of the last step the result: m runs along X's columns (X "across"), n along
// its rows (B "along").  A lane holds columns j + 16 m + 4 g + 0..3 of row i + 16 n + s.
template <typename Out, bool kPair, bool kLast, int kSize>
__global__ __launch_bounds__(kGemmThreads, kSize == kTile ? 1 : 2) void ortho_update_kernel(Table t, int turn, float a) {
  constexpr int kMT = kSize / 32, kNT = kSize / 32, kKind = 2;
  __shared__ __align__(1024) char lds[tile_lds(kSize)];
  Tiles tiles(t.total_tiles[kKind]);
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;

  Job<kSize, OrthoLoader<kPair, kSize>> job;
  Place at = {};
  auto start = [&] {
    job.steps = 0;
    if (!tiles.any()) return;
    at.entry = entry_of(t, tiles.at, [](const Entry& e) { return e.first_tile[kKind]; });
    const Entry& e = t.at[at.entry];
    const TileAt tile = tile_at(tiles.at - e.first_tile[kKind], static_cast<int>(tiles_of(e.r, kSize)),
                                static_cast<int>(tiles_of(e.pc, kSize)));
    at.i = tile.wide;
    at.j = tile.deep;
    const Pieces p = pieces_of<kPair>(e, turn);
    const int64_t i0 = static_cast<int64_t>(at.i) * kSize, j0 = static_cast<int64_t>(at.j) * kSize;
    const int64_t left_x = (static_cast<int64_t>(e.r) * e.pc - j0) * 2, left_b = (e.r - i0) * e.pr * 2;
    const uint16_t* const xh = p.from[0] + j0;
    const uint16_t* const bh = p.b[0] + i0 * e.pr;
    const int once = e.pr / kTileK;
    job.a.across(e.pc, wave, lane);
    job.b.along(e.pr, kSize, wave, lane);
    if constexpr (kPair) {
      const uint16_t* const xl = p.from[1] + j0;
      const uint16_t* const bl = p.b[1] + i0 * e.pr;
      job.a.aim(xl, left_x);
      job.a.parts(once, xh, xh, left_x);
      job.b.aim(bh, left_b);
      job.b.parts(once, bl, bh, left_b);
      job.steps = 3 * once;
    } else {
      job.a.aim(xh, left_x);
      job.b.aim(bh, left_b);
      job.steps = once;
    }
  };
  int parity = 0;
  start();
  if (job.steps > 0) job.copy(lds, wave);
  while (tiles.any()) {
    const Place here = at;
    Accumulators<kSize> acc = {};
    contract<true, false, true>(job, lds, parity, wave, lane, acc, [&] {
      tiles.next();
      start();
    });
    const Entry& e = t.at[here.entry];
    const Pieces p = pieces_of<kPair>(e, turn);
    const int i0 = here.i * kSize + (wave / 2) * (kSize / 2), j0 = here.j * kSize + (wave % 2) * (kSize / 2) + 4 * g;
    Out* const out = static_cast<Out*>(e.out);
    const bool vectors = e.c % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (4 * sizeof(Out)) == 0;
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      const int i = i0 + 16 * n + s;
      const bool row = i < e.r;
      const float factor = row ? a + p.e[i] : 0.0f;
#pragma unroll
      for (int m = 0; m < kMT; ++m) {
        const int j = j0 + 16 * m;
        if (!row || j >= e.pc) continue;
        const int64_t to = static_cast<int64_t>(i) * e.pc + j;
        const f32x4 x = *reinterpret_cast<const f32x4*>(p.x + to);
        float y[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = fmaf(factor, x[q], element(acc[m][n], q) * (1.0f / (kScaleA * kScaleX)));
        if constexpr (kLast) {
#pragma unroll
          for (int q = 0; q < 4; ++q) y[q] *= e.scale;
          if (!e.transposed) {
            store_result(out + static_cast<int64_t>(i) * e.c + j, y, e.c - j, vectors);
          } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (j + q >= e.c) continue;
              const int64_t back = static_cast<int64_t>(j + q) * e.r + i;
              if constexpr (sizeof(Out) == 4) out[back] = y[q];
              else out[back] = to_bf16(y[q]);
            }
          }
        } else {
          *reinterpret_cast<f32x4*>(p.x + to) = f32x4{y[0], y[1], y[2], y[3]};
#pragma unroll
          for (int q = 0; q < 4; ++q) y[q] *= kScaleX;
          v2u h, l;
          split4<kPair>(y, &h, &l);
          *reinterpret_cast<v2u*>(p.to[0] + to) = h;
          if constexpr (kPair) *reinterpret_cast<v2u*>(p.to[1] + to) = l;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy into LDS outlives the workgroup
}

// ---- The host's side. ----

Entry entry_for(const OrthoItem& item) {
  Entry e = {};
  e.in = item.in;
  e.out = item.out;
  e.transposed = item.rows > item.columns;
  e.r = static_cast<int32_t>(std::min(item.rows, item.columns));
  e.c = static_cast<int32_t>(std::max(item.rows, item.columns));
  e.pr = static_cast<int32_t>(round_up(e.r, kTileK));
  e.pc = static_cast<int32_t>(round_up(e.c, kTileK));
  e.scale = item.scale;
  return e;
}

// Matrices that are worked on together: as many of one type as a table and this bound hold.
constexpr int64_t kGroupElements = int64_t(1) << 28;

int64_t bytes_of(const OrthoItem& item, const Entry& e) {
  return round_up(item.bf16 ? piece_bytes<false>(e.r, e.pr, e.pc) : piece_bytes<true>(e.r, e.pr, e.pc), 256);
}

// Calls f(first, last) for each group of `items`, which are all of one type.
template <typename F>
void for_groups(const std::vector<OrthoItem>& items, F f) {
  size_t first = 0;
  while (first < items.size()) {
    int64_t elements = 0;
    size_t last = first;
    while (last < items.size() && last - first < static_cast<size_t>(Table::kMost)) {
      const int64_t n = items[last].rows * items[last].columns;
      if (last > first && elements + n > kGroupElements) break;
      elements += n;
      ++last;
    }
    f(first, last);
    first = last;
  }
}

std::vector<OrthoItem> of_type(const OrthoItem* items, int64_t count, bool bf16) {
  std::vector<OrthoItem> out;
  for (int64_t i = 0; i < count; ++i)
    if (items[i].bf16 == bf16) out.push_back(items[i]);
  return out;
}

constexpr size_t kPartialBytes = Table::kMost * kMostPartials * sizeof(double);

int64_t tiles_in(const Entry& e, int kind, int size) {
  const int64_t rows = tiles_of(e.r, size);
  return kind == 2 ? rows * tiles_of(e.pc, size) : rows * (rows + 1) / 2;
}

// Tiles of 256 or 128, by what their rounds take (round_cost).
int tile_for(const Table& t, int kind, int passes) {
  double best = INFINITY;
  int size = kTile;
  for (int candidate : {kTile, kSmallTile}) {
    double work = 0.0, tiles = 0.0;
    for (int i = 0; i < t.count; ++i) {
      const double n = static_cast<double>(tiles_in(t.at[i], kind, candidate));
      tiles += n;
      work += n * round_cost(candidate, (kind == 0 ? t.at[i].pc : t.at[i].pr) / kTileK * passes);
    }
    const double rounds = std::ceil(tiles / resident_tiles(candidate));
    const double cost = rounds * work / tiles;
    if (cost < best) {
      best = cost;
      size = candidate;
    }
  }
  return size;
}

template <bool kSquare, bool kPair>
hipError_t launch_symmetric(const Table& t, int size, int turn, const OrthoStep& p, hipStream_t st) {
  const dim3 grid(workgroups_of(t.total_tiles[kSquare ? 1 : 0], size)), block(kGemmThreads);
  if (size == kTile) hipLaunchKernelGGL((ortho_symmetric_kernel<kSquare, kPair, kTile>), grid, block, 0, st, t, turn, p.b, p.c);
  else hipLaunchKernelGGL((ortho_symmetric_kernel<kSquare, kPair, kSmallTile>), grid, block, 0, st, t, turn, p.b, p.c);
  return hipGetLastError();
}

template <typename Out, bool kPair, bool kLast>
hipError_t launch_update(const Table& t, int size, int turn, const OrthoStep& p, hipStream_t st) {
  const dim3 grid(workgroups_of(t.total_tiles[2], size)), block(kGemmThreads);
  if (size == kTile) hipLaunchKernelGGL((ortho_update_kernel<Out, kPair, kLast, kTile>), grid, block, 0, st, t, turn, p.a);
  else hipLaunchKernelGGL((ortho_update_kernel<Out, kPair, kLast, kSmallTile>), grid, block, 0, st, t, turn, p.a);
  return hipGetLastError();
}

template <typename T, bool kPair>
hipError_t launch_group(const OrthoItem* items, int count, const OrthoStep* steps, int step_count, float epsilon, char* ws,
                        hipStream_t st) {
  Table t = {};
  t.count = count;
  t.epsilon = epsilon;
  t.partials = reinterpret_cast<double*>(ws + kWsDataOffset);
  char* base = ws + round_up(kWsDataOffset, 256) + kPartialBytes;
  for (int i = 0; i < count; ++i) {
    Entry& e = t.at[i];
    e = entry_for(items[i]);
    e.base = base;
    base += bytes_of(items[i], e);
    const int64_t elements = static_cast<int64_t>(e.r) * e.c;
    e.first_partial = t.total_partials;
    e.partials = static_cast<int32_t>((elements + norm_chunk(elements) - 1) / norm_chunk(elements));
    t.total_partials += e.partials;
    e.first_block = t.total_blocks;
    t.total_blocks += static_cast<int32_t>(tiles_of(e.r, kScaleTile) * (e.pc / kScaleTile));
  }
  int size[3];
  for (int kind = 0; kind < 3; ++kind) {
    size[kind] = tile_for(t, kind, kPair ? 3 : 1);
    for (int i = 0; i < count; ++i) {
      t.at[i].first_tile[kind] = t.total_tiles[kind];
      t.total_tiles[kind] += static_cast<int32_t>(tiles_in(t.at[i], kind, size[kind]));
    }
  }
  hipLaunchKernelGGL(ortho_norm_kernel<T>, dim3(t.total_partials), dim3(kNormThreads), 0, st, t);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((ortho_scale_kernel<T, kPair>), dim3(t.total_blocks), dim3(kNormThreads), 0, st, t);
  e = hipGetLastError();
  for (int k = 0; k < step_count && e == hipSuccess; ++k) {
    const int turn = k % 2;
    e = launch_symmetric<false, kPair>(t, size[0], turn, steps[k], st);
    if (e == hipSuccess) e = launch_symmetric<true, kPair>(t, size[1], turn, steps[k], st);
    if (e == hipSuccess)
      e = k + 1 < step_count ? launch_update<T, kPair, false>(t, size[2], turn, steps[k], st)
                             : launch_update<T, kPair, true>(t, size[2], turn, steps[k], st);
  }
  return e;
}

}  // namespace

bool ortho_steps_ok(const OrthoStep* steps, int count) {
  double most = 1.0;  // the largest singular value that there may be
  for (int k = 0; k < count; ++k) {
    const double a = steps[k].a, b = steps[k].b, c = steps[k].c;
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    // B's eigenvalues b t + c t^2 over t in [0, most^2]: the ends, and the vertex between them.
    const double end = most * most;
    double low = std::min(0.0, b * end + c * end * end), high = std::max(0.0, b * end + c * end * end);
    if (c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < end) {
      low = std::min(low, -b * b / (4.0 * c));
      high = std::max(high, -b * b / (4.0 * c));
    }
    if (!(high - low <= kMostRange)) return false;
    // |a s + b s^3 + c s^5| over s in [0, most]: the end, and where a + 3 b t + 5 c t^2 = 0, t = s^2.
    auto value = [&](double s) { return std::fabs(s * (a + s * s * (b + s * s * c))); };
    double next = value(most);
    auto at = [&](double square) {
      if (square > 0.0 && square < end) next = std::max(next, value(std::sqrt(square)));
    };
    if (c != 0.0) {
      const double root = 9.0 * b * b - 20.0 * a * c;
      if (root >= 0.0) {
        at((-3.0 * b + std::sqrt(root)) / (10.0 * c));
        at((-3.0 * b - std::sqrt(root)) / (10.0 * c));
      }
    } else if (b != 0.0) {
      at(-a / (3.0 * b));
    }
    if (!(next <= kMostSingular)) return false;
    most = next;
  }
  return true;
}

size_t ortho_workspace_bytes(const OrthoItem* items, int64_t count) {
  int64_t most = 0;
  for (const bool bf16 : {true, false}) {
    const std::vector<OrthoItem> of = of_type(items, count, bf16);
    for_groups(of, [&](size_t first, size_t last) {
      int64_t bytes = 0;
      for (size_t i = first; i < last; ++i) bytes += bytes_of(of[i], entry_for(of[i]));
      most = std::max(most, bytes);
    });
  }
  return static_cast<size_t>(round_up(kWsDataOffset, 256) + static_cast<int64_t>(kPartialBytes) + most);
}

hipError_t launch_orthogonalize(const OrthoItem* items, int64_t count, const OrthoStep* steps, int step_count, float epsilon,
                                void* ws, hipStream_t st) {
  hipError_t e = hipSuccess;
  for (const bool bf16 : {true, false}) {
    const std::vector<OrthoItem> of = of_type(items, count, bf16);
    for_groups(of, [&](size_t first, size_t last) {
      if (e != hipSuccess) return;
      const int n = static_cast<int>(last - first);
      char* const base = static_cast<char*>(ws);
      e = bf16 ? launch_group<uint16_t, false>(of.data() + first, n, steps, step_count, epsilon, base, st)
               : launch_group<float, true>(of.data() + first, n, steps, step_count, epsilon, base, st);
    });
  }
  return e;
}

}  // namespace vtrace
