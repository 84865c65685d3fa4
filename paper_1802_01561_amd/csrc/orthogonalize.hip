// Matrices made nearly orthogonal by Newton-Schulz products: with X = G / max(|G|, epsilon),
// |G| the Frobenius norm, and `steps` times
//   A = X X^T,   B = b A + c A A,   X <- a X + B X,
// which takes every singular value s of X to a s + b s^3 + c s^5 and leaves the singular
// vectors.  X is kept with at most as many rows (r) as columns (c): a taller matrix is
// transposed when it is read, and back when the result is written.
//
// Numerics.  X is kept in 22 bits or more (of bfloat16 matrices its float16 operand and what
// that leaves, else float32), and the products' operands are float16, of fixed powers of
// two: singular values stay within a small range (the entry point checks the coefficients), so
// that bfloat16's exponents are not needed and float16's three more bits are had for
// nothing (bfloat16 operands: results 1.3e-2 to 3e-2 off, in relation to their norm).  The
// diagonals of A and B are far larger than the rest where the rows are nearly orthogonal; they
// are kept out of the operands, in float32:
//   with A = D + O:  B = b (D + O) + c (D D + D O + O D + O O),   B X = diag(B) X + offdiag(B) X,
// where only O O and offdiag(B) X are products on the matrix cores (with the diagonals in the
// operands 1.7e-3 to 2.8e-3 off, without 2e-4 to 7e-4, and one rounding to bfloat16 is 1.66e-3:
// results of 33 rows and more are 1.67e-3 to 1.85e-3 off, of 34 x 3194 1.96e-3).
// Float32 matrices have operands in two parts, high + low, and three products for each: 3e-7
// to 9e-7 off, from X's own rounding and the float32 sums (a library's float32 products 1.6e-6 to 3.6e-6:
// small singular values grow by 3.44 a step, and rounding errors beside the largest with them; where most
// are a hundredth of the largest, 2048 x 2048, 2.4e-6 and the library's 1.9e-5).
//
// Of matrices of a few values in large blocks the roundings are alike and do not cancel: results of bfloat16
// ones are up to 8.8e-3 off (steps one by one) and 1.9e-2 (the first two at once).  Of float32 ones tiles
// of 64 and 32, whose sums are over 256 k apiece, up to 1.8e-5, the others 1.9e-4 for 2048 x 2048, 3.2e-4 for 4096 x
// 8192 and 1.1e-3 for 65536 x 32768 (a library's products 8e-5 for 1024 x 1024, 5e-4 for 4096 x 4096, where this
// has 2.5e-6 and 3.4e-5).  Such sums in tiles of 256 have no registers; in tiles of 128 half of them go
// to scratch memory, and 4096 x 4096 takes 46% longer.
//
// A and B are symmetric: their tiles on and below the diagonal are computed, and stored twice.
#include "orthogonalize_few.hpp"
#include "orthogonalize_impl.hpp"

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <functional>
#include <numeric>
#include <string>

namespace vtrace {
namespace {

// A's and B's entries beside the diagonal are at most half the range of their eigenvalues.
constexpr double kMostSingular = 3.5, kMostRange = 12.0;

constexpr int kNormThreads = 256;
constexpr int64_t kNormChunk = 16384;  // least elements of a partial sum, a multiple of 8 vectors a thread
constexpr int64_t kMostPartials = 256;

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

// kFew: and A of the matrices of few rows, by the first workgroups.
template <typename In, bool kFew>
__global__ __launch_bounds__(kNormThreads) void ortho_norm_kernel(Table t) {
  constexpr int kPer = 16 / sizeof(In);
  const int id = kFew ? static_cast<int>(blockIdx.x) - t.few_chunks : blockIdx.x;
  if constexpr (kFew) {
    if (id < 0) {
      few_gram<In>(t, blockIdx.x);
      return;
    }
  }
  const Entry& g = t.at[entry_of(t, id, [](const Entry& e) { return e.first_partial; })];
  const int64_t elements = static_cast<int64_t>(g.r) * g.c, chunk = norm_chunk(elements);
  const int64_t from = (id - g.first_partial) * chunk, to = from + chunk < elements ? from + chunk : elements;
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
  if (threadIdx.x == 0) t.partials[id] = all;
}

constexpr int kScaleTile = 64;
// kFew: and the results of the matrices of few rows, by the first workgroups: theirs is the longest way.
template <typename In, bool kPair, bool kFew>
__global__ __launch_bounds__(kNormThreads) void ortho_scale_kernel(Table t, FewSteps steps) {
  union Lds {
    float tile[kScaleTile][kScaleTile + 1];
    char few[kFew ? kFewLds : 1];
  };
  __shared__ __align__(16) Lds lds;
  auto& s_tile = lds.tile;
  const int id = kFew ? static_cast<int>(blockIdx.x) - t.few_blocks : blockIdx.x;
  if constexpr (kFew) {
    if (id < 0) {
      few_apply<In>(t, steps, blockIdx.x, lds.few);
      return;
    }
  }
  const Entry& g = t.at[entry_of(t, id, [](const Entry& e) { return e.first_block; })];
  const int wide = g.pc / kScaleTile, block = id - g.first_block;
  const int i0 = block / wide * kScaleTile, j0 = block % wide * kScaleTile;
  const In* const in = static_cast<const In*>(g.in);
  constexpr int kPerPass = kNormThreads / kScaleTile, kPasses = kScaleTile / kPerPass;
  // Along the rows of the matrix as it is given; all of it under way before the norm is formed.
  const int y0 = g.transposed ? j0 : i0, x0 = g.transposed ? i0 : j0;
  const int rows = g.transposed ? g.c : g.r, columns = g.transposed ? g.r : g.c;
  const int row = threadIdx.x / kScaleTile, column = threadIdx.x % kScaleTile;
  // (Loads under a condition would be waited for one by one: places behind the ends are moved to them.)
  In given[kPasses];
#pragma unroll
  for (int k = 0; k < kPasses; ++k) {
    const int y = y0 + row + k * kPerPass, x = x0 + column;
    given[k] = in[static_cast<int64_t>(y < rows ? y : rows - 1) * columns + (x < columns ? x : columns - 1)];
  }
  const double squares = block_sum(static_cast<int>(threadIdx.x) < g.partials ? t.partials[g.first_partial + threadIdx.x] : 0.0);
  const double norm = sqrt(squares), least = t.epsilon;
  const double factor = 1.0 / (norm < least ? least : norm);  // a NaN norm stays
#pragma unroll
  for (int k = 0; k < kPasses; ++k) {
    const bool inside = y0 + row + k * kPerPass < rows && x0 + column < columns;
    const float v = inside ? static_cast<float>(static_cast<double>(logit_to_float(given[k])) * factor) : 0.0f;
    if (g.transposed) s_tile[column][row + k * kPerPass] = v;
    else s_tile[row + k * kPerPass][column] = v;
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
    if constexpr (kPair) *reinterpret_cast<f32x4*>(p.x + at) = f32x4{v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] *= kScaleX;
    const v2u high = high4(v);
    *reinterpret_cast<v2u*>(p.to[0] + at) = high;
    *reinterpret_cast<v2u*>((kPair ? p.to[1] : p.low) + at) = kPair ? low4(v, high) : left4(v, high);
  }
  if (!t.small) return;
  const TransposedPieces pt = transposed_of<kPair>(g, 1);
  for (int k = threadIdx.x / (kScaleTile / 4); k < kScaleTile; k += kNormThreads / (kScaleTile / 4)) {
    if (j0 + k >= g.c) break;
    const int64_t at = static_cast<int64_t>(j0 + k) * g.pr + i0 + j;
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = s_tile[j + q][k] * kScaleX;
    const v2u high = high4(v);
    *reinterpret_cast<v2u*>(pt.to[0] + at) = high;
    if constexpr (kPair) *reinterpret_cast<v2u*>(pt.to[1] + at) = low4(v, high);
  }
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
  // The small matrices' kernels write up to the pitches, zeros.
  const int64_t rows = tiles_of(size < kSmallTile ? e.pr : e.r, size);
  return kind == 2 ? rows * tiles_of(e.pc, size) : rows * (rows + 1) / 2;
}

// What a launch of one kind takes (us) in tiles of 256 or 128: rounds of as many as there is room for.
// Fewer than that take less a step, gradually (A of 64 and 128 steps, us a step): 36 to 72 tiles of 256 1.1
// (float32 1.2 to 1.35), 100 to 144 1.35 (1.45 to 1.5), 160 1.4 to 1.55 (1.65), 250 1.55 to 1.8 (1.75 to
// 1.85); of 128 36 to 144 0.45 to 0.5, 252 to 272 0.5 to 0.65, 360 to 410 0.85 to 0.9, 470 1.0.  Two values
// of each stand for that here, with the border between.  What a tile costs beside its steps is its fill
// and its stores.  bfloat16, x1 / x2 (steps one by one, the first two at once) in tiles of 64, 128, 256, us: 16 of
// 1024 x 1024 1063 / 1122, 728 / 785, 690 / 728; 2 of 2048 x 2048 812 / 853, 577 / 610, 851 / 924; 2 of 3000 x 3000
// 2699 / 2707, 1692 / 1783, 1602 / 1623; 8 of 1024 x 4096 1759 / 1575, 949 / 896, 1182 / 1132; float32 2 of 2048 x
// 2048 2132 / 2219, 1494 / 1600, 2195 / 2404.
//
// Tiles of equal steps that would leave a round behind theirs mostly empty are split along k, into up to
// as many pieces as fill it, if that is a fifth less with what their sums cost (us, of tiles of 256: five
// pieces of 13 steps take as long as one of 64, 20 to store and 12 a piece to join; six of 43 150 less
// than one of 256).  A of 4 matrices of 4096 x 4096 and 2 of 4096 x 16384, which has 16 of 272 long tiles too
// many: 1030 -> 790 us.  `split`: into so many wherever there are as many steps.
// `room`: bytes for the pieces' sums.
double tiles_cost(const Table& t, int kind, int size, int passes, int split, int64_t room, Units* units) {
  double all = 0.0;
  for (int i = 0; i < t.count; ++i) all += static_cast<double>(tiles_in(t.at[i], kind, size));
  const bool alone = size == kSmallTile && all <= kCus;
  const int64_t slots = alone ? kCus : resident_tiles(size);
  int64_t at = 0, open = 0;  // tiles so far, and those of a round that is not full
  // Of a round with so many tiles, and those that come behind.
  auto step = [&](int64_t there) {
    there += static_cast<int64_t>(all) - at;
    if (size == kTile) return there > 160 ? 1.56 : passes == 1 ? 1.0 : 1.15;
    return there > kCus ? 1.0 : 0.8;
  };
  auto beside = [&](int64_t there) {
    there += static_cast<int64_t>(all) - at;
    if (size == kTile) return kind == 2 ? 28.0 : 21.0;
    return there > kCus ? (kind == 2 ? 14.0 : 8.0) : kind == 2 ? 9.0 : 5.0;
  };
  const double to_store = size == kTile ? 20.0 : 10.0, to_join = size == kTile ? 12.0 : 6.0;
  *units = {};
  int splits = 0;
  int64_t sums = room / (size * size * static_cast<int64_t>(sizeof(float)));  // pieces that there is room for
  double us = 0.0, open_us = 0.0;
  for (int i = 0; i < t.count;) {
    auto steps_of = [&](int k) { return (kind == 0 ? t.at[k].pc : t.at[k].pr) / kTileK; };
    const int steps = steps_of(i);
    int64_t n = 0;
    for (; i < t.count && steps_of(i) == steps; ++i) n += tiles_in(t.at[i], kind, size);
    at += n;
    const double k = static_cast<double>(steps) * passes;
    auto cost = [&](int64_t there) { return step(there) * k + beside(there); };
    const int64_t full = (open + n) / slots, left = (open + n) % slots, own = std::min(left, n);
    if (full > 0) us += std::max(open_us, cost(slots)) + static_cast<double>(full - 1) * cost(slots);
    const double before = full > 0 ? 0.0 : open_us;
    open = left;
    open_us = left > 0 ? std::max(before, cost(left)) : 0.0;
    if (own == 0 || splits == Units::kSplits || kind == 2 || (passes == 3 && size == kTile && kind == 1)) continue;  // kWhole
    const double work = step(left) * k;
    int64_t pieces = std::min<int64_t>((slots - left + own) / own, split ? std::min(split, steps) : steps / 4);
    if (!split) pieces = std::min(pieces, std::max<int64_t>(1, std::lround(std::sqrt(work / to_join))));
    pieces = std::min(pieces, sums / own);
    if (pieces < 2) continue;
    const int64_t there = left + own * (pieces - 1);
    const double then = step(there) * k / static_cast<double>(pieces) + to_store + to_join * static_cast<double>(pieces);
    if (!split && then > 0.8 * work) continue;
    units->begin[splits] = static_cast<int>(at - own);
    units->end[splits] = static_cast<int>(at);
    units->pieces[splits++] = static_cast<int>(pieces);
    sums -= own * pieces;
    open = there;
    open_us = std::max(before, then + beside(there));
    if (open == slots) {
      us += open_us;
      open = 0;
      open_us = 0.0;
    }
  }
  units->total = static_cast<int>(at);
  for (int k = 0; k < Units::kSplits; ++k) {
    if (k >= splits) units->begin[k] = units->end[k] = 0x7fffffff;
    else units->total += (units->end[k] - units->begin[k]) * (units->pieces[k] - 1);
  }
  return us + open_us;
}

// The same in the small matrices' kernels' tiles of 64 or 32: a launch, and the tile that has a CU for
// itself, or all rounds of them.
// 1024 x 1024, us with tiles of 32, 64, 128: one bfloat16 matrix 192, 159, 279, four 511, 360, 301,
// eight 940, 587, 377; float32 270, 248, 625, two 439, 466, 633, four 758, 775, 651.
double small_cost(const Table& t, int kind, int size, bool pair) {
  double work = 0.0, longest = 0.0, tiles = 0.0;
  for (int i = 0; i < t.count; ++i) {
    const double steps = (kind == 0 ? t.at[i].pc : t.at[i].pr) / kTileK, n = static_cast<double>(tiles_in(t.at[i], kind, size));
    tiles += n;
    work += n * steps;
    longest = std::max(longest, steps);
  }
  // Two workgroups of a CU share its path into LDS.
  const double step = size == 64 ? (pair ? 0.5 : 0.26) : pair ? 0.25 : 0.13;
  const double beside = size == 64 ? (pair ? 6.0 : 2.5) : pair ? 0.5 : 0.8;
  const double alone = 2.5 + step * longest;
  if (tiles <= kCus) return 2.0 + alone;
  return 2.0 + std::max(alone, std::ceil(tiles / kCus) * (beside + step * work / tiles));
}

// VTRACE_KERNEL (ortho_32, ortho_64, ortho_128 or ortho_256, with x1 or x2 behind, and of the larger two k2 or k3
// behind that) forces the tiles, whether the first two steps are taken at once, and the pieces of tiles that do not
// fill a round, to cross-check them.
struct Forced {
  int size = 0, together = 0, split = 0;
};
Forced forced_kernel() {
  Forced f;
  const char* const k = std::getenv("VTRACE_KERNEL");
  if (k == nullptr) return f;
  for (const int size : {32, 64, kSmallTile, kTile})
    for (int together = 0; together <= 2; ++together)
      for (int split = 0; split <= 3; ++split)
        if (k == "ortho_" + std::to_string(size) + (together ? "x" + std::to_string(together) : "") +
                     (split ? "k" + std::to_string(split) : ""))
          f = {size, together, split};
  return f;
}

// A matrix's share of the workspace, whatever it is worked on with: its pieces, and spare bytes that hold
// X^T (the small matrices' kernels), or those of all matrices the sums of split tiles.  So the bytes for a
// list serve every list of some of its matrices, whose tiles may be others: of nine bfloat16 512 x
// 2048 tiles of 128, of eight of them tiles of 64.
// Where an X^T has more than that, tiles of 128 or 256 cost less than small ones in any list.
constexpr int64_t kMostSpare = int64_t(1) << 28;
int64_t transposed_of_entry(const Entry& e, bool pair) { return pair ? transposed_bytes<true>(e.c, e.pr) : transposed_bytes<false>(e.c, e.pr); }
int64_t spare_of(const Entry& e, bool pair) { return round_up(std::min(transposed_of_entry(e, pair), kMostSpare), 256); }
int64_t pieces_bytes(const Entry& e, bool pair) {
  return round_up(pair ? piece_bytes<true>(e.r, e.pr, e.pc) : piece_bytes<false>(e.r, e.pr, e.pc), 256);
}
int64_t few_bytes(const Entry& e) { return few_chunks(e.c) * static_cast<int64_t>(kFewRows * kFewRows * sizeof(double)); }
int64_t share_of(const Entry& e, bool pair) {
  const int64_t tiles = pieces_bytes(e, pair) + spare_of(e, pair);
  return e.r <= kFewRows ? std::max(tiles, few_bytes(e)) : tiles;
}
// For forced pieces as well: as many as a launch may have.
int64_t forced_spare() { return forced_kernel().split ? 2 * kCus * kTile * kTile * static_cast<int64_t>(sizeof(float)) : 0; }

// The entries of a group of matrices, all of one type.
Table table_of(const OrthoItem* items, int count, bool few_rows, char* ws) {
  Table t = {};
  const bool pair = !items[0].bf16;
  const Forced forced = forced_kernel();
  auto few = [&](const Entry& e) { return few_rows && e.r <= kFewRows && forced.size == 0; };
  for (int i = 0; i < count; ++i) t.at[i] = entry_for(items[i]);
  // Those of few rows last, and of the others the longest tiles first.
  std::stable_sort(t.at, t.at + count,
                   [&](const Entry& x, const Entry& y) { return few(x) != few(y) ? few(y) : x.pc > y.pc; });
  t.few = static_cast<int>(std::count_if(t.at, t.at + count, few));
  count -= t.few;
  t.count = count;
  int64_t room = forced_spare();
  bool small_fits = true;
  for (int i = 0; i < count; ++i) {
    Entry& e = t.at[i];
    room += spare_of(e, pair);
    small_fits = small_fits && transposed_of_entry(e, pair) <= kMostSpare;
    const int64_t elements = static_cast<int64_t>(e.r) * e.c;
    e.first_partial = t.total_partials;
    e.partials = static_cast<int32_t>((elements + norm_chunk(elements) - 1) / norm_chunk(elements));
    t.total_partials += e.partials;
    e.first_block = t.total_blocks;
    t.total_blocks += static_cast<int32_t>(tiles_of(e.r, kScaleTile) * (e.pc / kScaleTile));
  }
  if (count > 0) {
    const int passes = pair ? 3 : 1;
    double tiles[3], small[3];
    int small_size[3];
    for (int kind = 0; kind < 3; ++kind) {
      Units units;
      t.size[kind] = kTile;
      tiles[kind] = tiles_cost(t, kind, kTile, passes, 0, room, &t.units[kind]);
      const double of_small = tiles_cost(t, kind, kSmallTile, passes, 0, room, &units);
      if (of_small < tiles[kind]) {
        t.size[kind] = kSmallTile;
        tiles[kind] = of_small;
        t.units[kind] = units;
      }
      small_size[kind] = small_cost(t, kind, 32, pair) <= small_cost(t, kind, 64, pair) ? 32 : 64;
      small[kind] = small_cost(t, kind, small_size[kind], pair);
    }
    // The first two steps: A and X twice, or once and three products more of B's size.
    auto one_by_one = [](const double (&us)[3]) { return 2.0 * (us[0] + us[1] + us[2]); };
    auto together = [](const double (&us)[3]) { return us[0] + 5.0 * us[1] + us[2]; };
    t.small = small_fits && std::min(one_by_one(small), together(small)) < std::min(one_by_one(tiles), together(tiles));
    if (t.small) std::copy_n(small_size, 3, t.size);
    // The few rows' results go with the others' X, or with their first A if that takes as long as they do (five
    // float32 matrices of 16 to 513 rows 198 -> 191 us; beside a 64 x 64 matrix's A two 67 -> 69).
    t.few_later = t.small && small[0] > 8.0;
    t.twos = t.small ? together(small) < one_by_one(small) : together(tiles) < one_by_one(tiles);
  }
  if (forced.size) {
    const int size = small_fits ? forced.size : std::max(forced.size, kSmallTile);
    t.small = size < kSmallTile;
    t.few_later = false;
    std::fill_n(t.size, 3, size);
    for (int kind = 0; kind < 3 && !t.small; ++kind) {
      tiles_cost(t, kind, size, pair ? 3 : 1, forced.split, room, &t.units[kind]);
    }
  }
  if (forced.together) t.twos = forced.together == 2;
  int64_t at = round_up(kWsDataOffset, 256) + static_cast<int64_t>(kPartialBytes);
  t.partials = reinterpret_cast<double*>(reinterpret_cast<uintptr_t>(ws) + kWsDataOffset);
  for (int i = 0; i < count; ++i) {
    Entry& e = t.at[i];
    e.base = reinterpret_cast<char*>(reinterpret_cast<uintptr_t>(ws) + static_cast<uintptr_t>(at));
    at += pieces_bytes(e, pair);
    if (t.small) at += spare_of(e, pair);
    for (int kind = 0; kind < 3; ++kind) {
      e.first_tile[kind] = t.total_tiles[kind];
      t.total_tiles[kind] += static_cast<int32_t>(tiles_in(e, kind, t.size[kind]));
    }
  }
  t.counters = reinterpret_cast<unsigned*>(reinterpret_cast<uintptr_t>(ws) + kWsHeaderBytes);
  t.sums = reinterpret_cast<char*>(reinterpret_cast<uintptr_t>(ws) + static_cast<uintptr_t>(at));
  if (!t.small) at += room;
  // Every workgroup forms its Q, about 5 us: one tile each, then more (256 columns each, always: one float32
  // 32 x 4096 matrix 32 us, so 25; eight of 2 x 300 29 and 21).
  auto few_blocks = [&](int64_t block) {
    int64_t blocks = 0;
    for (int i = count; i < count + t.few; ++i) blocks += (t.at[i].c + block - 1) / block;
    return blocks;
  };
  t.few_block = kFewTile;
  while (t.few_block < 8 * kFewTile && few_blocks(t.few_block) > kFewMostBlocks) t.few_block *= 2;
  for (int i = count; i < count + t.few; ++i) {
    Entry& e = t.at[i];
    e.base = reinterpret_cast<char*>(reinterpret_cast<uintptr_t>(ws) + static_cast<uintptr_t>(at));
    e.partials = static_cast<int32_t>(few_chunks(e.c));
    at += few_bytes(e);
    e.first_partial = t.few_chunks;
    t.few_chunks += e.partials;
    e.first_block = t.few_blocks;
    t.few_blocks += (e.c + t.few_block - 1) / t.few_block;
  }
  return t;
}

// Whether singular values from [0, 1] stay within the operands' range.
bool singular_values_stay(const OrthoStep* steps, int count) {
  double most = 1.0;
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

// Whether the first two steps at once (launch_group) stay in the operands' range, singular values
// being at most 1 before them: the eigenvalues of what is formed are polynomials of t = s^2 of degree
// up to 12, whose range over [0, 1] is at most 1 / cos(12 pi / 128) times (5% over) that over 64
// Chebyshev points.
bool two_steps_ok(const OrthoStep& p, const OrthoStep& q) {
  constexpr int kPoints = 64;
  double low[3] = {0.0, 0.0, 0.0}, high[3] = {0.0, 0.0, 0.0};
  for (int i = 0; i < kPoints; ++i) {
    const double t = 0.5 * (1.0 + std::cos((2 * i + 1) * M_PI / (2 * kPoints)));
    const double first = p.a + t * (p.b + t * p.c), then = t * first * first;
    const double value[3] = {t * first, then, first * (q.a + then * (q.b + then * q.c)) - static_cast<double>(p.a) * q.a};
    for (int v = 0; v < 3; ++v) {
      low[v] = std::min(low[v], value[v]);
      high[v] = std::max(high[v], value[v]);
    }
  }
  for (int v = 0; v < 3; ++v)
    if (!(high[v] - low[v] <= kMostRange)) return false;
  return true;
}

// Whether A's own rounding errors stay small where it is stepped by itself: those beside small
// eigenvalues grow by a^2 a step, from 2^-50 to 2^-24 at most.  (Left to grow they turn an eigenvalue of
// zero into one that a polynomial with a maximum at zero takes out of its range.)
bool few_rows_ok(const OrthoStep* steps, int count) {
  double growth = 1.0;
  for (int k = 0; k < count; ++k) growth *= std::max(1.0, std::fabs(static_cast<double>(steps[k].a)));
  return growth <= 8192.0;
}

// Two steps at once.  With P = a I + B of the first, X' = P X has X' X'^T = P A P, so that both steps
// take one product with X each way, and the second's matrices come from the first's:
//   T = A P,   A' = T P,   B' = b' A' + c' A' A',   X'' = (a' I + B') (a I + B) X = (a a' I + Q) X,
//   Q = a' B + a B' + B' B.
// All are polynomials of A, and so commute and are symmetric: half their tiles are computed.
// Where X has more columns than rows, or its loads and stores take as long as products, that is
// less: 3 r^2 c operations and X twice against three products of r^3.
//
// The first two steps alone.  Their X is of norm 1, so that most singular values are small and Q with
// them, and the rounding errors are those of steps one by one (2048 x 2048 bfloat16 1.70e-3 off, of which
// one rounding is 1.66e-3).  Later most are near 1, Q is near -a a', and a result has its errors in full:
// with the last two of five at once as well 1.97e-3, of 4096 x 4096 2.28e-3 where this has 1.69e-3 (and 5 to 8%
// less time).  One layer of hidden size 4096 13.5 ms, one by one 14.15; 24 matrices of hidden size 1024 1565 us, 1665.
template <typename T, bool kPair>
hipError_t launch_group(const OrthoItem* items, int count, const OrthoStep* steps, int step_count, float epsilon, char* ws,
                        hipStream_t st) {
  Table t = table_of(items, count, few_rows_ok(steps, step_count), ws);
  t.epsilon = epsilon;
  const bool two_first = t.twos && step_count > 1 && two_steps_ok(steps[0], steps[1]);
  FewSteps few = {};
  std::copy_n(steps, step_count, few.at);
  few.count = step_count;
  const bool later = t.few > 0 && t.few_later, now = t.few > 0 && !later;
  const dim3 norms(t.total_partials + t.few_chunks), blocks(t.total_blocks + (now ? t.few_blocks : 0)), threads(kNormThreads);
  if (t.few > 0) hipLaunchKernelGGL((ortho_norm_kernel<T, true>), norms, threads, 0, st, t);
  else hipLaunchKernelGGL((ortho_norm_kernel<T, false>), norms, threads, 0, st, t);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (now) hipLaunchKernelGGL((ortho_scale_kernel<T, kPair, true>), blocks, threads, 0, st, t, few);
  else hipLaunchKernelGGL((ortho_scale_kernel<T, kPair, false>), blocks, threads, 0, st, t, few);
  e = hipGetLastError();
  if (t.count == 0) return e;
  int turn = 0;
  bool first = true;
  auto symmetric = [&](int of, const Product& p) {
    if (e != hipSuccess) return;
    e = t.small ? launch_ortho_small_symmetric(t, of, kPair, turn, p, later && first ? &few : nullptr, st) : launch_ortho_tiles_symmetric(t, of, kPair, turn, p, st);
    first = false;
  };
  for (int k = 0; k < step_count && e == hipSuccess;) {
    const int together = k == 0 && two_first ? 2 : 1, next = k + together;
    const OrthoStep& p = steps[k];
    symmetric(kOfX, {0, 0, 0, 0.0f, 0.0f, 0.0f});
    symmetric(kOfOne, {1, 0, 0, p.b, 0.0f, p.c});
    Update u = {1, p.a, next == step_count};
    if (together == 2) {
      const OrthoStep& q = steps[k + 1];
      symmetric(kOfTwo, {2, 0, 1, p.a, 0.0f, 1.0f});
      symmetric(kOfTwo, {0, 2, 1, p.a, 0.0f, 1.0f});
      symmetric(kOfOne, {2, 0, 0, q.b, 0.0f, q.c});
      symmetric(kOfTwo, {0, 2, 1, p.a, q.a, 1.0f});
      u.by = 0;
      u.of_x = p.a * q.a;
    }
    if (e == hipSuccess) e = t.small ? launch_ortho_small_update(t, kPair, turn, u, st) : launch_ortho_tiles_update(t, kPair, turn, u, st);
    turn ^= 1;
    k = next;
  }
  return e;
}

}  // namespace

bool ortho_steps_ok(const OrthoStep* steps, int count) { return singular_values_stay(steps, count); }

size_t ortho_workspace_bytes(const OrthoItem* items, int64_t count) {
  // The largest shares of a table, but not more than a group of several matrices may have: 32 bytes an
  // element of float32, and what the pitches add to 38 of 2^28 elements, less than 9 2^28 (half of both of
  // bfloat16).
  int64_t most = 0;
  for (const bool bf16 : {true, false}) {
    std::vector<int64_t> shares;
    for (int64_t i = 0; i < count; ++i)
      if (items[i].bf16 == bf16) shares.push_back(share_of(entry_for(items[i]), !bf16));
    std::sort(shares.begin(), shares.end(), std::greater<int64_t>());
    if (shares.size() > static_cast<size_t>(Table::kMost)) shares.resize(Table::kMost);
    const int64_t all = std::accumulate(shares.begin(), shares.end(), int64_t(0));
    if (!shares.empty()) most = std::max({most, shares[0], std::min(all, kGroupElements * (bf16 ? 21 : 42))});
  }
  return round_up(kWsDataOffset, 256) + kPartialBytes + static_cast<size_t>(most + forced_spare());
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
