// The products of Newton-Schulz steps in tiles of 256 or 128 (the contraction of the vocabulary
// layer's kernels, with float16 operands): large matrices, or many of them.
#include "orthogonalize_impl.hpp"

namespace vtrace {
namespace {

template <bool kPair, int kSize>
using OrthoLoader = std::conditional_t<kPair, PartsLoader<kSize>, Loader<kSize>>;

// A tile's entry and its place: (row, column) in tiles.
struct Place {
  int entry;
  int i, j;
  Unit unit;
};

// A tile whose k is split: the workgroup that is the last of its pieces has the sum of all, in their
// order, and true; the others leave their sums and have nothing more to do.  Sums go past the L2s by
// device-scope stores, which have completed before the tile's counter moves.
constexpr int kJoined = 16;  // sums of four in flight: registers hold no more
template <int kSize>
__device__ __forceinline__ bool join_pieces(const Table& t, const Unit& u, int* flag, Accumulators<kSize>& acc) {
  constexpr int kMT = kSize / 32, kNT = kSize / 32, kAll = kMT * kNT, kBatch = kAll < kJoined ? kAll : kJoined;
  constexpr int64_t kSums = static_cast<int64_t>(kSize) * kSize * 4;
  auto place = [&](int slot, int k) {
    return reinterpret_cast<unsigned long long*>(t.sums + slot * kSums + (static_cast<int64_t>(k) * kGemmThreads + threadIdx.x) * 16);
  };
#pragma unroll
  for (int k = 0; k < kAll; ++k) {
    unsigned long long* const to = place(u.slot, k);
    const f32x4& c = acc[k / kNT][k % kNT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t lo = __float_as_uint(element(c, 2 * h)), hi = __float_as_uint(element(c, 2 * h + 1));
      __hip_atomic_store(to + h, lo | hi << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  __atomic_signal_fence(__ATOMIC_SEQ_CST);  // keep the compiler from moving the stores past the wait
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);  // the stores have completed
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned* const counter = t.counters + u.counter;
    const bool last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<unsigned>(u.pieces) - 1;
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last;
  }
  __syncthreads();
  const bool last = __builtin_amdgcn_readfirstlane(*flag) != 0;
  __syncthreads();
  if (!last) return false;
  const int first = u.slot - u.piece;
#pragma unroll
  for (int k0 = 0; k0 < kAll; k0 += kBatch) {
#pragma unroll
    for (int k = k0; k < k0 + kBatch; ++k) acc[k / kNT][k % kNT] = f32x4{};
    for (int p = 0; p < u.pieces; ++p) {
      unsigned long long x[kBatch][2];
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) x[k][h] = __hip_atomic_load(place(first + p, k0 + k) + h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[(k0 + k) / kNT][(k0 + k) % kNT][q] += __uint_as_float(static_cast<uint32_t>(x[k][q / 2] >> (32 * (q % 2))));
    }
  }
  return true;
}

// A wave's 32 rows of half a tile's columns, to be read turned: 32-byte pieces exchanged within a row
// as in the stages, so that both kinds of access fall on all banks.
template <int kSize>
__device__ __forceinline__ int turned_swizzle(int row) {
  return swizzle_of(row) & (kSize / 32 - 1);
}
__device__ __forceinline__ s16x4 transposed_read(const char* lds) {
  typedef __attribute__((address_space(3))) s16x4* LdsVec;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVec)lds);
}

// Float16 products on the matrix cores and the operands' copies bound these kernels where k is long: A of 4
// matrices of 4096 x 4096 and 2 of 4096 x 16384 takes 790 us (1.04 PFLOP/s of the halves that are asked for,
// whose diagonal tiles are computed whole; matrix units busy 52%), A A 475 (0.87, 42%), A A of 24 matrices
// of hidden size 1024 55 (0.47, 23%: one round of 16 steps, 25 us, beside a tile's fill and stores).
//
// A symmetric matrix: the tiles (i, j), j <= i, of M N, rows of both "along".  A lane of the MFMA
// layout holds columns j + 8 g + 32 (m / 2) + 4 (m % 2) + 0..3 of row i + 16 n + s.
// kSplit: some tiles are split along k (which costs the others 4%).
template <int kOf, bool kPair, int kSize, bool kSplit>
__global__ __launch_bounds__(kGemmThreads, kSize == kTile ? 1 : 2) void ortho_symmetric_kernel(Table t, int turn, Product f) {
  constexpr int kMT = kSize / 32, kNT = kSize / 32, kKind = kOf == kOfX ? 0 : 1, kParts = kPair ? 2 : 1;
  constexpr int kTurnedBytes = 32 * kSize;  // of a wave: 32 rows of kSize / 2 columns, or 16 of both parts
  __shared__ __align__(1024) char lds[tile_lds(kSize) + 4 * kTurnedBytes];
  Tiles tiles(t.units[kKind].total);
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;

  Job<kSize, OrthoLoader<kPair, kSize>> job;
  Place at = {};
  auto start = [&] {
    job.steps = 0;
    if (!tiles.any()) return;
    at.unit = kSplit ? unit_at(t.units[kKind], tiles.at) : Unit{tiles.at, 0, 1, 0, 0};
    at.entry = entry_of(t, at.unit.tile, [](const Entry& e) { return e.first_tile[kKind]; });
    const Entry& e = t.at[at.entry];
    const TileAt tile = triangle_at(at.unit.tile - e.first_tile[kKind]);
    at.i = tile.wide;
    at.j = tile.deep;
    const Pieces p = pieces_of<kPair>(e, turn);
    const int64_t pitch = kOf == kOfX ? e.pc : e.pr;
    const int all = static_cast<int>(pitch / kTileK);
    const int begin = all * at.unit.piece / at.unit.pieces, once = all * (at.unit.piece + 1) / at.unit.pieces - begin;
    auto operand = [&](int matrix, int k) { return (kOf == kOfX ? p.from[k] : symmetric_of<kPair>(e, p, matrix, k)) + begin * kTileK; };
    const int64_t ia = static_cast<int64_t>(at.j) * kSize, ib = static_cast<int64_t>(at.i) * kSize;
    const int64_t left_a = ((e.r - ia) * pitch - begin * kTileK) * 2, left_b = ((e.r - ib) * pitch - begin * kTileK) * 2;
    const uint16_t* const a = operand(f.n, 0) + ia * pitch;
    const uint16_t* const b = operand(f.m, 0) + ib * pitch;
    job.a.along(pitch, kSize, wave, lane);
    job.b.along(pitch, kSize, wave, lane);
    if constexpr (kPair) {
      job.a.aim(operand(f.n, 1) + ia * pitch, left_a);
      job.a.parts(once, a, a, left_a);
      job.b.aim(b, left_b);
      job.b.parts(once, operand(f.m, 1) + ib * pitch, b, left_b);
      job.steps = 3 * once;
    } else {
      job.a.aim(a, left_a);
      job.b.aim(b, left_b);
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
    if constexpr (kSplit) {
      if (here.unit.pieces > 1 && !join_pieces<kSize>(t, here.unit, reinterpret_cast<int*>(lds + tile_lds(kSize)), acc)) continue;
    }
    const Entry& e = t.at[here.entry];
    const Pieces p = pieces_of<kPair>(e, turn);
    const int i0 = here.i * kSize + (wave / 2) * (kSize / 2), j0 = here.j * kSize + (wave % 2) * (kSize / 2);
    const bool mirrored = here.i != here.j;
    uint16_t* const out[kParts] = {symmetric_of<kPair>(e, p, f.out, 0)};
    if constexpr (kPair) const_cast<uint16_t*&>(out[kParts - 1]) = symmetric_of<kPair>(e, p, f.out, 1);
    char* const turned = lds + tile_lds(kSize) + wave * kTurnedBytes;
    const float* const dm = diagonal_of(e, p, f.m);
    const float* const dn = diagonal_of(e, p, f.n);
    float* const d_out = diagonal_of(e, p, f.out);
    // Eight elements of a row of M (and N), as they lie: of the next 16 rows, while these are stored,
    // or (two matrices in two parts, which the registers do not hold beside a tile of 256) where they
    // are used.
    constexpr bool kLate = kOf == kOfTwo && kPair && kSize == kTile;
    constexpr int kMatrices = kOf == kOfTwo ? 2 : 1, kBuffers = kLate ? 1 : 2, kPieces = kLate ? 1 : kMT / 2;
    v4u o[kBuffers][kMatrices][kParts][kPieces];
    float di[kNT] = {}, dj[kMT / 2][8];
    auto load_piece = [&](int n, int m) {
      const int i = i0 + 16 * n + s < e.r ? i0 + 16 * n + s : e.r - 1, j = j0 + 8 * g + 32 * m;
      const int64_t from = static_cast<int64_t>(i) * e.pr + (j < e.pr ? j : 0);
#pragma unroll
      for (int w = 0; w < kMatrices; ++w)
#pragma unroll
        for (int k = 0; k < kParts; ++k)
          o[n % kBuffers][w][k][m % kPieces] = *reinterpret_cast<const v4u*>(symmetric_of<kPair>(e, p, w == 0 ? f.m : f.n, k) + from);
    };
    auto load_row = [&](int n) {
#pragma unroll
      for (int m = 0; m < kMT / 2; ++m) load_piece(n, m);
    };
    if constexpr (kOf != kOfX) {
      if (!kLate) load_row(0);
#pragma unroll
      for (int m = 0; m < kMT / 2; ++m)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int j = j0 + 8 * g + 32 * m + q;
          dj[m][q] = dn[j < e.r ? j : e.r - 1];
        }
#pragma unroll
      for (int n = 0; n < kNT; ++n) di[n] = dm[i0 + 16 * n + s < e.r ? i0 + 16 * n + s : e.r - 1];
    }
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      const int i = i0 + 16 * n + s;
      const bool row = i < e.r;
      if constexpr (kOf != kOfX) {
        if (!kLate && n + 1 < kNT) load_row(n + 1);
      }
#pragma unroll
      for (int m = 0; m < kMT / 2; ++m) {
        const int j = j0 + 8 * g + 32 * m;
        if constexpr (kLate) load_piece(n, m);
        float y[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float sum = element(acc[2 * m + q / 4][n], q % 4);
          const bool in = row && j + q < e.r;
          if constexpr (kOf == kOfX) {
            y[q] = sum * (1.0f / (kScaleX * kScaleX));
            if (in && i == j + q) d_out[i] = y[q];
          } else {
            // With M = D + O and N = D' + O': M N without its diagonal is D O' + O D' + O O'.
            const float oo = sum * (1.0f / (kScaleA * kScaleA));
            float off[kMatrices];
#pragma unroll
            for (int w = 0; w < kMatrices; ++w) {
              off[w] = high_of(o[n % kBuffers][w][0][m % kPieces][q / 2], q % 2);
              if constexpr (kPair) off[w] += high_of(o[n % kBuffers][w][kParts - 1][m % kPieces][q / 2], q % 2);
              off[w] *= 1.0f / kScaleA;
            }
            y[q] = product_off<kOf>(f, off[0], off[kMatrices - 1], di[n], dj[m][q], oo);
            if (in && i == j + q) d_out[i] = product_diagonal<kOf>(f, di[n], dj[m][q], oo);
          }
          y[q] = in && i != j + q ? y[q] * kScaleA : 0.0f;
        }
        v4u part[2];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          part[0][q] = high2(y[2 * q], y[2 * q + 1]);
          if constexpr (kPair) part[1][q] = low2(y[2 * q], y[2 * q + 1], part[0][q]);
        }
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
          if (row && j < e.pr) *reinterpret_cast<v4u*>(out[k] + static_cast<int64_t>(i) * e.pr + j) = part[k];
          if (mirrored) {
            const int at = 16 * (kPair ? k : n % 2) + s, piece = 2 * m + g / 2;
            *reinterpret_cast<v4u*>(turned + at * kSize + ((piece ^ turned_swizzle<kSize>(at)) * 32) + (g % 2) * 16) = part[k];
          }
        }
      }
      if (mirrored && (kPair || n % 2 == 1)) {
        // The wave's last rows, turned: a lane has eight (float32 matrices: four) consecutive elements
        // of a row above the diagonal.  A wave's accesses to LDS are in order.
        asm volatile("" ::: "memory");
        constexpr int kHalves = kPair ? 1 : 2;
        const int back = i0 + 16 * (n + 1 - kHalves) + 4 * kHalves * g;
#pragma unroll
        for (int k = 0; k < (kPair ? 2 : 1); ++k)
#pragma unroll
          for (int block = 0; block < kSize / 32; ++block) {
            s16x4 half[kHalves];
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
              const int at = 16 * k + 4 * kHalves * g + 4 * h + s / 4;
              half[h] = transposed_read(turned + at * kSize + ((block ^ turned_swizzle<kSize>(at)) * 32) + (s % 4) * 8);
            }
            const int j = j0 + 16 * block + s;
            if (j >= e.r || back >= e.pr) continue;
            uint16_t* const to = out[k] + static_cast<int64_t>(j) * e.pr + back;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) *reinterpret_cast<s16x4*>(to + 4 * h) = half[h];
          }
        asm volatile("" ::: "memory");
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy into LDS outlives the workgroup
}

// 4 of 4096 x 4096 and 2 of 4096 x 16384 1500 us (1.10 PFLOP/s, matrix units busy 52%), 24 matrices of hidden size
// 1024 166 (0.62, 27%: X's 8 bytes an element beside 16 steps of products; four columns a lane, 8-byte loads and
// stores, took 9 and 20% more; rows fetched further ahead, and workgroups that start at different times, gain nothing).
// X <- a X + B X, or of the last step the result: m runs along X's columns (X "across"), n along
// its rows (B "along").  A lane holds columns j + 8 g + 32 (m / 2) + 4 (m % 2) + 0..3 of row i + 16 n + s.
template <typename Out, bool kPair, bool kLast, int kSize>
__global__ __launch_bounds__(kGemmThreads, kSize == kTile ? 1 : 2) void ortho_update_kernel(Table t, int turn, Update f) {
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
    const uint16_t* const bh = symmetric_of<kPair>(e, p, f.by, 0) + i0 * e.pr;
    const int once = e.pr / kTileK;
    job.a.across(e.pc, wave, lane);
    job.b.along(e.pr, kSize, wave, lane);
    if constexpr (kPair) {
      const uint16_t* const xl = p.from[1] + j0;
      const uint16_t* const bl = symmetric_of<kPair>(e, p, f.by, 1) + i0 * e.pr;
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
    const Entry& e = t.at[here.entry];
    const Pieces p = pieces_of<kPair>(e, turn);
    const int i0 = here.i * kSize + (wave / 2) * (kSize / 2), j0 = here.j * kSize + (wave % 2) * (kSize / 2) + 8 * g;
    const float* const diagonal = diagonal_of(e, p, f.by);
    Out* const out = static_cast<Out*>(e.out);
    const bool vectors = e.c % 8 == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
    // X's rows are fetched kAhead times 16 ahead, the first of them during the last step of k.
    constexpr int kAhead = 1, kBuffers = kAhead + 1;
    f32x4 x[kBuffers][kPair ? kMT : 1];
    v4u part[kBuffers][2][kPair ? 1 : kMT / 2];
    float of_row[kBuffers];
    auto load_rows = [&](int n) {
      const int i = i0 + 16 * n + s < e.r ? i0 + 16 * n + s : e.r - 1;
      of_row[n % kBuffers] = diagonal[i];
#pragma unroll
      for (int m = 0; m < kMT; m += 2) {
        const int j = j0 + 16 * m;
        const int64_t from = static_cast<int64_t>(i) * e.pc + (j < e.pc ? j : 0);
        if constexpr (kPair) {
          x[n % kBuffers][m] = *reinterpret_cast<const f32x4*>(p.x + from);
          x[n % kBuffers][m + 1] = *reinterpret_cast<const f32x4*>(p.x + from + 4);
        } else {
          part[n % kBuffers][0][m / 2] = *reinterpret_cast<const v4u*>(p.from[0] + from);
          part[n % kBuffers][1][m / 2] = *reinterpret_cast<const v4u*>(p.low + from);
        }
      }
    };
    contract<true, false, true, true>(job, lds, parity, wave, lane, acc, [&] {
#pragma unroll
      for (int n = 0; n < kAhead; ++n) load_rows(n);
      tiles.next();
      start();
    });
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      if (n + kAhead < kNT) load_rows(n + kAhead);
      const int i = i0 + 16 * n + s;
      const bool row = i < e.r;
      const float factor = f.of_x + of_row[n % kBuffers];
#pragma unroll
      for (int m = 0; m < kMT; m += 2) {
        const int j = j0 + 16 * m;
        float y[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float before;
            if constexpr (kPair) {
              before = x[n % kBuffers][m + h][q];
            } else {
              const v4u high = part[n % kBuffers][0][m / 2], left = part[n % kBuffers][1][m / 2];
              before = whole_of(v2u{high[2 * h], high[2 * h + 1]}, v2u{left[2 * h], left[2 * h + 1]}, q) * (1.0f / kScaleX);
            }
            y[h][q] = fmaf(factor, before, element(acc[m + h][n], q) * (1.0f / (kScaleA * kScaleX)));
          }
        }
        if (!row || j >= e.pc) continue;
        if constexpr (kLast) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) y[h][q] *= e.scale;
          if (!e.transposed) {
            store_results(out + static_cast<int64_t>(i) * e.c + j, y, e.c - j, vectors);
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              if (j + k >= e.c) continue;
              const int64_t back = static_cast<int64_t>(j + k) * e.r + i;
              if constexpr (sizeof(Out) == 4) out[back] = y[k / 4][k % 4];
              else out[back] = to_bf16(y[k / 4][k % 4]);
            }
          }
        } else {
          const int64_t to = static_cast<int64_t>(i) * e.pc + j;
          v2u high[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if constexpr (kPair) *reinterpret_cast<f32x4*>(p.x + to + 4 * h) = f32x4{y[h][0], y[h][1], y[h][2], y[h][3]};
#pragma unroll
            for (int q = 0; q < 4; ++q) y[h][q] *= kScaleX;
            high[h] = high4(y[h]);
          }
          auto both = [](v2u u, v2u v) { return v4u{u[0], u[1], v[0], v[1]}; };
          *reinterpret_cast<v4u*>(p.to[0] + to) = both(high[0], high[1]);
          if constexpr (kPair) *reinterpret_cast<v4u*>(p.to[1] + to) = both(low4(y[0], high[0]), low4(y[1], high[1]));
          else *reinterpret_cast<v4u*>(p.low + to) = both(left4(y[0], high[0]), left4(y[1], high[1]));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy into LDS outlives the workgroup
}

template <int kOf, bool kPair>
hipError_t launch_symmetric(const Table& t, int turn, const Product& p, hipStream_t st) {
  const int kind = kOf == kOfX ? 0 : 1;
  const Units& u = t.units[kind];
  const dim3 grid(workgroups_of(u.total, t.size[kind])), block(kGemmThreads);
  const bool split = u.total != t.total_tiles[kind];
  if constexpr (!kWhole<kPair, kTile, kOf == kOfX ? 0 : 1>) {
    if (t.size[kind] == kTile && split) {
      hipLaunchKernelGGL((ortho_symmetric_kernel<kOf, kPair, kTile, true>), grid, block, 0, st, t, turn, p);
      return hipGetLastError();
    }
  }
  if (t.size[kind] == kTile) hipLaunchKernelGGL((ortho_symmetric_kernel<kOf, kPair, kTile, false>), grid, block, 0, st, t, turn, p);
  else if (split) hipLaunchKernelGGL((ortho_symmetric_kernel<kOf, kPair, kSmallTile, true>), grid, block, 0, st, t, turn, p);
  else hipLaunchKernelGGL((ortho_symmetric_kernel<kOf, kPair, kSmallTile, false>), grid, block, 0, st, t, turn, p);
  return hipGetLastError();
}

template <typename Out, bool kLast>
hipError_t launch_update(const Table& t, int turn, const Update& u, hipStream_t st) {
  constexpr bool kPair = sizeof(Out) == 4;
  const dim3 grid(workgroups_of(t.total_tiles[2], t.size[2])), block(kGemmThreads);
  if (t.size[2] == kTile) hipLaunchKernelGGL((ortho_update_kernel<Out, kPair, kLast, kTile>), grid, block, 0, st, t, turn, u);
  else hipLaunchKernelGGL((ortho_update_kernel<Out, kPair, kLast, kSmallTile>), grid, block, 0, st, t, turn, u);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_ortho_tiles_symmetric(const Table& t, int of, bool pair, int turn, const Product& p, hipStream_t st) {
  if (of == kOfX) return pair ? launch_symmetric<kOfX, true>(t, turn, p, st) : launch_symmetric<kOfX, false>(t, turn, p, st);
  if (of == kOfOne) return pair ? launch_symmetric<kOfOne, true>(t, turn, p, st) : launch_symmetric<kOfOne, false>(t, turn, p, st);
  return pair ? launch_symmetric<kOfTwo, true>(t, turn, p, st) : launch_symmetric<kOfTwo, false>(t, turn, p, st);
}

hipError_t launch_ortho_tiles_update(const Table& t, bool pair, int turn, const Update& u, hipStream_t st) {
  if (pair) return u.last ? launch_update<float, true>(t, turn, u, st) : launch_update<float, false>(t, turn, u, st);
  return u.last ? launch_update<uint16_t, true>(t, turn, u, st) : launch_update<uint16_t, false>(t, turn, u, st);
}

}  // namespace vtrace
