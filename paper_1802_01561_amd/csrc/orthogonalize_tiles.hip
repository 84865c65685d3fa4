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

}  // namespace

hipError_t launch_ortho_tiles_symmetric(const Table& t, bool square, bool pair, int size, int turn, const OrthoStep& p,
                                        hipStream_t st) {
  if (square) return pair ? launch_symmetric<true, true>(t, size, turn, p, st) : launch_symmetric<true, false>(t, size, turn, p, st);
  return pair ? launch_symmetric<false, true>(t, size, turn, p, st) : launch_symmetric<false, false>(t, size, turn, p, st);
}

hipError_t launch_ortho_tiles_update(const Table& t, bool pair, bool last, int size, int turn, const OrthoStep& p,
                                     hipStream_t st) {
  if (pair) return last ? launch_update<float, true, true>(t, size, turn, p, st) : launch_update<float, true, false>(t, size, turn, p, st);
  return last ? launch_update<uint16_t, false, true>(t, size, turn, p, st) : launch_update<uint16_t, false, false>(t, size, turn, p, st);
}

}  // namespace vtrace
