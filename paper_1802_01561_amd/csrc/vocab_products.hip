// The two products of vtrace_vocab_grad with G = dL/dz of one piece of the vocabulary:
//   d_weight[v, h] = sum_n G[n, v] x[n, h],   d_hidden[n, h] += sum_v G[n, v] weight[v, h].
// In both, m runs along h, so that a lane holds four consecutive elements of a row of
// the result.  G's low parts, where there are any, are a second pass over k.
#include "vocab_impl.hpp"

namespace vtrace {
namespace {

__device__ __forceinline__ int64_t active_rows64(const VocabArgs& a) {
  return (static_cast<int64_t>(*a.active_count) + kTileK - 1) / kTileK * kTileK;
}

template <typename Out>
__device__ __forceinline__ void store4(Out* p, f32x4 x) {
  if constexpr (sizeof(Out) == 4) {
    *reinterpret_cast<f32x4*>(p) = x;
  } else {
    v2u w;
    w.x = pack_bf16x2(x[0], x[1]);
    w.y = pack_bf16x2(x[2], x[3]);
    *reinterpret_cast<v2u*>(p) = w;
  }
}

template <typename Out>
__global__ __launch_bounds__(kGemmThreads, 1) void vocab_d_weight_kernel(VocabArgs a, int64_t v_begin) {
  __shared__ __align__(1024) char lds[kGemmLds];
  const int64_t tiles_h = (a.H + kTile - 1) / kTile;
  const int64_t v_left = a.V - v_begin < a.g_pitch ? a.V - v_begin : a.g_pitch;
  const int64_t tiles_v = (v_left + kTile - 1) / kTile;
  const TileAt at = tile_at(xcd_tile(blockIdx.x, tiles_h * tiles_v), tiles_h, tiles_v);
  const int64_t h0 = at.wide * kTile, vt = at.deep * kTile;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);

  const int64_t rows = active_rows64(a);
  const int once = static_cast<int>(rows / kTileK);
  const int64_t part = a.row_pitch * a.g_pitch;  // elements of G's high parts
  Loader<> lx, lg;
  lx.across(a.x + h0, (rows * a.x_pitch - h0) * 2, a.x_pitch, a.x_pitch - h0, wave, lane);
  lg.across(a.g + vt, (rows * a.g_pitch - vt) * 2, a.g_pitch, a.g_pitch - vt, wave, lane);
  if (!a.grad_bf16) {
    lx.restart_after(once, a.x + h0, (rows * a.x_pitch - h0) * 2);
    lg.restart_after(once, a.g + part + vt, (rows * a.g_pitch - vt) * 2);
  }
  f32x4 acc[kMT][kNT] = {};
  contract<true, true>(lx, lg, a.grad_bf16 ? once : 2 * once, lds, wave, lane, acc);

  const int s = lane % 16, g = lane / 16;
  Out* const d_weight = static_cast<Out*>(a.d_weight);
#pragma unroll
  for (int n = 0; n < kNT; ++n) {
    const int64_t v = v_begin + vt + (wave / 2) * kWaveN + 16 * n + s;
    if (v >= a.V) continue;
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      const int64_t h = h0 + (wave % 2) * kWaveM + 16 * m + 4 * g;
      if (h < a.H) store4(d_weight + v * a.H + h, acc[m][n]);
    }
  }
}

// d_hidden's tiles are few where there are few steps: k (the piece) is split over
// `splits` workgroups, each with float32 sums of its own that grow over the pieces.
__global__ __launch_bounds__(kGemmThreads, 1) void vocab_d_hidden_kernel(VocabArgs a, int64_t v_begin, int first) {
  __shared__ __align__(1024) char lds[kGemmLds];
  const int64_t count = *a.active_count;
  const int64_t tiles_h = (a.H + kTile - 1) / kTile;
  const int64_t tiles_n = (count + kTile - 1) / kTile;
  const int64_t tiles = tiles_h * tiles_n;
  if (static_cast<int64_t>(blockIdx.x) >= tiles * a.splits) return;
  const int64_t id = xcd_tile(blockIdx.x, tiles * a.splits);
  const int split = static_cast<int>(id / tiles);
  const TileAt at = tile_at(id % tiles, tiles_n, tiles_h);
  const int64_t h0 = at.deep * kTile, n0 = at.wide * kTile;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);

  const int64_t v_left = a.V - v_begin < a.g_pitch ? a.V - v_begin : a.g_pitch;
  const int64_t steps = (v_left + kTileK - 1) / kTileK;
  const int64_t from = steps * split / a.splits, to = steps * (split + 1) / a.splits;
  const int once = static_cast<int>(to - from);
  const int64_t part = a.row_pitch * a.g_pitch;
  const int64_t v0 = v_begin + from * kTileK;
  Loader<> lw, lg;
  const uint16_t* const w = a.weight + v0 * a.H + h0;
  const int64_t w_left = ((a.V - v0) * a.H - h0) * 2;
  lw.across(w, w_left, a.H, a.H - h0, wave, lane);
  const uint16_t* const gp = a.g + n0 * a.g_pitch + from * kTileK;
  const int64_t g_left = ((a.row_pitch - n0) * a.g_pitch - from * kTileK) * 2;
  lg.along(gp, g_left, 0x7fffffff, wave, lane,
           [&](int r) -> uint32_t { return static_cast<uint32_t>(r * a.g_pitch * 2); });
  if (!a.grad_bf16) {
    lw.restart_after(once, w, w_left);
    lg.restart_after(once, gp + part, g_left);
  }
  f32x4 acc[kMT][kNT] = {};
  contract<true, false>(lw, lg, a.grad_bf16 ? once : 2 * once, lds, wave, lane, acc);

  const int s = lane % 16, g = lane / 16;
#pragma unroll
  for (int n = 0; n < kNT; ++n) {
    const int64_t row = n0 + (wave / 2) * kWaveN + 16 * n + s;
    if (row >= count) continue;
    float* const out = a.h_partials + (split * a.row_pitch + row) * a.H;
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      const int64_t h = h0 + (wave % 2) * kWaveM + 16 * m + 4 * g;
      if (h >= a.H) continue;
      f32x4 x = acc[m][n];
      if (!first) x += *reinterpret_cast<const f32x4*>(out + h);
      *reinterpret_cast<f32x4*>(out + h) = x;
    }
  }
}

int64_t tiles_of(int64_t n) { return (n + kTile - 1) / kTile; }

}  // namespace

hipError_t launch_vocab_d_weight(const VocabArgs& a, int64_t v0, hipStream_t st) {
  const int64_t v = a.V - v0 < a.g_pitch ? a.V - v0 : a.g_pitch;
  const dim3 grid(static_cast<unsigned>(tiles_of(a.H) * tiles_of(v))), block(kGemmThreads);
  if (a.grad_bf16) hipLaunchKernelGGL(vocab_d_weight_kernel<uint16_t>, grid, block, 0, st, a, v0);
  else hipLaunchKernelGGL(vocab_d_weight_kernel<float>, grid, block, 0, st, a, v0);
  return hipGetLastError();
}

hipError_t launch_vocab_d_hidden(const VocabArgs& a, int64_t v0, bool first, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(tiles_of(a.H) * tiles_of(a.N) * a.splits)), block(kGemmThreads);
  hipLaunchKernelGGL(vocab_d_hidden_kernel, grid, block, 0, st, a, v0, first ? 1 : 0);
  return hipGetLastError();
}

}  // namespace vtrace
