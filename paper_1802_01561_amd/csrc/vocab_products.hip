// The two products of vtrace_vocab_grad with G = dL/dz of one piece of the vocabulary:
//   d_weight[v, h] = sum_n G[n, v] x[n, h],   d_hidden[n, h] += sum_v G[n, v] weight[v, h].
// In both, m runs along h, so that a lane holds four consecutive elements of a row of
// the result.  G's low parts, where there are any, are a second pass over k: G = high + low
// to 2^-17 of itself (half a step of bfloat16 twice), for float32 outputs.
//
// Measured: 4096 steps, H = 4096, V = 131072, bfloat16, in eight pieces (4.4 TFLOP each)
// d_weight 3.31 ms, 1.33 PFLOP/s, d_hidden 3.22 ms, 1.37.
#include "vocab_impl.hpp"

namespace vtrace {
namespace {

__device__ __forceinline__ int64_t active_rows64(const VocabArgs& a) {
  return (static_cast<int64_t>(*a.active_count) + kTileK - 1) / kTileK * kTileK;
}

__device__ __forceinline__ f32x4 load4(Rsrc r, uint32_t offset) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, offset, 0, 0));
}

template <typename Out>
__device__ __forceinline__ void store4(Rsrc r, uint32_t offset, const f32x4& x) {
  if constexpr (sizeof(Out) == 4) {
    const f32x4 w = {element(x, 0), element(x, 1), element(x, 2), element(x, 3)};
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, w), r, offset, 0, 0);
  } else {
    v2u w;
    w.x = pack_bf16x2(element(x, 0), element(x, 1));
    w.y = pack_bf16x2(element(x, 2), element(x, 3));
    __builtin_amdgcn_raw_buffer_store_b64(w, r, offset, 0, 0);
  }
}

template <typename Out, int kSize>
__global__ __launch_bounds__(kGemmThreads, kSize == kTile ? 1 : 2) void vocab_d_weight_kernel(VocabArgs a, int64_t v_begin) {
  constexpr int kMT = kSize / 32, kNT = kSize / 32;
  __shared__ __align__(1024) char lds[tile_lds(kSize)];
  const int tiles_h = static_cast<int>((a.H + kSize - 1) / kSize);
  const int64_t v_left = a.V - v_begin < a.g_pitch ? a.V - v_begin : a.g_pitch;
  const int tiles_v = static_cast<int>((v_left + kSize - 1) / kSize);
  Tiles tiles(static_cast<int64_t>(tiles_h) * tiles_v);
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;
  const int64_t rows = active_rows64(a);
  const int once = rows == 0 ? 1 : static_cast<int>(rows / kTileK);  // no rows: a step of nothing
  const int64_t part = a.row_pitch * a.g_pitch;  // elements of G's high parts

  Job<kSize> job;
  job.a.across(a.x_pitch, wave, lane);
  job.b.across(a.g_pitch, wave, lane);
  TileAt at;
  auto start = [&] {
    job.steps = 0;
    if (!tiles.any()) return;
    at = tile_at(tiles.at, tiles_h, tiles_v);
    const int64_t h0 = static_cast<int64_t>(at.wide) * kSize, vt = static_cast<int64_t>(at.deep) * kSize;
    job.a.aim(a.x + h0, (rows * a.x_pitch - h0) * 2);
    job.b.aim(a.g + vt, (rows * a.g_pitch - vt) * 2);
    job.steps = once;
    if (!a.grad_bf16) {
      job.a.restart_after(once, a.x + h0, (rows * a.x_pitch - h0) * 2);
      job.b.restart_after(once, a.g + part + vt, (rows * a.g_pitch - vt) * 2);
      job.steps = 2 * once;
    }
  };
  int parity = 0;
  start();
  if (job.steps > 0) job.copy(lds, wave);
  while (tiles.any()) {
    const int64_t h0 = static_cast<int64_t>(at.wide) * kSize, vt = static_cast<int64_t>(at.deep) * kSize;
    Accumulators<kSize> acc = {};
    contract<true>(job, lds, parity, wave, lane, acc, [&] {
      tiles.next();
      start();
    });
    // Rows behind the vocabulary's end lie behind the array's; columns behind a row's end
    // are pointed there.
    const int64_t first = (v_begin + vt) * a.H;
    const Rsrc out = make_rsrc(static_cast<Out*>(a.d_weight) + first, (a.V * a.H - first) * static_cast<int>(sizeof(Out)));
    const int64_t h = h0 + (wave % 2) * (kSize / 2) + 4 * g;
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      const uint32_t row = static_cast<uint32_t>((((wave / 2) * (kSize / 2) + 16 * n + s) * a.H + h) * sizeof(Out));
#pragma unroll
      for (int m = 0; m < kMT; ++m)
        store4<Out>(out, h + 16 * m < a.H ? row + 16 * m * static_cast<uint32_t>(sizeof(Out)) : kOutOfRange, acc[m][n]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy into LDS outlives the workgroup
}

// d_hidden's tiles are few where there are few steps: k (the piece) is split into `splits`
// parts, each with float32 sums of its own that grow over the pieces (how many parts is
// chosen on the device: best_split).
template <int kSize>
__global__ __launch_bounds__(kGemmThreads, kSize == kTile ? 1 : 2) void vocab_d_hidden_kernel(VocabArgs a, int64_t v_begin, int first) {
  __shared__ __align__(1024) char lds[tile_lds(kSize)];
  constexpr int kMT = kSize / 32, kNT = kSize / 32;
  const int count = *a.active_count;
  const int tiles_h = static_cast<int>((a.H + kSize - 1) / kSize);
  const int tiles_n = (count + kSize - 1) / kSize;
  const int per_split = tiles_h * tiles_n, splits = *a.splits;
  Tiles tiles(static_cast<int64_t>(per_split) * splits);
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;
  const int64_t v_left = a.V - v_begin < a.g_pitch ? a.V - v_begin : a.g_pitch;
  const int all_steps = static_cast<int>((v_left + kTileK - 1) / kTileK);
  const int64_t part = a.row_pitch * a.g_pitch;

  struct Part {
    int64_t h0, n0;
    int split, from, to;
  };
  auto part_of = [&](int id) {
    const int split = id / per_split;
    const TileAt at = tile_at(id % per_split, tiles_n, tiles_h);
    return Part{static_cast<int64_t>(at.deep) * kSize, static_cast<int64_t>(at.wide) * kSize, split,
                static_cast<int>(static_cast<int64_t>(all_steps) * split / splits),
                static_cast<int>(static_cast<int64_t>(all_steps) * (split + 1) / splits)};
  };
  const int passes = a.grad_bf16 ? 1 : 2;
  auto once_of = [&](const Part& p) { return p.to == p.from ? 1 : p.to - p.from; };  // nothing left: a step of nothing
  Feed<kSize> ws(tiles), gs(tiles);
  ws.load.across(a.H, wave, lane);
  ws.load.step /= 2;
  gs.load.along(a.g_pitch, kSize, wave, lane);
  auto start_w = [&](Feed<kSize>& f) {
    const Part p = part_of(f.tiles.at);
    const int64_t v0 = v_begin + static_cast<int64_t>(p.from) * kTileK;
    const uint16_t* const w = a.weight + v0 * a.H + p.h0;
    const int64_t left = p.to == p.from ? 0 : ((a.V - v0) * a.H - p.h0) * 2;
    f.load.aim(w, left);
    if (passes == 2) f.load.restart_after(2 * once_of(p), w, left);
    return 2 * passes * once_of(p);
  };
  auto start_g = [&](Feed<kSize>& f) {
    const Part p = part_of(f.tiles.at);
    const uint16_t* const gp = a.g + p.n0 * a.g_pitch + static_cast<int64_t>(p.from) * kTileK;
    const int64_t left = ((a.row_pitch - p.n0) * a.g_pitch - static_cast<int64_t>(p.from) * kTileK) * 2;
    f.load.aim(gp, left);
    if (passes == 2) f.load.restart_after(once_of(p), gp + part, left);
    return passes * once_of(p);
  };
  int parity = 0;
  if (tiles.any()) start_halves(ws, gs, lds, wave, start_w, start_g);
  for (; tiles.any(); tiles.next()) {
    const Part p = part_of(tiles.at);
    const int64_t h0 = p.h0, n0 = p.n0;
    float* const sums = a.h_partials + static_cast<int64_t>(p.split) * tiles_n * kSize * a.H;
    Accumulators<kSize> acc = {};
    contract_halves(passes * once_of(p), ws, gs, lds, parity, wave, lane, acc, start_w, start_g);
    // Later pieces add to what the earlier ones left: the next step's row is fetched while
    // this one's is added to.
    const Rsrc out = make_rsrc(sums + n0 * a.H, (count - n0) * a.H * 4);
    const Rsrc before = make_rsrc(sums + n0 * a.H, first ? 0 : (count - n0) * a.H * 4);
    const int64_t h = h0 + (wave % 2) * (kSize / 2) + 4 * g;
    auto place = [&](int n, int m) -> uint32_t {
      const int row = (wave / 2) * (kSize / 2) + 16 * n + s;
      return h + 16 * m < a.H ? static_cast<uint32_t>((row * a.H + h + 16 * m) * 4) : kOutOfRange;
    };
    f32x4 was[2][kMT];
#pragma unroll
    for (int m = 0; m < kMT; ++m) was[0][m] = load4(before, place(0, m));
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      if (n + 1 < kNT) {
#pragma unroll
        for (int m = 0; m < kMT; ++m) was[(n + 1) % 2][m] = load4(before, place(n + 1, m));
      }
#pragma unroll
      for (int m = 0; m < kMT; ++m) {
        f32x4 x = was[n % 2][m];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += element(acc[m][n], i);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, x), out, place(n, m), 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy into LDS outlives the workgroup
}

template <typename Out, int kSize>
hipError_t launch_d_weight(const VocabArgs& a, int64_t v0, hipStream_t st) {
  const int64_t v = a.V - v0 < a.g_pitch ? a.V - v0 : a.g_pitch;
  const dim3 grid(workgroups_of(tiles_of(a.H, kSize) * tiles_of(v, kSize), kSize)), block(kGemmThreads);
  hipLaunchKernelGGL((vocab_d_weight_kernel<Out, kSize>), grid, block, 0, st, a, v0);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_vocab_d_weight(const VocabArgs& a, int64_t v0, hipStream_t st) {
  if (a.grad_bf16)
    return a.small_weight ? launch_d_weight<uint16_t, kSmallTile>(a, v0, st) : launch_d_weight<uint16_t, kTile>(a, v0, st);
  return a.small_weight ? launch_d_weight<float, kSmallTile>(a, v0, st) : launch_d_weight<float, kTile>(a, v0, st);
}

hipError_t launch_vocab_d_hidden(const VocabArgs& a, int64_t v0, bool first, hipStream_t st) {
  // How many tiles there are is known on the device: as many workgroups as fit.
  const dim3 grid(resident_tiles(a.small_hidden ? kSmallTile : kTile)), block(kGemmThreads);
  if (a.small_hidden) hipLaunchKernelGGL(vocab_d_hidden_kernel<kSmallTile>, grid, block, 0, st, a, v0, first ? 1 : 0);
  else hipLaunchKernelGGL(vocab_d_hidden_kernel<kTile>, grid, block, 0, st, a, v0, first ? 1 : 0);
  return hipGetLastError();
}

}  // namespace vtrace
