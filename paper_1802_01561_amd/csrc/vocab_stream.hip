// vtrace_vocab_log_probs for few steps (up to 128): the vocabulary layer is read once, and
// that is what bounds it.  Two kernels; which one takes a call is chosen in vocab.hip.
//
// Up to 64 steps of a small layer: rows from memory straight into matrix-core operands.
// A workgroup of four waves takes 16 R tokens and all steps.  The waves share out the
// hidden units, 64 (a 128-byte line of each row) at a time; their partial logits meet
// in LDS, where each wave takes some of the 16 x 16 pieces, adds the bias and forms the
// softmax statistics as in vocab_logits.hip.  20 steps, H = 256, V = 32768 (17 MB) 8 us and 4
// for the join.
#include "vocab_impl.hpp"

namespace vtrace {
namespace {

constexpr int kStreamThreads = 256;
constexpr int kStreamWaves = 4;

template <int R, int NT, bool kDot>
__global__ __launch_bounds__(kStreamThreads) void vocab_stream_kernel(VocabArgs a) {
  __shared__ f32x4 s_part[kStreamWaves][R * NT][kWave];
  __shared__ float s_stat[3][R][NT * 16];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;
  const int64_t H = a.H;
  const int64_t tiles = (a.V + 16 * R - 1) / (16 * R);
  const int steps = static_cast<int>((H + 63) / 64);
  const Rsrc rx = make_rsrc(a.hidden, a.N * H * 2);
  uint32_t ow[R], ox[NT];
#pragma unroll
  for (int r = 0; r < R; ++r) ow[r] = static_cast<uint32_t>((16 * r + s) * H * 2) + 16 * g;
#pragma unroll
  for (int n = 0; n < NT; ++n)
    ox[n] = 16 * n + s < a.N ? static_cast<uint32_t>((16 * n + s) * H * 2) + 16 * g : kOutOfRange;

  v4u w[2][R], x[2][NT];
  // Rows behind the vocabulary's end lie behind the descriptor's.
  auto load = [&](int64_t tile, int step) {
    const Rsrc rw = make_rsrc(a.weight + tile * (16 * R) * H, (a.V - tile * (16 * R)) * H * 2);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const int k = step * 64 + kk * 32;
      const bool in = k + 8 * g < H;
#pragma unroll
      for (int r = 0; r < R; ++r)
        w[kk][r] = __builtin_amdgcn_raw_buffer_load_b128(rw, in ? ow[r] + 2 * k : kOutOfRange, 0, 0);
#pragma unroll
      for (int n = 0; n < NT; ++n)
        x[kk][n] = __builtin_amdgcn_raw_buffer_load_b128(rx, in ? ox[n] + 2 * k : kOutOfRange, 0, 0);
    }
  };
  // This thread's row of the statistics, over the workgroup's tiles.
  float run_c = -INFINITY, run_sum = 0.0f, run_dot = 0.0f;
  if (wave < steps) load(blockIdx.x, wave);
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t v0 = tile * (16 * R);
    f32x4 acc[R][NT] = {};
    for (int step = wave; step < steps; step += kStreamWaves) {
      bf16x8 wa[2][R], xb[2][NT];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
        for (int r = 0; r < R; ++r) wa[kk][r] = __builtin_bit_cast(bf16x8, w[kk][r]);
#pragma unroll
        for (int n = 0; n < NT; ++n) xb[kk][n] = __builtin_bit_cast(bf16x8, x[kk][n]);
      }
      // The next step, or the next tile's first (its loads are in flight over the epilogue).
      if (step + kStreamWaves < steps) load(tile, step + kStreamWaves);
      else if (tile + gridDim.x < tiles) load(tile + gridDim.x, wave);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            acc[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[kk][r], xb[kk][n], acc[r][n], 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int n = 0; n < NT; ++n) s_part[wave][r * NT + n][lane] = acc[r][n];
    __syncthreads();

    for (int q = wave; q < R * NT; q += kStreamWaves) {
      const int r = q / NT, n = q % NT;
      f32x4 z = s_part[0][q][lane] + s_part[1][q][lane] + (s_part[2][q][lane] + s_part[3][q][lane]);
      const int64_t v = v0 + 16 * r + 4 * g;  // tokens v .. v + 3 of step 16 n + s
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[i] += start_of_logit(a, v + i);
        top = fmaxf(top, z[i]);
      }
      top = group_max(top);
      const float c = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f, dot = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float d = log2_ratio(z[i], c);
        const float e = __builtin_amdgcn_exp2f(d);
        sum += e;
        dot = fmaf(e, fmaxf(d, kLeastLog), dot);
      }
      sum = group_sum(sum);
      if constexpr (kDot) dot = group_sum(dot);
      const int row = 16 * n + s;
      if (g == 0) {
        // A piece of nothing but -inf logits has no maximum.
        s_stat[0][r][row] = sum == 0.0f ? -INFINITY : c;
        s_stat[1][r][row] = sum;
        if constexpr (kDot) s_stat[2][r][row] = dot;
      }
      const int32_t token = row < a.N ? a.tokens[row] : kNoToken;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (token >= 0 && token == v + i && v + i < a.V) a.token_logit[row] = z[i];
    }
    __syncthreads();
    if (threadIdx.x < NT * 16) {
      const int row = threadIdx.x;
      float c = run_c;
#pragma unroll
      for (int r = 0; r < R; ++r) c = fmaxf(c, s_stat[0][r][row]);
      auto add = [&](float part_c, float part, float part_dot) {
        const float d = part_c == -INFINITY ? 0.0f : log2_ratio(part_c, c);
        const float e = __builtin_amdgcn_exp2f(d), p = part * e;
        run_sum += p;
        if constexpr (kDot) run_dot += fmaf(p, d, part_dot * e);
      };
      const float was_sum = run_sum, was_dot = run_dot;
      run_sum = 0.0f;
      run_dot = 0.0f;
      add(run_c, was_sum, was_dot);
#pragma unroll
      for (int r = 0; r < R; ++r) add(s_stat[0][r][row], s_stat[1][r][row], kDot ? s_stat[2][r][row] : 0.0f);
      run_c = c;
    }
  }
  if (threadIdx.x < a.N) {
    const int64_t o = static_cast<int64_t>(threadIdx.x) * a.pieces + blockIdx.x;
    a.part_max[o] = run_c == -INFINITY ? 0.0f : run_c;
    a.part_sum[o] = run_sum;
    if constexpr (kDot) a.part_dot[o] = run_dot;
  }
}

// Up to 128 steps of a large layer: the layer passes through LDS, copied there two or more
// steps of 64 hidden units ahead, so that the copies take no registers and the hidden
// states are fetched once for 128 or 256 tokens (in the kernel above they weigh as much as
// the rows: 48 steps, H = 2048, V = 100003 (410 MB) 131 -> 85 to 92 us, 4.4 to 4.8 TB/s; one step,
// H = 4096, V = 131072 (1.07 GB) 212 us, 5.1 TB/s, where plain reads of this pattern reach 4.7
// to 5.9).  Each wave has 32 of the tile's tokens and all steps, and
// keeps their statistics in registers from tile to tile.  A tile holds as many tokens as
// share the vocabulary out evenly over the resident workgroups; up to 64 steps these are
// mostly two a CU of four waves each, whose barriers do not meet (one of eight waves: 104 us
// instead of 93).  The copies run on across the tiles: the sequence of (tile, step) is flat.
template <int kRows, int kWaves, int kPerCu, bool kDot>
__global__ __launch_bounds__(kWaves* kWave, kPerCu* kWaves / 4) void vocab_narrow_kernel(VocabArgs a) {
  constexpr int NT = kRows / 16;
  constexpr int kTileTokens = 32 * kWaves;
  constexpr int kWBytes = kTileTokens * kTileK * 2;
  constexpr int kStage = kWBytes + kRows * kTileK * 2;
  constexpr int kNarrowStages = 160 * 1024 / kPerCu / kStage;  // all of LDS, between the CU's workgroups
  __shared__ __align__(1024) char lds[kNarrowStages * kStage];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;
  const int64_t H = a.H;
  const int tokens = a.tile_tokens;
  const int64_t tiles = (a.V + tokens - 1) / tokens;
  const int steps = static_cast<int>((H + kTileK - 1) / kTileK);

  Loader<kTileTokens, kWaves> lw;
  Loader<kRows, kWaves> lx;
  lw.along(H, tokens, wave, lane);
  lx.along(H, static_cast<int>(a.N), wave, lane);
  int64_t load_tile = blockIdx.x;
  int load_step = 0;
  auto start_tile = [&] {
    const int64_t v0 = load_tile * tokens;
    const bool any = load_tile < tiles;
    lw.aim(a.weight + v0 * H, any ? (a.V - v0) * H * 2 : 0, static_cast<int>(H));
    lx.aim(a.hidden, any ? a.N * H * 2 : 0, static_cast<int>(H));
  };
  // Behind the last tile everything is out of range: the number of copies in flight stays
  // the same, and with it what a wait for the oldest means.
  auto copy = [&](int stage) {
    char* const to = lds + stage * kStage;
    lw.copy(to, wave);
    lx.copy(to + kWBytes, wave);
    if (++load_step == steps) {
      load_step = 0;
      load_tile += gridDim.x;
      start_tile();
    }
  };
  constexpr int kCopies = Loader<kTileTokens, kWaves>::kCopies + Loader<kRows, kWaves>::kCopies;
  constexpr int kInFlight = kCopies * (kNarrowStages - 2);
  static_assert(kInFlight < 64, "vmcnt's six bits");
  // vmcnt(kInFlight) lgkmcnt(0)
  constexpr int kWaitOldest = (kInFlight & 15) | (kInFlight >> 4) << 14 | 0x0070;

  Reader<false, true, 2> rw;
  Reader<false, false, NT> rx;
  rw.start(wave * 32, s, g);
  rx.start(0, s, g);
  float run_c[NT], run_sum[NT], run_dot[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    run_c[n] = -INFINITY;
    run_sum[n] = 0.0f;
    run_dot[n] = 0.0f;
  }
  start_tile();
  for (int i = 0; i < kNarrowStages - 1; ++i) copy(i);
  int stage = 0;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t v0 = tile * tokens + wave * 32 + 8 * g;
    f32x4 acc[2][NT];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      f32x4 b;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        b[i] = wave * 32 + 8 * g + 4 * m + i < tokens ? start_of_logit(a, v0 + 4 * m + i) : -INFINITY;
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[m][n] = b;
    }
    for (int step = 0; step < steps; ++step) {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(kWaitOldest);
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      copy(stage == 0 ? kNarrowStages - 1 : stage - 1);
      const char* const cur = lds + stage * kStage;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        bf16x8 w[2], x[NT];
#pragma unroll
        for (int m = 0; m < 2; ++m) w[m] = rw.read(cur, m, kk);
#pragma unroll
        for (int n = 0; n < NT; ++n) x[n] = rx.read(cur + kWBytes, n, kk);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[m], x[n], acc[m][n], 0, 0, 0);
      }
      stage = stage == kNarrowStages - 1 ? 0 : stage + 1;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = 16 * n + s;
      const int32_t token = row < a.N ? a.tokens[row] : kNoToken;
      float top = -INFINITY;
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          top = fmaxf(top, acc[m][n][i]);
          if (token >= 0 && token < a.V && token == v0 + 4 * m + i && wave * 32 + 8 * g + 4 * m + i < tokens)
            a.token_logit[row] = acc[m][n][i];
        }
      top = group_max(top);
      const float c = fmaxf(run_c[n], top), zero = c == -INFINITY ? 0.0f : c;
      float sum = 0.0f, dot = 0.0f;
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float d = log2_ratio(acc[m][n][i], zero);
          const float e = __builtin_amdgcn_exp2f(d);
          sum += e;
          if constexpr (kDot) dot = fmaf(e, fmaxf(d, kLeastLog), dot);
        }
      // The lane's sums so far, moved to the new maximum.
      const float d = run_c[n] == -INFINITY ? 0.0f : log2_ratio(run_c[n], c);
      const float e = __builtin_amdgcn_exp2f(d), p = run_sum[n] * e;
      if constexpr (kDot) run_dot[n] = fmaf(p, d, run_dot[n] * e) + dot;
      run_sum[n] = p + sum;
      run_c[n] = c;
    }
  }
  // The waves' statistics of each step, joined in LDS (behind the last copies).
  __builtin_amdgcn_s_waitcnt(kWaitAll);
  __syncthreads();
  float* const s_stat = reinterpret_cast<float*>(lds);  // [3][kWaves][kRows]
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const float sum = group_sum(run_sum[n]);
    const float dot = kDot ? group_sum(run_dot[n]) : 0.0f;
    if (g == 0) {
      float* const p = s_stat + wave * kRows + 16 * n + s;
      p[0] = run_c[n];
      p[kWaves * kRows] = sum;
      p[2 * kWaves * kRows] = dot;
    }
  }
  __syncthreads();
  const int row = threadIdx.x;
  if (row >= a.N) return;
  float c = -INFINITY, sum = 0.0f, dot = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) c = fmaxf(c, s_stat[w * kRows + row]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float* const p = s_stat + w * kRows + row;
    const float d = p[0] == -INFINITY ? 0.0f : log2_ratio(p[0], c);
    const float e = __builtin_amdgcn_exp2f(d), part = p[kWaves * kRows] * e;
    sum += part;
    dot += fmaf(part, d, p[2 * kWaves * kRows] * e);
  }
  const int64_t o = row * a.pieces + blockIdx.x;
  a.part_max[o] = c == -INFINITY ? 0.0f : c;
  a.part_sum[o] = sum;
  if constexpr (kDot) a.part_dot[o] = dot;
}

// A plan that a kernel does not cover (its steps would be left without statistics) is refused.
template <int R, int NT, bool kDot>
hipError_t launch_stream(const VocabArgs& a, hipStream_t st) {
  if (a.N > 16 * NT || a.tile_tokens != 16 * R) return hipErrorInvalidValue;
  hipLaunchKernelGGL((vocab_stream_kernel<R, NT, kDot>), dim3(static_cast<unsigned>(a.pieces)), dim3(kStreamThreads), 0,
                     st, a);
  return hipGetLastError();
}
template <int R, bool kDot>
hipError_t launch_stream_rows(const VocabArgs& a, hipStream_t st) {
  if (a.N <= 16) return launch_stream<R, 1, kDot>(a, st);
  if constexpr (R == 4) return launch_stream<R, 2, kDot>(a, st);
  else return a.N <= 32 ? launch_stream<R, 2, kDot>(a, st) : launch_stream<R, 4, kDot>(a, st);
}
template <int kRows, int kWaves, int kPerCu, bool kDot>
hipError_t launch_narrow(const VocabArgs& a, hipStream_t st) {
  if (a.N > kRows || a.tile_tokens > 32 * kWaves) return hipErrorInvalidValue;
  hipLaunchKernelGGL((vocab_narrow_kernel<kRows, kWaves, kPerCu, kDot>), dim3(static_cast<unsigned>(a.pieces)),
                     dim3(kWaves * kWave), 0, st, a);
  return hipGetLastError();
}
template <bool kDot>
hipError_t launch(const VocabArgs& a, hipStream_t st) {
  if (a.narrow && a.N <= 32 && a.narrow_per_cu == 1) return launch_narrow<32, 4, 1, kDot>(a, st);
  if (a.narrow && a.N <= 32) return launch_narrow<32, 4, 2, kDot>(a, st);
  if (a.narrow && a.N <= 64) return launch_narrow<64, 4, 2, kDot>(a, st);
  if (a.narrow) return launch_narrow<128, 8, 1, kDot>(a, st);
  if (a.tile_tokens == 64) return launch_stream_rows<4, kDot>(a, st);
  if (a.tile_tokens == 32) return launch_stream_rows<2, kDot>(a, st);
  return launch_stream_rows<1, kDot>(a, st);
}

}  // namespace

hipError_t launch_vocab_few(const VocabArgs& a, hipStream_t st) {
  return a.entropy ? launch<true>(a, st) : launch<false>(a, st);
}

}  // namespace vtrace
