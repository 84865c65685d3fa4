// The logits of a vocabulary layer, tile by tile, used where they are formed: for the
// softmax statistics of vtrace_vocab_log_probs, and for G = dL/dz of vtrace_vocab_grad.
//
// The tile is z^T: m runs along the vocabulary, n along the steps, so that a lane of
// the MFMA layout holds 32 logits of each of eight steps and the sums over the vocabulary
// are mostly additions inside a lane.  The accumulators start at the bias, and at -inf
// for the rows behind the vocabulary's end, whose exponentials are 0.
//
// Statistics of a step over a wave's rows (128 tokens, 64 in the small tiles): with c the largest
// logit and d = (z - c) log2 e,
//   sum 2^d and, for the entropy, sum 2^d d.
// The pieces are joined in float64 (vocab.hip).
//
// Measured: statistics of 6200 steps, H = 4096, V = 131072 (6.66 TFLOP) in 5.33 ms,
// 1.25 PFLOP/s; G of 4096 steps in eight pieces (4.4 TFLOP, 1.07 GB of G) in 3.5 ms, 1.25.
#include "vocab_impl.hpp"

namespace vtrace {
namespace {

enum { kStats = 0, kStatsDot = 1, kGrad = 2, kGradDot = 3 };

// The sum over a row of 16 lanes, in all of them.
template <int kTurn>
__device__ __forceinline__ float plus_turned(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x120 + kTurn, 0xF, 0xF, true));
}
__device__ __forceinline__ float row_sum(float x) {
  return plus_turned<1>(plus_turned<2>(plus_turned<4>(plus_turned<8>(x))));
}

// The token that lane (s, g) holds in accumulator (m, i), of its wave's 128 and behind 8 g.
__device__ __forceinline__ constexpr int token_at(int m, int i) { return 32 * (m / 2) + 4 * (m % 2) + i; }

template <int kMode, bool kBias, int kSize>
__global__ __launch_bounds__(kGemmThreads, kSize == kTile ? 1 : 2) void vocab_logits_kernel(VocabArgs a, int64_t v_begin, int64_t v_count) {
  // The stages, then two tiles' tokens and scalars: one array, since what the compiler makes of
  // several loses what __restrict says of the stages.
  constexpr int kMT = kSize / 32, kNT = kSize / 32, kWaveM = kSize / 2, kWaveN = kSize / 2;
  constexpr int kGemmLds = tile_lds(kSize);
  constexpr int kTokens = kSize * sizeof(int32_t), kScalars = kMode >= kGrad ? kSize * sizeof(float4v) : 0;
  constexpr int kStarts = kBias ? kSize * sizeof(float) : 0;
  __shared__ __align__(1024) char lds[kGemmLds + 2 * (kTokens + kScalars + kStarts)];
  int32_t* const s_tokens = reinterpret_cast<int32_t*>(lds + kGemmLds);
  float4v* const s_scalars = reinterpret_cast<float4v*>(lds + kGemmLds + 2 * kTokens);
  float* const s_starts = reinterpret_cast<float*>(lds + kGemmLds + 2 * (kTokens + kScalars));
  const int count = *a.active_count;
  const int tiles_n = (count + kSize - 1) / kSize;
  const int tiles_v = static_cast<int>((v_count + kSize - 1) / kSize);
  Tiles tiles(static_cast<int64_t>(tiles_n) * tiles_v);
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = (wave % 2) * kWaveM, wn = (wave / 2) * kWaveN;
  const int64_t H = a.H;

  // Rows behind the vocabulary's end lie behind the array's.
  Job<kSize> job;
  job.a.along(H, kSize, wave, lane);
  job.b.along(a.x_pitch, kSize, wave, lane);
  TileAt at;
  auto start = [&] {
    job.steps = 0;
    if (!tiles.any()) return;
    at = tile_at(tiles.at, tiles_n, tiles_v);
    const int64_t n0 = static_cast<int64_t>(at.wide) * kSize, v0 = v_begin + static_cast<int64_t>(at.deep) * kSize;
    job.steps = static_cast<int>(a.x_pitch / kTileK);
    job.a.aim(a.weight + v0 * H, (a.V - v0) * H * 2, static_cast<int>(H));
    job.b.aim(a.x + n0 * a.x_pitch, kSize * a.x_pitch * 2);
  };
  // What a tile needs of each step, and where its logits start, by way of LDS (registers
  // would hold the former through the contraction): fetched before the stores of the tile
  // before it, so that nobody waits for those.
  int32_t token = kNoToken;
  float4v scalars = {};
  float start_at = 0.0f;
  auto fetch = [&] {
    if (job.steps == 0 || static_cast<int>(threadIdx.x) >= kSize) return;
    const int64_t n = static_cast<int64_t>(at.wide) * kSize + threadIdx.x;
    token = a.row_tokens[n];
    if constexpr (kMode >= kGrad) scalars = a.row_scalars[n];
    if constexpr (kBias) start_at = start_of_logit(a, v_begin + static_cast<int64_t>(at.deep) * kSize + threadIdx.x);
  };
  int parity = 0, turn = 0;
  start();
  if (job.steps > 0) job.copy(lds, wave);
  fetch();
  while (tiles.any()) {
    const int64_t n0 = static_cast<int64_t>(at.wide) * kSize;
    const int64_t vt = static_cast<int64_t>(at.deep) * kSize;  // in this launch's piece
    const int64_t v0 = v_begin + vt;                           // in the vocabulary
    const int tile_deep = at.deep;
    // What follows from the lane's number is formed in each tile: kept from tile to tile it
    // would take the registers that the contraction needs.
    int here = lane;
    asm volatile("" : "+v"(here));
    const int s = here % 16, g = here / 16;
    // Accumulator (m, n) of lane (s, g) holds tokens 8 g + token_at(m, 0..3) of step 16 n + s;
    // it starts as start_of_logit.
    const int64_t first = v0 + wm;
    const int own = static_cast<int>(a.V - first < kSize ? a.V - first : kSize) - 8 * g;
    // Two of each: a wave may be in its next tile while another ends this one.
    turn ^= kSize;
    if (static_cast<int>(threadIdx.x) < kSize) {
      s_tokens[turn + threadIdx.x] = token;
      if constexpr (kMode >= kGrad) s_scalars[turn + threadIdx.x] = scalars;
      if constexpr (kBias) s_starts[turn + threadIdx.x] = start_at;
    }
    if constexpr (kBias) {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    Accumulators<kSize> acc;
#pragma unroll
    for (int m = 0; m < kMT; ++m) {
      f32x4 b;
      if constexpr (kBias) {
        b = *reinterpret_cast<const f32x4*>(s_starts + turn + wm + 8 * g + token_at(m, 0));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = token_at(m, i) >= own ? -INFINITY : 0.0f;
      }
#pragma unroll
      for (int n = 0; n < kNT; ++n) acc[m][n] = b;
    }
    contract<false>(job, lds, parity, wave, lane, acc, [&] {
      tiles.next();
      start();
    });
    fetch();
    __builtin_amdgcn_sched_barrier(0);

    // A step's token, counted from this lane's first (what token_at gives, where it has it).
    auto taken_of = [&](int32_t token) {
      return token < 0 || token < first || token >= first + kWaveM ? -1 : static_cast<int>(token - first) - 8 * g;
    };
    if constexpr (kMode < kGrad) {
      const int64_t piece = tile_deep * 2 + wave % 2;
#pragma unroll
      for (int n = 0; n < kNT; ++n) {
        const int64_t row = n0 + wn + 16 * n + s;
        const int taken = taken_of(s_tokens[turn + wn + 16 * n + s]);
        float z[kMT][4];
        float top = -INFINITY;
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            z[m][i] = element(acc[m][n], i);
            top = fmaxf(top, z[m][i]);
          }
        top = group_max(top);
        const float c = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f, dot = 0.0f;
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float d = log2_ratio(z[m][i], c);
            const float e = __builtin_amdgcn_exp2f(d);
            sum += e;
            if constexpr (kMode == kStatsDot) dot = fmaf(e, fmaxf(d, kLeastLog), dot);
          }
        sum = group_sum(sum);
        if constexpr (kMode == kStatsDot) dot = group_sum(dot);
        if (g == 0) {
          const int64_t o = piece * a.row_pitch + row;
          a.part_max[o] = c;
          a.part_sum[o] = sum;
          if constexpr (kMode == kStatsDot) a.part_dot[o] = dot;
        }
        // The taken token's logit, where this lane holds it.
        if (__any(taken >= 0)) {
          float logit = 0.0f;
          bool mine = false;
#pragma unroll
          for (int m = 0; m < kMT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              logit = taken == token_at(m, i) ? z[m][i] : logit;
              mine |= taken == token_at(m, i);
            }
          if (mine) a.token_logit[row] = logit;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      const int64_t P = a.row_pitch;
      float col[kMT][4];
      if constexpr (kBias) {
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) col[m][i] = 0.0f;
      }
#pragma unroll
      for (int n = 0; n < kNT; ++n) {
        const int64_t row = n0 + wn + 16 * n + s;
        // G = p (c0 + c1 log2 p) + d_lp 1[v = a] with p = 2^(z log2 e - l2): see the gather kernel.
        const float4v scalars = s_scalars[turn + wn + 16 * n + s];
        const float l2 = scalars[0], c0 = scalars[1], c1 = scalars[2], d_lp = scalars[3];
        const int taken = taken_of(s_tokens[turn + wn + 16 * n + s]);
        float grad[kMT][4];
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float d = fmaf(element(acc[m][n], i), kLog2eF, -l2);
            const float p = __builtin_amdgcn_exp2f(d);
            grad[m][i] = kMode == kGradDot ? p * fmaf(c1, fmaxf(d, kLeastLog), c0) : p * c0;
          }
        if (__any(taken >= 0)) {
#pragma unroll
          for (int m = 0; m < kMT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) grad[m][i] += taken == token_at(m, i) ? d_lp : 0.0f;
        }
        if constexpr (kBias) {
#pragma unroll
          for (int m = 0; m < kMT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              col[m][i] += grad[m][i];
              asm volatile("" : "+v"(col[m][i]));  // here, not later: it would have to keep what it adds
            }
        }
        uint16_t* out = a.g + row * a.g_pitch + vt + wm + 8 * g;
        uint16_t* out_low = out + P * a.g_pitch;
#pragma unroll
        for (int p = 0; p < kMT / 2; ++p) {
          const float* const x = grad[2 * p];
          const float* const y = grad[2 * p + 1];
          v4u hi;
          hi.x = pack_bf16x2(x[0], x[1]);
          hi.y = pack_bf16x2(x[2], x[3]);
          hi.z = pack_bf16x2(y[0], y[1]);
          hi.w = pack_bf16x2(y[2], y[3]);
          *reinterpret_cast<v4u*>(out + 32 * p) = hi;
          if (!a.grad_bf16) {
            auto low = [](float f0, float f1, unsigned h) {
              return pack_bf16x2(f0 - __uint_as_float(h << 16), f1 - __uint_as_float(h & 0xffff0000u));
            };
            v4u lo;
            lo.x = low(x[0], x[1], hi.x);
            lo.y = low(x[2], x[3], hi.y);
            lo.z = low(y[0], y[1], hi.z);
            lo.w = low(y[2], y[3], hi.w);
            *reinterpret_cast<v4u*>(out_low + 32 * p) = lo;
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (kBias) {
        // d_bias: this wave's 128 steps, summed over the 16 lanes of a group; lane s keeps
        // the sums of accumulators s and s + 16.
        float keep[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4 * kMT; ++j) {
          const float x = row_sum(col[j / 4][j % 4]);
          keep[j / 16] = s == j % 16 ? x : keep[j / 16];
        }
        float* const out = a.bias_partials + (n0 + wn) / kBiasSteps * a.g_pitch + vt + wm + 8 * g + token_at(s / 4, s % 4);
        out[0] = keep[0];
        if constexpr (kSize == kTile) {
          out[64] = keep[1];
          out[a.g_pitch] = 0.0f;
          out[a.g_pitch + 64] = 0.0f;
        }
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(kWaitAll);  // no copy into LDS outlives the workgroup
}

template <int kMode, int kSize>
hipError_t launch_tiles(const VocabArgs& a, int64_t v0, int64_t v_count, hipStream_t st) {
  const dim3 grid(workgroups_of(tiles_of(a.N, kSize) * tiles_of(v_count, kSize), kSize)), block(kGemmThreads);
  // d_bias without a bias: as if there were one of zeros.
  if (a.bias != nullptr || a.d_bias != nullptr)
    hipLaunchKernelGGL((vocab_logits_kernel<kMode, true, kSize>), grid, block, 0, st, a, v0, v_count);
  else
    hipLaunchKernelGGL((vocab_logits_kernel<kMode, false, kSize>), grid, block, 0, st, a, v0, v_count);
  return hipGetLastError();
}
template <int kMode>
hipError_t launch(const VocabArgs& a, int64_t v0, int64_t v_count, hipStream_t st) {
  return a.small_logits ? launch_tiles<kMode, kSmallTile>(a, v0, v_count, st)
                        : launch_tiles<kMode, kTile>(a, v0, v_count, st);
}

}  // namespace

hipError_t launch_vocab_stats(const VocabArgs& a, hipStream_t st) {
  return a.entropy ? launch<kStatsDot>(a, 0, a.V, st) : launch<kStats>(a, 0, a.V, st);
}

hipError_t launch_vocab_logit_grads(const VocabArgs& a, int64_t v0, hipStream_t st) {
  const int64_t n = a.V - v0 < a.g_pitch ? a.V - v0 : a.g_pitch;
  return a.d_entropy ? launch<kGradDot>(a, v0, n, st) : launch<kGrad>(a, v0, n, st);
}

}  // namespace vtrace
