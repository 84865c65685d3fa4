// The logits of a vocabulary layer, tile by tile, used where they are formed: for the
// softmax statistics of vtrace_vocab_log_probs, and for G = dL/dz of vtrace_vocab_grad.
//
// The tile is z^T: m runs along the vocabulary, n along the steps, so that a lane of
// the MFMA layout holds 32 logits of each of four steps and the sums over the vocabulary
// are mostly additions inside a lane.  The accumulators start at the bias, and at -inf
// for the rows behind the vocabulary's end, whose exponentials are 0.
//
// Statistics of a step over 128 tokens (a wave's rows): with d = z log2 e - c, c the
// rounded maximum of z log2 e,
//   sum 2^d and, for the entropy, sum 2^d d.
// They are exact about c (not about the maximum before rounding), and the pieces are
// joined in float64 (vocab.hip).
#include "vocab_impl.hpp"

namespace vtrace {
namespace {

enum { kStats = 0, kStatsDot = 1, kGrad = 2, kGradDot = 3 };

template <int kMode>
__global__ __launch_bounds__(kGemmThreads, 1) void vocab_logits_kernel(VocabArgs a, int64_t v_begin, int64_t v_count) {
  __shared__ __align__(1024) char lds[kGemmLds];
  const int64_t count = *a.active_count;
  const int64_t tiles_n = (count + kTile - 1) / kTile;
  const int64_t tiles_v = (v_count + kTile - 1) / kTile;
  if (static_cast<int64_t>(blockIdx.x) >= tiles_n * tiles_v) return;
  const TileAt at = tile_at(xcd_tile(blockIdx.x, tiles_n * tiles_v), tiles_n, tiles_v);
  const int64_t n0 = at.wide * kTile;
  const int64_t vt = at.deep * kTile;    // in this launch's piece
  const int64_t v0 = v_begin + vt;       // in the vocabulary
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int s = lane % 16, g = lane / 16;
  const int wm = (wave % 2) * kWaveM, wn = (wave / 2) * kWaveN;

  Loader<> lw, lx;
  const int64_t H = a.H;
  lw.along(a.weight + v0 * H, (a.V - v0) * H * 2, static_cast<int>(H), wave, lane, [&](int r) -> uint32_t {
    return v0 + r < a.V ? static_cast<uint32_t>(r * H * 2) : kOutOfRange;
  });
  if constexpr (kMode >= kGrad) {
    lx.along(a.x + n0 * a.x_pitch, kTile * a.x_pitch * 2, static_cast<int>(a.x_pitch), wave, lane,
             [&](int r) -> uint32_t { return static_cast<uint32_t>(r * a.x_pitch * 2); });
  } else {
    lx.along(a.hidden, a.N * H * 2, static_cast<int>(H), wave, lane, [&](int r) -> uint32_t {
      return n0 + r < count ? static_cast<uint32_t>(static_cast<int64_t>(a.active[n0 + r]) * H * 2) : kOutOfRange;
    });
  }

  // Lane (s, g) holds tokens v(m, i) = 32 (m / 2) + 8 g + 4 (m % 2) + i of steps 16 n + s.
  f32x4 acc[kMT][kNT];
#pragma unroll
  for (int m = 0; m < kMT; ++m) {
    f32x4 b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t v = v0 + wm + 32 * (m / 2) + 8 * g + 4 * (m % 2) + i;
      b[i] = start_of_logit(a, v);
    }
#pragma unroll
    for (int n = 0; n < kNT; ++n) acc[m][n] = b;
  }
  const int steps = static_cast<int>((H + kTileK - 1) / kTileK);
  contract<false, false>(lw, lx, steps, lds, wave, lane, acc);

  if constexpr (kMode < kGrad) {
    const int64_t piece = at.deep * 2 + wave % 2;
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      const int64_t row = n0 + wn + 16 * n + s;
      float top = -INFINITY;
#pragma unroll
      for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, acc[m][n][i]);
      top = group_max(top);
      const float c = top == -INFINITY ? 0.0f : top * kLog2eF;
      float sum = 0.0f, dot = 0.0f;
#pragma unroll
      for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float d = fmaf(acc[m][n][i], kLog2eF, -c);
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
      const int32_t token = row < count ? a.tokens[a.active[row]] : kNoToken;
      const int64_t in = token - (v0 + wm);
      if (__any(token >= 0 && in >= 0 && in < kWaveM)) {
#pragma unroll
        for (int m = 0; m < kMT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (in == 32 * (m / 2) + 8 * g + 4 * (m % 2) + i) a.token_logit[row] = acc[m][n][i];
      }
    }
  } else {
    const int64_t P = a.row_pitch;
    float col[kMT][4];
#pragma unroll
    for (int m = 0; m < kMT; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) col[m][i] = 0.0f;
    const bool edge = n0 + kTile > count;
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
      const int64_t row = n0 + wn + 16 * n + s;
      const float lse = a.row_scalars[row], c0 = a.row_scalars[P + row];
      const float c1 = kMode == kGradDot ? a.row_scalars[2 * P + row] : 0.0f;
      const float d_lp = a.row_scalars[3 * P + row];
      const int32_t token = __float_as_int(a.row_scalars[4 * P + row]);
      const int64_t in = token - (v0 + wm);
      const bool here = __any(token >= 0 && in >= 0 && in < kWaveM);
#pragma unroll
      for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lp = acc[m][n][i] - lse;
          const float p = __builtin_amdgcn_exp2f(lp * kLog2eF);
          float d = kMode == kGradDot ? p * fmaf(c1, fmaxf(lp, kLeastLog), c0) : p * c0;
          if (edge && row >= count) d = 0.0f;
          if (here && in == 32 * (m / 2) + 8 * g + 4 * (m % 2) + i) d += d_lp;
          acc[m][n][i] = d;
          col[m][i] += d;
        }
      uint16_t* out = a.g + row * a.g_pitch + vt + wm + 8 * g;
      uint16_t* out_low = out + P * a.g_pitch;
#pragma unroll
      for (int p = 0; p < kMT / 2; ++p) {
        v4u hi;
        const f32x4 x = acc[2 * p][n], y = acc[2 * p + 1][n];
        hi.x = pack_bf16x2(x[0], x[1]);
        hi.y = pack_bf16x2(x[2], x[3]);
        hi.z = pack_bf16x2(y[0], y[1]);
        hi.w = pack_bf16x2(y[2], y[3]);
        *reinterpret_cast<v4u*>(out + 32 * p) = hi;
        if (!a.grad_bf16) {
          auto low = [](float f, unsigned h) { return f - __uint_as_float(h << 16); };
          auto low2 = [&](float f0, float f1, unsigned h) {
            return pack_bf16x2(low(f0, h & 0xffffu), low(f1, h >> 16));
          };
          v4u lo;
          lo.x = low2(x[0], x[1], hi.x);
          lo.y = low2(x[2], x[3], hi.y);
          lo.z = low2(y[0], y[1], hi.z);
          lo.w = low2(y[2], y[3], hi.w);
          *reinterpret_cast<v4u*>(out_low + 32 * p) = lo;
        }
      }
    }
    if (a.d_bias != nullptr) {
      // d_bias: this wave's 128 steps, summed over the 16 lanes of a group.
#pragma unroll
      for (int m = 0; m < kMT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = col[m][i];
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) x += __shfl_xor(x, o, 16);
          if (s == 0)
            a.bias_partials[(at.wide * (kTile / kWaveN) + wave / 2) * a.g_pitch + vt + wm + 32 * (m / 2) + 8 * g + 4 * (m % 2) + i] = x;
        }
    }
  }
}

template <int kMode>
hipError_t launch(const VocabArgs& a, int64_t v0, int64_t v_count, hipStream_t st) {
  const int64_t tiles = (a.row_pitch / kTile) * ((v_count + kTile - 1) / kTile);
  hipLaunchKernelGGL(vocab_logits_kernel<kMode>, dim3(static_cast<unsigned>(tiles)), dim3(kGemmThreads), 0, st, a, v0,
                     v_count);
  return hipGetLastError();
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
