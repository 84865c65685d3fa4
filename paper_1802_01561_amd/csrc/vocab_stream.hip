// vtrace_vocab_log_probs for few steps (up to 64): the vocabulary layer is read once,
// from memory straight into matrix-core operands, and nothing else matters.
//
// A workgroup of four waves takes 16 R tokens and all steps.  The waves share out the
// hidden units, 64 (a 128-byte line of each row) at a time; their partial logits meet
// in LDS, where each wave takes some of the 16 x 16 pieces, adds the bias and forms the
// softmax statistics as in vocab_logits.hip.
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
  const int64_t v0 = static_cast<int64_t>(blockIdx.x) * (16 * R);
  const Rsrc rw = make_rsrc(a.weight + v0 * H, (a.V - v0) * H * 2);
  const Rsrc rx = make_rsrc(a.hidden, a.N * H * 2);
  uint32_t ow[R], ox[NT];
#pragma unroll
  for (int r = 0; r < R; ++r)
    ow[r] = v0 + 16 * r + s < a.V ? static_cast<uint32_t>((16 * r + s) * H * 2) + 16 * g : kOutOfRange;
#pragma unroll
  for (int n = 0; n < NT; ++n)
    ox[n] = 16 * n + s < a.N ? static_cast<uint32_t>((16 * n + s) * H * 2) + 16 * g : kOutOfRange;

  f32x4 acc[R][NT] = {};
  v4u w[2][R], x[2][NT];
  const int steps = static_cast<int>((H + 63) / 64);
  auto load = [&](int step) {
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
  if (wave < steps) load(wave);
  for (int step = wave; step < steps; step += kStreamWaves) {
    bf16x8 wa[2][R], xb[2][NT];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int r = 0; r < R; ++r) wa[kk][r] = __builtin_bit_cast(bf16x8, w[kk][r]);
#pragma unroll
      for (int n = 0; n < NT; ++n) xb[kk][n] = __builtin_bit_cast(bf16x8, x[kk][n]);
    }
    if (step + kStreamWaves < steps) load(step + kStreamWaves);
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
    const float c = top == -INFINITY ? 0.0f : top * kLog2eF;
    float sum = 0.0f, dot = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float d = fmaf(z[i], kLog2eF, -c);
      const float e = __builtin_amdgcn_exp2f(d);
      sum += e;
      dot = fmaf(e, fmaxf(d, kLeastLog), dot);
    }
    sum = group_sum(sum);
    if constexpr (kDot) dot = group_sum(dot);
    const int row = 16 * n + s;
    if (g == 0) {
      s_stat[0][r][row] = c;
      s_stat[1][r][row] = sum;
      if constexpr (kDot) s_stat[2][r][row] = dot;
    }
    const int32_t token = row < a.N ? a.tokens[row] : kNoToken;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (token >= 0 && token == v + i && v + i < a.V) a.token_logit[row] = z[i];
  }
  __syncthreads();
  for (int row = threadIdx.x; row < NT * 16; row += kStreamThreads) {
    // A piece of nothing but -inf logits (sum 0) has no maximum.
    float c = -INFINITY;
#pragma unroll
    for (int r = 0; r < R; ++r) c = fmaxf(c, s_stat[1][r][row] == 0.0f ? -INFINITY : s_stat[0][r][row]);
    c = c == -INFINITY ? 0.0f : c;
    float sum = 0.0f, dot = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float d = s_stat[1][r][row] == 0.0f ? 0.0f : s_stat[0][r][row] - c;
      const float e = __builtin_amdgcn_exp2f(d), part = s_stat[1][r][row] * e;
      sum += part;
      if constexpr (kDot) dot += s_stat[2][r][row] * e + part * d;
    }
    const int64_t o = static_cast<int64_t>(blockIdx.x) * a.row_pitch + row;
    a.part_max[o] = c;
    a.part_sum[o] = sum;
    if constexpr (kDot) a.part_dot[o] = dot;
  }
}

template <int R, int NT>
hipError_t launch(const VocabArgs& a, hipStream_t st) {
  const unsigned blocks = static_cast<unsigned>((a.V + 16 * R - 1) / (16 * R));
  if (a.entropy)
    hipLaunchKernelGGL((vocab_stream_kernel<R, NT, true>), dim3(blocks), dim3(kStreamThreads), 0, st, a);
  else
    hipLaunchKernelGGL((vocab_stream_kernel<R, NT, false>), dim3(blocks), dim3(kStreamThreads), 0, st, a);
  return hipGetLastError();
}

template <int R>
hipError_t launch_rows(const VocabArgs& a, hipStream_t st) {
  if (a.N <= 16) return launch<R, 1>(a, st);
  if (a.N <= 32) return launch<R, 2>(a, st);
  return launch<R, 4>(a, st);
}

}  // namespace

hipError_t launch_vocab_stream(const VocabArgs& a, hipStream_t st) {
  return a.pieces == (a.V + 63) / 64 ? launch_rows<4>(a, st) : launch_rows<1>(a, st);
}

}  // namespace vtrace
