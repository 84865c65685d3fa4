// Host-side declarations of the vocabulary layer's kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace vtrace {

typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int64_t kVocabMaxTokens = int64_t(1) << 24;
constexpr int64_t kVocabMaxHidden = 32768;
// Hidden states are addressed with 31-bit byte offsets.
constexpr int64_t kVocabMaxHiddenElements = (int64_t(1) << 30) - 1;
constexpr int32_t kNoToken = -1;
// Steps of one partial sum of d_bias.
constexpr int kBiasSteps = 64;

// Everything the kernels of one call need.  N = T B steps; "active" steps are
// those whose token is not kNoToken, numbered in their order.
struct VocabArgs {
  int64_t N, V, H;
  const uint16_t* hidden;  // [N,H] bfloat16
  const uint16_t* weight;  // [V,H] bfloat16
  const float* bias;       // [V] or null
  const int32_t* tokens;   // [N]
  // vtrace_vocab_log_probs
  float* log_probs;  // [N]
  float* log_sums;   // [N]
  float* entropy;    // [N] or null
  // vtrace_vocab_grad
  const float* in_log_sums;  // [N]
  const float* in_entropy;   // [N] or null
  const float* d_log_probs;  // [N]
  const float* d_entropy;    // [N] or null
  void* d_hidden;            // [N,H]
  void* d_weight;            // [V,H]
  float* d_bias;             // [V] or null
  int grad_bf16;
  bool small_logits, small_weight, small_hidden;  // tiles of 128 instead of 256
  // workspace pieces
  unsigned int* error_flag;
  int32_t* active_count;  // in the header
  int32_t* active;        // [N] the active steps
  // log_probs: statistics of vocabulary pieces, [pieces, row_pitch] each ([N, pieces] from
  // the kernel for few steps)
  float* part_max;
  float* part_sum;
  float* part_dot;        // or null
  float* token_logit;     // [row_pitch]
  int64_t row_pitch;
  int64_t pieces;         // grad: of the vocabulary
  int tile_tokens;        // of the kernels for few steps
  bool narrow;            // the one of the two that goes through LDS
  int narrow_per_cu;      // its workgroups a CU
  // tiles: the active steps' hidden states, zeros around, and tokens
  uint16_t* x;            // [row_pitch, x_pitch]
  int64_t x_pitch;
  int32_t* row_tokens;    // [row_pitch]
  // grad
  float4v* row_scalars;   // [row_pitch]: log-sum (log2 units), c0, c1, d_log_probs
  uint16_t* g;            // [1 or 2, row_pitch, g_pitch] G of one piece: high (and low) parts
  int64_t g_pitch;        // tokens of a piece, a multiple of the tile
  float* bias_partials;   // [row_pitch / kBiasSteps, g_pitch]
  float* h_partials;      // [*splits, count rounded up to tiles, H]
  int32_t* splits;        // in the header: parts of d_hidden's product
};

struct VocabPlan {
  bool few;        // log_probs: the kernels for few steps
  int64_t pieces;  // log_probs: statistics per step; grad: of the vocabulary
  int tile_tokens;
  bool narrow;
  int narrow_per_cu;
  bool small_logits, small_weight, small_hidden;
  int64_t row_pitch, x_pitch, g_pitch;
  int64_t split_rows;
  size_t bytes;
};
VocabPlan plan_vocab_log_probs(int64_t N, int64_t V, int64_t H);
VocabPlan plan_vocab_grad(int64_t N, int64_t V, int64_t H, bool grad_bf16);
void attach_vocab_log_probs(VocabArgs* a, const VocabPlan& p, void* ws);
void attach_vocab_grad(VocabArgs* a, const VocabPlan& p, void* ws);
hipError_t launch_vocab_log_probs(const VocabArgs& a, const VocabPlan& p, hipStream_t s);
hipError_t launch_vocab_grad(const VocabArgs& a, const VocabPlan& p, hipStream_t s);

// The launches of one translation unit each.
hipError_t launch_vocab_stats(const VocabArgs& a, hipStream_t s);
hipError_t launch_vocab_few(const VocabArgs& a, hipStream_t s);
hipError_t launch_vocab_logit_grads(const VocabArgs& a, int64_t v0, hipStream_t s);
hipError_t launch_vocab_d_weight(const VocabArgs& a, int64_t v0, hipStream_t s);
hipError_t launch_vocab_d_hidden(const VocabArgs& a, int64_t v0, bool first, hipStream_t s);

}  // namespace vtrace
