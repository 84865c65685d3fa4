// C ABI of the token-policy operators (vtrace_tokens.h): argument validation and launch.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "checks.hpp"
#include "clip.hpp"
#include "log_prob_loss.hpp"
#include "vocab.hpp"
#include "vtrace_tokens.h"

namespace {

using vtrace::aligned;
using vtrace::as_hip;

// So that tiles are numbered by 32 bits, and their products and sums fit 64.
constexpr int64_t kVocabMostSteps = int64_t(1) << 25;
constexpr int64_t kVocabMostLogits = int64_t(1) << 38;

bool vocab_shape_ok(int64_t T, int64_t B, int64_t V, int64_t H) {
  if (T < 1 || B < 1 || V < 1 || V > vtrace::kVocabMaxTokens) return false;
  if (H < 8 || H > vtrace::kVocabMaxHidden || H % 8 != 0) return false;
  if (T > kVocabMostSteps || B > kVocabMostSteps / T) return false;
  const int64_t n = T * B;
  return n <= vtrace::kVocabMaxHiddenElements / H && n <= kVocabMostLogits / V;
}

vtrace_status status_of(hipError_t e) { return e == hipSuccess ? VTRACE_OK : VTRACE_ERR_HIP; }

vtrace::VocabArgs vocab_args(int64_t T, int64_t B, int64_t V, int64_t H, const void* hidden, const void* vocab_weight,
                             const float* vocab_bias, const int32_t* tokens) {
  vtrace::VocabArgs a;
  std::memset(&a, 0, sizeof(a));
  a.N = T * B;
  a.V = V;
  a.H = H;
  a.hidden = static_cast<const uint16_t*>(hidden);
  a.weight = static_cast<const uint16_t*>(vocab_weight);
  a.bias = vocab_bias;
  a.tokens = tokens;
  return a;
}

}  // namespace

extern "C" {

size_t vtrace_vocab_workspace_bytes(int64_t T, int64_t B, int64_t V, int64_t H) {
  if (!vocab_shape_ok(T, B, V, H)) return 0;
  return vtrace::plan_vocab_log_probs(T * B, V, H).bytes;
}

vtrace_status vtrace_vocab_log_probs(int64_t T, int64_t B, int64_t V, int64_t H, const void* hidden,
                                     const void* vocab_weight, const float* vocab_bias, const int32_t* tokens,
                                     float* log_probs, float* log_sums, float* entropy, void* workspace,
                                     size_t workspace_bytes, vtrace_stream_t stream) {
  if (!hidden || !vocab_weight || !tokens || !log_probs || !log_sums) return VTRACE_ERR_NULL;
  if (!vocab_shape_ok(T, B, V, H)) return VTRACE_ERR_SHAPE;
  if (!aligned(hidden, 16) || !aligned(vocab_weight, 16)) return VTRACE_ERR_ALIGN;
  if (!aligned(vocab_bias, 4) || !aligned(tokens, 4) || !aligned(log_probs, 4) || !aligned(log_sums, 4) ||
      !aligned(entropy, 4))
    return VTRACE_ERR_ALIGN;
  if (!workspace) return VTRACE_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return VTRACE_ERR_ALIGN;
  const vtrace::VocabPlan plan = vtrace::plan_vocab_log_probs(T * B, V, H);
  if (workspace_bytes < plan.bytes) return VTRACE_ERR_WORKSPACE;
  vtrace::VocabArgs a = vocab_args(T, B, V, H, hidden, vocab_weight, vocab_bias, tokens);
  a.log_probs = log_probs;
  a.log_sums = log_sums;
  a.entropy = entropy;
  vtrace::attach_vocab_log_probs(&a, plan, workspace);
  (void)hipGetLastError();  // do not report an earlier, unrelated error
  return status_of(vtrace::launch_vocab_log_probs(a, plan, as_hip(stream)));
}

size_t vtrace_vocab_grad_workspace_bytes(int64_t T, int64_t B, int64_t V, int64_t H, vtrace_dtype grad_dtype) {
  if (!vocab_shape_ok(T, B, V, H) || (grad_dtype != VTRACE_F32 && grad_dtype != VTRACE_BF16)) return 0;
  return vtrace::plan_vocab_grad(T * B, V, H, grad_dtype == VTRACE_BF16).bytes;
}

vtrace_status vtrace_vocab_grad(int64_t T, int64_t B, int64_t V, int64_t H, vtrace_dtype grad_dtype,
                                const void* hidden, const void* vocab_weight, const float* vocab_bias,
                                const int32_t* tokens, const float* log_sums, const float* entropy,
                                const float* d_log_probs, const float* d_entropy, void* d_hidden, void* d_weight,
                                float* d_bias, void* workspace, size_t workspace_bytes, vtrace_stream_t stream) {
  if (!hidden || !vocab_weight || !tokens || !log_sums || !d_log_probs || !d_hidden || !d_weight)
    return VTRACE_ERR_NULL;
  if (d_entropy && !entropy) return VTRACE_ERR_NULL;
  if (!vocab_shape_ok(T, B, V, H)) return VTRACE_ERR_SHAPE;
  if (grad_dtype != VTRACE_F32 && grad_dtype != VTRACE_BF16) return VTRACE_ERR_DTYPE;
  if (!aligned(hidden, 16) || !aligned(vocab_weight, 16) || !aligned(d_hidden, 16) || !aligned(d_weight, 16))
    return VTRACE_ERR_ALIGN;
  if (!aligned(vocab_bias, 4) || !aligned(tokens, 4) || !aligned(log_sums, 4) || !aligned(entropy, 4) ||
      !aligned(d_log_probs, 4) || !aligned(d_entropy, 4) || !aligned(d_bias, 4))
    return VTRACE_ERR_ALIGN;
  if (!workspace) return VTRACE_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return VTRACE_ERR_ALIGN;
  const vtrace::VocabPlan plan = vtrace::plan_vocab_grad(T * B, V, H, grad_dtype == VTRACE_BF16);
  if (workspace_bytes < plan.bytes) return VTRACE_ERR_WORKSPACE;
  vtrace::VocabArgs a = vocab_args(T, B, V, H, hidden, vocab_weight, vocab_bias, tokens);
  a.in_log_sums = log_sums;
  a.in_entropy = entropy;
  a.d_log_probs = d_log_probs;
  a.d_entropy = d_entropy;
  a.d_hidden = d_hidden;
  a.d_weight = d_weight;
  a.d_bias = d_bias;
  a.grad_bf16 = grad_dtype == VTRACE_BF16;
  vtrace::attach_vocab_grad(&a, plan, workspace);
  (void)hipGetLastError();
  return status_of(vtrace::launch_vocab_grad(a, plan, as_hip(stream)));
}

size_t vtrace_log_prob_workspace_bytes(int64_t T, int64_t B) {
  if (!vtrace::shape_ok(T, B, 1) || B > vtrace::kLogProbMaxLanes) return 0;
  return vtrace::log_prob_workspace_bytes(T, B);
}

vtrace_status vtrace_log_prob_loss_grad(int64_t T, int64_t B, const float* target_log_probs,
                                        const float* behaviour_log_probs, const float* entropy, const float* rewards,
                                        const float* discounts, const float* values, const float* bootstrap_value,
                                        const int32_t* lengths, float rho_bar, float c_bar, float lambda,
                                        float baseline_cost, float entropy_cost, const vtrace_variant* variant,
                                        float* losses, float* d_log_probs, float* d_entropy, float* d_values,
                                        float* vs, float* pg_advantages, void* workspace, size_t workspace_bytes,
                                        vtrace_stream_t stream) {
  if (!target_log_probs || !behaviour_log_probs || !rewards || !discounts || !values || !bootstrap_value || !losses ||
      !d_log_probs || !d_values)
    return VTRACE_ERR_NULL;
  if (!vtrace::shape_ok(T, B, 1) || B > vtrace::kLogProbMaxLanes) return VTRACE_ERR_SHAPE;
  if (!vtrace::truncation_ok(rho_bar) || !vtrace::truncation_ok(c_bar)) return VTRACE_ERR_PARAM;
  if (std::isnan(lambda) || lambda < 0.0f || lambda > 1.0f) return VTRACE_ERR_PARAM;
  if (!std::isfinite(baseline_cost) || !std::isfinite(entropy_cost)) return VTRACE_ERR_PARAM;
  vtrace::Variant v;
  const vtrace_status st = vtrace::parse_variant(variant, &v);
  if (st != VTRACE_OK) return st;
  const void* const arrays[] = {target_log_probs, behaviour_log_probs, entropy, rewards, discounts,
                                values, bootstrap_value, lengths, losses, d_log_probs,
                                d_entropy, d_values, vs, pg_advantages};
  for (const void* p : arrays)
    if (!aligned(p, 4)) return VTRACE_ERR_ALIGN;
  if (!workspace) return VTRACE_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return VTRACE_ERR_ALIGN;
  if (workspace_bytes < vtrace::log_prob_workspace_bytes(T, B)) return VTRACE_ERR_WORKSPACE;
  vtrace::LogProbArgs a;
  std::memset(&a, 0, sizeof(a));
  a.step.T = T;
  a.step.B = B;
  a.step.rewards = rewards;
  a.step.discounts = discounts;
  a.step.values = values;
  a.step.bootstrap_value = bootstrap_value;
  a.step.rho_bar = rho_bar;
  a.step.c_bar = c_bar;
  a.step.lambda = lambda;
  a.step.baseline_cost = baseline_cost;
  a.step.entropy_cost = entropy_cost;
  a.step.correction = v.correction;
  a.step.q_estimate = v.q_estimate;
  a.step.epsilon = v.epsilon;
  a.step.reward_transform = v.reward_transform;
  a.step.losses = losses;
  a.step.d_values = d_values;
  a.step.vs = vs;
  a.step.pg_adv = pg_advantages;
  a.target = target_log_probs;
  a.behaviour = behaviour_log_probs;
  a.entropy = entropy;
  a.lengths = lengths;
  a.d_log_probs = d_log_probs;
  a.d_entropy = d_entropy;
  vtrace::attach_log_prob_workspace(&a, workspace);
  (void)hipGetLastError();
  return status_of(vtrace::launch_log_prob_loss(a, as_hip(stream)));
}

vtrace_status vtrace_clip_grad_norm(int64_t count, const void* const* gradients, void* const* outputs,
                                    const int64_t* sizes, const int32_t* dtypes, float max_norm, float* norm,
                                    void* workspace, size_t workspace_bytes, vtrace_stream_t stream) {
  if (!norm || (count > 0 && (!gradients || !sizes || !dtypes))) return VTRACE_ERR_NULL;
  if (count < 0 || count > vtrace::kClipMostTensors) return VTRACE_ERR_SHAPE;
  if (outputs && (std::isnan(max_norm) || max_norm < 0.0f)) return VTRACE_ERR_PARAM;
  if (!aligned(norm, 4)) return VTRACE_ERR_ALIGN;
  if (!workspace) return VTRACE_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return VTRACE_ERR_ALIGN;
  if (workspace_bytes < vtrace::clip_workspace_bytes()) return VTRACE_ERR_WORKSPACE;
  static_assert(VTRACE_CLIP_WORKSPACE_BYTES == vtrace::kWsDataOffset + 8 * vtrace::kClipMostBlocks, "header states the size");
  try {
    // What is read and what is written, to find outputs that overlap anything.
    struct Range {
      uintptr_t begin, end;
      bool written;
      int64_t item;
    };
    std::vector<vtrace::ClipItem> items;
    std::vector<Range> ranges;
    items.reserve(static_cast<size_t>(count));
    if (outputs) {
      ranges.reserve(2 * static_cast<size_t>(count) + 2);
      const auto n = reinterpret_cast<uintptr_t>(norm), w = reinterpret_cast<uintptr_t>(workspace);
      ranges.push_back({n, n + 4, true, -1});
      ranges.push_back({w, w + workspace_bytes, true, -2});
    }
    for (int64_t i = 0; i < count; ++i) {
      if (sizes[i] < 0 || sizes[i] > vtrace::kClipMostElements) return VTRACE_ERR_SHAPE;
      if (dtypes[i] != VTRACE_F32 && dtypes[i] != VTRACE_BF16) return VTRACE_ERR_DTYPE;
      if (sizes[i] == 0) continue;
      const uintptr_t bytes = dtypes[i] == VTRACE_F32 ? 4 : 2;
      if (!gradients[i] || (outputs && !outputs[i])) return VTRACE_ERR_NULL;
      if (!aligned(gradients[i], bytes) || (outputs && !aligned(outputs[i], bytes))) return VTRACE_ERR_ALIGN;
      items.push_back({gradients[i], outputs ? outputs[i] : nullptr, sizes[i], dtypes[i] == VTRACE_BF16});
      if (!outputs) continue;
      const auto in = reinterpret_cast<uintptr_t>(gradients[i]), out = reinterpret_cast<uintptr_t>(outputs[i]);
      const uintptr_t n = static_cast<uintptr_t>(sizes[i]) * bytes;
      ranges.push_back({out, out + n, true, i});
      if (in != out) ranges.push_back({in, in + n, false, i});
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range& x, const Range& y) { return x.begin < y.begin; });
    uintptr_t written_to = 0, read_to = 0;
    for (const Range& r : ranges) {
      if (r.begin < written_to || (r.written && r.begin < read_to)) return VTRACE_ERR_PARAM;
      if (r.written) written_to = std::max(written_to, r.end);
      else read_to = std::max(read_to, r.end);
    }
    (void)hipGetLastError();
    return status_of(vtrace::launch_clip(items.data(), static_cast<int64_t>(items.size()), outputs != nullptr, max_norm,
                                         norm, workspace, as_hip(stream)));
  } catch (const std::bad_alloc&) {
    return VTRACE_ERR_HIP;
  }
}

}  // extern "C"
