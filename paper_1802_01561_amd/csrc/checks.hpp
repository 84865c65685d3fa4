// Argument checks shared by the C entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "vtrace.h"

namespace vtrace {

constexpr int64_t kMaxElements = int64_t(1) << 40;

inline bool shape_ok(int64_t T, int64_t B, int64_t A) {
  if (T < 1 || B < 1 || A < 1) return false;
  if (T > kMaxElements || B > kMaxElements || A > kMaxElements) return false;
  const __int128 n = static_cast<__int128>(T) * B * A;
  return n <= kMaxElements;
}

inline bool aligned(const void* p, uintptr_t k) { return (reinterpret_cast<uintptr_t>(p) % k) == 0; }

inline bool truncation_ok(float x) { return !std::isnan(x) && x >= 0.0f; }

inline hipStream_t as_hip(vtrace_stream_t s) { return reinterpret_cast<hipStream_t>(s); }

// A caller's variant, checked (NULL = V-trace with float32 gradients).
struct Variant {
  int correction = VTRACE_CORRECTION_VTRACE;
  int q_estimate = VTRACE_Q_VTRACE;
  float epsilon = 0.0f;
  int behaviour_log_probs = 0;
  int reward_transform = VTRACE_REWARD_RAW;
  int grad_bf16 = 0;
};

inline vtrace_status parse_variant(const vtrace_variant* v, Variant* out) {
  *out = Variant{};
  if (v == nullptr) return VTRACE_OK;
  if (v->correction < VTRACE_CORRECTION_VTRACE || v->correction > VTRACE_CORRECTION_ONE_STEP_IS)
    return VTRACE_ERR_PARAM;
  if (v->q_estimate != VTRACE_Q_VTRACE && v->q_estimate != VTRACE_Q_BASELINE) return VTRACE_ERR_PARAM;
  if (v->correction == VTRACE_CORRECTION_EPSILON && !(std::isfinite(v->epsilon) && v->epsilon > 0.0f))
    return VTRACE_ERR_PARAM;
  if (v->behaviour_input != VTRACE_BEHAVIOUR_LOGITS && v->behaviour_input != VTRACE_BEHAVIOUR_LOG_PROBS)
    return VTRACE_ERR_PARAM;
  if (v->reward_transform < VTRACE_REWARD_RAW || v->reward_transform > VTRACE_REWARD_ASYMMETRIC)
    return VTRACE_ERR_PARAM;
  if (v->grad_dtype != VTRACE_F32 && v->grad_dtype != VTRACE_BF16) return VTRACE_ERR_DTYPE;
  out->correction = v->correction;
  out->q_estimate = v->q_estimate;
  out->epsilon = v->epsilon;
  out->behaviour_log_probs = v->behaviour_input == VTRACE_BEHAVIOUR_LOG_PROBS;
  out->reward_transform = v->reward_transform;
  out->grad_bf16 = v->grad_dtype == VTRACE_BF16;
  return VTRACE_OK;
}

}  // namespace vtrace
