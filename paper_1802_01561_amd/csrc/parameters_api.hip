// C ABI of the calls on a token policy's parameters (vtrace_parameters.h): argument validation
// and launch.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "checks.hpp"
#include "embed.hpp"
#include "launch.hpp"
#include "orthogonalize.hpp"
#include "vocab.hpp"
#include "vtrace_parameters.h"

namespace {

using vtrace::aligned;
using vtrace::as_hip;

constexpr int64_t kEmbedMostSteps = int64_t(1) << 25;
constexpr int64_t kEmbedMostElements = int64_t(1) << 37;
constexpr int64_t kOrthoMostElements = int64_t(1) << 31;

bool embed_shape_ok(int64_t T, int64_t B, int64_t V, int64_t H) {
  if (T < 1 || B < 1 || V < 1 || V > vtrace::kVocabMaxTokens) return false;
  if (H < 8 || H > vtrace::kVocabMaxHidden || H % 8 != 0) return false;
  if (T > kEmbedMostSteps || B > kEmbedMostSteps / T) return false;
  return T * B <= kEmbedMostElements / H && V <= kEmbedMostElements / H;
}

bool dtype_ok(int32_t d) { return d == VTRACE_F32 || d == VTRACE_BF16; }

vtrace_status status_of(hipError_t e) { return e == hipSuccess ? VTRACE_OK : VTRACE_ERR_HIP; }

vtrace::EmbedArgs embed_args(int64_t T, int64_t B, int64_t V, int64_t H, const int32_t* tokens, float scale, bool table_bf16,
                             bool steps_bf16) {
  vtrace::EmbedArgs a;
  std::memset(&a, 0, sizeof(a));
  a.N = T * B;
  a.V = V;
  a.H = H;
  a.tokens = tokens;
  a.scale = scale;
  a.table_bf16 = table_bf16;
  a.steps_bf16 = steps_bf16;
  return a;
}

// The matrices of a list that have elements; in and out may be NULL.
vtrace_status ortho_items(int64_t count, const void* const* matrices, void* const* outputs, const int64_t* rows,
                          const int64_t* columns, const int32_t* dtypes, const float* scales, bool pointers,
                          std::vector<vtrace::OrthoItem>* items) {
  items->reserve(static_cast<size_t>(count));
  for (int64_t i = 0; i < count; ++i) {
    if (rows[i] < 0 || rows[i] > vtrace::kOrthoMostSize || columns[i] < 0 || columns[i] > vtrace::kOrthoMostSize ||
        rows[i] * columns[i] > kOrthoMostElements)
      return VTRACE_ERR_SHAPE;
    if (!dtype_ok(dtypes[i])) return VTRACE_ERR_DTYPE;
    if (scales && !std::isfinite(scales[i])) return VTRACE_ERR_PARAM;
    if (rows[i] * columns[i] == 0) continue;
    if (pointers) {
      const uintptr_t bytes = dtypes[i] == VTRACE_F32 ? 4 : 2;
      if (!matrices[i] || !outputs[i]) return VTRACE_ERR_NULL;
      if (!aligned(matrices[i], bytes) || !aligned(outputs[i], bytes)) return VTRACE_ERR_ALIGN;
    }
    items->push_back({pointers ? matrices[i] : nullptr, pointers ? outputs[i] : nullptr, rows[i], columns[i],
                      scales ? scales[i] : 1.0f, dtypes[i] == VTRACE_BF16});
  }
  return VTRACE_OK;
}

}  // namespace

extern "C" {

vtrace_status vtrace_vocab_embed(int64_t T, int64_t B, int64_t V, int64_t H, vtrace_dtype weight_dtype,
                                 vtrace_dtype embedded_dtype, const void* vocab_weight, const int32_t* tokens, float scale,
                                 void* embedded, void* workspace, size_t workspace_bytes, vtrace_stream_t stream) {
  if (!vocab_weight || !tokens || !embedded) return VTRACE_ERR_NULL;
  if (!embed_shape_ok(T, B, V, H)) return VTRACE_ERR_SHAPE;
  if (!dtype_ok(weight_dtype) || !dtype_ok(embedded_dtype)) return VTRACE_ERR_DTYPE;
  if (!std::isfinite(scale)) return VTRACE_ERR_PARAM;
  if (!aligned(vocab_weight, 16) || !aligned(embedded, 16) || !aligned(tokens, 4)) return VTRACE_ERR_ALIGN;
  if (workspace && !aligned(workspace, 16)) return VTRACE_ERR_ALIGN;
  if (workspace && workspace_bytes < vtrace::kWsHeaderBytes) return VTRACE_ERR_WORKSPACE;
  vtrace::EmbedArgs a = embed_args(T, B, V, H, tokens, scale, weight_dtype == VTRACE_BF16, embedded_dtype == VTRACE_BF16);
  a.table = vocab_weight;
  a.rows = embedded;
  if (workspace) a.error_flag = reinterpret_cast<unsigned int*>(static_cast<char*>(workspace) + vtrace::kWsFlagOffset);
  (void)hipGetLastError();  // do not report an earlier, unrelated error
  return status_of(vtrace::launch_embed(a, as_hip(stream)));
}

size_t vtrace_vocab_embed_grad_workspace_bytes(int64_t T, int64_t B, int64_t V, int64_t H) {
  if (!embed_shape_ok(T, B, V, H)) return 0;
  return vtrace::plan_embed_grad(T * B, V, H).bytes;
}

vtrace_status vtrace_vocab_embed_grad(int64_t T, int64_t B, int64_t V, int64_t H, vtrace_dtype embedded_dtype,
                                      vtrace_dtype grad_dtype, const void* d_embedded, const int32_t* tokens, float scale,
                                      int32_t accumulate, void* d_weight, void* workspace, size_t workspace_bytes,
                                      vtrace_stream_t stream) {
  if (!d_embedded || !tokens || !d_weight) return VTRACE_ERR_NULL;
  if (!embed_shape_ok(T, B, V, H)) return VTRACE_ERR_SHAPE;
  if (!dtype_ok(embedded_dtype) || !dtype_ok(grad_dtype)) return VTRACE_ERR_DTYPE;
  if (!std::isfinite(scale)) return VTRACE_ERR_PARAM;
  if (!aligned(d_embedded, 16) || !aligned(d_weight, 16) || !aligned(tokens, 4)) return VTRACE_ERR_ALIGN;
  if (!workspace) return VTRACE_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return VTRACE_ERR_ALIGN;
  const vtrace::EmbedPlan plan = vtrace::plan_embed_grad(T * B, V, H);
  if (workspace_bytes < plan.bytes) return VTRACE_ERR_WORKSPACE;
  vtrace::EmbedArgs a = embed_args(T, B, V, H, tokens, scale, grad_dtype == VTRACE_BF16, embedded_dtype == VTRACE_BF16);
  a.d_rows = d_embedded;
  a.d_table = d_weight;
  a.accumulate = accumulate != 0;
  vtrace::attach_embed_grad(&a, plan, workspace);
  (void)hipGetLastError();
  return status_of(vtrace::launch_embed_grad(a, plan, as_hip(stream)));
}

size_t vtrace_orthogonalize_workspace_bytes(int64_t count, const int64_t* rows, const int64_t* columns, const int32_t* dtypes) {
  if (count < 0 || count > vtrace::kOrthoMostMatrices || (count > 0 && (!rows || !columns || !dtypes))) return 0;
  try {
    std::vector<vtrace::OrthoItem> items;
    if (ortho_items(count, nullptr, nullptr, rows, columns, dtypes, nullptr, false, &items) != VTRACE_OK) return 0;
    return vtrace::ortho_workspace_bytes(items.data(), static_cast<int64_t>(items.size()));
  } catch (const std::bad_alloc&) {
    return 0;
  }
}

vtrace_status vtrace_orthogonalize(int64_t count, const void* const* matrices, void* const* outputs, const int64_t* rows,
                                   const int64_t* columns, const int32_t* dtypes, const float* scales, int32_t steps,
                                   const float* coefficients, float epsilon, void* workspace, size_t workspace_bytes,
                                   vtrace_stream_t stream) {
  if (!coefficients || (count > 0 && (!matrices || !outputs || !rows || !columns || !dtypes))) return VTRACE_ERR_NULL;
  if (count < 0 || count > vtrace::kOrthoMostMatrices) return VTRACE_ERR_SHAPE;
  if (steps < 1 || steps > vtrace::kOrthoMostSteps) return VTRACE_ERR_PARAM;
  if (!std::isfinite(epsilon) || !(epsilon > 0.0f)) return VTRACE_ERR_PARAM;
  vtrace::OrthoStep step[vtrace::kOrthoMostSteps];
  for (int k = 0; k < steps; ++k) step[k] = {coefficients[3 * k], coefficients[3 * k + 1], coefficients[3 * k + 2]};
  if (!vtrace::ortho_steps_ok(step, steps)) return VTRACE_ERR_PARAM;
  if (!workspace) return VTRACE_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return VTRACE_ERR_ALIGN;
  try {
    std::vector<vtrace::OrthoItem> items;
    const vtrace_status st = ortho_items(count, matrices, outputs, rows, columns, dtypes, scales, true, &items);
    if (st != VTRACE_OK) return st;
    const int64_t n = static_cast<int64_t>(items.size());
    if (workspace_bytes < vtrace::ortho_workspace_bytes(items.data(), n)) return VTRACE_ERR_WORKSPACE;
    // What is read and what is written, to find outputs that overlap anything.
    struct Range {
      uintptr_t begin, end;
      bool written;
    };
    std::vector<Range> ranges;
    ranges.reserve(2 * items.size() + 1);
    const auto w = reinterpret_cast<uintptr_t>(workspace);
    ranges.push_back({w, w + workspace_bytes, true});
    for (const vtrace::OrthoItem& item : items) {
      const auto in = reinterpret_cast<uintptr_t>(item.in), out = reinterpret_cast<uintptr_t>(item.out);
      const uintptr_t bytes = static_cast<uintptr_t>(item.rows * item.columns) * (item.bf16 ? 2 : 4);
      ranges.push_back({out, out + bytes, true});
      if (in != out) ranges.push_back({in, in + bytes, false});
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range& x, const Range& y) { return x.begin < y.begin; });
    uintptr_t written_to = 0, read_to = 0;
    for (const Range& r : ranges) {
      if (r.begin < written_to || (r.written && r.begin < read_to)) return VTRACE_ERR_PARAM;
      if (r.written) written_to = std::max(written_to, r.end);
      else read_to = std::max(read_to, r.end);
    }
    (void)hipGetLastError();
    return status_of(vtrace::launch_orthogonalize(items.data(), n, step, steps, epsilon, workspace, as_hip(stream)));
  } catch (const std::bad_alloc&) {
    return VTRACE_ERR_HIP;
  }
}

}  // extern "C"
