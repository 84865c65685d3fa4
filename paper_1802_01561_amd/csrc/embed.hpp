// Host-side declarations of the vocabulary's rows as inputs, and their gradient.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace vtrace {

// Everything the kernels of one call need.  N = T B steps.
struct EmbedArgs {
  int64_t N, V, H;
  const int32_t* tokens;  // [N]
  float scale;
  bool table_bf16, steps_bf16;
  const void* table;  // embed: [V,H]
  void* rows;         // embed: [N,H]
  const void* d_rows;  // grad: [N,H]
  void* d_table;       // grad: [V,H]
  bool accumulate;     // grad: added to what d_table holds
  // workspace pieces
  unsigned int* error_flag;  // or null (embed)
  // The steps in the order of their tokens, those without a token of the vocabulary last:
  // tokens as unsigned, and the steps' numbers; a second pair for the passes of a long sort.
  uint32_t* keys[2];   // [N]
  uint32_t* steps[2];  // [N]
  uint32_t* counts;    // [digits, blocks of a pass]
  float* partials;     // [chunks, 2, H]
  int chunk;           // sorted steps of a chunk
};

struct EmbedPlan {
  bool ranks;  // sorted by ranks, in one launch
  int chunk;
  size_t keys_at[2], steps_at[2], counts_at, partials_at, bytes;
};
EmbedPlan plan_embed_grad(int64_t N, int64_t V, int64_t H);
void attach_embed_grad(EmbedArgs* a, const EmbedPlan& p, void* ws);
hipError_t launch_embed(const EmbedArgs& a, hipStream_t s);
hipError_t launch_embed_grad(const EmbedArgs& a, const EmbedPlan& p, hipStream_t s);

}  // namespace vtrace
