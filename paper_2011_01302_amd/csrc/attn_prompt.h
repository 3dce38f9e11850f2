// Shared by the 16-bit and the float32 prompt attention.
#pragma once

#include "attn_join.h"

namespace ios {

constexpr int kBM = 128;                 // queries of a workgroup
constexpr int kFloatKeys = 32;           // keys of a float32 tile

struct PromptArgs {
  int heads, ratio, dim, seqs, causal;
  float scale;
  ios_tokens q, k, v, out;
  float *lse;
  const int32_t *cu_q, *cu_k;
  float *part;                   // parts of the rows' keys, chunk tiles each (null: whole rows)
  int chunk;
};

hipError_t launch_attn_prompt_float(const PromptArgs &a, bool two, int splits, hipStream_t s);

}  // namespace ios
