// Shared by the 16-bit and the float32 prompt attention.
#pragma once

#include "attn_join.h"

namespace ios {

// queries of a workgroup and keys of its tiles
constexpr int kRows = 128, kKeys = 64, kFloatRows = 64, kFloatKeys = 32;

struct PromptArgs {
  int heads, ratio, dim, seqs, causal;
  float scale;
  ios_tokens q, k, v, out;
  float *lse;
  const int32_t *cu_q, *cu_k;
  float *part;                   // parts of the rows' keys, chunk tiles each (null: whole rows)
  int chunk;
  int rows, keys;                // of a workgroup and of a tile
};

#if defined(__HIPCC__)
// The workgroup's head and its tile of a.rows queries: sequence i has tiles from cu_q[i] / rows + i on.  All heads' last
// tiles, which see most keys, go first (with a whole head after the other, the last head's longest tile began when the
// others' were done: a third of the time of 8192 causal tokens), and heads that share keys go to one XCD (workgroups
// go to the eight in turn), whose L2 they share.
__device__ __forceinline__ int prompt_block(const PromptArgs &a, int64_t *tile) {
  const unsigned h = blockIdx.x % a.heads;
  *tile = (gridDim.x - 1 - blockIdx.x) / a.heads;
  return a.heads % 8 ? h : h % 8 * (a.heads / 8) + h / 8;
}
#endif

hipError_t launch_attn_prompt_float(const PromptArgs &a, int splits, hipStream_t s);

}  // namespace ios
