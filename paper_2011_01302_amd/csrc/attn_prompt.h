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
// bf16 and float32 values reach to float32's largest, and weights to 2^8: where a row's sum leaves the range, the keys
// are walked again with weights times kDown (a power of two: every other result stays as it was, to the bit, unless it
// is below 2^-86).  2^28 keys then stay within the range.
constexpr float kDown = 0x1p-40f, kUp = 0x1p40f;

// What scores are multiplied by, never 0 (-infinity times 0 is a NaN, and hidden scores are that): for a scale of 0 the
// least number, with which finite scores come to 2^-21 at most.
__device__ __forceinline__ float multiplier(float scale) { return fmaxf(__builtin_fabsf(scale) * kLog2e, 0x1p-149f); }

constexpr uint32_t kOutside = 0x80000000u;       // byte offset past every buffer: reads as 0
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, 0x7FFFFFFF, 0x00020000);
}

// The head, sequence and first query of this workgroup; false: none.  Heads that share keys go to one XCD (workgroups
// go to the eight in turn), whose L2 they share.  All heads' longest tiles go first: with a whole head after the other,
// the last head's longest tile began when the others were done, a third of the time of 8192 causal tokens.  The last
// tiles of a sequence see most keys; of up to 64 sequences (a lane each) those with most keys come first, more are
// taken from the last one on.
__device__ __forceinline__ bool prompt_block(const PromptArgs &a, int *head, int *seq, int64_t *q0) {
  const unsigned h = blockIdx.x % a.heads;
  *head = a.heads % 8 ? h : h % 8 * (a.heads / 8) + h / 8;
  int64_t x = blockIdx.x / a.heads;
  if (a.seqs > 64) {
    x = gridDim.x / a.heads - 1 - x;
    // sequence i has tiles from cu_q[i] / rows + i on
    auto start = [&](int i) { return clip(a.cu_q[i], a.q.tokens) / a.rows + i; };
    *seq = find_owner(a.seqs, x, start);
    *q0 = (x - start(*seq)) * a.rows;
    return *q0 >= 0;                                              // rows before the first sequence, offsets that descend
  }
  const int lane = threadIdx.x & 63, i = min(lane, a.seqs - 1);
  const int64_t lq = clip(a.cu_q[i + 1], a.q.tokens) - clip(a.cu_q[i], a.q.tokens);
  const int lk = (int)(clip(a.cu_k[i + 1], a.k.tokens) - clip(a.cu_k[i], a.k.tokens));
  const int tiles = lane < a.seqs && lq > 0 ? (int)((lq + a.rows - 1) / a.rows) : 0;
  int before = 0;
  for (int j = 0; j < a.seqs; ++j) {
    const int k = __builtin_amdgcn_readlane(lk, j), t = __builtin_amdgcn_readlane(tiles, j);
    before += k > lk || (k == lk && j < lane) ? t : 0;
  }
  const uint64_t mine = __ballot(x >= before && x < (int64_t)before + tiles);
  if (mine == 0) return false;
  const int own = __builtin_ctzll(mine);
  *seq = own;
  *q0 = (int64_t)(__builtin_amdgcn_readlane(before, own) + __builtin_amdgcn_readlane(tiles, own) - 1 - (int)x) * a.rows;
  return true;
}
#endif

hipError_t launch_attn_prompt_float(const PromptArgs &a, int splits, hipStream_t s);

}  // namespace ios
