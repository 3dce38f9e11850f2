// Internal to the decoder operators (attention, the 4-bit key-value cache and
// its pages): what their kernels and entry points share.
#pragma once

#include "ios_internal.h"

namespace ios {

// ---- the cache's layout in memory
//
// A page of one layer is [kv_heads][page_tokens / 32] tiles of 32 tokens of
// one head.  With G = head_dim / 32 groups of 32 values, a tile is 1280 G
// bytes, laid out as the matrix instruction v_mfma_f32_16x16x32_f16 takes its
// operands, so that the attention loads them as they are:
//   K codes    [2 blocks of 16 keys][64 lanes][G words]; lane l holds key
//              l % 16, word g values 32 g + 8 (l / 16) .. + 7 of it
//   V codes    [2G / VW][64 lanes][VW words], VW = 4 (2 where G is odd): word
//              t, lane l holds value 16 t + l % 16 of keys 4 q .. 4 q + 3 and
//              16 + 4 q .. + 3, q = l / 16
//   K scales   [G][32 keys] halves
//   K zeros    [32 keys][G] halves (z sum(q) is a product of its own)
//   V params   [G][4 q][8 s, 8 z] halves, in the order of a word's keys
// A word's element j (0 .. 7) is its nibble j / 2 + 4 (j % 2): (w >> 4 i) &
// 0x000F000F are elements 2 i and 2 i + 1, one in each half.
constexpr int kTileKeys = 32;
constexpr int kGroup = 32;
__host__ __device__ constexpr int tile_bytes(int g) { return 1280 * g; }
__host__ __device__ constexpr int v_words(int g) { return g % 2 ? 2 : 4; }
// word offsets inside a tile
__host__ __device__ constexpr int k_word(int g, int key, int octet, int group) {
  return ((key >> 4) * 64 + (key & 15) + 16 * octet) * g + group;
}
__host__ __device__ constexpr int v_word(int g, int t, int lane) {
  return 128 * g + (t / v_words(g) * 64 + lane) * v_words(g) + t % v_words(g);
}
// half offsets of K's parameters, word offset of V's
__host__ __device__ constexpr int k_scale(int g, int group, int key) { return 512 * g + group * 32 + key; }
__host__ __device__ constexpr int k_zero(int g, int group, int key) { return 544 * g + key * g + group; }
__host__ __device__ constexpr int v_param(int g, int group, int q) { return 288 * g + group * 32 + q * 8; }
// key of a tile -> quarter q and element j of its V words
__host__ __device__ constexpr int v_quarter(int key) { return (key & 15) >> 2; }
__host__ __device__ constexpr int v_elem(int key) { return (key & 3) + 4 * (key >> 4); }
__host__ __device__ constexpr int nibble_shift(int j) { return 4 * ((j >> 1) + 4 * (j & 1)); }

// A cache as its kernels see one layer of it.
struct CacheView {
  unsigned char *pool;        // the layer's pages
  const int32_t *table, *lens;
  int64_t page_bytes;
  int32_t head_bytes;         // page_tokens / 32 tiles
  int32_t pages, slots, row, heads;
  int32_t page_lg;            // log2 page_tokens
};

// Words of a cache's workspace: flags, the number of pages to copy, the number
// of live ones, then four words a page and two a slot.
enum { CW_FLAGS = 0, CW_COPIES = 1, CW_LIVE = 2, CW_HEAD = 16 };
enum { CACHE_NO_PAGES = 1, CACHE_NO_ENTRIES = 2, CACHE_CHILD_USED = 4 };
constexpr int64_t cache_work_words(int64_t pages, int64_t slots) { return CW_HEAD + 4 * pages + 2 * slots; }

// ---- device helpers
#if defined(__HIPCC__)

// The unit of work x belongs to: sequence i < n owns units start(i) ..
// start(i + 1) - 1; start ascends from start(0) = 0.  64 sequences a step.
template <class F>
__device__ __forceinline__ int find_owner(int n, int64_t x, F start) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) >> 6, i = lo + lane * step;
    const int c = __builtin_popcountll(__ballot(i < hi && start(i < hi ? i : lo) <= x));
    lo += (c > 0 ? c - 1 : 0) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The same by halves, for a thread by itself.
template <class F>
__device__ __forceinline__ int find_row(int n, int64_t x, F start) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start(mid) <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int64_t clip(int64_t v, int64_t n) { return v < 0 ? 0 : v > n ? n : v; }

// One head's tile that holds token `pos` of a slot; null where the table has
// no page for it.
__device__ __forceinline__ unsigned char *cache_tile(const CacheView &c, int slot, int pos, int head, int tile_b) {
  const int page = c.table[(int64_t)slot * c.row + (pos >> c.page_lg)];
  if ((unsigned)page >= (unsigned)c.pages) return nullptr;
  return c.pool + page * c.page_bytes + (int64_t)head * c.head_bytes +
         ((pos & ((1 << c.page_lg) - 1)) / kTileKeys) * tile_b;
}

// Tokens of a slot (0 for one that does not exist).
__device__ __forceinline__ int cache_len(const CacheView &c, int slot) {
  if ((unsigned)slot >= (unsigned)c.slots) return 0;
  const int64_t n = clip(c.lens[slot], (int64_t)c.row << c.page_lg);
  return (int)n;
}
#endif

// ---- launches (the entry points have checked every size)
hipError_t launch_append(const CacheView &c, int groups, int dtype, const ios_tokens &k, const ios_tokens &v, int n,
                         const int32_t *seqs, const int32_t *cu, hipStream_t s);
hipError_t launch_read(const CacheView &c, int groups, int dtype, const ios_tokens &k, const ios_tokens &v, int n,
                       const int32_t *seqs, const int32_t *cu, hipStream_t s);
hipError_t launch_attn_cache(const CacheView &c, const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &out,
                             float *lse, const int32_t *seqs, void *work, int splits, hipStream_t s);
hipError_t launch_attn_prompt(const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &k, const ios_tokens &v,
                              const ios_tokens &out, float *lse, const int32_t *cu_q, const int32_t *cu_k,
                              void *work, int splits, hipStream_t s);
hipError_t launch_reserve(const ios_cache &c, int64_t page_bytes, int n, const int32_t *seqs, const int32_t *add,
                          hipStream_t s);
hipError_t launch_fork(const ios_cache &c, int n, const int32_t *parents, const int32_t *children, hipStream_t s);
hipError_t launch_free(const ios_cache &c, int n, const int32_t *seqs, hipStream_t s);
hipError_t launch_compact(const ios_cache &c, int64_t page_bytes, int32_t *live, hipStream_t s);
hipError_t launch_copy(const ios_cache &c, int64_t page_bytes, int n, const int32_t *src, const int32_t *dst,
                       hipStream_t s);

// Over how many workgroups the keys of a row are spread (1: no workspace).
int cache_splits(const ios_attn_desc &d);
int prompt_splits(const ios_attn_desc &d, int64_t q_tokens);

}  // namespace ios
