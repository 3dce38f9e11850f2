// What the attentions over the 4-bit cache share: tiles copied to LDS, codes as operands of the matrix instruction,
// rows' statistics.
#pragma once

#include <type_traits>

#include "attn_join.h"

namespace ios {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfx8 __attribute__((ext_vector_type(8)));

constexpr int kCols = 16;                // queries (rows that read one head of keys) of a product

typedef __attribute__((address_space(3))) void lds_void;
// one tile in the ring, whole 1024-byte loads
constexpr int stage_loads(int g) { return (tile_bytes(g) + 1023) / 1024; }
constexpr int stage_bytes(int g) { return stage_loads(g) * 1024; }

template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "vmcnt is 6 bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Copy a tile to LDS, 16 bytes a lane and load, through no register (the compiler does not see the write); what is
// past `bytes` reads as 0.
template <int G>
__device__ __forceinline__ void copy_tile(const unsigned char *tile, unsigned char *lds, int lane) {
  const __amdgpu_buffer_rsrc_t r =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(tile), (short)0, tile_bytes(G), 0x00020000);
#pragma unroll
  for (int i = 0; i < stage_loads(G); ++i)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(lds + i * 1024), 16, lane * 16 + i * 1024, 0, 0, 0);
}
// A row's weights are p = 2^(score - m) with m kTop below the largest score when it was last followed, and m is only
// followed when a score passes it by kTop + 2: then p is at most 2^15, and f16 holds weights down to 2^-38 of the
// largest (without kTop those below 2^-25 would be lost, which 10^5 keys together would show).
constexpr float kTop = 13.f, kSlack = kTop + 2.f;

// How T is computed: parts of q, parts of p s (0: values rounded to f16).
template <class T> constexpr int kQParts = std::is_same_v<T, float> ? 2 : 1;
template <class T> constexpr int kPParts = std::is_same_v<T, float> ? 3 : std::is_same_v<T, _Float16> ? 2 : 0;

// 8 codes of a word in operand order, as the 16-bit numbers 2^k + c that `base` | c is in two halves: one
// instruction to shift and one to mask and set two codes, if the mask is in a vector register (`mask`).
__device__ __forceinline__ uintx4 codes_over(uint32_t w, uint32_t mask, uint32_t base) {
  uintx4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (w >> (4 * i) & mask) | base;
  return r;
}
// As f16 numbers 0 .. 15 (0x6400 | c is 1024 + c) ...
__device__ __forceinline__ halfx8 codes(uint32_t w, uint32_t mask) {
  return __builtin_bit_cast(halfx8, codes_over(w, mask, 0x64006400u)) - (_Float16)1024;
}
// ... as bf16 numbers 128 + c ...
__device__ __forceinline__ bfx8 codes_128(uint32_t w, uint32_t mask) {
  return __builtin_bit_cast(bfx8, codes_over(w, mask, 0x43004300u));
}
// ... or c itself.
__device__ __forceinline__ bfx8 codes_bf(uint32_t w) {
  bfx8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (__bf16)(float)(w >> nibble_shift(e) & 15);
  return r;
}

// Maximum and sum over the 4 lanes that hold a column (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float col_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float col_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

}  // namespace ios
