// What the attentions over the 4-bit cache share: tiles copied to LDS, a column's maximum and sum.
#pragma once

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
