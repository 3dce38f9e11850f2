// Single-token attention over the 4-bit cache (ios_attn_cache).
//
// Per key and head it reads 5/4 head_dim bytes and does 4 head_dim products
// for each of its queries: bound by memory, if the 4-bit codes become operands
// of the matrix instruction with few instructions.  A workgroup takes up to 16
// queries that share a head of keys (one column of the product each) and a
// range of the sequence; its eight waves take tiles of 32 keys in turn and are
// joined at the end, the ranges in a second launch.
//
// 32 sequences of 8192 .. 32031 tokens, 8 heads of 128, 4 queries each: 823 MB in
// 176 us, 4.7 TB/s (a large copy moves 4.95), and 5 for the join; the loads alone
// take 152 us.  Results in f16 take 239 us, in float32 382 (more products, and
// codes converted one by one).  One sequence of 131072 tokens and 2 such heads:
// 14 us, and 4 for the join.  Tiles
// reach LDS through a ring of direct copies per wave, two tiles deep: with
// 16 waves a CU about 80 KB are on their way, and no barrier is needed before
// the end (registers and no ring: 595 us; four waves and three tiles: 220).
//
// Scores: with q summed over the values of a group, q . (z + s c) = z sum(q) +
// s (c . q), c exact in f16 and q too (bf16 after scaling a row by a power of two;
// float32 as two f16 parts, 22 bits).  sum(q) meets z in two f16 parts as well
// (22 bits, where one product takes all groups); the rest is summed in 32 bits.
// The second product for bf16 results rounds p and the values z + s c to f16
// (2^-12 each, against 2^-9 of the result).  For f16 and float32 that would
// show in the result, so there the codes stay exact and p s is split into two
// or three bf16 parts (which keep float32's range), the zero points are summed
// in 32 bits.
#include <type_traits>

#include "attn_join.h"

namespace ios {

namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfx8 __attribute__((ext_vector_type(8)));

constexpr int kCols = 16;                // queries (heads of one key head) of a workgroup
constexpr int kWavesA = 8, kThreadsA = 64 * kWavesA;
constexpr int kStages = 2;               // tiles of a wave's ring
// Parts of a sequence's keys (bf16; us of both sides): kWantBlocks workgroups, twice what the chip holds at once, as they
// end at different times (for 512, 1024 and 2048: 32 sequences of 8k .. 32k keys 195, 188, 193; 16 of 16000 71, 70, 73; but
// 16 of 5000 27, 30, 38 and 4 of 16000 17, 21, 21); at least kMinKeys keys each, a tile for every wave (for 128, 256 and 512:
// one sequence of 5000 9.9, 10.4, 11.8; 4 of 1300 9.2, 9.7, 12.0; 16 of 1300 21, 18, 15); at most kMaxSplits (131072 keys in
// 64 parts and their join 22.7, in 128 18.4); and none, so no second launch, below kOneKeys (in one part and in several: 600
// keys 8.5 and 10.1, 785 9.9 and 10.0, 1000 11.2 and 10.1, 1300 12.8 and 10.1; 16 sequences of 785 10.6 and 13.9).
constexpr int kMaxSplits = kMaxParts, kWantBlocks = 1024, kMinKeys = 256, kOneKeys = 1024;
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

template <class T, int G>
__global__ __launch_bounds__(kThreadsA) void attn_cache_kernel(CacheView c, int heads, int ratio, float scale, ios_tokens q,
                                                         ios_tokens out, float *lse, const int32_t *seqs,
                                                         int chunk, float *part) {
  constexpr int D = 32 * G, NT = 2 * G, VW = v_words(G);
  constexpr int NL = stage_loads(G), SB = stage_bytes(G), RB = (kWavesA * kCols * (D + 1) + kWavesA * 2 * kCols) * 4;
  __shared__ __align__(16) unsigned char lds[kWavesA * kStages * SB > RB ? kWavesA * kStages * SB : RB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, kq = lane >> 4;
  const int split = blockIdx.x, splits = gridDim.x, i = blockIdx.z;
  const int blocks = (ratio + kCols - 1) / kCols;                 // of kCols queries per key head
  const int kvh = blockIdx.y / blocks, c0 = blockIdx.y % blocks * kCols;
  const int cols = min(ratio - c0, kCols), head0 = kvh * ratio + c0;
  // What the first loads depend on is fetched side by side: the length, the pages of the wave's first tiles (through
  // the scalar cache: the vector loads' counter is the ring's) and the queries.
  typedef const __attribute__((address_space(4))) int32_t const_i32;
  const int slot = ((const_i32 *)seqs)[i], at = min(max(slot, 0), c.slots - 1);
  const int first = split * chunk + wave, tile_lg = c.page_lg - 5;
  const_i32 *pages = (const_i32 *)(c.table + (int64_t)at * c.row);
  auto page_of = [&](int k) { return pages[min((first + k * kWavesA) >> tile_lg, c.row - 1)]; };
  int page[kStages];
#pragma unroll
  for (int k = 0; k < kStages; ++k) page[k] = page_of(k);
  const int held = ((const_i32 *)c.lens)[at];
  struct alignas(16) Row { T v[8]; } rows[G];
  const T *src = (const T *)q.data + (int64_t)i * q.token_stride + (int64_t)(head0 + min(col, cols - 1)) * q.head_stride;
#pragma unroll
  for (int g = 0; g < G; ++g) rows[g] = *(const Row *)(src + 32 * g + 8 * kq);

  const int len = slot == at ? (int)clip(held, (int64_t)c.row << c.page_lg) : 0;
  const int tiles = (len + kTileKeys - 1) / kTileKeys;
  const int t1 = split + 1 == splits ? tiles : min(split * chunk + chunk, tiles);
  if (part && split * chunk >= t1) return;                        // the parts' count leaves this one out
  // a ring of kStages tiles per wave: while one is worked on, the others are on their way
  const int n = first < t1 ? (t1 - first + kWavesA - 1) / kWavesA : 0;
  unsigned char *ring = lds + wave * (kStages * SB);
  uint32_t sound = 0;                                             // bit j: the j-th last tile issued has a page
  auto issue = [&](int k, int page) {
    const int t = first + k * kWavesA;
    const bool ok = (unsigned)page < (unsigned)c.pages;
    const unsigned char *tile = c.pool + (ok ? page : 0) * c.page_bytes + (int64_t)kvh * c.head_bytes +
                                (t & ((1 << tile_lg) - 1)) * tile_bytes(G);
    sound = sound << 1 | (ok ? 1u : 0u);
    copy_tile<G>(tile, ring + k % kStages * SB, lane);
  };
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k)
    if (k < n) issue(k, page[k]);

  // the queries as f16 operands: multiplied by a power of two that brings the row's largest value to 2^8 .. 2^9 (so
  // that sums of 32 fit too; values below 2^-22 of the largest lose bits), which the scores are multiplied back by;
  // the sign of the scale goes into them
  constexpr int QP = kQParts<T>, PP = kPParts<T>;
  halfx8 qf[G][QP];
  float qs[G], mul;
  {
    float f[G][8], m = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[g][e] = (float)rows[g].v[e];
        m = fmaxf(m, __builtin_fabsf(f[g][e]));
      }
    m = col_max(m);
    const int ex = __builtin_bit_cast(int, m) >> 23;              // biased exponent, 0 .. 255
    const int sh = ex == 0 || ex == 255 ? 0 : min(8 + 127 - ex, 126);
    float up = __builtin_bit_cast(float, (uint32_t)(127 + sh) << 23);
    mul = fmaxf(__builtin_fabsf(scale) * kLog2e / up, 1e-30f);    // not 0; scores of scaled queries are below 2^36
    up = scale < 0.f ? -up : up;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = f[g][e] * up;
        s += x;
#pragma unroll
        for (int k = 0; k < QP; ++k) {
          qf[g][k][e] = (_Float16)x;
          x -= (float)qf[g][k][e];
        }
      }
      qs[g] = col_sum(s);
    }
  }
  // their sums by group as an operand, in two f16 parts: slot 4 kq + g of the product with a key's zero points
  halfx4 qz = {0, 0, 0, 0};
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const _Float16 hi = (_Float16)qs[g];
    qz[g] = kq == 0 ? hi : kq == 1 ? (_Float16)(qs[g] - (float)hi) : (_Float16)0;
  }
  uint32_t mask = 0x000F000Fu;
  asm("" : "+v"(mask));

  float m = -INFINITY, l = 0.f;
  floatx4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  float zs[G] = {};                                               // PP > 0: sum of p (z - offset s), this lane's keys

  int next = page[kStages - 1];
  for (int k = 0; k < n; ++k) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // the reads of the slot that is loaded next
    const int ahead = min(kStages - 1, n - 1 - k);                // tiles issued after this one
    if (k + kStages - 1 < n) {
      issue(k + kStages - 1, next);
      next = page_of(k + kStages);
      wait_loads<NL *(kStages - 1)>();
    } else {
      static_assert(kStages == 2, "a longer ring has other tiles on their way behind this one");
      wait_loads<0>();
    }
    if (!(sound >> ahead & 1)) continue;
    const uint32_t *tile = (const uint32_t *)(ring + k % kStages * SB);
    const int left = len - (first + k * kWavesA) * kTileKeys;     // keys of the tile, when below 32
    const _Float16 *half = (const _Float16 *)tile;
    if (left < kTileKeys) {                                       // what is past the last token may be anything
      for (int x = lane; x < G * kTileKeys; x += 64) {
        const int key = x & 31;
        _Float16 *vp = (_Float16 *)const_cast<uint32_t *>(tile + v_param(G, x >> 5, v_quarter(key))) + v_elem(key);
        if (key >= left) vp[0] = vp[8] = (_Float16)0;
      }
    }
    // scores: lane holds keys 16 b + 4 kq + r of query col
    floatx4 s[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      halfx4 kz = {0, 0, 0, 0};
#pragma unroll
      for (int g = 0; g < G; ++g) kz[g] = half[k_zero(G, g, 16 * b + col)];
      s[b] = __builtin_amdgcn_mfma_f32_16x16x16f16(kz, qz, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const halfx8 kc = codes(tile[(b * 64 + lane) * G + g], mask);
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < QP; ++k) x = __builtin_amdgcn_mfma_f32_16x16x32_f16(kc, qf[g][k], x, 0, 0, 0);
        const halfx4 ks = *(const halfx4 *)(half + k_scale(G, g, 16 * b + 4 * kq));
#pragma unroll
        for (int r = 0; r < 4; ++r) s[b][r] = fmaf((float)ks[r], x[r], s[b][r]);
      }
    }
    if (left < kTileKeys) {
      asm volatile("");                                           // a branch, not selects in every tile
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[b][r] = 16 * b + 4 * kq + r < left ? s[b][r] : -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[b][r]);
    mx *= mul;
    if (__any(mx > m + kSlack)) {
      // each row by its own scores alone, so that no row's result depends on another's
      const float rm = col_max(mx), mn = rm > m + kSlack ? rm - kTop : m;
      const float a = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= a;
#pragma unroll
      for (int t2 = 0; t2 < NT; ++t2) o[t2] *= a;
#pragma unroll
      for (int g = 0; g < G; ++g) zs[g] *= a;
    }
    const float mu = m == -INFINITY ? 0.f : m;
    float p[8];
    halfx8 ph;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], mul, -mu));
      l += p[e];
      ph[e] = (_Float16)p[e];
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const halfx8 vs = *(const halfx8 *)(tile + v_param(G, g, kq)), vz = *(const halfx8 *)(tile + v_param(G, g, kq) + 4);
      bfx8 pp[PP > 0 ? PP : 1];
      if constexpr (PP > 0) {
        constexpr float offset = PP == 2 ? 128.f : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          zs[g] = fmaf(p[e], (float)vz[e] - offset * (float)vs[e], zs[g]);
          float x = p[e] * (float)vs[e];
#pragma unroll
          for (int k = 0; k < PP; ++k) {
            pp[k][e] = (__bf16)x;
            x -= (float)pp[k][e];
          }
        }
      }
#pragma unroll
      for (int t2 = 2 * g; t2 < 2 * g + 2; ++t2) {
        const uint32_t w = tile[128 * G + (t2 / VW * 64 + lane) * VW + t2 % VW];
        if constexpr (PP > 0) {
          const bfx8 vc = PP == 2 ? codes_128(w, mask) : codes_bf(w);
#pragma unroll
          for (int k = 0; k < PP; ++k) o[t2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vc, pp[k], o[t2], 0, 0, 0);
        } else {
          o[t2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes(w, mask) * vs + vz, ph, o[t2], 0, 0, 0);
        }
      }
    }
  }

  // join the waves: o[t][r] is value 16 t + 4 kq + r of query col
  l = col_sum(l);
  if constexpr (PP > 0) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float z = col_sum(zs[g]);
      o[2 * g] += z;
      o[2 * g + 1] += z;
    }
  }
  __syncthreads();                                                // the rings are done with
  auto *red_o = (float(*)[kCols][D + 1])lds;
  auto *red_m = (float(*)[kCols])(lds + kWavesA * kCols * (D + 1) * 4);
  auto *red_l = red_m + kWavesA;
  if (kq == 0) red_m[wave][col] = m;
  __syncthreads();
  float mm = m;
#pragma unroll
  for (int w = 0; w < kWavesA; ++w) mm = fmaxf(mm, red_m[w][col]);
  const float f = mm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mm);
  if (kq == 0) red_l[wave][col] = l * f;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) red_o[wave][col][16 * t + 4 * kq + r] = o[t][r] * f;
  __syncthreads();
#pragma unroll 1
  for (int x = threadIdx.x; x < cols * D; x += kThreadsA) {
    const int h = x / D, d = x % D;
    float ll = 0.f, v = 0.f, top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWavesA; ++w) {
      top = fmaxf(top, red_m[w][h]);
      ll += red_l[w][h];
      v += red_o[w][h][d];
    }
    const int64_t row = (int64_t)i * heads + head0 + h;
    if (part) {
      part[(row * splits + split) * D + d] = v;
      if (d == 0) {
        float *ml = part + (int64_t)q.tokens * heads * splits * D + (row * splits + split) * 2;
        ml[0] = top;
        ml[1] = ll;
      }
    } else {
      ((T *)out.data)[(int64_t)i * out.token_stride + (int64_t)(head0 + h) * out.head_stride + d] =
          (T)(ll == 0.f ? 0.f : v / ll);
      if (lse && d == 0) lse[(int64_t)(head0 + h) * q.tokens + i] = (top + __builtin_log2f(ll)) * kLn2;
    }
  }
}

template <class T, int G>
__global__ __launch_bounds__(256) void attn_join_kernel(CacheView c, int heads, int splits, int chunk, ios_tokens out,
                                                        float *lse, const int32_t *seqs, const float *part) {
  const int64_t i = blockIdx.x / heads, h = blockIdx.x % heads;
  join_parts<T, false>(blockIdx.x, out.tokens * heads, 32 * G, splits, part,
                       [&] {
                         const int tiles = (cache_len(c, seqs[i]) + kTileKeys - 1) / kTileKeys;
                         return min((tiles + chunk - 1) / chunk, splits);
                       },
                       (T *)out.data + i * out.token_stride + h * out.head_stride, lse ? lse + h * out.tokens + i : nullptr);
}

int64_t keys_of(const ios_attn_desc &d) { return d.max_keys ? d.max_keys : 1 << 16; }

template <class T, int G>
hipError_t run(const CacheView &c, const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &out, float *lse,
               const int32_t *seqs, float *part, int splits, hipStream_t s) {
  const int ratio = d.heads / d.kv_heads, blocks = (ratio + kCols - 1) / kCols;
  // tiles of a part; a sequence longer than max_keys makes its last part longer
  const int chunk = (int)std::max<int64_t>(1, (keys_of(d) + (int64_t)kTileKeys * splits - 1) / ((int64_t)kTileKeys * splits));
  hipLaunchKernelGGL((attn_cache_kernel<T, G>), dim3(splits, d.kv_heads * blocks, d.seqs), dim3(kThreadsA), 0, s, c,
                     d.heads, ratio, d.scale, q, out, lse, seqs, chunk, splits > 1 ? part : nullptr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((attn_join_kernel<T, G>), dim3((unsigned)((int64_t)d.seqs * d.heads)), dim3(256), 0, s, c, d.heads,
                     splits, chunk, out, lse, seqs, part);
  return hipGetLastError();
}

template <class T>
hipError_t for_groups(const CacheView &c, const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &out,
                      float *lse, const int32_t *seqs, float *part, int splits, hipStream_t s) {
  switch (d.head_dim / kGroup) {
    case 1: return run<T, 1>(c, d, q, out, lse, seqs, part, splits, s);
    case 2: return run<T, 2>(c, d, q, out, lse, seqs, part, splits, s);
    case 3: return run<T, 3>(c, d, q, out, lse, seqs, part, splits, s);
    default: return run<T, 4>(c, d, q, out, lse, seqs, part, splits, s);
  }
}

}  // namespace

int cache_splits(const ios_attn_desc &d) {
  const int ratio = d.heads / d.kv_heads;
  const int64_t blocks = (int64_t)d.seqs * d.kv_heads * ((ratio + kCols - 1) / kCols);
  if (keys_of(d) < kOneKeys) return 1;
  const int64_t parts = std::min<int64_t>((kWantBlocks + blocks - 1) / blocks, keys_of(d) / kMinKeys);
  return (int)std::max<int64_t>(1, std::min<int64_t>(parts, kMaxSplits));
}

hipError_t launch_attn_cache(const CacheView &c, const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &out,
                             float *lse, const int32_t *seqs, void *work, int splits, hipStream_t s) {
  if (d.dtype == IOS_F32) return for_groups<float>(c, d, q, out, lse, seqs, (float *)work, splits, s);
  if (d.dtype == IOS_F16) return for_groups<_Float16>(c, d, q, out, lse, seqs, (float *)work, splits, s);
  return for_groups<__bf16>(c, d, q, out, lse, seqs, (float *)work, splits, s);
}

}  // namespace ios
