// Single-token attention over the 4-bit cache (ios_attn_cache).
//
// Per key and head it reads 5/4 head_dim bytes and does 4 head_dim products
// for each of its queries: bound by memory, if the 4-bit codes become operands
// of the matrix instruction with few instructions.  A workgroup takes up to 16
// queries that share a head of keys (one column of the product each) and a
// range of the sequence; its four waves take tiles of 32 keys in turn and are
// joined at the end, the ranges in a second launch.
//
// Scores are exact up to 32-bit sums: with q summed over the values of a
// group, s . (z + s_k c) = z sum(q) + s_k (c . q), c exact in f16 and q too
// (bf16 after scaling a row by a power of two; float32 as two f16 parts).
// The second product for bf16 results rounds p and the values z + s c to f16
// (2^-12 each, against 2^-9 of the result).  For f16 and float32 that would
// show in the result, so there the codes stay exact and p s is split into two
// or three bf16 parts (which keep float32's range), the zero points are summed
// in 32 bits.
#include <type_traits>

#include "decoder.h"

namespace ios {

namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bfx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kCols = 16;                // queries (heads of one key head) of a workgroup
constexpr int kWavesA = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// a row's maximum is only followed when it grows by more than 2^8: p stays below 2^8, sums in 32 bits
constexpr float kSlack = 8.f;

// How T is computed: parts of q, parts of p s (0: values rounded to f16).
template <class T> constexpr int kQParts = std::is_same_v<T, float> ? 2 : 1;
template <class T> constexpr int kPParts = std::is_same_v<T, float> ? 3 : std::is_same_v<T, _Float16> ? 2 : 0;

// 8 codes of a word as exact f16 numbers 0 .. 15, in operand order.
__device__ __forceinline__ halfx8 codes(uint32_t w) {
  halfx8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // 0x6400 | c is the f16 1024 + c
    const halfx2 h = __builtin_bit_cast(halfx2, (w >> (4 * i) & 0x000F000Fu) | 0x64006400u) - (_Float16)1024;
    r[2 * i] = h[0];
    r[2 * i + 1] = h[1];
  }
  return r;
}

// 8 codes as bf16 numbers, 128 + c (0x4300 | c is the bf16 128 + c) ...
__device__ __forceinline__ bfx8 codes_128(uint32_t w) {
  uintx4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (w >> (4 * i) & 0x000F000Fu) | 0x43004300u;
  return __builtin_bit_cast(bfx8, r);
}
// ... or c itself.
__device__ __forceinline__ bfx8 codes_bf(uint32_t w) {
  bfx8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (__bf16)(float)(w >> nibble_shift(e) & 15);
  return r;
}

__device__ __forceinline__ float half_of(uint32_t w, int hi) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(hi ? w >> 16 : w));
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
__global__ __launch_bounds__(256) void attn_cache_kernel(CacheView c, int heads, int ratio, float scale, ios_tokens q,
                                                         ios_tokens out, float *lse, const int32_t *seqs,
                                                         float *part) {
  constexpr int D = 32 * G, NT = 2 * G, VW = v_words(G);
  __shared__ float red_o[kWavesA][kCols][D + 1];
  __shared__ float red_ml[kWavesA][2][kCols];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, kq = lane >> 4;
  const int split = blockIdx.x, splits = gridDim.x, i = blockIdx.z;
  const int blocks = (ratio + kCols - 1) / kCols;                 // of kCols queries per key head
  const int kvh = blockIdx.y / blocks, c0 = blockIdx.y % blocks * kCols;
  const int cols = min(ratio - c0, kCols), head0 = kvh * ratio + c0;
  const int slot = seqs[i], len = cache_len(c, slot);
  const int tiles = (len + kTileKeys - 1) / kTileKeys;
  const int t0 = (int)((int64_t)tiles * split / splits), t1 = (int)((int64_t)tiles * (split + 1) / splits);

  // the queries as f16 operands: multiplied by a power of two that brings the row's largest value to 2^14 .. 2^15,
  // so that bf16 values fit (those below 2^-28 of the largest lose bits); the scores are multiplied back
  constexpr int QP = kQParts<T>, PP = kPParts<T>;
  halfx8 qf[G][QP];
  float qs[G], mul;
  {
    float f[G][8], m = 0.f;
    const T *src = (const T *)q.data + (int64_t)i * q.token_stride + (int64_t)(head0 + min(col, cols - 1)) * q.head_stride;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      struct alignas(16) { T v[8]; } r = *(const decltype(r) *)(src + 32 * g + 8 * kq);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[g][e] = (float)r.v[e];
        m = fmaxf(m, __builtin_fabsf(f[g][e]));
      }
    }
    m = col_max(m);
    const int ex = __builtin_bit_cast(int, m) >> 23;              // biased exponent, 0 .. 255
    const int sh = ex == 0 || ex == 255 ? 0 : min(14 + 127 - ex, 126);
    const float up = __builtin_bit_cast(float, (uint32_t)(127 + sh) << 23);
    mul = scale * kLog2e / up;
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

  float m = -INFINITY, l = 0.f;
  floatx4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  float zs[G] = {};                                               // PP > 0: sum of p (z - offset s), this lane's keys

  for (int t = t0 + wave; t < t1; t += kWavesA) {
    const uint32_t *tile = (const uint32_t *)cache_tile(c, slot, t * kTileKeys, kvh, tile_bytes(G));
    if (!tile) continue;
    const int left = len - t * kTileKeys;                         // keys of the tile, when below 32
    // scores: lane holds keys 16 b + 4 kq + r of query col
    float s[2][4];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint32_t w = tile[(b * 64 + lane) * G + g];
        const halfx8 kc = codes(w);
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < QP; ++k) x = __builtin_amdgcn_mfma_f32_16x16x32_f16(kc, qf[g][k], x, 0, 0, 0);
        const uintx4 p = *(const uintx4 *)(tile + k_param(G, g, 16 * b + 4 * kq));
#pragma unroll
        for (int r = 0; r < 4; ++r)
          acc[r] = fmaf(half_of(p[r], 0), x[r], fmaf(half_of(p[r], 1), qs[g], acc[r]));
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) s[b][r] = 16 * b + 4 * kq + r < left ? acc[r] * mul : -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[b][r]);
    if (__any(mx > m + kSlack)) {
      // each row by its own scores alone, so that no row's result depends on another's
      const float rm = col_max(mx), mn = rm > m + kSlack ? rm : m;
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
      p[e] = __builtin_amdgcn_exp2f(s[e >> 2][e & 3] - mu);
      l += p[e];
      ph[e] = (_Float16)p[e];
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      halfx8 vs = *(const halfx8 *)(tile + v_param(G, g, kq)), vz = *(const halfx8 *)(tile + v_param(G, g, kq) + 4);
      if (left < kTileKeys) {                                     // what is past the last token may be anything
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (4 * kq + (e & 3) + 16 * (e >> 2) >= left) vs[e] = vz[e] = (_Float16)0;
      }
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
          const bfx8 vc = PP == 2 ? codes_128(w) : codes_bf(w);
#pragma unroll
          for (int k = 0; k < PP; ++k) o[t2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vc, pp[k], o[t2], 0, 0, 0);
        } else {
          o[t2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes(w) * vs + vz, ph, o[t2], 0, 0, 0);
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
  if (kq == 0) {
    red_ml[wave][0][col] = m;
    red_ml[wave][1][col] = l;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) red_o[wave][col][16 * t + 4 * kq + r] = o[t][r];
  __syncthreads();
  for (int x = threadIdx.x; x < cols * D; x += 256) {
    const int h = x / D, d = x % D;
    float mm = -INFINITY, ll = 0.f, v = 0.f;
#pragma unroll
    for (int w = 0; w < kWavesA; ++w) mm = fmaxf(mm, red_ml[w][0][h]);
    const float mu = mm == -INFINITY ? 0.f : mm;
#pragma unroll
    for (int w = 0; w < kWavesA; ++w) {
      const float a = __builtin_amdgcn_exp2f(red_ml[w][0][h] - mu);
      ll = fmaf(a, red_ml[w][1][h], ll);
      v = fmaf(a, red_o[w][h][d], v);
    }
    const int64_t row = (int64_t)i * heads + head0 + h;
    if (part) {
      float *p = part + (row * splits + split) * (D + 2);
      p[2 + d] = v;
      if (d == 0) {
        p[0] = mm;
        p[1] = ll;
      }
    } else {
      ((T *)out.data)[(int64_t)i * out.token_stride + (int64_t)(head0 + h) * out.head_stride + d] =
          (T)(ll == 0.f ? 0.f : v / ll);
      if (lse && d == 0) lse[(int64_t)(head0 + h) * q.tokens + i] = (mm + __builtin_log2f(ll)) * kLn2;
    }
  }
}

// Join the splits of a row: one workgroup per row, a thread per value.
template <class T>
__global__ __launch_bounds__(128) void attn_join_kernel(int heads, int dim, int splits, ios_tokens out, float *lse,
                                                        const float *part) {
  const int64_t row = blockIdx.x, i = row / heads, h = row % heads;
  const float *p = part + row * splits * (dim + 2);
  float mm = -INFINITY;
  for (int s = 0; s < splits; ++s) mm = fmaxf(mm, p[(int64_t)s * (dim + 2)]);
  const float mu = mm == -INFINITY ? 0.f : mm;
  float ll = 0.f, v = 0.f;
  for (int s = 0; s < splits; ++s) {
    const float *ps = p + (int64_t)s * (dim + 2);
    const float a = __builtin_amdgcn_exp2f(ps[0] - mu);
    ll = fmaf(a, ps[1], ll);
    if ((int)threadIdx.x < dim) v = fmaf(a, ps[2 + threadIdx.x], v);
  }
  if ((int)threadIdx.x < dim)
    ((T *)out.data)[i * out.token_stride + h * out.head_stride + threadIdx.x] = (T)(ll == 0.f ? 0.f : v / ll);
  if (lse && threadIdx.x == 0) lse[h * out.tokens + i] = (mm + __builtin_log2f(ll)) * kLn2;
}

template <class T, int G>
hipError_t run(const CacheView &c, const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &out, float *lse,
               const int32_t *seqs, float *part, int splits, hipStream_t s) {
  const int ratio = d.heads / d.kv_heads, blocks = (ratio + kCols - 1) / kCols;
  hipLaunchKernelGGL((attn_cache_kernel<T, G>), dim3(splits, d.kv_heads * blocks, d.seqs), dim3(64 * kWavesA), 0, s, c,
                     d.heads, ratio, d.scale, q, out, lse, seqs, splits > 1 ? part : nullptr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((attn_join_kernel<T>), dim3((unsigned)((int64_t)d.seqs * d.heads)), dim3(128), 0, s, d.heads,
                     d.head_dim, splits, out, lse, part);
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
  const int64_t keys = d.max_keys ? d.max_keys : 1 << 16;
  return (int)std::max<int64_t>(1, std::min((1024 + blocks - 1) / blocks, (keys + 255) / 256));
}

hipError_t launch_attn_cache(const CacheView &c, const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &out,
                             float *lse, const int32_t *seqs, void *work, int splits, hipStream_t s) {
  if (d.dtype == IOS_F32) return for_groups<float>(c, d, q, out, lse, seqs, (float *)work, splits, s);
  if (d.dtype == IOS_F16) return for_groups<_Float16>(c, d, q, out, lse, seqs, (float *)work, splits, s);
  return for_groups<__bf16>(c, d, q, out, lse, seqs, (float *)work, splits, s);
}

}  // namespace ios
