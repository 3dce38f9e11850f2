// Keys and values to and from the 4-bit cache (ios_cache_append, ios_cache_read).
//
// A workgroup owns one tile (32 tokens of one head) and builds or reads it in
// LDS: the V codes of 8 tokens share a word, so a tile is the smallest piece
// that is written whole.  Where the tile already holds earlier tokens it is
// read first.  2 D values in and 5/4 D bytes out per token and head.  35472 tokens
// of 8 heads of 128: read as float32 72 us (336 MB, 4.7 TB/s: memory); append 71
// us (190 MB, 52 .. 66 if the input stays in the 256 MB cache: the quantiser's
// vector instructions, 66 per cent busy).  32 single tokens 5.6 and 3.8 us, a
// chain of dependent loads (offsets, slot, length, page, values).
#include "decoder.h"

namespace ios {

namespace {

constexpr float kLimit = 61440.f;       // so that z + s c never leaves f16
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

template <class T>
struct alignas(16) Row8 {
  T v[8];
};

// What both kernels need to know of the tile of this workgroup.
struct TileJob {
  unsigned char *tile;        // null: nothing to do
  int lo, hi;                 // tokens of the tile in the call, [lo, hi)
  int64_t row;                // row of the call that is the tile's token 0 (may be negative)
};

// Sequence i has tiles from unit cu[i] / 32 + 2 i on: L tokens touch at most
// L / 32 + 2 tiles.
__device__ __forceinline__ TileJob find_tile(const CacheView &c, int tile_b, int n, const int32_t *seqs,
                                             const int32_t *cu, int64_t tokens, int head, int *seq) {
  TileJob j{nullptr, 0, 0, 0};
  auto start = [&](int i) { return clip(cu[i], tokens) / kTileKeys + 2 * (int64_t)i; };
  const int i = find_owner(n, blockIdx.x, start);
  *seq = i;
  const int64_t a = clip(cu[i], tokens), b = clip(cu[i + 1], tokens);
  const int slot = seqs[i], len = cache_len(c, slot);
  const int64_t first = (int64_t)len - (b - a);              // position of the call's first token
  const int64_t p0 = first < 0 ? 0 : first;
  const int64_t t0 = (p0 / kTileKeys + (blockIdx.x - start(i))) * kTileKeys;
  if (b <= a || blockIdx.x < start(i) || t0 >= len) return j;  // units before the first sequence, offsets that descend
  j.tile = cache_tile(c, slot, (int)t0, head, tile_b);
  j.lo = p0 > t0 ? (int)(p0 - t0) : 0;
  j.hi = len - t0 < kTileKeys ? (int)(len - t0) : kTileKeys;
  j.row = a + t0 - first;
  return j;
}

// 32 values of a group, 8 in each of 4 neighbouring lanes: codes of this
// lane's, scale and zero point.
struct Quant {
  uint32_t word;              // 8 codes
  uint32_t param;             // s | z << 16
};
template <class T>
__device__ __forceinline__ Quant quantise(const Row8<T> &r) {
  float x[8], lo = kLimit, hi = -kLimit;
  int nan = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float f = (float)r.v[e];
    nan |= f != f;
    x[e] = fminf(fmaxf(f, -kLimit), kLimit);
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
  }
#pragma unroll
  for (int m = 1; m < 4; m <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, m));
    hi = fmaxf(hi, __shfl_xor(hi, m));
    nan |= __shfl_xor(nan, m);
  }
  float step = (hi - lo) * (float)(1.0 / 15.0);
  asm("" : "+v"(step));       // rounded to f32 before f16: the compiler may otherwise multiply and convert in one step
  const _Float16 z = (_Float16)lo, s = (_Float16)step;
  // (x - z) / s as the division rounds it, from the rounded reciprocal: each step takes the exact remainder (one fused
  // operation) times the reciprocal; the first makes the quotient one of the two nearest numbers, the second the nearest
  // (Markstein, 1990).  5 operations a value, a division takes 11.
  const float fz = (float)z, fs = (float)s, inv = 1.f / fs;
  Quant q{0, 0};
  if (!nan) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = x[e] - fz;
      float v = t * inv;
      v = fmaf(fmaf(-v, fs, t), inv, v);
      v = fmaf(fmaf(-v, fs, t), inv, v);
      const float c = fs > 0.f ? fminf(fmaxf(rintf(v), 0.f), 15.f) : 0.f;
      q.word |= (uint32_t)c << nibble_shift(e);
    }
    q.param = __builtin_bit_cast(uint16_t, s) | (uint32_t)__builtin_bit_cast(uint16_t, z) << 16;
  } else {
    q.param = 0x7E007E00u;
  }
  return q;
}

template <class T, int G>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheView c, ios_tokens k, ios_tokens v, int n,
                                                           const int32_t *seqs, const int32_t *cu) {
  __shared__ uint32_t img[tile_bytes(G) / 4];
  __shared__ uint32_t vc[kTileKeys * 4 * G];                 // codes of V by key and octet of values
  const int tid = threadIdx.x, head = blockIdx.y;
  int seq;
  const TileJob j = find_tile(c, tile_bytes(G), n, seqs, cu, k.tokens, head, &seq);
  if (!j.tile || j.lo >= j.hi) return;
  // every load first: the tokens' values (a thread has up to N octets of K and of V) and the tile, if it holds some
  constexpr int N = (kTileKeys * 4 * G + 255) / 256;
  Row8<T> kr[N], vr[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int o = tid + 256 * u, key = min(max(o / (4 * G), j.lo), j.hi - 1), oct = o % (4 * G);
    const int64_t row = j.row + key;
    kr[u] = *(const Row8<T> *)((const T *)k.data + row * k.token_stride + head * k.head_stride + oct * 8);
    vr[u] = *(const Row8<T> *)((const T *)v.data + row * v.token_stride + head * v.head_stride + oct * 8);
  }
  uintx4 *gt = (uintx4 *)j.tile, *li = (uintx4 *)img;
  for (int i = tid; i < tile_bytes(G) / 16; i += 256) li[i] = j.lo > 0 ? gt[i] : uintx4{0, 0, 0, 0};
  __syncthreads();
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int o = tid + 256 * u, key = o / (4 * G), oct = o % (4 * G), g = oct / 4, q = oct % 4;
    if (key < j.lo || key >= j.hi) continue;                 // the 4 lanes of a group agree
    const Quant a = quantise(kr[u]);
    img[k_word(G, key, q, g)] = a.word;
    const Quant b = quantise(vr[u]);
    vc[o] = b.word;
    if (q == 0) {
      ((uint16_t *)img)[k_scale(G, g, key)] = (uint16_t)a.param;
      ((uint16_t *)img)[k_zero(G, g, key)] = (uint16_t)(a.param >> 16);
      uint16_t *p = (uint16_t *)(img + v_param(G, g, v_quarter(key))) + v_elem(key);
      p[0] = (uint16_t)b.param;
      p[8] = (uint16_t)(b.param >> 16);
    }
  }
  __syncthreads();
  for (int w = tid; w < 128 * G; w += 256) {
    const int t = w >> 6, lane = w & 63, d = 16 * t + (lane & 15), q = lane >> 4;
    uint32_t word = img[v_word(G, t, lane)];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = 4 * q + (e & 3) + 16 * (e >> 2);
      if (key < j.lo || key >= j.hi) continue;
      const uint32_t code = vc[key * 4 * G + d / 8] >> nibble_shift(d & 7) & 15;
      word = (word & ~(15u << nibble_shift(e))) | code << nibble_shift(e);
    }
    img[v_word(G, t, lane)] = word;
  }
  __syncthreads();
  for (int i = tid; i < tile_bytes(G) / 16; i += 256) gt[i] = li[i];
}

template <class T>
__device__ __forceinline__ T held(uint32_t param, uint32_t code) {
  const float s = (float)__builtin_bit_cast(_Float16, (uint16_t)param);
  const float z = (float)__builtin_bit_cast(_Float16, (uint16_t)(param >> 16));
  return (T)(z + s * (float)code);
}

template <class T, int G>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheView c, ios_tokens k, ios_tokens v, int n,
                                                         const int32_t *seqs, const int32_t *cu) {
  __shared__ uint32_t img[tile_bytes(G) / 4];
  const int tid = threadIdx.x, head = blockIdx.y;
  int seq;
  const TileJob j = find_tile(c, tile_bytes(G), n, seqs, cu, k.tokens, head, &seq);
  const int64_t a = clip(cu[seq], k.tokens), b = clip(cu[seq + 1], k.tokens);
  auto store = [&](const ios_tokens &t, int64_t row, int oct, const Row8<T> &r) {
    *(Row8<T> *)((T *)t.data + row * t.token_stride + head * t.head_stride + oct * 8) = r;
  };
  const Row8<T> zero{};
  if (blockIdx.x == a / kTileKeys + 2 * seq) {               // rows for which the sequence has no token
    const int64_t missing = (b - a) - cache_len(c, seqs[seq]);
    for (int64_t o = tid; o < missing * (4 * G); o += 256) {
      store(k, a + o / (4 * G), (int)(o % (4 * G)), zero);
      store(v, a + o / (4 * G), (int)(o % (4 * G)), zero);
    }
  }
  if (j.hi <= j.lo) return;
  if (j.tile)
    for (int i = tid; i < tile_bytes(G) / 16; i += 256) ((uintx4 *)img)[i] = ((const uintx4 *)j.tile)[i];
  else                                                       // no page: reads as 0
    for (int i = tid; i < tile_bytes(G) / 16; i += 256) ((uintx4 *)img)[i] = uintx4{0, 0, 0, 0};
  __syncthreads();
  for (int o = tid; o < kTileKeys * 4 * G; o += 256) {
    const int key = o / (4 * G), oct = o % (4 * G), g = oct / 4, q = oct % 4;
    if (key < j.lo || key >= j.hi) continue;
    const uint16_t *half = (const uint16_t *)img;
    const uint32_t kw = img[k_word(G, key, q, g)], kp = half[k_scale(G, g, key)] | (uint32_t)half[k_zero(G, g, key)] << 16;
    const uint16_t *p = (const uint16_t *)(img + v_param(G, g, v_quarter(key))) + v_elem(key);
    const uint32_t vp = p[0] | (uint32_t)p[8] << 16;
    Row8<T> kr, vr;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      kr.v[e] = held<T>(kp, kw >> nibble_shift(e) & 15);
      const int d = oct * 8 + e;
      const uint32_t vw = img[v_word(G, d >> 4, (d & 15) + 16 * v_quarter(key))];
      vr.v[e] = held<T>(vp, vw >> nibble_shift(v_elem(key)) & 15);
    }
    store(k, j.row + key, oct, kr);
    store(v, j.row + key, oct, vr);
  }
}

template <class F>
hipError_t for_type(int dtype, F f) {
  if (dtype == IOS_F32) return f(float{});
  if (dtype == IOS_F16) return f(_Float16{});
  return f(__bf16{});
}

}  // namespace

#define IOS_FOR_GROUPS(kernel)                                                                          \
  for_type(dtype, [&](auto t) {                                                                         \
    using T = decltype(t);                                                                              \
    const dim3 grid((unsigned)(k.tokens / kTileKeys + 2 * (int64_t)n), c.heads);                        \
    if (groups == 1) hipLaunchKernelGGL((kernel<T, 1>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu);   \
    else if (groups == 2) hipLaunchKernelGGL((kernel<T, 2>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu); \
    else if (groups == 3) hipLaunchKernelGGL((kernel<T, 3>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu); \
    else hipLaunchKernelGGL((kernel<T, 4>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu);               \
    return hipGetLastError();                                                                           \
  })

hipError_t launch_append(const CacheView &c, int groups, int dtype, const ios_tokens &k, const ios_tokens &v, int n,
                         const int32_t *seqs, const int32_t *cu, hipStream_t s) {
  return IOS_FOR_GROUPS(cache_append_kernel);
}

hipError_t launch_read(const CacheView &c, int groups, int dtype, const ios_tokens &k, const ios_tokens &v, int n,
                       const int32_t *seqs, const int32_t *cu, hipStream_t s) {
  return IOS_FOR_GROUPS(cache_read_kernel);
}

}  // namespace ios
