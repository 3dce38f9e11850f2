// Keys and values to and from the 4-bit cache (ios_cache_append, ios_cache_append_rotary, ios_cache_keep, ios_cache_read).
//
// A workgroup owns one tile (32 tokens of one head) and builds or reads it in
// LDS: the V codes of 8 tokens share a word, so a tile is the smallest piece
// that is written whole.  Where the tile already holds earlier tokens it is
// read first.  2 D values in and 5/4 D bytes out per token and head.  35472 tokens
// of 8 heads of 128: read as float32 72 us (336 MB, 4.7 TB/s: memory); append 71
// us (190 MB, 52 .. 66 if the input stays in the 256 MB cache: the quantiser's
// vector instructions, 66 per cent busy).  32 single tokens 5.6 and 3.8 us, a
// chain of dependent loads (offsets, slot, length, page, values).  With rotation, 19136 tokens of 8 heads of 64 and 16 of
// queries: 50 us for 130 MB (queries 23, keys and values 27, 17 unturned: vector units 60 per cent busy; every head's workgroup
// makes its own table of the tile's cosines), in float32 72; 32 single tokens 6.2.
// Accepted drafts of 256 sequences, 2048 tiles: 12.6 us, the same chain; with a sequence's tiles beside each other 17, as every
// other workgroup, and so half of the XCDs, had none.
#include "rotary.h"

namespace ios {

namespace {

constexpr float kLimit = 61440.f;       // so that z + s c never leaves f16
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

template <class T>
using Row8 = Octet8<T>;

// What both kernels need to know of the tile of this workgroup.
struct TileJob {
  unsigned char *tile;        // null: nothing to do
  int lo, hi;                 // tokens of the tile in the call, [lo, hi)
  int64_t row;                // row of the call that is the tile's token 0 (may be negative)
  int pos;                    // place of the tile's token 0 in the sequence
};

// Sequence i has tiles from unit cu[i] / 32 + 2 i on: L tokens touch at most
// L / 32 + 2 tiles.
__device__ __forceinline__ TileJob find_tile(const CacheView &c, int tile_b, int n, const int32_t *seqs,
                                             const int32_t *cu, int64_t tokens, int head, int *seq) {
  TileJob j{nullptr, 0, 0, 0, 0};
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
  j.pos = (int)t0;
  return j;
}

// The same for the accepted drafts of sequence i, rows path[i * most ..] of the call.
// j.row is then the place in the list that is the tile's token 0.
__device__ __forceinline__ TileJob find_kept(const CacheView &c, int tile_b, int n, const int32_t *seqs,
                                             const int32_t *count, int most, int head, int *seq) {
  TileJob j{nullptr, 0, 0, 0, 0};
  const int i = (int)blockIdx.x % n, x = (int)blockIdx.x / n;  // first tiles first: the others are mostly not touched
  *seq = i;
  const int slot = seqs[i], len = cache_len(c, slot), kept = (int)clip(count[i], most), first = len - kept;
  const int p0 = max(first, 0), t0 = (p0 / kTileKeys + x) * kTileKeys;
  if (kept == 0 || t0 >= len) return j;
  j.tile = cache_tile(c, slot, t0, head, tile_b);
  j.lo = max(p0 - t0, 0);
  j.hi = min(len - t0, kTileKeys);
  j.row = t0 - first;
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

// Where a call's tokens come from: rows behind each other, the same with keys to be turned and queries beside them, or
// rows by a list.
enum { ROWS = 0, TURNED = 1, KEPT = 2 };
template <int M> struct Source {};
template <> struct Source<TURNED> {
  ios_rotary r;
  ios_tokens q, qo;
  int heads;
};
template <> struct Source<KEPT> {
  const int32_t *count;
  int most;
};
constexpr int kQueryHeads = 8;          // heads of queries that a workgroup turns

// Cosines and sines of a tile's tokens, [token][pair].
__device__ __forceinline__ void turns_of(const ios_rotary &r, const TileJob &j, int half, float2 *cs) {
  for (int y = threadIdx.x; y < (j.hi - j.lo) * half; y += 256)
    cs[y] = turn_of(j.pos + j.lo + y / half, r.freq[y % half], r.amplitude);
}

// The queries of a tile's tokens, up to kQueryHeads heads from head0 on.
template <class T>
__device__ __forceinline__ void turn_queries(const Source<TURNED> &x, const TileJob &j, int dim, int head0, float2 *cs) {
  constexpr int N = 4;                                       // units on their way at once
  const RotaryUnits u(x.r, dim);
  const int heads = min(x.heads - head0, kQueryHeads), units = (j.hi - j.lo) * heads * u.all;
  RotaryUnit<T> unit[N];
  int at[N], key[N], head[N];
  auto row = [&](const ios_tokens &a, int e) {
    return (T *)a.data + (j.row + j.lo + key[e]) * a.token_stride + (head0 + head[e]) * a.head_stride;
  };
  auto load = [&](int y0) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int y = min(y0 + 256 * e, units - 1), z = y / u.all;
      at[e] = y - z * u.all;
      key[e] = z / heads;
      head[e] = z - key[e] * heads;
      unit[e].load(u, row(x.q, e), at[e]);
    }
  };
  load(threadIdx.x);
  turns_of(x.r, j, u.half, cs);
  __syncthreads();
  for (int y0 = threadIdx.x; y0 < units; y0 += 256 * N) {
    if (y0 != (int)threadIdx.x) load(y0);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (y0 + 256 * e < units) {
        unit[e].turn_by(u, cs + key[e] * u.half, at[e]);
        unit[e].store(u, row(x.qo, e), at[e]);
      }
  }
}

// The tile's keys, octet tid + 256 u of them in kr[u].
template <class T, int G, int N>
__device__ __forceinline__ void turn_keys(const ios_rotary &r, const TileJob &j, Row8<T> (&kr)[N], T *rows, float2 *cs) {
  const RotaryUnits u(r, 32 * G);
  const int tid = threadIdx.x, keys = j.hi - j.lo;
  turns_of(r, j, u.half, cs);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (tid + 256 * e < kTileKeys * 4 * G) *(Row8<T> *)(rows + (tid + 256 * e) * 8) = kr[e];
  __syncthreads();
  for (int y = tid; y < keys * u.turned; y += 256) {
    const int key = y / u.turned, at = y - key * u.turned;
    T *row = rows + (j.lo + key) * 32 * G;
    RotaryUnit<T> unit;
    unit.load(u, row, at);
    unit.turn_by(u, cs + key * u.half, at);
    unit.store(u, row, at);
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (tid + 256 * e < kTileKeys * 4 * G) kr[e] = *(const Row8<T> *)(rows + (tid + 256 * e) * 8);
}

// For M == KEPT `cu` is the list of rows.
template <class T, int G, int M>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheView c, ios_tokens k, ios_tokens v, int n,
                                                           const int32_t *seqs, const int32_t *cu, Source<M> from) {
  __shared__ uint32_t img[tile_bytes(G) / 4];
  __shared__ uint32_t vc[kTileKeys * 4 * G];                 // codes of V by key and octet of values
  __shared__ __align__(16) T turned[M == TURNED ? kTileKeys * 32 * G : 1];
  __shared__ float2 cs[M == TURNED ? kTileKeys * 16 * G : 1];
  const int tid = threadIdx.x, head = blockIdx.y;
  int seq;
  TileJob j;
  if constexpr (M == KEPT) j = find_kept(c, tile_bytes(G), n, seqs, from.count, from.most, head, &seq);
  else j = find_tile(c, tile_bytes(G), n, seqs, cu, k.tokens, M == TURNED ? min(head, c.heads - 1) : head, &seq);
  if ((!j.tile && !(M == TURNED && head >= c.heads)) || j.lo >= j.hi) return;
  if constexpr (M == TURNED) {
    if (head >= c.heads) {
      turn_queries<T>(from, j, 32 * G, (head - c.heads) * kQueryHeads, cs);
      return;
    }
  }
  // every load first: the tile, if it holds tokens, and the tokens' values (a thread has up to N octets of K and of V)
  constexpr int I = (tile_bytes(G) / 16 + 255) / 256;
  uintx4 *gt = (uintx4 *)j.tile, *li = (uintx4 *)img, old[I];
#pragma unroll
  for (int u = 0; u < I; ++u)
    old[u] = j.lo > 0 ? gt[min(tid + 256 * u, tile_bytes(G) / 16 - 1)] : uintx4{0, 0, 0, 0};
  constexpr int N = (kTileKeys * 4 * G + 255) / 256;
  Row8<T> kr[N], vr[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int o = tid + 256 * u, key = min(max(o / (4 * G), j.lo), j.hi - 1), oct = o % (4 * G);
    int64_t row = j.row + key;
    if constexpr (M == KEPT) {
      if (key != o / (4 * G)) continue;
      row = cu[(int64_t)seq * from.most + row];
    }
    if (M == KEPT && (row < 0 || row >= k.tokens)) {         // no such row: the token is 0
      kr[u] = vr[u] = Row8<T>{};
      continue;
    }
    kr[u] = *(const Row8<T> *)((const T *)k.data + row * k.token_stride + head * k.head_stride + oct * 8);
    vr[u] = *(const Row8<T> *)((const T *)v.data + row * v.token_stride + head * v.head_stride + oct * 8);
  }
  if constexpr (M == TURNED) turn_keys<T, G, N>(from.r, j, kr, turned, cs);
#pragma unroll
  for (int u = 0; u < I; ++u)
    if (tid + 256 * u < tile_bytes(G) / 16) li[tid + 256 * u] = old[u];
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

// The tiles that the tokens of n sequences can touch.
unsigned tiles_of(int64_t tokens, int n) { return (unsigned)(tokens / kTileKeys + 2 * (int64_t)n); }

template <int M>
hipError_t append(const CacheView &c, int groups, int dtype, dim3 grid, const ios_tokens &k, const ios_tokens &v, int n,
                  const int32_t *seqs, const int32_t *cu, const Source<M> &from, hipStream_t s) {
  return for_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (groups == 1) hipLaunchKernelGGL((cache_append_kernel<T, 1, M>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu, from);
    else if (groups == 2) hipLaunchKernelGGL((cache_append_kernel<T, 2, M>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu, from);
    else if (groups == 3) hipLaunchKernelGGL((cache_append_kernel<T, 3, M>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu, from);
    else hipLaunchKernelGGL((cache_append_kernel<T, 4, M>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu, from);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_append(const CacheView &c, int groups, int dtype, const ios_tokens &k, const ios_tokens &v, int n,
                         const int32_t *seqs, const int32_t *cu, hipStream_t s) {
  return append<ROWS>(c, groups, dtype, dim3(tiles_of(k.tokens, n), c.heads), k, v, n, seqs, cu, {}, s);
}

hipError_t launch_append_rotary(const CacheView &c, int groups, int dtype, const ios_rotary &r, const ios_tokens *q,
                                const ios_tokens *qo, int heads, const ios_tokens &k, const ios_tokens &v, int n,
                                const int32_t *seqs, const int32_t *cu, hipStream_t s) {
  Source<TURNED> from{r, {}, {}, 0};
  if (q) from.q = *q, from.qo = *qo, from.heads = heads;
  const dim3 grid(tiles_of(k.tokens, n), c.heads + (from.heads + kQueryHeads - 1) / kQueryHeads);
  return append<TURNED>(c, groups, dtype, grid, k, v, n, seqs, cu, from, s);
}

hipError_t launch_keep(const CacheView &c, int groups, int dtype, const ios_tokens &k, const ios_tokens &v, int n,
                       const int32_t *seqs, const int32_t *path, int most, const int32_t *count, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)n * (most / kTileKeys + 2)), c.heads);
  return append<KEPT>(c, groups, dtype, grid, k, v, n, seqs, path, {count, most}, s);
}

hipError_t launch_read(const CacheView &c, int groups, int dtype, const ios_tokens &k, const ios_tokens &v, int n,
                       const int32_t *seqs, const int32_t *cu, hipStream_t s) {
  return for_type(dtype, [&](auto t) {
    using T = decltype(t);
    const dim3 grid(tiles_of(k.tokens, n), c.heads);
    if (groups == 1) hipLaunchKernelGGL((cache_read_kernel<T, 1>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu);
    else if (groups == 2) hipLaunchKernelGGL((cache_read_kernel<T, 2>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu);
    else if (groups == 3) hipLaunchKernelGGL((cache_read_kernel<T, 3>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu);
    else hipLaunchKernelGGL((cache_read_kernel<T, 4>), grid, dim3(256), 0, s, c, k, v, n, seqs, cu);
    return hipGetLastError();
  });
}

}  // namespace ios
