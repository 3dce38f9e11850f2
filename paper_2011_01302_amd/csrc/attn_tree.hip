// Attention of drafted tokens over the 4-bit cache and their ancestors (ios_attn_tree).
//
// The rows of a sequence that read one head of keys, draft by draft and head by head, are columns of the products, as
// in single-token attention; a workgroup takes up to NB blocks of 16 of them and a range of the cached keys, so that a
// tile's codes become operands once for all of them.  Its eight waves take tiles of 32 keys in turn.  The drafts' own
// keys, at most two tiles, come as they are, masked by ancestry, and belong to the first range.
#include "attn_codes.h"

namespace ios {

namespace {

constexpr int kWavesT = 8, kThreadsT = 64 * kWavesT;
constexpr int kStagesT = 2;              // tiles of a wave's ring
constexpr int kWantTree = 512, kMinTree = 256, kOneTree = 1024;

typedef float floatx8 __attribute__((ext_vector_type(8)));

template <class T> struct Octet { typedef T type __attribute__((ext_vector_type(8))); };

// Which drafts of its sequence draft `lane` sees: itself and its ancestors.  A parent that is not an earlier draft is
// none.  Each step doubles the distance that is covered.
__device__ __forceinline__ uint64_t ancestors(const int32_t *parent, int m) {
  const int lane = threadIdx.x & 63;
  const int p = lane < m ? parent[lane] : -1;
  int up = p >= 0 && p < lane ? p : -1;
  uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int from = max(up, 0);
    const uint32_t l = __shfl(lo, from), h = __shfl(hi, from);
    const int next = __shfl(up, from);
    lo |= up >= 0 ? l : 0u;
    hi |= up >= 0 ? h : 0u;
    up = up >= 0 ? next : -1;
  }
  return (uint64_t)hi << 32 | lo;
}

template <class T, int G, int NB>
__global__ __launch_bounds__(kThreadsT) void attn_tree_kernel(CacheView c, int heads, int ratio, float scale, ios_tokens q,
                                                              ios_tokens k, ios_tokens v, ios_tokens out, float *lse,
                                                              const int32_t *seqs, const int32_t *cu,
                                                              const int32_t *parent, int most, int chunk, float *part) {
  constexpr int D = 32 * G, NT = 2 * G, VW = v_words(G), W = kCols * NB;
  constexpr int NL = stage_loads(G), SB = stage_bytes(G);
  constexpr int RO = kWavesT * kCols * (D + 1) * 4, RB = RO + kWavesT * kCols * 4 + kWavesT * W * 4;
  __shared__ __align__(16) unsigned char lds[kWavesT * kStagesT * SB > RB ? kWavesT * kStagesT * SB : RB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, kq = lane >> 4;
  const int split = blockIdx.x, splits = gridDim.x, i = blockIdx.z;
  const int blocks = (most * ratio + W - 1) / W;
  const int kvh = blockIdx.y / blocks, r0 = blockIdx.y % blocks * W;
  typedef const __attribute__((address_space(4))) int32_t const_i32;
  const int64_t a = clip(((const_i32 *)cu)[i], q.tokens), b = clip(((const_i32 *)cu)[i + 1], q.tokens);
  const int m = (int)min(max(b - a, (int64_t)0), (int64_t)most), rows = m * ratio;
  if (r0 >= rows) return;
  const int slot = ((const_i32 *)seqs)[i], at = min(max(slot, 0), c.slots - 1);
  const int first = split * chunk + wave, tile_lg = c.page_lg - 5;
  const_i32 *pages = (const_i32 *)(c.table + (int64_t)at * c.row);
  auto page_of = [&](int x) { return pages[min((first + x * kWavesT) >> tile_lg, c.row - 1)]; };
  int page[kStagesT];
#pragma unroll
  for (int x = 0; x < kStagesT; ++x) page[x] = page_of(x);
  const int held = ((const_i32 *)c.lens)[at];
  const int len = slot == at ? (int)clip(held, (int64_t)c.row << c.page_lg) : 0;
  const int tiles = (len + kTileKeys - 1) / kTileKeys;
  const int t1 = split + 1 == splits ? tiles : min(split * chunk + chunk, tiles);
  if (split > 0 && split * chunk >= t1) return;                   // the parts' count leaves this one out

  // row of this lane's column of block n, and its query
  auto row_of = [&](int n) { return min(r0 + 16 * n + col, rows - 1); };
  auto query = [&](int n) {
    const int r = row_of(n), t = r / ratio, h = r - t * ratio;
    return (const T *)q.data + (a + t) * q.token_stride + (int64_t)(kvh * ratio + h) * q.head_stride;
  };
  typedef typename Octet<T>::type octet;

  // a ring of kStagesT tiles per wave: while one is worked on, the others are on their way
  const int n_tiles = first < t1 ? (t1 - first + kWavesT - 1) / kWavesT : 0;
  unsigned char *ring = lds + wave * (kStagesT * SB);
  uint32_t sound = 0;                                             // bit j: the j-th last tile issued has a page
  auto issue = [&](int x, int page) {
    const int t = first + x * kWavesT;
    const bool ok = (unsigned)page < (unsigned)c.pages;
    const unsigned char *tile = c.pool + (ok ? page : 0) * c.page_bytes + (int64_t)kvh * c.head_bytes +
                                (t & ((1 << tile_lg) - 1)) * tile_bytes(G);
    sound = sound << 1 | (ok ? 1u : 0u);
    copy_tile<G>(tile, ring + x % kStagesT * SB, lane);
  };
#pragma unroll
  for (int x = 0; x < kStagesT - 1; ++x)
    if (x < n_tiles) issue(x, page[x]);

  // the queries as f16 operands, scaled by a power of two per row (as in single-token attention), and their sums by
  // group in two f16 parts
  constexpr int QP = kQParts<T>, PP = kPParts<T>;
  halfx8 qf[NB][G][QP];
  halfx4 qz[NB];
  float mul[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const T *src = query(n);
    float f[G][8], top = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const octet row = *(const octet *)(src + 32 * g + 8 * kq);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[g][e] = (float)row[e];
        top = fmaxf(top, __builtin_fabsf(f[g][e]));
      }
    }
    top = col_max(top);
    const int ex = __builtin_bit_cast(int, top) >> 23;            // biased exponent, 0 .. 255
    const int sh = ex == 0 || ex == 255 ? 0 : min(8 + 127 - ex, 126);
    float up = __builtin_bit_cast(float, (uint32_t)(127 + sh) << 23);
    mul[n] = fmaxf(__builtin_fabsf(scale) * kLog2e / up, 1e-30f);
    up = scale < 0.f ? -up : up;
    qz[n] = halfx4{0, 0, 0, 0};
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = f[g][e] * up;
        s += x;
#pragma unroll
        for (int p = 0; p < QP; ++p) {
          qf[n][g][p][e] = (_Float16)x;
          x -= (float)qf[n][g][p][e];
        }
      }
      s = col_sum(s);
      const _Float16 hi = (_Float16)s;
      qz[n][g] = kq == 0 ? hi : kq == 1 ? (_Float16)(s - (float)hi) : (_Float16)0;
    }
  }
  uint32_t mask = 0x000F000Fu;
  asm("" : "+v"(mask));

  float mx_[NB], l[NB];                                           // reference and sum of a row's weights
  floatx4 o[NB][NT];
  float zs[NB][G] = {};                                           // PP > 0: sum of p (z - offset s), this lane's keys
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    mx_[n] = -INFINITY;
    l[n] = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) o[n][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  auto rescale = [&](int n, float to) {
    const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mx_[n] - to);
    mx_[n] = to;
    l[n] *= f;
#pragma unroll
    for (int t = 0; t < NT; ++t) o[n][t] *= f;
#pragma unroll
    for (int g = 0; g < G; ++g) zs[n][g] *= f;
  };

  int next = page[kStagesT - 1];
  for (int x = 0; x < n_tiles; ++x) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // the reads of the slot that is loaded next
    const int ahead = min(kStagesT - 1, n_tiles - 1 - x);         // tiles issued after this one
    if (x + kStagesT - 1 < n_tiles) {
      issue(x + kStagesT - 1, next);
      next = page_of(x + kStagesT);
      wait_loads<NL *(kStagesT - 1)>();
    } else {
      static_assert(kStagesT == 2, "a longer ring has other tiles on their way behind this one");
      wait_loads<0>();
    }
    if (!(sound >> ahead & 1)) continue;
    const uint32_t *tile = (const uint32_t *)(ring + x % kStagesT * SB);
    const int left = len - (first + x * kWavesT) * kTileKeys;     // keys of the tile, when below 32
    const _Float16 *half = (const _Float16 *)tile;
    if (left < kTileKeys) {                                       // what is past the last token may be anything
      for (int y = lane; y < G * kTileKeys; y += 64) {
        const int key = y & 31;
        _Float16 *vp = (_Float16 *)const_cast<uint32_t *>(tile + v_param(G, y >> 5, v_quarter(key))) + v_elem(key);
        if (key >= left) vp[0] = vp[8] = (_Float16)0;
      }
    }
    // scores: lane holds keys 16 b + 4 kq + r of query col of every block
    floatx4 s[NB][2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      halfx4 kz = {0, 0, 0, 0};
#pragma unroll
      for (int g = 0; g < G; ++g) kz[g] = half[k_zero(G, g, 16 * b + col)];
#pragma unroll
      for (int n = 0; n < NB; ++n)
        s[n][b] = __builtin_amdgcn_mfma_f32_16x16x16f16(kz, qz[n], floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const halfx8 kc = codes(tile[(b * 64 + lane) * G + g], mask);
        const halfx4 ks = *(const halfx4 *)(half + k_scale(G, g, 16 * b + 4 * kq));
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          floatx4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int p = 0; p < QP; ++p) y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kc, qf[n][g][p], y, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) s[n][b][r] = fmaf((float)ks[r], y[r], s[n][b][r]);
        }
      }
    }
    if (left < kTileKeys) {
      asm volatile("");                                           // a branch, not selects in every tile
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[n][b][r] = 16 * b + 4 * kq + r < left ? s[n][b][r] : -INFINITY;
    }
    float p[NB][8];
    halfx8 ph[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      float mx = s[n][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, s[n][e >> 2][e & 3]);
      mx *= mul[n];
      if (__any(mx > mx_[n] + kSlack)) {
        // each row by its own scores alone, so that no row's result depends on another's
        const float rm = col_max(mx);
        rescale(n, rm > mx_[n] + kSlack ? rm - kTop : mx_[n]);
      }
      const float mu = mx_[n] == -INFINITY ? 0.f : mx_[n];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[n][e] = __builtin_amdgcn_exp2f(fmaf(s[n][e >> 2][e & 3], mul[n], -mu));
        l[n] += p[n][e];
        ph[n][e] = (_Float16)p[n][e];
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const halfx8 vs = *(const halfx8 *)(tile + v_param(G, g, kq)), vz = *(const halfx8 *)(tile + v_param(G, g, kq) + 4);
      bfx8 pp[NB][PP > 0 ? PP : 1];
      if constexpr (PP > 0) {
        constexpr float offset = PP == 2 ? 128.f : 0.f;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            zs[n][g] = fmaf(p[n][e], (float)vz[e] - offset * (float)vs[e], zs[n][g]);
            float y = p[n][e] * (float)vs[e];
#pragma unroll
            for (int k2 = 0; k2 < PP; ++k2) {
              pp[n][k2][e] = (__bf16)y;
              y -= (float)pp[n][k2][e];
            }
          }
      }
#pragma unroll
      for (int t = 2 * g; t < 2 * g + 2; ++t) {
        const uint32_t w = tile[128 * G + (t / VW * 64 + lane) * VW + t % VW];
        if constexpr (PP > 0) {
          const bfx8 vc = PP == 2 ? codes_128(w, mask) : codes_bf(w);
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int k2 = 0; k2 < PP; ++k2) o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vc, pp[n][k2], o[n][t], 0, 0, 0);
        } else {
          const halfx8 vv = codes(w, mask) * vs + vz;
#pragma unroll
          for (int n = 0; n < NB; ++n) o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, ph[n], o[n][t], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NB; ++n) {                                  // o[n][t][r] is value 16 t + 4 kq + r of row col
    l[n] = col_sum(l[n]);
    if constexpr (PP > 0) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float z = col_sum(zs[n][g]);
        zs[n][g] = 0.f;
        o[n][2 * g] += z;
        o[n][2 * g + 1] += z;
      }
    }
  }

  // the drafts' own keys: the last waves of the first range, which have the fewest tiles
  const int k0 = (kWavesT - 1 - wave) * kTileKeys;
  if (split == 0 && k0 < m) {
    const uint64_t mine = ancestors(parent + a, m);
    const T *kd = (const T *)k.data + a * k.token_stride + kvh * k.head_stride;
    const T *vd = (const T *)v.data + a * v.token_stride + kvh * v.head_stride;
    const int keys = min(m - k0, kTileKeys);
    // keys with values that the weights' usual reference would lead out of float32, and whether there are infinities or NaN
    uint32_t big = 0;
    bool odd = false;
    for (int y = lane; y < keys * (D / 8); y += 64) {
      const int key = y / (D / 8);
      const octet x = *(const octet *)(vd + (k0 + key) * v.token_stride + y % (D / 8) * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = __builtin_fabsf((float)x[e]);
        odd |= !(f < INFINITY);
        big |= f > 0x1p90f && f < INFINITY ? 1u << key : 0u;
      }
    }
    odd = __any(odd);
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) big |= __shfl_xor(big, y);
    const float by = scale * kLog2e;
    float p[NB][8];
    uint32_t seen[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int t = row_of(n) / ratio;
      const uint32_t lo = __shfl((uint32_t)mine, t), hi = __shfl((uint32_t)(mine >> 32), t);
      seen[n] = k0 ? hi : lo;
      const T *src = query(n);
      floatx4 s[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const T *key = kd + min(k0 + 16 * b + col, m - 1) * k.token_stride;
        floatx4 y = {0.f, 0.f, 0.f, 0.f};
        if constexpr (std::is_same_v<T, float>) {
#pragma unroll
          for (int ch = 0; ch < D / 16; ++ch) {
            const floatx4 kk = *(const floatx4 *)(key + 16 * ch + 4 * kq), qq = *(const floatx4 *)(src + 16 * ch + 4 * kq);
#pragma unroll
            for (int e = 0; e < 4; ++e) y = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[e], qq[e], y, 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const octet kk = *(const octet *)(key + 32 * g + 8 * kq), qq = *(const octet *)(src + 32 * g + 8 * kq);
            if constexpr (std::is_same_v<T, _Float16>) y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk, qq, y, 0, 0, 0);
            else y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qq, y, 0, 0, 0);
          }
        }
        s[b] = y;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = seen[n] >> (16 * (e >> 2) + 4 * kq + (e & 3)) & 1 ? s[e >> 2][e & 3] * by : -INFINITY;
        s[e >> 2][e & 3] = x;
        mx = fmaxf(mx, x);
      }
      const float rm = col_max(mx);
      rescale(n, big & seen[n] ? fmaxf(mx_[n], rm) + 24.f         // weights up to 2^-24
                 : rm > mx_[n] + kSlack ? rm - kTop : mx_[n]);
      const float mu = mx_[n] == -INFINITY ? 0.f : mx_[n];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[n][e] = __builtin_amdgcn_exp2f(s[e >> 2][e & 3] - mu);
        sum += p[n][e];
      }
      l[n] += col_sum(sum);
    }
    // the product with the values: 16-bit weights in two parts
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      T val[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = 4 * kq + (e & 3) + 16 * (e >> 2);
        const T x = vd[min(k0 + key, m - 1) * v.token_stride + 16 * t + col];
        val[e] = key < keys && __builtin_fabsf((float)x) < INFINITY ? x : (T)0;
      }
      if constexpr (std::is_same_v<T, float>) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) o[n][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(val[e], p[n][e], o[n][t], 0, 0, 0);
      } else {
        octet vv;
#pragma unroll
        for (int e = 0; e < 8; ++e) vv[e] = val[e];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          octet hi, lo;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            hi[e] = (T)p[n][e];
            lo[e] = (T)(p[n][e] - (float)hi[e]);
          }
          if constexpr (std::is_same_v<T, _Float16>) {
            o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, hi, o[n][t], 0, 0, 0);
            o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, lo, o[n][t], 0, 0, 0);
          } else {
            o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, hi, o[n][t], 0, 0, 0);
            o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, lo, o[n][t], 0, 0, 0);
          }
        }
      }
    }
    if (odd) {                                                    // infinities and NaN, to the rows that see them
#pragma unroll 1
      for (int key = 0; key < keys; ++key)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = (float)vd[(k0 + key) * v.token_stride + 16 * t + 4 * kq + r];
#pragma unroll
            for (int n = 0; n < NB; ++n)
              if (!(__builtin_fabsf(x) < INFINITY) && (seen[n] >> key & 1)) o[n][t][r] += x;
          }
    }
  }

  // join the waves, a block of rows at a time
  __syncthreads();                                                // the rings are done with
  auto *red_o = (float(*)[kCols][D + 1])lds;
  auto *red_l = (float(*)[kCols])(lds + RO);
  auto *red_m = (float(*)[W])(lds + RO + kWavesT * kCols * 4);
  if (kq == 0) {
#pragma unroll
    for (int n = 0; n < NB; ++n) red_m[wave][16 * n + col] = mx_[n];
  }
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int cols = min(rows - r0 - 16 * n, kCols);
    if (cols <= 0) break;
    __syncthreads();                                              // red_m, and the block before
    float mm = mx_[n];
#pragma unroll
    for (int w = 0; w < kWavesT; ++w) mm = fmaxf(mm, red_m[w][16 * n + col]);
    const float f = mm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx_[n] - mm);
    if (kq == 0) red_l[wave][col] = l[n] * f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) red_o[wave][col][16 * t + 4 * kq + r] = weighed(o[n][t][r], f);
    __syncthreads();
#pragma unroll 1
    for (int x = threadIdx.x; x < cols * D; x += kThreadsT) {
      const int h = x / D, d = x % D, r = r0 + 16 * n + h, t = r / ratio, head = kvh * ratio + r - t * ratio;
      float ll = 0.f, y = 0.f, top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWavesT; ++w) {
        top = fmaxf(top, red_m[w][16 * n + h]);
        ll += red_l[w][h];
        y += red_o[w][h][d];
      }
      const int64_t row = (a + t) * heads + head;
      if (part) {
        part[(row * splits + split) * D + d] = y;
        if (d == 0) {
          float *ml = part + q.tokens * heads * splits * D + (row * splits + split) * 2;
          ml[0] = top;
          ml[1] = ll;
        }
      } else {
        ((T *)out.data)[(a + t) * out.token_stride + (int64_t)head * out.head_stride + d] = mean_odd<T>(y, ll);
        if (lse && d == 0) lse[(int64_t)head * q.tokens + a + t] = (top + __builtin_log2f(ll)) * kLn2;
      }
    }
  }
}

template <class T, int G>
__global__ __launch_bounds__(256) void attn_tree_join_kernel(CacheView c, int heads, int seqs_n, int most, int splits,
                                                             int chunk, ios_tokens out, float *lse, const int32_t *seqs,
                                                             const int32_t *cu, const float *part) {
  const int64_t row = blockIdx.x, t = row / heads, h = row % heads;
  const int i = find_owner(seqs_n, t, [&](int x) { return clip(cu[x], out.tokens); });
  const int64_t a = clip(cu[i], out.tokens), b = clip(cu[i + 1], out.tokens);
  if (t < a || t >= b || t >= a + most) return;                   // a row of no sequence, or past the last draft
  join_parts<T, false, true>(row, out.tokens * heads, 32 * G, splits, part,
                             [&] {
                               const int tiles = (cache_len(c, seqs[i]) + kTileKeys - 1) / kTileKeys;
                               return max(1, min((tiles + chunk - 1) / chunk, splits));
                             },
                             (T *)out.data + t * out.token_stride + h * out.head_stride,
                             lse ? lse + h * out.tokens + t : nullptr);
}

int64_t keys_of(const ios_attn_desc &d) { return d.max_keys ? d.max_keys : 1 << 16; }

// Blocks of 16 rows that a workgroup takes.
int row_blocks(const ios_attn_desc &d, int most) {
  const int rows = most * (d.heads / d.kv_heads);
  return rows <= 16 ? 1 : 2;
}

struct Call {
  CacheView c;
  const ios_attn_desc *d;
  ios_tokens q, k, v, out;
  float *lse;
  const int32_t *seqs, *cu, *parent;
  int most, splits;
  float *part;
  hipStream_t s;
};

template <class T, int G, int NB>
hipError_t run(const Call &x) {
  const ios_attn_desc &d = *x.d;
  const int ratio = d.heads / d.kv_heads, blocks = (x.most * ratio + 16 * NB - 1) / (16 * NB), splits = x.splits;
  // tiles of a part; a sequence longer than max_keys makes its last part longer
  const int chunk = (int)std::max<int64_t>(1, (keys_of(d) + (int64_t)kTileKeys * splits - 1) / ((int64_t)kTileKeys * splits));
  hipLaunchKernelGGL((attn_tree_kernel<T, G, NB>), dim3(splits, d.kv_heads * blocks, d.seqs), dim3(kThreadsT), 0, x.s, x.c,
                     d.heads, ratio, d.scale, x.q, x.k, x.v, x.out, x.lse, x.seqs, x.cu, x.parent, x.most, chunk,
                     splits > 1 ? x.part : nullptr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((attn_tree_join_kernel<T, G>), dim3((unsigned)(x.q.tokens * d.heads)), dim3(256), 0, x.s, x.c, d.heads,
                     d.seqs, x.most, splits, chunk, x.out, x.lse, x.seqs, x.cu, x.part);
  return hipGetLastError();
}

template <class T, int G>
hipError_t for_blocks(const Call &x) {
  return row_blocks(*x.d, x.most) == 1 ? run<T, G, 1>(x) : run<T, G, 2>(x);
}

template <class T>
hipError_t for_groups(const Call &x) {
  switch (x.d->head_dim / kGroup) {
    case 1: return for_blocks<T, 1>(x);
    case 2: return for_blocks<T, 2>(x);
    case 3: return for_blocks<T, 3>(x);
    default: return for_blocks<T, 4>(x);
  }
}

}  // namespace

int tree_splits(const ios_attn_desc &d, int most) {
  const int rows = most * (d.heads / d.kv_heads), w = 16 * row_blocks(d, most);
  const int64_t blocks = (int64_t)d.seqs * d.kv_heads * ((rows + w - 1) / w);
  if (keys_of(d) < kOneTree || rows == 0) return 1;
  const int64_t parts = std::min<int64_t>((kWantTree + blocks - 1) / blocks, keys_of(d) / kMinTree);
  return (int)std::max<int64_t>(1, std::min<int64_t>(parts, kMaxParts));
}

hipError_t launch_attn_tree(const CacheView &c, const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &k,
                            const ios_tokens &v, const ios_tokens &out, float *lse, const int32_t *seqs,
                            const int32_t *cu, const int32_t *parent, int most, void *work, int splits, hipStream_t s) {
  const Call x{c, &d, q, k, v, out, lse, seqs, cu, parent, most, splits, (float *)work, s};
  if (d.dtype == IOS_F32) return for_groups<float>(x);
  if (d.dtype == IOS_F16) return for_groups<_Float16>(x);
  return for_groups<__bf16>(x);
}

}  // namespace ios
