// Attention of drafted tokens over the 4-bit cache and their ancestors (ios_attn_tree).
//
// The rows of a sequence that read one head of keys, draft by draft and head by head, are columns of the products, as
// in single-token attention; a workgroup takes a block of up to NB times 16 of them and a range of the cached keys, so
// that a tile's codes become operands once for all of them.  Its eight waves take tiles of 32 keys in turn.  The drafts'
// own keys, at most two tiles, come as they are, masked by ancestry, and belong to the first range.
//
// Sequences differ in length and trees in size, so the ranges are laid out on the device: all blocks' steps (eight tiles
// each) one after another, cut into equal shares, one for each workgroup that the card holds at a time.  A block that
// lies in several shares leaves its parts in the workspace, at most two a workgroup, for a second launch.  (Parts by the
// longest sequence's length left workgroups idle for 39 per cent of the time on 32 sequences of 8192 to 32031 tokens.)
//
// Those under 16 drafts of 32 heads (64 rows a head of keys, bf16): 290 us, 823 MB of cache and 169 GFLOP.  Matrix cores are
// busy for 25 and vector units (codes to numbers and the softmax) for 50 per cent, waves wait for 38: a tile's scores, weights
// and values follow each other, and two waves a SIMD, as many as the sums' registers leave room for, do not cover that.  f16
// takes 530 (values formed in 32 bits and split one by one, three products for one), float32 880.  Under 4 drafts (16 rows)
// 166 us: memory.  One sequence of 131072 tokens under 32 drafts of 16 heads 76 us, four blocks of rows that each turn the same
// codes into numbers.  A small call is latency: 28x28 tokens under 7 drafts 19 us, four tiles a wave one after the other, before
// and after them the queries, the drafts and the join of the waves with code that no cache holds yet.
//
// Every workgroup reads all sequences' offsets and lengths to find its share, and steps over those without rows one by one: 32
// drafts behind 32 sequences of 40 tokens 15 us, behind 32 of 4096 94 and of 65535 1435 (39 and 330 without a workspace).
#include "attn_codes.h"

namespace ios {

namespace {

constexpr int kWavesT = 8, kThreadsT = 64 * kWavesT;
constexpr int kStagesT = 3;              // tiles of a wave's ring
constexpr int kStepTiles = kWavesT;      // tiles of a step: one a wave
// Steps that a block of rows costs beside its keys (us for 1, 3 and 6: one sequence of 131072 tokens 80.5, 75.8, 76.4, the maps
// in f16 29.8, 31.0, 35.3, in bf16 26.4, 25.9, 28.4); the fewest of a share (for 1, 3 and 6: the maps 30.9, 31.0, 34.3, one
// sequence of 3100 tokens under 13 drafts 16.6, 19.9, 22.2, one of 20000 under 4 16.4, 16.9, 18.5, the others the same); and the
// keys from which blocks are cut, so that there is a second launch (whole and cut: one sequence of 600 keys in float32 16.0 and
// 18.7, 1000 21.1 and 20.7, 1300 24.6 and 20.7, in bf16 1000 13.4 and 16.7, 2000 17.3 and 18.0; 16 sequences of 300 21.4 and
// 23.1, 600 25.1 and 23.0, 1000 30.9 and 26.9).  The maps: 16 sequences of 1 to 3100 tokens under 0 to 64 drafts of 16 heads.
constexpr int kItemSteps = 3, kShareSteps = 3, kOneTree = 1024;

// How the products over the cache are computed, for results in T:
// bf16: keys and values z + s c rounded to f16 (2^-11 at most, against 2^-8 of the result), weights to f16
// f16: scores z sum(q) + s (c . q) with exact codes; values and weights in two f16 parts each, of whose products the one of
//      both second parts is left out (2^-22)
// f32: the same scores with q in three f16 parts; p s in three bf16 parts times exact codes, zero points in 32 bits.  Codes
//      are taken from 8 on, (z + 8 s) + s (c - 8), so that no term is much larger than the value (with the zero point at the
//      least value results were 1.2e-6 of their size off over 785 tokens, elementary operations in float32 5e-7)
template <class T> constexpr bool kHeldKeys = std::is_same_v<T, __bf16>;
template <class T> constexpr int kQueryParts = std::is_same_v<T, float> ? 3 : 1;

// The largest weight is 2^kTopTree when its row's reference is set, and the reference is set anew when one would pass 2^6
// times that: rows whose largest score grows by less than 6 (base 2) from the first tile on, which are nearly all, keep the
// first.  A 16-bit weight is off by at most 2^-25, so 2^-34 of the largest: 10^6 keys together by 2^-14 (2^-38 in single-token
// attention, whose rows follow their largest score sooner).  Float32's need no such room, and scores near the reference are the
// more exact the nearer they are.
template <class T> constexpr float kTopTree = std::is_same_v<T, float> ? 0.f : 9.f;
template <class T> constexpr float kFarTree = kTopTree<T> + 6.f;

// Rows in which a draft's value times such a weight would come near float32's largest hold their sums 2^-kApart times as
// large.  Float32 simply takes a reference so much higher; in bf16 the cached tokens' weights go to f16, which has no room
// for that (weights of 2^-24 and less are its last subnormal number or 0, and the row's ordinary values lose most of what the
// wave that has the drafts adds, an eighth), so there the weights stay as they are and the products of such rows are taken
// by themselves.  The test for them costs 1 per cent (one sequence of 131072 tokens 75.7 and 76.3 us).
template <class T> constexpr float kApart = kTopTree<T> + 24.f;
template <class T> constexpr bool kApartSums = std::is_same_v<T, __bf16>;

template <class T> struct Octet { typedef T type __attribute__((ext_vector_type(8))); };

// Which drafts of its sequence draft `lane` sees: itself and its ancestors.  A parent that is not an earlier draft is
// none.  Each step doubles the distance that is covered.
__device__ __forceinline__ uint64_t ancestors(const int32_t *parent, int m) {
  const int lane = threadIdx.x & 63;
  const int p = lane < m ? parent[lane] : -1;
  int up = p >= 0 && p < lane ? p : -1;
  uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
  for (int d = 1; d < m; d <<= 1) {
    const int from = max(up, 0);
    const uint32_t l = __shfl(lo, from), h = __shfl(hi, from);
    const int next = __shfl(up, from);
    lo |= up >= 0 ? l : 0u;
    hi |= up >= 0 ? h : 0u;
    up = up >= 0 ? next : -1;
  }
  return (uint64_t)hi << 32 | lo;
}

// Codes of a word as in codes(), with one shift: f16 numbers 1024 + c and 64 + c are c in their last bits, or four further up.
struct CodeMasks {
  uint32_t lo, hi;                       // in vector registers
  __device__ __forceinline__ CodeMasks() : lo(0x000F000Fu), hi(0x00F000F0u) { asm("" : "+v"(lo), "+v"(hi)); }
  // C less than the codes
  template <int C = 0>
  __device__ __forceinline__ halfx8 codes(uint32_t w) const {
    const uint32_t w8 = w >> 8;
    const uintx4 r = {(w & lo) | 0x64006400u, (w & hi) | 0x54005400u, (w8 & lo) | 0x64006400u, (w8 & hi) | 0x54005400u};
    return __builtin_bit_cast(halfx8, r) - halfx8{1024 + C, 1024 + C, 64 + C, 64 + C, 1024 + C, 1024 + C, 64 + C, 64 + C};
  }
};

// A sequence of the call.
struct TreeSeq {
  int64_t row;                           // its first
  int m, len, place;                     // drafts, cached tokens, slot (one that does not exist: some other's, and no tokens)
  TreeSeq() = default;
  template <class I>
  __device__ __forceinline__ TreeSeq(const CacheView &c, const I *seqs, const I *cu, const I *lens, int i, int64_t tokens,
                                     int most) {
    row = clip(cu[i], tokens);
    m = (int)min(max(clip(cu[i + 1], tokens) - row, (int64_t)0), (int64_t)most);
    const int slot = seqs[i];
    place = min(max(slot, 0), c.slots - 1);
    const int held = lens[place];
    len = slot == place ? (int)clip(held, (int64_t)c.row << c.page_lg) : 0;
  }
  // steps of one block of rows, and of all of them
  __device__ __forceinline__ int block_steps() const {
    return kItemSteps + (len + kStepTiles * kTileKeys - 1) / (kStepTiles * kTileKeys);
  }
  __device__ __forceinline__ int64_t steps(int ratio, int w, int kv_heads) const {
    return (int64_t)((m * ratio + w - 1) / w * kv_heads) * block_steps();
  }
};

// A block of rows' first part and their number.  A workgroup's parts are 2 g and, where its share begins inside another
// block, 2 g + 1; the workgroups behind the first go on with part 2 g.
struct PartRef {
  int32_t first, count;
};

__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32)) << 32 |
                   (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x));
}

// The workspace holds [parts][W][D] sums of weighed values, [parts][W][2] references and sums of weights, and a PartRef
// for every block of rows at its first row's place of [tokens][heads].
template <class T, int G, int NB>
__global__ __launch_bounds__(kThreadsT) void attn_tree_kernel(CacheView c, int heads, int ratio, float scale, ios_tokens q,
                                                              ios_tokens k, ios_tokens v, ios_tokens out, float *lse,
                                                              const int32_t *seqs, const int32_t *cu,
                                                              const int32_t *parent, int n_seqs, int most, float *part) {
  constexpr int D = 32 * G, NT = 2 * G, VW = v_words(G), W = kCols * NB;
  constexpr int NL = stage_loads(G), SB = stage_bytes(G);
  constexpr int RO = kWavesT * kCols * (D / 4 + 1) * 16;
  // behind the ring the queries' operands, which stay in registers where there are few
  constexpr int QP = kQueryParts<T>, RING = kWavesT * kStagesT * SB;
  constexpr bool QL = NB * QP > 2;
  static_assert(RO + kWavesT * kCols * 4 + kWavesT * W * 4 <= RING, "what joins the waves takes the ring's place");
  __shared__ __align__(16) unsigned char lds[RING + NB * G * QP * 1024];
  __shared__ halfx4 sums_of[kHeldKeys<T> ? 1 : NB][64];
  __shared__ float mul_of[W];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, kq = lane >> 4, tile_lg = c.page_lg - 5;
  typedef const __attribute__((address_space(4))) int32_t const_i32;
  typedef typename Octet<T>::type octet;

  // the share: `left` steps from step `at` of sequence i on; without a workspace one block of rows
  int64_t share = 1, left = 1, at = blockIdx.x;
  int i = blockIdx.y;
  TreeSeq seq;
  if (part) {
    struct Begin {
      int64_t sums[kWavesT], at;
      TreeSeq seq;
      int i;
    };
    Begin &begin = *(Begin *)lds;
    const int per = (n_seqs + kThreadsT - 1) / kThreadsT, i0 = threadIdx.x * per, i1 = min(i0 + per, n_seqs);
    auto steps_of = [&](int x) { return TreeSeq(c, seqs, cu, c.lens, x, q.tokens, most).steps(ratio, W, c.heads); };
    int64_t mine = 0;
    for (int x = i0; x < i1; ++x) mine += steps_of(x);
    int64_t upto = mine, all = 0;
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) {
      const int64_t z = __shfl_up(upto, y);
      upto += lane >= y ? z : 0;
    }
    if (lane == 63) begin.sums[wave] = upto;
    __syncthreads();
    upto -= mine;
#pragma unroll
    for (int w = 0; w < kWavesT; ++w) {
      upto += w < wave ? begin.sums[w] : 0;
      all += begin.sums[w];
    }
    all = uniform(all);
    share = max((all + gridDim.x - 1) / gridDim.x, (int64_t)kShareSteps);
    int64_t from = share * blockIdx.x;
    if (from >= all) return;
    left = min(share, all - from);
    if (from >= upto && from < upto + mine) {
      from -= upto;
      int x = i0;
      for (int64_t n; x + 1 < i1 && from >= (n = steps_of(x)); ++x) from -= n;
      begin.i = x;
      begin.at = from;
      begin.seq = TreeSeq(c, seqs, cu, c.lens, x, q.tokens, most);
    }
    __syncthreads();
    i = __builtin_amdgcn_readfirstlane(begin.i);
    at = uniform(begin.at);
    seq.row = uniform(begin.seq.row);
    seq.m = __builtin_amdgcn_readfirstlane(begin.seq.m);
    seq.len = __builtin_amdgcn_readfirstlane(begin.seq.len);
    seq.place = __builtin_amdgcn_readfirstlane(begin.seq.place);
    __syncthreads();                                              // before the ring is filled
  }

  bool known = part != nullptr;                                   // seq is sequence i
  for (int turn = 0; left > 0 && i < n_seqs;) {
    if (!known) seq = TreeSeq(c, (const_i32 *)seqs, (const_i32 *)cu, (const_i32 *)c.lens, i, q.tokens, most);
    known = true;
    const int64_t a = seq.row;
    const int m = seq.m, len = seq.len, rows = m * ratio, tiles = (len + kTileKeys - 1) / kTileKeys, all = seq.block_steps();
    // which block and head of keys, from which of its steps on (the quotient is below 2^31, so its floor is right)
    const int block = part ? (int)((double)at / (double)all) : (int)at, from = part ? (int)(at - (int64_t)block * all) : 0;
    const int r0 = block / c.heads * W, kvh = block % c.heads;
    if (r0 >= rows) {
      if (!part) return;
      ++i;
      at = 0;
      known = false;
      continue;
    }
    const int steps = part ? (int)min((int64_t)(all - from), left) : all;
    const int first = max(from - kItemSteps, 0) * kStepTiles + wave;
    const int end = min(max(from + steps - kItemSteps, 0) * kStepTiles, tiles);
    const_i32 *pages = (const_i32 *)(c.table + (int64_t)seq.place * c.row);
    auto page_of = [&](int x) { return pages[min((first + x * kWavesT) >> tile_lg, c.row - 1)]; };
    int page[kStagesT];
#pragma unroll
    for (int x = 0; x < kStagesT; ++x) page[x] = page_of(x);
    const int64_t slot = steps == all ? -1 : 2 * (int64_t)blockIdx.x + (turn > 0 ? 1 : 0);
    if (part && from == 0 && threadIdx.x == 0) {
      const int64_t rest = all - steps;
      PartRef *refs = (PartRef *)(part + 2 * (int64_t)gridDim.x * W * (D + 2));
      refs[(a + r0 / ratio) * heads + kvh * ratio + r0 % ratio] = {(int32_t)slot, (int32_t)(1 + (rest + share - 1) / share)};
    }

    // a ring of kStagesT tiles per wave: while one is worked on, the others are on their way
    const int n_tiles = first < end ? (end - first + kWavesT - 1) / kWavesT : 0;
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
    // group in three f16 parts, slot 4 kq + g of the product with a key's zero points: a wave for each 16 rows
    auto query = [&](int r) {
      const int t = r / ratio;
      return (const T *)q.data + (a + t) * q.token_stride + (int64_t)(kvh * ratio + r - t * ratio) * q.head_stride;
    };
    auto q_at = [&](int n, int g, int p) { return (halfx8 *)(lds + RING) + ((n * G + g) * QP + p) * 64 + lane; };
    if (wave < NB) {
      const T *src = query(min(r0 + 16 * wave + col, rows - 1));
      octet in[G];
      float top = 0.f;
#pragma unroll
      for (int g = 0; g < G; ++g) in[g] = *(const octet *)(src + 32 * g + 8 * kq);
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, __builtin_fabsf((float)in[g][e]));
      top = col_max(top);
      const int ex = __builtin_bit_cast(int, top) >> 23;          // biased exponent, 0 .. 255
      const int sh = ex == 0 || ex == 255 ? 0 : min(8 + 127 - ex, 126);
      float up = __builtin_bit_cast(float, (uint32_t)(127 + sh) << 23);
      if (kq == 0) mul_of[16 * wave + col] = fmaxf(__builtin_fabsf(scale) * kLog2e / up, 1e-30f);
      up = scale < 0.f ? -up : up;
      halfx4 z = {0, 0, 0, 0};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float s = 0.f;
        halfx8 parts[QP];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x = (float)in[g][e] * up;
          s += x;
#pragma unroll
          for (int p = 0; p < QP; ++p) {
            parts[p][e] = (_Float16)x;
            x -= (float)parts[p][e];
          }
        }
#pragma unroll
        for (int p = 0; p < QP; ++p) *q_at(wave, g, p) = parts[p];
        if constexpr (!kHeldKeys<T>) {
          s = col_sum(s);
          const _Float16 hi = (_Float16)s, lo = (_Float16)(s - (float)hi);
          z[g] = kq == 0 ? hi : kq == 1 ? lo : kq == 2 ? (_Float16)(s - (float)hi - (float)lo) : (_Float16)0;
        }
      }
      if constexpr (!kHeldKeys<T>) sums_of[wave][lane] = z;
    }
    float mx_[NB], l[NB];                                           // reference and sum of a row's weights
    floatx4 o[NB][NT];
    constexpr bool ZS = std::is_same_v<T, float>;
    float zs[NB][ZS ? G : 1] = {};                                  // float32: sum of p (z + 8 s), this lane's keys
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      mx_[n] = -INFINITY;
      l[n] = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[n][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    // the drafts' own keys, a tile of them and 16 rows for each wave, from the last wave on; every load first
    constexpr float kDown = 1.0 / (1ull << (int)kApart<T>);
    uint64_t apart = 0;                                             // lanes of rows `my` whose sums are kDown times as large
    const int my = (kWavesT - 1 - wave) % NB, k0 = (kWavesT - 1 - wave) / NB * kTileKeys;
    if (from == 0 && k0 < m && r0 + 16 * my < rows) {
      const T *kd = (const T *)k.data + a * k.token_stride + kvh * k.head_stride;
      const T *vd = (const T *)v.data + a * v.token_stride + kvh * v.head_stride;
      const int keys = min(m - k0, kTileKeys);
      const int row = min(r0 + 16 * my + col, rows - 1), draft = row / ratio;
      const T *src = query(row);
      T val[NT][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const T *x = vd + min(k0 + 4 * kq + (e & 3) + 16 * (e >> 2), m - 1) * v.token_stride + col;
#pragma unroll
        for (int t = 0; t < NT; ++t) val[t][e] = x[16 * t];
      }
      floatx4 s[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const T *key = kd + min(k0 + 16 * b + col, m - 1) * k.token_stride;
        s[b] = floatx4{0.f, 0.f, 0.f, 0.f};
        if constexpr (ZS) {
#pragma unroll
          for (int ch = 0; ch < D / 16; ++ch) {
            const floatx4 kk = *(const floatx4 *)(key + 16 * ch + 4 * kq), qq = *(const floatx4 *)(src + 16 * ch + 4 * kq);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[e], qq[e], s[b], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const octet kk = *(const octet *)(key + 32 * g + 8 * kq), qq = *(const octet *)(src + 32 * g + 8 * kq);
            if constexpr (std::is_same_v<T, _Float16>) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk, qq, s[b], 0, 0, 0);
            else s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qq, s[b], 0, 0, 0);
          }
        }
      }
      const uint64_t mine = ancestors(parent + a, m);
      const uint32_t lo = __shfl((uint32_t)mine, draft), hi = __shfl((uint32_t)(mine >> 32), draft), seen = k0 ? hi : lo;
      // the values' sizes by key, and whether there are infinities or NaN, which take no part in the products
      constexpr bool BIG = !std::is_same_v<T, _Float16>;
      float top[BIG ? 8 : 1] = {}, check = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float f = (float)val[t][e];
          check = fmaf(f, 0.f, check);
          if constexpr (BIG) top[e] = fmaxf(top[e], __builtin_fabsf(f));
        }
      const bool odd = __any(check != 0.f);
      if (odd) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 8; ++e) val[t][e] = __builtin_fabsf((float)val[t][e]) < INFINITY ? val[t][e] : (T)0;
      }
      const float by = scale * kLog2e;
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = seen >> (16 * (e >> 2) + 4 * kq + (e & 3)) & 1 ? s[e >> 2][e & 3] * by : -INFINITY;
        s[e >> 2][e & 3] = x;
        mx = fmaxf(mx, x);
      }
      mx = col_max(mx);
      float ref = mx - kTopTree<T>;
      if constexpr (BIG) {
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, top[e]);
        if (__any(most > 0x1p90f)) {
          // (a large value of no weight leaves its rows as they are)
          float far = -INFINITY;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float x = top[e] < INFINITY ? top[e] : 0x1.fffffep127f;
#pragma unroll
            for (int y = 1; y < 16; y <<= 1) x = fmaxf(x, __shfl_xor(x, y));
            far = fmaxf(far, __builtin_log2f(x) + (s[e >> 2][e & 3] - mx));
          }
          far = col_max(far);
          if constexpr (kApartSums<T>) apart = __ballot(far > 100.f);
          else if (far > 100.f) ref += kApart<T>;
        }
      }
      float p[8], sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f(s[e >> 2][e & 3] - (ref == -INFINITY ? 0.f : ref));
        sum += p[e];
      }
      if (kApartSums<T> && apart) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] *= apart >> lane & 1 ? kDown : 1.f;
      }
      floatx4 od[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        od[t] = floatx4{0.f, 0.f, 0.f, 0.f};
        if constexpr (ZS) {
#pragma unroll
          for (int e = 0; e < 8; ++e) od[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(val[t][e], p[e], od[t], 0, 0, 0);
        } else {                                                    // 16-bit weights in two parts
          octet vv, hi8, lo8;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            vv[e] = val[t][e];
            hi8[e] = (T)p[e];
            lo8[e] = (T)(p[e] - (float)hi8[e]);
          }
          if constexpr (std::is_same_v<T, _Float16>) {
            od[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, hi8, od[t], 0, 0, 0);
            od[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, lo8, od[t], 0, 0, 0);
          } else {
            od[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, hi8, od[t], 0, 0, 0);
            od[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, lo8, od[t], 0, 0, 0);
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
              if (!(__builtin_fabsf(x) < INFINITY) && (seen >> key & 1)) od[t][r] += x;
            }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
        if (n == my) {
          mx_[n] = ref;
          l[n] = sum;
#pragma unroll
          for (int t = 0; t < NT; ++t) o[n][t] = od[t];
        }
    }
    __syncthreads();                                              // the queries' operands
    halfx8 qr[QL ? 1 : NB][G][QP];
    halfx4 qz[NB];
    float mul[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      mul[n] = mul_of[16 * n + col];
      if constexpr (!kHeldKeys<T>) qz[n] = sums_of[n][lane];
      if constexpr (!QL)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int p = 0; p < QP; ++p) qr[n][g][p] = *q_at(n, g, p);
    }
    const CodeMasks masks;

    auto rescale = [&](int n, float to) {
      const float f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mx_[n] - to);
      // an infinity or NaN stays one where its weight comes to 0, and finite values come to less than 2^-72
      const float f1 = f == 0.f ? 0x1p-100f : f, f2 = f == 0.f ? 0x1p-100f : 1.f;
      mx_[n] = to;
      l[n] *= f;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[n][t] = o[n][t] * f1 * f2;
#pragma unroll
      for (int g = 0; g < (ZS ? G : 1); ++g) zs[n][g] *= f;
    };

    int next = page[kStagesT - 1];
    for (int x = 0; x < n_tiles; ++x) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // the reads of the slot that is loaded next
      const int ahead = min(kStagesT - 1, n_tiles - 1 - x);         // tiles issued after this one
      if (x + kStagesT - 1 < n_tiles) {
        issue(x + kStagesT - 1, next);
        next = page_of(x + kStagesT);
      }
      static_assert(kStagesT <= 3, "a wait for every number of tiles behind this one");
      if (ahead >= 2) wait_loads<2 * NL>();
      else if (ahead == 1) wait_loads<NL>();
      else wait_loads<0>();
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
      halfx4 kz[2] = {};
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        halfx8 middle = {};                                         // float32: z + 8 s in two parts
#pragma unroll
        for (int g = 0; g < G; ++g) {
          kz[b][g] = half[k_zero(G, g, 16 * b + col)];
          if constexpr (ZS) {
            const float y = fmaf(8.f, (float)half[k_scale(G, g, 16 * b + col)], (float)kz[b][g]);
            middle[g] = (_Float16)y;
            middle[4 + g] = (_Float16)(y - (float)middle[g]);
          }
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          s[n][b] = floatx4{0.f, 0.f, 0.f, 0.f};
          if constexpr (!kHeldKeys<T> && !ZS) s[n][b] = __builtin_amdgcn_mfma_f32_16x16x16f16(kz[b], qz[n], s[n][b], 0, 0, 0);
          if constexpr (ZS)
            s[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(middle, __builtin_shufflevector(qz[n], qz[n], 0, 1, 2, 3, 4, 5, 6, 7), s[n][b], 0, 0, 0);
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        halfx8 kc[2];
        halfx4 ks[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          kc[b] = masks.template codes<ZS ? 8 : 0>(tile[(b * 64 + lane) * G + g]);
          if constexpr (kHeldKeys<T>) kc[b] = kc[b] * half[k_scale(G, g, 16 * b + col)] + kz[b][g];
          else ks[b] = *(const halfx4 *)(half + k_scale(G, g, 16 * b + 4 * kq));
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          halfx8 qq[QP];
#pragma unroll
          for (int p = 0; p < QP; ++p) qq[p] = QL ? *q_at(n, g, p) : qr[QL ? 0 : n][g][p];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            floatx4 y = kHeldKeys<T> ? s[n][b] : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < QP; ++p) y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kc[b], qq[p], y, 0, 0, 0);
            if constexpr (kHeldKeys<T>) s[n][b] = y;
            else
#pragma unroll
              for (int r = 0; r < 4; ++r) s[n][b][r] = fmaf((float)ks[b][r], y[r], s[n][b][r]);
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
      float p[ZS ? NB : 1][8];                                      // float32: the weights themselves
      halfx8 ph[ZS ? 1 : NB], pl[std::is_same_v<T, _Float16> ? NB : 1];
      float mx[NB];
      bool far = false;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        mx[n] = s[n][0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx[n] = fmaxf(mx[n], s[n][e >> 2][e & 3]);
        mx[n] *= mul[n];
        far |= mx[n] > mx_[n] + kFarTree<T>;
      }
      if (__any(far) || apart) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {                              // each row by its own scores alone
          const float rm = col_max(mx[n]);
          rescale(n, rm > mx_[n] + kFarTree<T> ? rm - kTopTree<T> : mx_[n]);
        }
        if (kApartSums<T> && apart) {                               // products by themselves, no weight in those below
          halfx8 pa = {};
#pragma unroll
          for (int n = 0; n < NB; ++n)
            if (n == my) {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float y = s[n][e >> 2][e & 3];
                const float x = apart >> lane & 1 ? __builtin_amdgcn_exp2f(fmaf(y, mul[n], -mx_[n])) : 0.f;
                l[n] += x;
                pa[e] = (_Float16)x;
                s[n][e >> 2][e & 3] = apart >> lane & 1 ? -INFINITY : y;
              }
            }
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            asm volatile("" ::: "memory");                          // one after the other: few registers
            const halfx8 vs = *(const halfx8 *)(tile + v_param(G, t / 2, kq)), vz = *(const halfx8 *)(tile + v_param(G, t / 2, kq) + 4);
            const halfx8 vv = masks.codes(tile[128 * G + (t / VW * 64 + lane) * VW + t % VW]) * vs + vz;
            const floatx4 y = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, pa, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int n = 0; n < NB; ++n)
              if (n == my) o[n][t] += y * kDown;
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float mu = mx_[n] == -INFINITY ? 0.f : mx_[n];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[n][e >> 2][e & 3], mul[n], -mu));
          l[n] += x;
          if constexpr (ZS) p[n][e] = x;
          else ph[n][e] = (_Float16)x;
          if constexpr (std::is_same_v<T, _Float16>) pl[n][e] = (_Float16)(x - (float)ph[n][e]);
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const halfx8 vs = *(const halfx8 *)(tile + v_param(G, g, kq)), vz = *(const halfx8 *)(tile + v_param(G, g, kq) + 4);
        bfx8 pp[ZS ? NB : 1][3];
        if constexpr (ZS) {
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              zs[n][g] = fmaf(p[n][e], fmaf(8.f, (float)vs[e], (float)vz[e]), zs[n][g]);
              float y = p[n][e] * (float)vs[e];
#pragma unroll
              for (int k2 = 0; k2 < 3; ++k2) {
                pp[n][k2][e] = (__bf16)y;
                y -= (float)pp[n][k2][e];
              }
            }
        }
#pragma unroll
        for (int t = 2 * g; t < 2 * g + 2; ++t) {
          const uint32_t w = tile[128 * G + (t / VW * 64 + lane) * VW + t % VW];
          if constexpr (ZS) {
            bfx8 vc;
#pragma unroll
            for (int e = 0; e < 8; ++e) vc[e] = (__bf16)(float)((int)((w ^ 0x88888888u) << (28 - nibble_shift(e))) >> 28);      // c - 8
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
              for (int k2 = 0; k2 < 3; ++k2) o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vc, pp[n][k2], o[n][t], 0, 0, 0);
          } else if constexpr (std::is_same_v<T, _Float16>) {
            const halfx8 vc = masks.codes(w);
            halfx8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float y = fmaf((float)vc[e], (float)vs[e], (float)vz[e]);      // exact but for the sum's last bit
              hi[e] = (_Float16)y;
              lo[e] = (_Float16)(y - (float)hi[e]);
            }
#pragma unroll
            for (int n = 0; n < NB; ++n) {
              o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, ph[n], o[n][t], 0, 0, 0);
              o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, pl[n], o[n][t], 0, 0, 0);
              o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, ph[n], o[n][t], 0, 0, 0);
            }
          } else {
            const halfx8 vv = masks.codes(w) * vs + vz;
#pragma unroll
            for (int n = 0; n < NB; ++n) o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, ph[n], o[n][t], 0, 0, 0);
          }
        }
      }
    }
    if (kApartSums<T> && apart) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
        if (n == my && (apart >> lane & 1)) {
          l[n] *= kDown;
          mx_[n] += kApart<T>;
        }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {                                  // o[n][t][r] is value 16 t + 4 kq + r of row col
      l[n] = col_sum(l[n]);
      if constexpr (ZS) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float z = col_sum(zs[n][g]);
          o[n][2 * g] += z;
          o[n][2 * g + 1] += z;
        }
      }
    }

    // join the waves, 16 rows at a time
    __syncthreads();                                                // the rings are done with
    auto *red_o = (floatx4(*)[kCols][D / 4 + 1])lds;
    auto *red_l = (float(*)[kCols])(lds + RO);
    auto *red_m = (float(*)[W])(lds + RO + kWavesT * kCols * 4);
    if (kq == 0) {
#pragma unroll
      for (int n = 0; n < NB; ++n) red_m[wave][16 * n + col] = mx_[n];
    }
#pragma unroll 1
    for (int n = 0; r0 + 16 * n < rows && n < NB; ++n) {
      __syncthreads();                                              // red_m, and the rows before
#pragma unroll
      for (int x = 0; x < NB; ++x)
        if (x == n) {
          float mm = mx_[x];
#pragma unroll
          for (int w = 0; w < kWavesT; ++w) mm = fmaxf(mm, red_m[w][16 * x + col]);
          const float f = mm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx_[x] - mm);
          const float f1 = f == 0.f ? 0x1p-100f : f, f2 = f == 0.f ? 0x1p-100f : 1.f;      // as in rescale
          if (kq == 0) red_l[wave][col] = l[x] * f;
#pragma unroll
          for (int t = 0; t < NT; ++t) red_o[wave][col][4 * t + kq] = o[x][t] * f1 * f2;
        }
      __syncthreads();
      const int h = threadIdx.x / (D / 4), d4 = threadIdx.x % (D / 4), r = r0 + 16 * n + h;
      if (h < kCols && r < rows) {
        const int t = r / ratio, head = kvh * ratio + r - t * ratio;
        float ll = 0.f, top = -INFINITY;
        floatx4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWavesT; ++w) {
          top = fmaxf(top, red_m[w][16 * n + h]);
          ll += red_l[w][h];
          y += red_o[w][h][d4];
        }
        if (slot >= 0) {
          const int64_t to = slot * W + 16 * n + h;
          *(floatx4 *)(part + to * D + 4 * d4) = y;
          if (d4 == 0) *(float2 *)(part + 2 * (int64_t)gridDim.x * W * D + to * 2) = float2{top, ll};
        } else {
          struct alignas(4 * sizeof(T)) { T v[4]; } z;
#pragma unroll
          for (int e = 0; e < 4; ++e) z.v[e] = mean_odd<T>(y[e], ll);
          *(decltype(z) *)((T *)out.data + (a + t) * out.token_stride + (int64_t)head * out.head_stride + 4 * d4) = z;
          if (lse && d4 == 0) lse[(int64_t)head * q.tokens + a + t] = (top + __builtin_log2f(ll)) * kLn2;
        }
      }
    }
    __syncthreads();                                                // before the ring is filled again
    left -= part ? steps : 1;
    at += steps;
    ++turn;
  }
}

// One row by TPR threads, 256 / TPR rows a workgroup: four values a thread, the parts spread over the threads; every sum
// in a fixed order.
template <class T, int G, int TPR>
__global__ __launch_bounds__(256) void attn_tree_join_kernel(int heads, int ratio, int seqs_n, int most, int w,
                                                             int64_t parts, ios_tokens out, float *lse, const int32_t *cu,
                                                             const float *part) {
  constexpr int D = 32 * G, Q = D / 4, N = TPR / Q;               // N threads share four values
  __shared__ floatx4 sum[TPR > 64 ? N : 1][Q];
  __shared__ float red[2][4];
  const int64_t row = (int64_t)blockIdx.x * (256 / TPR) + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  const int64_t t = row / heads;
  if (t >= out.tokens) return;
  const int h = (int)(row % heads), tid = threadIdx.x % TPR, lane = threadIdx.x & 63;
  const int i = find_owner(seqs_n, t, [&](int x) { return clip(cu[x], out.tokens); });
  const int64_t a = clip(cu[i], out.tokens), b = clip(cu[i + 1], out.tokens);
  if (t < a || t >= b || t >= a + most) return;                   // a row of no sequence, or past the last draft
  const int r = (int)(t - a) * ratio + h % ratio, r0 = r / w * w;
  const PartRef ref = ((const PartRef *)(part + parts * w * (D + 2)))[(a + r0 / ratio) * heads + h / ratio * ratio + r0 % ratio];
  if (ref.count <= 1) return;                                     // its workgroup has written it
  auto place = [&](int x) { return (int64_t)(x == 0 ? ref.first : (ref.first & ~1) + 2 * x) * w + (r - r0); };
  const float2 *ml = (const float2 *)(part + parts * w * D);
  const int d4 = tid % Q, n = tid / Q, mine = n < N ? ref.count : 0;
  floatx4 z[2];                                                   // the first values beside the references
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (n + u * N < mine) z[u] = *(const floatx4 *)(part + place(n + u * N) * D + 4 * d4);
  float top = -INFINITY, ll = 0.f;
  for (int x = tid; x < ref.count; x += TPR) top = fmaxf(top, ml[place(x)].x);
#pragma unroll
  for (int y = 1; y < 64; y <<= 1) top = fmaxf(top, __shfl_xor(top, y));
  if constexpr (TPR > 64) {
    if (lane == 0) red[0][threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  }
  const float mu = top == -INFINITY ? 0.f : top;
  for (int x = tid; x < ref.count; x += TPR) {
    const float2 y = ml[place(x)];
    ll += __builtin_amdgcn_exp2f(y.x - mu) * y.y;
  }
#pragma unroll
  for (int y = 1; y < 64; y <<= 1) ll += __shfl_xor(ll, y);
  if constexpr (TPR > 64) {
    if (lane == 0) red[1][threadIdx.x >> 6] = ll;
    __syncthreads();
    ll = red[1][0] + red[1][1] + red[1][2] + red[1][3];
  }
  floatx4 y = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](int x, const floatx4 &v) {
    const float f = __builtin_amdgcn_exp2f(ml[place(x)].x - mu);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += weighed(v[e], f);
  };
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (n + u * N < mine) add(n + u * N, z[u]);
#pragma unroll 4
  for (int x = n + 2 * N; x < mine; x += N) add(x, *(const floatx4 *)(part + place(x) * D + 4 * d4));
  if constexpr (TPR > 64) {
    if (n < N) sum[n][d4] = y;
    __syncthreads();
    if (tid < Q)
#pragma unroll
      for (int x = 1; x < N; ++x) y += sum[x][d4];
  } else {
    floatx4 all = y;
#pragma unroll
    for (int x = 1; x < N; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) all[e] += __shfl(y[e], (lane + x * Q) & 63);
    y = all;
  }
  if (tid < Q) {
    struct alignas(4 * sizeof(T)) { T v[4]; } z;
#pragma unroll
    for (int e = 0; e < 4; ++e) z.v[e] = mean_odd<T>(y[e], ll);
    *(decltype(z) *)((T *)out.data + t * out.token_stride + h * out.head_stride + 4 * tid) = z;
  }
  if (lse && tid == 0) lse[h * out.tokens + t] = (top + __builtin_log2f(ll)) * kLn2;
}

int64_t keys_of(const ios_attn_desc &d) { return d.max_keys ? d.max_keys : 1 << 16; }

// Steps of the whole call at most, with blocks of w rows: no more blocks have rows than every sequence's most, nor than all
// rows make.
int64_t steps_of(const ios_attn_desc &d, int64_t q_tokens, int most, int w) {
  const int ratio = d.heads / d.kv_heads;
  const int64_t blocks = std::min<int64_t>((int64_t)d.seqs * ((most * ratio + w - 1) / w), q_tokens * ratio / w + d.seqs);
  return d.kv_heads * blocks * (kItemSteps + (keys_of(d) + kStepTiles * kTileKeys - 1) / (kStepTiles * kTileKeys));
}

// 16-row groups of a block.  Four read the cache once for 64 rows, but each wave then begins and ends with twice the work of
// two: 32 sequences under 64 rows each 286 us against 370 (bf16; f16 530 against 578), one under 256 rows 76 against 78.5
// (f16 121 against 122), but maps of 1 to 3100 tokens 32.3 against 25.9 (f16 38.6 against 31.0).  So four where every workgroup
// has 12 steps; float32's three parts of the queries and weights leave registers for two.
int row_groups(const ios_attn_desc &d, int64_t q_tokens, int most) {
  const int rows = most * (d.heads / d.kv_heads);
  if (rows <= 16) return 1;
  return rows <= 32 || d.dtype == IOS_F32 || steps_of(d, q_tokens, most, 64) < 12 * 256 ? 2 : 4;
}

struct Call {
  CacheView c;
  const ios_attn_desc *d;
  ios_tokens q, k, v, out;
  float *lse;
  const int32_t *seqs, *cu, *parent;
  int most, groups;
  float *part;
  hipStream_t s;
};

template <class T, int G, int NB>
hipError_t run(const Call &x) {
  const ios_attn_desc &d = *x.d;
  constexpr int W = 16 * NB;
  const int ratio = d.heads / d.kv_heads;
  const dim3 grid = x.groups ? dim3(x.groups) : dim3(d.kv_heads * ((x.most * ratio + W - 1) / W), d.seqs);
  hipLaunchKernelGGL((attn_tree_kernel<T, G, NB>), grid, dim3(kThreadsT), 0, x.s, x.c, d.heads, ratio, d.scale, x.q, x.k, x.v,
                     x.out, x.lse, x.seqs, x.cu, x.parent, d.seqs, x.most, x.groups ? x.part : nullptr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !x.groups) return e;
  const int64_t rows = x.q.tokens * d.heads, parts = 2 * (int64_t)x.groups;
  // A wave for each row where it has few parts (a wave and a workgroup each: the maps in bf16 25.9 and 29.9 us, 32 long
  // sequences 284 and 299, but one of 131072 tokens under a single draft 28.3 and 23.5); always from 2048 rows on.
  if (parts * W <= 16 * rows)
    hipLaunchKernelGGL((attn_tree_join_kernel<T, G, 64>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, x.s, d.heads, ratio,
                       d.seqs, x.most, W, parts, x.out, x.lse, x.cu, x.part);
  else
    hipLaunchKernelGGL((attn_tree_join_kernel<T, G, 256>), dim3((unsigned)rows), dim3(256), 0, x.s, d.heads, ratio, d.seqs,
                       x.most, W, parts, x.out, x.lse, x.cu, x.part);
  return hipGetLastError();
}

template <class T, int G>
hipError_t for_blocks(const Call &x) {
  switch (row_groups(*x.d, x.q.tokens, x.most)) {
    case 1: return run<T, G, 1>(x);
    case 2: return run<T, G, 2>(x);
    default:
      if constexpr (std::is_same_v<T, float>) return run<T, G, 2>(x);
      else return run<T, G, 4>(x);
  }
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

// Workgroups that share the keys, one a CU at most (0: each takes a block of rows with all of its keys).
int groups_of(const ios_attn_desc &d, int64_t q_tokens, int most) {
  if (keys_of(d) < kOneTree) return 0;
  const int64_t steps = steps_of(d, q_tokens, most, 16 * row_groups(d, q_tokens, most));
  return (int)std::min<int64_t>(256, (steps + kShareSteps - 1) / kShareSteps);
}

}  // namespace

int64_t tree_bytes(const ios_attn_desc &d, int64_t q_tokens, int most) {
  const int64_t groups = groups_of(d, q_tokens, most), w = 16 * row_groups(d, q_tokens, most);
  return groups ? 2 * groups * w * (d.head_dim + 2) * (int64_t)sizeof(float) + q_tokens * d.heads * (int64_t)sizeof(PartRef) : 0;
}

hipError_t launch_attn_tree(const CacheView &c, const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &k,
                            const ios_tokens &v, const ios_tokens &out, float *lse, const int32_t *seqs,
                            const int32_t *cu, const int32_t *parent, int most, void *work, hipStream_t s) {
  const Call x{c, &d, q, k, v, out, lse, seqs, cu, parent, most, work ? groups_of(d, q.tokens, most) : 0, (float *)work, s};
  if (d.dtype == IOS_F32) return for_groups<float>(x);
  if (d.dtype == IOS_F16) return for_groups<_Float16>(x);
  return for_groups<__bf16>(x);
}

}  // namespace ios
