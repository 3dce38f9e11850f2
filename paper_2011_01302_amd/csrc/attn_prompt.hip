// Attention over packed prompts in f16 and bf16 (ios_attn_prompt).
//
// A workgroup takes 128 queries of one head, 32 a wave, and walks the keys they
// see in tiles of 64, keeping the running maximum and sum of the softmax and
// the output in registers; the scores never leave them.  Both products are
// computed transposed, S^T = K Q^T and O^T = V^T P^T, on
// v_mfma_f32_32x32x16: a lane then holds one query's scores, its statistics
// need one exchange between the two half waves, and the scores are the second
// product's operand as they stand (keys 8 i + 4 h + 0 .. 3 of a tile lie in
// half h; V is read in that order).
//
// Bound by power for heads of 96 and 128 (16384 causal tokens, 32 heads of 128:
// 1.97 ms, 1120 TFLOP/s at 1.73 GHz, matrix cores 56 and vector units 51 per
// cent busy; a large matrix product of the library reaches 1130 .. 1220 at 1.72),
// by the exponentials and the other vector instructions of the softmax for
// smaller heads (4096 causal tokens, 16 heads of 64: 61 us, 560 TFLOP/s), by its
// longest rows where prompts of different lengths are packed.
#include <type_traits>

#include "attn_prompt.h"

namespace ios {

namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

constexpr int kBM = kRows, kBN = kKeys;
// Fewer than kFewBlocks workgroups: the keys of a row are spread over workgroups (a second launch joins them), in parts
// of at least kPartKeys keys (32 heads of 128 over 6000 keys: 256 rows, 96 workgroups, 65 us, 90 in one part; 512 rows,
// 160 workgroups, 105 and 92; 1 row 18.8 us).  Up to kTwoGroups workgroups, and from kTwoKeys keys on: over two groups of
// waves of one workgroup (16 heads of 64, 2048 causal tokens, 272 workgroups: 27.5 us, 32.3 with one group; 32 heads of
// 128, 288 workgroups: 27.7 and 28.6, 416: 40.2 and 41.2, 544: 58.1 and 54.3).
constexpr int kFewBlocks = 129, kPartKeys = 256, kTwoGroups = 320, kTwoKeys = 1024;
// p = 2^(score - m), m kTop below the row's largest score when it was last followed, which it is when a score passes it
// by kTop + 2 (sums are in 32 bits).  f16 then holds p from 2^15 down to 2^-38 of the largest.
template <class T> constexpr float kTop = std::is_same_v<T, _Float16> ? 13.f : 0.f;

template <class T>
__device__ __forceinline__ floatx16 mfma(shortx8 a, shortx8 b, floatx16 c) {
  if constexpr (std::is_same_v<T, _Float16>)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bfx8, a), __builtin_bit_cast(bfx8, b), c, 0, 0, 0);
}

// 16-byte chunk c of row r of a tile in LDS is stored at chunk c ^ swz(r), so
// that the reads below spread over the banks: K rows are read 16 at a time
// at one chunk, V four rows at a time at four chunks.
template <int DP>
__device__ __forceinline__ int swz_k(int r) {
  return DP == 128 ? r & 15 : DP == 64 ? r >> 1 & 7 : r >> 2 & 3;
}
template <int DP>
__device__ __forceinline__ int swz_v(int r) {
  return DP == 128 ? 4 * (r & 3) : DP == 64 ? 4 * (r >> 1 & 1) : 0;
}

// Direct global -> LDS load of 16 bytes a lane, l the same for every lane
// (readers wait for vmcnt(0) and a barrier).
__device__ __forceinline__ void lds_copy16(__amdgpu_buffer_rsrc_t r, unsigned char *l, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)l, 16, (int)off, 0, 0, 0);
}


// The two halves of a wave hold different keys of the same queries: this
// lane's value and the other half's.  (The swap exchanges two registers; given
// one twice it would exchange it with itself, hence the copy.)
__device__ __forceinline__ float other_half(float v) {
  int a = __builtin_bit_cast(int, v), b = a;
  asm("" : "+v"(b));
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return __builtin_bit_cast(float, threadIdx.x & 32 ? r[0] : r[1]);
}

// KG groups of four waves take the tiles in turn and are joined at the end.
template <class T, int DP, int KG>
__global__ __launch_bounds__(256 * KG, 2) void attn_prompt_kernel(PromptArgs a) {
  constexpr int CH = DP / 8, KS = DP / 16, DB = DP / 32, LOADS = kBN * CH / 256;
  // the only array in LDS: with a second one the compiler tells them apart, and waits for every copy in flight before
  // it reads from either
  __shared__ __align__(16) unsigned char stage[KG][2][2][kBN * DP * 2];   // [group][buffer][K, V]
  const int tid = threadIdx.x & 255, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  auto &lds = stage[group];
  const int half = lane >> 5, l31 = lane & 31, l15 = lane & 15;

  int head, seq;
  int64_t first_query;
  if (!prompt_block(a, &head, &seq, &first_query)) return;
  const int64_t qa = clip(a.cu_q[seq], a.q.tokens), ka = clip(a.cu_k[seq], a.k.tokens);
  const int lq = (int)(clip(a.cu_q[seq + 1], a.q.tokens) - qa);
  const int lk = max((int)(clip(a.cu_k[seq + 1], a.k.tokens) - ka), 0);
  if (first_query >= lq) return;
  const int q0 = (int)first_query, r0 = q0 + 32 * wave;
  const int kvh = head / a.ratio;

  // last key that a row sees (-1: none); rows past the sequence see what its last row sees
  const int64_t diff = (int64_t)lk - lq;
  auto last_key = [&](int row) { return a.causal ? (int)min((int64_t)min(row, lq - 1) + diff, (int64_t)lk - 1) : lk - 1; };
  const int lim = max(last_key(r0 + l31), -1);
  const int lim_lo = last_key(r0), lim_hi = r0 < lq ? last_key(r0 + 31) : -1;   // waves past the sequence sit out
  int tiles = max(last_key(q0 + kBM - 1) + kBN, 0) / kBN;
  const int split = blockIdx.z, t0 = split * a.chunk;
  if (a.part) {
    if (split > 0 && t0 >= tiles) return;
    if (split + 1 < (int)gridDim.z) tiles = min(tiles, t0 + a.chunk);
  }

  // queries, the sign of the scale folded in
  shortx8 qf[KS];
  const float mul = multiplier(a.scale);
  {
    const T *src = (const T *)a.q.data + (qa + min(r0 + l31, lq - 1)) * a.q.token_stride + head * a.q.head_stride;
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = 16 * s + 8 * half;
      uintx4 w = {0, 0, 0, 0};
      if (d < a.dim) w = *(const uintx4 *)(src + d);
      qf[s] = __builtin_bit_cast(shortx8, w ^ flip);
    }
  }

  // what this thread copies of a tile: rows and byte offsets of its chunks
  uint32_t koff[LOADS], voff[LOADS];
  int row_of[LOADS];
#pragma unroll
  for (int p = 0; p < LOADS; ++p) {
    const int s = p * 256 + tid, r = s / CH, pos = s % CH;
    row_of[p] = r;
    const int kc = pos ^ swz_k<DP>(r), vc = pos ^ swz_v<DP>(r);
    koff[p] = kc * 8 < a.dim ? (uint32_t)(r * (int)a.k.token_stride + kc * 8) * 2 : kOutside;
    voff[p] = vc * 8 < a.dim ? (uint32_t)(r * (int)a.v.token_stride + vc * 8) * 2 : kOutside;
  }
  const T *kbase = (const T *)a.k.data + ka * a.k.token_stride + kvh * a.k.head_stride;
  const T *vbase = (const T *)a.v.data + ka * a.v.token_stride + kvh * a.v.head_stride;
  auto issue = [&](const T *base, int64_t stride, const uint32_t *off, int t, unsigned char *to) {
    const __amdgpu_buffer_rsrc_t r = buffer(base + (int64_t)t * kBN * stride);
    const int left = lk - t * kBN;                           // rows past the sequence's last key read as 0
#pragma unroll
    for (int p = 0; p < LOADS; ++p)
      lds_copy16(r, to + (p * 256 + wave * 64) * 16, row_of[p] < left ? off[p] : kOutside);
  };
  auto issue_k = [&](int t, int buf) { issue(kbase, a.k.token_stride, koff, t, lds[buf][0]); };
  auto issue_v = [&](int t, int buf) { issue(vbase, a.v.token_stride, voff, t, lds[buf][1]); };

  float m, l;
  floatx16 o[DB];
  const floatx16 zero = {};

  // scores of a tile, transposed: keys 32 b + (r & 3) + 8 (r >> 2) + 4 half of query l31
  auto scores = [&](const unsigned char *sk, floatx16 *s, int lane) {
    const int half = lane >> 5, l31 = lane & 31;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s[b] = zero;
      const int r = 32 * b + l31;
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        const shortx8 kf = *(const shortx8 *)(sk + r * (CH * 16) + ((2 * i + half) ^ swz_k<DP>(r)) * 16);
        s[b] = mfma<T>(kf, qf[i], s[b]);
      }
    }
  };
  auto hide = [&](int t, floatx16 *s, int half, int lim) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (t * kBN + 32 * b + (r & 3) + 8 * (r >> 2) + 4 * half > lim) s[b][r] = -INFINITY;
  };
  auto largest = [&](const floatx16 *s) {
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
    return mx;
  };
  // follow the rows' maxima where they have grown, each row by its own scores alone, so that no row's result depends on
  // another's; in the walk with care o may hold infinities and NaN
  auto follow = [&](float mx, auto care) {
    mx *= mul;
    if (__any(mx > m + (kTop<T> + 2.f))) {
      const float rm = fmaxf(mx, other_half(mx)), mn = rm > m + (kTop<T> + 2.f) ? rm - kTop<T> : m;
      const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        if constexpr (decltype(care)::value) {
#pragma unroll
          for (int r = 0; r < 16; ++r) o[i][r] = weighed(o[i][r], f);
        } else {
          o[i] *= f;
        }
      }
    }
  };
  auto weights = [&](const floatx16 *s, shortx8 *pf, float by) {
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[b][r], mul, -mu));
        l += e;
        pf[2 * b + (r >> 3)][r & 7] = __builtin_bit_cast(short, (T)(e * by));  // p as the inputs' type: 2^-9 (2^-12) each
      }
  };
  auto values = [&](const unsigned char *sv, int i, int ks, int lane) {
    const int half = lane >> 5, l15 = lane & 15;
    const int r = 16 * ks + 4 * half + (l15 >> 2), c = 4 * i + 2 * (lane >> 4 & 1) + ((l15 & 3) >> 1);
    const unsigned char *p = sv + r * (CH * 16) + (c ^ swz_v<DP>(r)) * 16 + 8 * (l15 & 1);
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)p);
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(p + 8 * CH * 16));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto clear = [&] {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = zero;
  };
  // this wave's loads have landed, and every wave is done with what they replace
  auto arrived = [] {
    __builtin_amdgcn_s_waitcnt(0x0070);                      // vmcnt = lgkmcnt = 0
    asm volatile("s_barrier" ::: "memory");
  };
  auto masked = [&](int t) { return t * kBN + kBN - 1 > lim_lo; };

  // The walk over the keys.  A wave issues a product every 32 cycles at most, and the vector units are free between:
  // the next tile's scores are computed while this tile's become weights, this tile's output while the next one's
  // maxima are looked for.  The compiler keeps that order (it would do one after the other).
  typedef const __attribute__((address_space(3))) shortx8 lds_shortx8;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)&lds[0][0][0];
  const uint32_t klane = lds0 + l31 * (CH * 16) + (half ^ swz_k<DP>(l31)) * 16;
  const int vrow = 4 * half + (l15 >> 2), vchunk = 2 * (lane >> 4 & 1) + ((l15 & 3) >> 1);
  const uint32_t vlane = lds0 + kBN * DP * 2 + vrow * (CH * 16) + (vchunk ^ swz_v<DP>(vrow)) * 16 + 8 * (l15 & 1);
  constexpr uint32_t kBuffer = 2 * kBN * DP * 2;
  // operand c of K Q^T: values 16 (c / 2) .. + 15 of keys 32 (c % 2) .. + 31
  auto k_operand = [&](uint32_t base, int c) {
    constexpr int flip = DP == 128 ? 7 : DP == 64 ? 3 : 1;      // the chunk bits that the swizzle covers
    const int i = c >> 1;
    return *(lds_shortx8 *)(uintptr_t)((base ^ ((i & flip) << 5)) + ((i & ~flip) << 5) + (c & 1) * 32 * CH * 16);
  };
  // operand c of V^T P^T: values 32 (c % DB) .. + 31 of keys 16 (c / DB) .. + 15
  auto v_operand = [&](uint32_t base, int c) {
    const int i = c % DB, ks = c / DB;
    const uint32_t p = (DP == 96 ? base + (i << 6) : base ^ (i << 6)) + ks * 16 * CH * 16;
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(uintptr_t)p);
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(uintptr_t)(p + 8 * CH * 16));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  clear();
  {
    const int first = t0 + group;
    // past the last tile that a row of this wave sees there is nothing to do but to load and to wait
    const int end = min(tiles, (lim_hi + kBN) / kBN);
    // tile k of this group, whose scores are s; leaves those of the next in sn
    auto step = [&](int k, floatx16 *s, floatx16 *sn) __attribute__((always_inline)) {
      const int t = first + k * KG, next = t + KG;
      arrived();
      if (next < tiles) issue_v(next, (k + 1) & 1);
      if (next + KG < tiles) issue_k(next + KG, k & 1);
      if (t >= end) return;
      const uint32_t kb = klane + ((k + 1) & 1) * kBuffer, vb = vlane + (k & 1) * kBuffer;
      constexpr int NK = 2 * KS, NV = 4 * DB, AHEAD = 3;
      shortx8 f[AHEAD + 1], pf[4];
      const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int c = 0; c < AHEAD; ++c) f[c] = k_operand(kb, c);
#pragma unroll
      for (int c = 0; c < NK; ++c) {                         // scores of no tile, and not used, after the last one
        if (c + AHEAD < NK) f[(c + AHEAD) % (AHEAD + 1)] = k_operand(kb, c + AHEAD);
        else f[(c + AHEAD) % (AHEAD + 1)] = v_operand(vb, c + AHEAD - NK);
        sn[c & 1] = mfma<T>(f[c % (AHEAD + 1)], qf[c >> 1], c < 2 ? zero : sn[c & 1]);
#pragma unroll
        for (int x = c * 32 / NK; x < (c + 1) * 32 / NK; ++x) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[x >> 4][x & 15], mul, -mu));
          l += e;
          pf[x >> 3][x & 7] = __builtin_bit_cast(short, (T)e);                // p as the inputs' type: 2^-9 (2^-12) each
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        if (c + AHEAD < NV) f[(c + NK + AHEAD) % (AHEAD + 1)] = v_operand(vb, c + AHEAD);
        o[c % DB] = mfma<T>(f[(c + NK) % (AHEAD + 1)], pf[c / DB], o[c % DB]);
#pragma unroll
        for (int x = c * 32 / NV; x < (c + 1) * 32 / NV; ++x) mx = fmaxf(mx, sn[x & 1][x >> 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (next < end) {
        if (masked(next)) {
          hide(next, sn, half, lim);
          mx = largest(sn);
        }
        follow(mx, std::false_type{});
      }
    };
    floatx16 s[2], sn[2];
    if (first < tiles) issue_k(first, 0);
    arrived();
    if (first < tiles) issue_v(first, 0);
    if (first + KG < tiles) issue_k(first + KG, 1);
    if (first < end) {
      scores(lds[0][0], s, lane);
      if (masked(first)) hide(first, s, half, lim);
      follow(largest(s), std::false_type{});
    }
    for (int k = 0; t0 + k * KG < tiles; k += 2) {
      step(k, s, sn);
      if (t0 + (k + 1) * KG < tiles) step(k + 1, sn, s);
    }
  }
  // From here on the lane's place is worked out anew: the walk is short of registers.
  const int ln = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), lnh = ln >> 5;
  const int lim2 = max(last_key(r0 + (ln & 31)), -1);
  // whether any wave of the workgroup found a number that is not finite
  auto odd = [&]() __attribute__((always_inline)) {
    int x = 0;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) x |= !(__builtin_fabsf(o[i][r]) < INFINITY);
    int *found = (int *)stage;
    __syncthreads();                                         // the tiles are done with
    x = __any(x);
    if (ln == 0) found[group * 4 + wave] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4 * KG; ++w) x |= found[w];
    return __builtin_amdgcn_readfirstlane(x);
  };
  // Again, with care: infinities and NaN among the values are kept out of the product (0 times one of them is a NaN, and
  // a weight may come to 0 as well as be hidden) and reach the rows that see them by counts.  And once more if a sum has
  // left float32's range (f16 values stay far below).  (As a loop over both the kernel for heads of 128 spills registers.)
  float up = 1.f;
  const bool again = odd();
  if (again) {
    auto careful = [&](float by) __attribute__((always_inline)) {
      clear();
      for (int k = 0; t0 + k * KG < tiles; ++k) {
        const int t = t0 + k * KG + group;
        __syncthreads();
        if (t < tiles) {
          issue_k(t, 0);
          issue_v(t, 0);
        }
        arrived();
        if (t >= tiles || t * kBN > lim_hi) continue;
        floatx16 s[2];
        shortx8 pf[4];
        scores(lds[0][0], s, ln);
        hide(t, s, lnh, lim2);
        follow(largest(s), std::true_type{});
        weights(s, pf, by);
#pragma unroll
        for (int i = 0; i < DB; ++i) {
          floatx16 above = zero, below = zero;               // infinities of both signs (a NaN is both) that a row sees
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            shortx8 vf = values(lds[0][1], i, ks, ln);
            constexpr int inf = std::is_same_v<T, _Float16> ? 0x7C00 : 0x7F80;
            const short one = __builtin_bit_cast(short, (T)1.f);
            shortx8 va, vb, seen;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int mag = vf[e] & 0x7FFF;
              va[e] = mag > inf || vf[e] == inf ? one : 0;
              vb[e] = mag > inf || (mag == inf && vf[e] < 0) ? one : 0;
              if (mag >= inf) vf[e] = 0;
              seen[e] = t * kBN + 16 * ks + 4 * lnh + (e & 3) + 8 * (e >> 2) <= lim2 ? one : 0;
            }
            above = mfma<T>(va, seen, above);
            below = mfma<T>(vb, seen, below);
            o[i] = mfma<T>(vf, pf[ks], o[i]);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if (above[r] > 0.f) o[i][r] += INFINITY;
            if (below[r] > 0.f) o[i][r] -= INFINITY;
          }
        }
      }
    };
    careful(1.f);
    if constexpr (!std::is_same_v<T, _Float16>) {
      if (odd()) {
        careful(kDown);
        up = kUp;
      }
    }
  }

  l += other_half(l);
  if constexpr (KG > 1) {                                    // the second group's rows go through LDS to the first
    static_assert(KG == 2 && sizeof(stage) >= (4 * DB * 16 * 64 + 512) * 4, "one other group");
    __syncthreads();                                         // the tiles are done with
    float *oo = (float *)stage + wave * (DB * 16 * 64) + ln, *ml = (float *)stage + 4 * DB * 16 * 64 + wave * 64 + ln;
    if (group == 1) {
      ml[0] = m;
      ml[256] = l;
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) oo[(i * 16 + r) * 64] = o[i][r];
    }
    __syncthreads();
    if (group == 1) return;
    const float m1 = ml[0], mm = fmaxf(m, m1), mu = mm == -INFINITY ? 0.f : mm;
    float f0 = __builtin_amdgcn_exp2f(m - mu), f1 = __builtin_amdgcn_exp2f(m1 - mu);
    m = mm;
    l = l * f0 + ml[256] * f1;
    const float inv = l == 0.f ? 0.f : 0.5f / l;               // half means: they stay below float32's largest
    f0 *= inv;
    f1 *= inv;
    if (again) {
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = joined_odd(o[i][r], f0, oo[(i * 16 + r) * 64], f1) * up;
    } else {
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = joined(o[i][r], f0, oo[(i * 16 + r) * 64], f1);
    }
  } else {
    const float inv = l == 0.f && m == -INFINITY ? 0.f : 0.5f / l;  // no key seen (m is +infinity where scores overflow)
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = o[i][r] * inv * up;
  }
  const int row = r0 + (ln & 31);
  if (row >= lq) return;
  if (a.part) {
    const int64_t x = (qa + row) * a.heads + head;
    float *dst = a.part + (x * gridDim.z + split) * a.dim;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        if (32 * i + 8 * r4 + 4 * lnh < a.dim)
          *(floatx4 *)(dst + 32 * i + 8 * r4 + 4 * lnh) =
              floatx4{o[i][4 * r4], o[i][4 * r4 + 1], o[i][4 * r4 + 2], o[i][4 * r4 + 3]};
    if (lnh == 0) {
      float *ml = a.part + (int64_t)a.q.tokens * a.heads * gridDim.z * a.dim + (x * gridDim.z + split) * 2;
      ml[0] = m;
      ml[1] = l;
    }
    return;
  }
  T *dst = (T *)a.out.data + (qa + row) * a.out.token_stride + head * a.out.head_stride;
  auto store = [&](auto number) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int d = 32 * i + 8 * r4 + 4 * lnh;
        if (d < a.dim) {
          struct alignas(8) { T v[4]; } w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w.v[e] = number(o[i][4 * r4 + e]);
          *(decltype(w) *)(dst + d) = w;
        }
      }
  };
  if (again) store([](float x) { return doubled_odd<T>(x); });
  else store([](float x) { return doubled<T>(x); });
  if (a.lse && lnh == 0) a.lse[(int64_t)head * a.q.tokens + qa + row] = (m + __builtin_log2f(l)) * kLn2;
}

// The rows' parts: a workgroup per row.  Rows of no sequence are passed over.
template <class T>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a, int splits) {
  const int64_t i = blockIdx.x / a.heads, h = blockIdx.x % a.heads;
  if (i < clip(a.cu_q[0], a.q.tokens) || i >= clip(a.cu_q[a.seqs], a.q.tokens)) return;
  join_parts<T, true>(blockIdx.x, a.q.tokens * a.heads, a.dim, splits, a.part,
                      [&] {
                        // the workgroup's tiles, as the first launch counted them
                        const int seq = find_row(a.seqs, i, [&](int s) { return clip(a.cu_q[s], a.q.tokens); });
                        const int64_t qa = clip(a.cu_q[seq], a.q.tokens), ka = clip(a.cu_k[seq], a.k.tokens);
                        const int64_t lq = clip(a.cu_q[seq + 1], a.q.tokens) - qa;
                        const int64_t lk = max(clip(a.cu_k[seq + 1], a.k.tokens) - ka, (int64_t)0);
                        const int64_t row = (i - qa) / a.rows * a.rows + a.rows - 1;
                        const int64_t last = a.causal ? min(min(row, lq - 1) + lk - lq, lk - 1) : lk - 1;
                        const int64_t tiles = max(last + a.keys, (int64_t)0) / a.keys;
                        return (int)min(max((tiles + a.chunk - 1) / a.chunk, (int64_t)1), (int64_t)splits);
                      },
                      (T *)a.out.data + i * a.out.token_stride + h * a.out.head_stride,
                      a.lse ? a.lse + h * a.q.tokens + i : nullptr);
}

template <class T>
hipError_t join(const PromptArgs &a, int splits, hipStream_t s) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((prompt_join_kernel<T>), dim3((unsigned)(a.q.tokens * a.heads)), dim3(256), 0, s, a, splits);
  return hipGetLastError();
}

int64_t prompt_blocks(const ios_attn_desc &d, int64_t q_tokens) {
  return (q_tokens / (d.dtype == IOS_F32 ? kFloatRows : kRows) + d.seqs) * d.heads;
}

template <class T, int DP>
hipError_t run(const PromptArgs &a, bool two, int splits, hipStream_t s) {
  const dim3 grid((unsigned)((a.q.tokens / kBM + a.seqs) * a.heads), 1, splits);
  if (two) hipLaunchKernelGGL((attn_prompt_kernel<T, DP, 2>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((attn_prompt_kernel<T, DP, 1>), grid, dim3(256), 0, s, a);
  return join<T>(a, splits, s);
}
template <class T>
hipError_t for_dim(const PromptArgs &a, bool two, int splits, hipStream_t s) {
  if (a.dim <= 32) return run<T, 32>(a, two, splits, s);
  if (a.dim <= 64) return run<T, 64>(a, two, splits, s);
  if (a.dim <= 96) return run<T, 96>(a, two, splits, s);
  return run<T, 128>(a, two, splits, s);
}

}  // namespace

int prompt_splits(const ios_attn_desc &d, int64_t q_tokens) {
  const int64_t blocks = prompt_blocks(d, q_tokens);
  if (blocks >= kFewBlocks || blocks == 0) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / blocks, d.max_keys / kPartKeys), kMaxParts));
}

hipError_t launch_attn_prompt(const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &k, const ios_tokens &v,
                              const ios_tokens &out, float *lse, const int32_t *cu_q, const int32_t *cu_k, void *work,
                              int splits, hipStream_t s) {
  const bool f32 = d.dtype == IOS_F32;
  PromptArgs a{d.heads, d.heads / d.kv_heads, d.head_dim, d.seqs, d.causal, d.scale, q, k, v, out, lse, cu_q, cu_k,
               splits > 1 ? (float *)work : nullptr, 1 << 24, f32 ? kFloatRows : kRows, f32 ? kFloatKeys : kKeys};
  if (splits > 1) a.chunk = std::max(1, (int)(((int64_t)d.max_keys + (int64_t)a.keys * splits - 1) / ((int64_t)a.keys * splits)));
  if (f32) {
    const hipError_t e = launch_attn_prompt_float(a, splits, s);
    return e == hipSuccess ? join<float>(a, splits, s) : e;
  }
  const bool two = splits == 1 && d.max_keys >= kTwoKeys && prompt_blocks(d, q.tokens) <= kTwoGroups;
  return d.dtype == IOS_F16 ? for_dim<_Float16>(a, two, splits, s) : for_dim<__bf16>(a, two, splits, s);
}

}  // namespace ios
