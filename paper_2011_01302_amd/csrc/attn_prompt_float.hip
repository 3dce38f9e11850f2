// Attention over packed prompts in float32 (ios_attn_prompt): the walk of
// attn_prompt.hip on v_mfma_f32_32x32x2_f32, every number in 32 bits.  Bound by
// the fp32 matrix rate, a seventh of the 16-bit one: tiles of 32 keys go through
// registers to LDS, the next one's on its way.  Three packed maps (1225, 784 and
// 193 tokens, 12 heads of 96): 115 us, 86 TFLOP/s of the 153 that a large matrix
// product reaches, matrix cores 52 per cent busy; what is lost is mostly the
// workgroups' uneven number per CU.
#include <type_traits>

#include "attn_prompt.h"

namespace ios {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));

// a row's maximum is only followed when it grows by more than 2^8 (p stays below 2^8)
constexpr float kSlack = 8.f;
constexpr int kBM = kFloatRows, kBN = kFloatKeys, kRW = kBM / 32, kGroupThreads = 64 * kRW, KG = 2;


__device__ __forceinline__ floatx4 load16(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t more) {
  return __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, (int)more, 0));
}

// Two waves of 32 queries, and two groups of such waves that take the tiles in turn and are joined at the end: the
// matrix cores are what bounds, so the work is cut small enough to come out even over them.
template <int DP>
__global__ __launch_bounds__(kGroupThreads * KG, 2) void attn_prompt_float_kernel(PromptArgs a) {
  constexpr int CH = DP / 4, DB = DP / 32, PITCH = DP + 4, LOADS = kBN * CH / kGroupThreads;
  __shared__ __align__(16) float stage[KG][2][kBN * PITCH];
  __shared__ float other_o[kGroupThreads][17], other_ml[kGroupThreads][2];
  __shared__ int odd_rows[KG][2][kBN];            // of this tile and the next: waves may be a tile apart
  const int tid = threadIdx.x % kGroupThreads, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / kGroupThreads);
  float *sk = stage[group][0], *sv = stage[group][1];
  const int half = lane >> 5, l31 = lane & 31;

  int head, seq;
  int64_t first_query;
  if (!prompt_block(a, &head, &seq, &first_query)) return;
  const int64_t qa = clip(a.cu_q[seq], a.q.tokens), ka = clip(a.cu_k[seq], a.k.tokens);
  const int lq = (int)(clip(a.cu_q[seq + 1], a.q.tokens) - qa);
  const int lk = max((int)(clip(a.cu_k[seq + 1], a.k.tokens) - ka), 0);
  if (first_query >= lq) return;
  const int q0 = (int)first_query, r0 = q0 + 32 * wave;
  const int kvh = head / a.ratio;
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

  // Q: values 8 i + 4 half + e of query l31 (the order in which K's are read)
  float qf[DP / 2];
  const float mul = multiplier(a.scale), sign = a.scale < 0.f ? -1.f : 1.f;
  {
    const float *src = (const float *)a.q.data + (qa + min(r0 + l31, lq - 1)) * a.q.token_stride + head * a.q.head_stride;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) {
      const int d = 8 * i + 4 * half;
      floatx4 w = {0.f, 0.f, 0.f, 0.f};
      if (d < a.dim) w = *(const floatx4 *)(src + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) qf[4 * i + e] = w[e] * sign;
    }
  }
  const float *kbase = (const float *)a.k.data + ka * a.k.token_stride + kvh * a.k.head_stride;
  const float *vbase = (const float *)a.v.data + ka * a.v.token_stride + kvh * a.v.head_stride;

  float m, l;
  floatx16 o[DB];
  const floatx16 zero = {};

  // what this thread loads of a tile, through descriptors (past their end, and past the sequence's last key, reads as 0).
  // For heads of 128, where registers are short, one offset and what all threads add to it (2048 keys and queries, 12
  // heads, not causal: 292 us, 318 with offsets of their own; heads of 64, causal: 111 and 110).
  constexpr int ROWS = DP == 128 ? kGroupThreads / CH : 0, OFFS = ROWS ? 1 : LOADS;
  uint32_t koff[OFFS], voff[OFFS];
#pragma unroll
  for (int p = 0; p < OFFS; ++p) {
    const int s = p * kGroupThreads + tid, r = s / CH, d = s % CH * 4;
    koff[p] = d < a.dim ? (uint32_t)(r * (int)a.k.token_stride + d) * 4 : kOutside;
    voff[p] = d < a.dim ? (uint32_t)(r * (int)a.v.token_stride + d) * 4 : kOutside;
  }
  floatx4 nk[LOADS], nv[LOADS];                              // the next tile, on its way
  auto load = [&](int t) {
    const __amdgpu_buffer_rsrc_t kr = buffer(kbase + (int64_t)t * kBN * a.k.token_stride);
    const __amdgpu_buffer_rsrc_t vr = buffer(vbase + (int64_t)t * kBN * a.v.token_stride);
#pragma unroll
    for (int p = 0; p < LOADS; ++p) {
      const bool in = t * kBN + (p * kGroupThreads + tid) / CH < lk;
      const int at = ROWS ? 0 : p, more = p * ROWS * 4;
      nk[p] = load16(kr, in ? koff[at] : kOutside, more * (int)a.k.token_stride);
      nv[p] = load16(vr, in ? voff[at] : kOutside, more * (int)a.v.token_stride);
    }
  };
  auto walk = [&](auto again) {
    constexpr bool kAgain = decltype(again)::value;
    constexpr float by = kAgain ? kDown : 1.f;
    int wtid = tid;                                            // addresses of the first walk are not kept for the second
    asm("" : "+v"(wtid));
    const int half = wtid >> 5 & 1, l31 = wtid & 31;
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = zero;
    if (!kAgain && t0 + group < tiles) load(t0 + group);
    for (int k = 0; t0 + k * KG < tiles; ++k) {
      const int t = t0 + k * KG + group;
      int *odd_row = odd_rows[group][k & 1];
      if (kAgain && t < tiles) load(t);
      if (tid < kBN) odd_row[tid] = 0;
      __syncthreads();
#pragma unroll
      for (int p = 0; p < LOADS; ++p) {
        const int s = p * kGroupThreads + wtid, r = s / CH, d = s % CH * 4;
        *(floatx4 *)(sk + r * PITCH + d) = nk[p];
        // an infinity or NaN (or four values whose sum is beyond float32): they stay out of the products, see below
        const float sum = __builtin_fabsf(nv[p][0]) + __builtin_fabsf(nv[p][1]) + __builtin_fabsf(nv[p][2]) + __builtin_fabsf(nv[p][3]);
        if (!(sum < INFINITY)) {
          odd_row[r] = 1;
#pragma unroll
          for (int e = 0; e < 4; ++e) nv[p][e] = __builtin_fabsf(nv[p][e]) < INFINITY ? nv[p][e] : 0.f;
        }
        *(floatx4 *)(sv + r * PITCH + d) = nv[p];
      }
      __syncthreads();
      if (!kAgain && t + KG < tiles) load(t + KG);
      if (t >= tiles || t * kBN > lim_hi) continue;
      floatx16 s = zero;
#pragma unroll
      for (int i = 0; i < DP / 8; ++i) {
        const floatx4 kf = *(const floatx4 *)(sk + l31 * PITCH + 8 * i + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[4 * i + e], s, 0, 0, 0);
      }
      const bool masked = t * kBN + kBN - 1 > lim_lo;
      if (masked) {
        asm volatile("");                                    // a branch, not selects in every tile
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t * kBN + (r & 3) + 8 * (r >> 2) + 4 * half > lim) s[r] = -INFINITY;
      }
      float mx = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
      mx *= mul;
      if (__any(mx > m + kSlack)) {
        // each row by its own scores alone, so that no row's result depends on another's
        const float rm = fmaxf(mx, __shfl_xor(mx, 32)), mn = rm > m + kSlack ? rm : m;
        const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= f;
#pragma unroll
        for (int i = 0; i < DB; ++i) {
          if constexpr (kAgain) {                            // o may hold infinities and NaN
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] = weighed(o[i][r], f);
          } else {
            o[i] *= f;
          }
        }
      }
      const float mu = m == -INFINITY ? 0.f : m;
      auto weight = [&](int r) {
        s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], mul, -mu));
        l += s[r];
        s[r] *= by;
      };
      float vf[3][DB];                                       // values of keys on their way from LDS
      auto fetch = [&](int r) {
#pragma unroll
        for (int i = 0; i < DB; ++i) vf[r % 3][i] = sv[((r & 3) + 8 * (r >> 2) + 4 * half) * PITCH + 32 * i + l31];
      };
      fetch(0);
      fetch(1);
      weight(0);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (r + 2 < 16) fetch(r + 2);
        if (r + 1 < 16) weight(r + 1);
#pragma unroll
        for (int i = 0; i < DB; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[r % 3][i], s[r], o[i], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      // The infinities and NaN that were left out (0 times one of them is a NaN, also for rows that do not see the key):
      // added to the rows that see them.
      if (__any(odd_row[l31])) {
        for (int key = 0; key < kBN; ++key) {
          if (!__builtin_amdgcn_readfirstlane(odd_row[key])) continue;
          const bool seen = t * kBN + key <= lim;
          const float *src = vbase + (int64_t)(t * kBN + key) * a.v.token_stride + 4 * half;
#pragma unroll
          for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
              if (32 * i + 8 * r4 + 4 * half >= a.dim) continue;
              const floatx4 x = *(const floatx4 *)(src + 32 * i + 8 * r4);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (seen && !(__builtin_fabsf(x[e]) < INFINITY)) o[i][4 * r4 + e] += x[e];
            }
        }
      }
    }
  };
  walk(std::false_type{});
  int odd = 0;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd |= !(__builtin_fabsf(o[i][r]) < INFINITY);
  float up = 1.f;
  const bool again = __builtin_amdgcn_readfirstlane(__syncthreads_or(odd));
  if (again) {                                               // rows see an infinity or NaN, or a sum has left float32's range
    walk(std::true_type{});
    up = kUp;
  }

  l += __shfl_xor(l, 32);
  {                                                          // the second group's rows go through LDS to the first
    if (group == 1) {
      other_ml[tid][0] = m;
      other_ml[tid][1] = l;
    }
    __syncthreads();
    const float m1 = other_ml[tid][0], mm = fmaxf(m, m1), mu = mm == -INFINITY ? 0.f : mm;
    float f0 = __builtin_amdgcn_exp2f(m - mu), f1 = __builtin_amdgcn_exp2f(m1 - mu);
    m = mm;
    l = l * f0 + other_ml[tid][1] * f1;
    const float inv = l == 0.f ? 0.f : 0.5f / l;             // half means: they stay below float32's largest
    f0 *= inv;
    f1 *= inv;
#pragma unroll
    for (int i = 0; i < DB; ++i) {
      if (group == 1) {
#pragma unroll
        for (int r = 0; r < 16; ++r) other_o[tid][r] = o[i][r];
      }
      __syncthreads();
      if (group == 0) {
        if (again) {
#pragma unroll
          for (int r = 0; r < 16; ++r) o[i][r] = joined_odd(o[i][r], f0, other_o[tid][r], f1) * up;
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) o[i][r] = joined(o[i][r], f0, other_o[tid][r], f1);
        }
      }
      __syncthreads();
    }
    if (group == 1) return;
  }
  const int row = r0 + l31;
  if (row >= lq) return;
  if (a.part) {
    const int64_t x = (qa + row) * a.heads + head;
    float *dst = a.part + (x * gridDim.z + split) * a.dim;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        if (32 * i + 8 * r4 + 4 * half < a.dim)
          *(floatx4 *)(dst + 32 * i + 8 * r4 + 4 * half) =
              floatx4{o[i][4 * r4], o[i][4 * r4 + 1], o[i][4 * r4 + 2], o[i][4 * r4 + 3]};
    if (half == 0) {
      float *ml = a.part + (int64_t)a.q.tokens * a.heads * gridDim.z * a.dim + (x * gridDim.z + split) * 2;
      ml[0] = m;
      ml[1] = l;
    }
    return;
  }
  float *dst = (float *)a.out.data + (qa + row) * a.out.token_stride + head * a.out.head_stride;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int d = 32 * i + 8 * r4 + 4 * half;
      if (d < a.dim) {
        floatx4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = doubled_odd<float>(o[i][4 * r4 + e]);
        *(floatx4 *)(dst + d) = w;
      }
    }
  if (a.lse && half == 0) a.lse[(int64_t)head * a.q.tokens + qa + row] = (m + __builtin_log2f(l)) * kLn2;
}

template <int DP>
hipError_t run(const PromptArgs &a, int splits, hipStream_t s) {
  const dim3 grid((unsigned)((a.q.tokens / kBM + a.seqs) * a.heads), 1, splits);
  hipLaunchKernelGGL((attn_prompt_float_kernel<DP>), grid, dim3(kGroupThreads * KG), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_prompt_float(const PromptArgs &a, int splits, hipStream_t s) {
  if (a.dim <= 32) return run<32>(a, splits, s);
  if (a.dim <= 64) return run<64>(a, splits, s);
  if (a.dim <= 96) return run<96>(a, splits, s);
  return run<128>(a, splits, s);
}

}  // namespace ios
