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
#include <type_traits>

#include "decoder.h"

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

constexpr int kBM = 128, kBN = 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// the maximum is only followed when it grows by more than 2^8 (p stays below 2^8, the sums are in 32 bits)
constexpr float kSlack = 8.f;
constexpr uint32_t kOutside = 0x80000000u;       // byte offset past every buffer: reads as 0

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

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, 0x7FFFFFFF, 0x00020000);
}
// Direct global -> LDS load of 16 bytes a lane, l the same for every lane; the
// compiler does not see the write (readers wait for vmcnt(0) and a barrier).
__device__ __forceinline__ void lds_copy16(__amdgpu_buffer_rsrc_t r, unsigned char *l, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)l, 16, (int)off, 0, 0, 0);
}

struct PromptArgs {
  int heads, ratio, dim, seqs, causal;
  float scale;
  ios_tokens q, k, v, out;
  float *lse;
  const int32_t *cu_q, *cu_k;
};

// The two halves of a wave hold different keys of the same queries: this
// lane's value and the other half's.  (The swap exchanges two registers; given
// one twice it would exchange it with itself, hence the copy.)
__device__ __forceinline__ float other_half(float v) {
  int a = __builtin_bit_cast(int, v), b = a;
  asm("" : "+v"(b));
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  return __builtin_bit_cast(float, threadIdx.x & 32 ? r[0] : r[1]);
}

template <class T, int DP>
__global__ __launch_bounds__(256, 2) void attn_prompt_kernel(PromptArgs a) {
  constexpr int CH = DP / 8, KS = DP / 16, DB = DP / 32, LOADS = kBN * CH / 256;
  __shared__ __align__(16) unsigned char lds[2][2][kBN * DP * 2];      // [buffer][K, V]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l31 = lane & 31, l15 = lane & 15;

  // 128-query tiles: sequence i has tiles from cu_q[i] / 128 + i on; the last tiles, which see most keys, go first
  const int64_t x = gridDim.x - 1 - blockIdx.x;
  auto start = [&](int i) { return clip(a.cu_q[i], a.q.tokens) / kBM + i; };
  const int seq = find_owner(a.seqs, x, start);
  const int64_t qa = clip(a.cu_q[seq], a.q.tokens), ka = clip(a.cu_k[seq], a.k.tokens);
  const int lq = (int)(clip(a.cu_q[seq + 1], a.q.tokens) - qa);
  const int lk = max((int)(clip(a.cu_k[seq + 1], a.k.tokens) - ka), 0);
  const int64_t tile = x - start(seq);
  if (tile * kBM >= lq) return;
  const int q0 = (int)tile * kBM, r0 = q0 + 32 * wave;
  const int head = blockIdx.y, kvh = head / a.ratio;

  // last key that a row sees (-1: none); rows past the sequence see what its last row sees
  const int64_t diff = (int64_t)lk - lq;
  auto last_key = [&](int row) { return a.causal ? (int)min((int64_t)min(row, lq - 1) + diff, (int64_t)lk - 1) : lk - 1; };
  const int lim = max(last_key(r0 + l31), -1);
  const int lim_lo = last_key(r0), lim_hi = last_key(r0 + 31);
  const int tiles = max(last_key(q0 + kBM - 1) + kBN, 0) / kBN;

  // queries, the sign of the scale folded in
  shortx8 qf[KS];
  const float mul = fmaxf(__builtin_fabsf(a.scale) * kLog2e, 1e-30f);
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
  auto issue = [&](int t, int buf) {
    const __amdgpu_buffer_rsrc_t kr = buffer(kbase + (int64_t)t * kBN * a.k.token_stride);
    const __amdgpu_buffer_rsrc_t vr = buffer(vbase + (int64_t)t * kBN * a.v.token_stride);
    const int left = lk - t * kBN;                           // rows past the sequence's last key read as 0
#pragma unroll
    for (int p = 0; p < LOADS; ++p) {
      unsigned char *dk = &lds[buf][0][(p * 256 + wave * 64) * 16], *dv = &lds[buf][1][(p * 256 + wave * 64) * 16];
      lds_copy16(kr, dk, row_of[p] < left ? koff[p] : kOutside);
      lds_copy16(vr, dv, row_of[p] < left ? voff[p] : kOutside);
    }
  };

  float m, l;
  floatx16 o[DB];
  const floatx16 zero = {};

  // One walk over the keys.  careful: infinities and NaN among the values of a tile that not every row sees whole
  // are kept out of the product (0 times one of them is a NaN) and reach the rows that see them by counts.
  auto walk = [&](auto careful) {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = zero;
    if (tiles > 0) issue(0, 0);
    for (int t = 0; t < tiles; ++t) {
      // this wave's loads have landed, and every wave is done with the other buffer
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (t + 1 < tiles) issue(t + 1, (t + 1) & 1);
      if (t * kBN > lim_hi) continue;                        // no row of this wave sees the tile
      const unsigned char *sk = lds[t & 1][0], *sv = lds[t & 1][1];
      const bool masked = t * kBN + kBN - 1 > lim_lo;
      floatx16 s[2];
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
      if (masked) {
        asm volatile("");                                    // a branch: selects in every tile took a quarter of the walk
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (t * kBN + 32 * b + (r & 3) + 8 * (r >> 2) + 4 * half > lim) s[b][r] = -INFINITY;
      }
      float mx = s[0][0];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
      mx *= mul;
      if (__any(mx > m + kSlack)) {
        // each row by its own scores alone, so that no row's result depends on another's
        const float rm = fmaxf(mx, other_half(mx)), mn = rm > m + kSlack ? rm : m;
        const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= f;
#pragma unroll
        for (int i = 0; i < DB; ++i) o[i] *= f;
      }
      const float mu = m == -INFINITY ? 0.f : m;
      shortx8 pf[4];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[b][r], mul, -mu));
          l += e;
          pf[2 * b + (r >> 3)][r & 7] = __builtin_bit_cast(short, (T)e);      // p as the inputs' type: 2^-9 (2^-12) each
        }
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        floatx16 nan = zero, up = zero, down = zero;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const int r = 16 * ks + 4 * half + (l15 >> 2), c = 4 * i + 2 * (lane >> 4 & 1) + ((l15 & 3) >> 1);
          const unsigned char *p = sv + r * (CH * 16) + (c ^ swz_v<DP>(r)) * 16 + 8 * (l15 & 1);
          const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)p);
          const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4 *)(p + 8 * CH * 16));
          shortx8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          if constexpr (careful) {
            if (masked) {
              constexpr int inf = std::is_same_v<T, _Float16> ? 0x7C00 : 0x7F80;
              const short one = __builtin_bit_cast(short, (T)1.f);
              shortx8 vn, vu, vd, seen;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int mag = vf[e] & 0x7FFF;
                vn[e] = mag > inf ? one : 0;
                vu[e] = vf[e] == inf ? one : 0;
                vd[e] = mag == inf && vf[e] < 0 ? one : 0;
                if (mag >= inf) vf[e] = 0;
                seen[e] = t * kBN + 16 * ks + 4 * half + (e & 3) + 8 * (e >> 2) <= lim ? one : 0;
              }
              nan = mfma<T>(vn, seen, nan);
              up = mfma<T>(vu, seen, up);
              down = mfma<T>(vd, seen, down);
            }
          }
          o[i] = mfma<T>(vf, pf[ks], o[i]);
        }
        if constexpr (careful) {
          if (masked) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
              o[i][r] += nan[r] > 0.f || (up[r] > 0.f && down[r] > 0.f) ? NAN
                         : up[r] > 0.f ? INFINITY : down[r] > 0.f ? -INFINITY : 0.f;
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
  if (__syncthreads_or(odd)) walk(std::true_type{});

  l += other_half(l);
  const int row = r0 + l31;
  if (row >= lq) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T *dst = (T *)a.out.data + (qa + row) * a.out.token_stride + head * a.out.head_stride;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int d = 32 * i + 8 * r4 + 4 * half;
      if (d < a.dim) {
        struct alignas(8) { T v[4]; } w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w.v[e] = (T)(o[i][4 * r4 + e] * inv);
        *(decltype(w) *)(dst + d) = w;
      }
    }
  if (a.lse && half == 0) a.lse[(int64_t)head * a.q.tokens + qa + row] = (m + __builtin_log2f(l)) * kLn2;
}

template <class T, int DP>
hipError_t run(const PromptArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((attn_prompt_kernel<T, DP>), dim3((unsigned)(a.q.tokens / kBM + a.seqs), a.heads), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <class T>
hipError_t for_dim(const PromptArgs &a, hipStream_t s) {
  if (a.dim <= 32) return run<T, 32>(a, s);
  if (a.dim <= 64) return run<T, 64>(a, s);
  if (a.dim <= 96) return run<T, 96>(a, s);
  return run<T, 128>(a, s);
}

}  // namespace

hipError_t launch_attn_prompt_float(const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &k,
                                    const ios_tokens &v, const ios_tokens &out, float *lse, const int32_t *cu_q,
                                    const int32_t *cu_k, hipStream_t s);

int prompt_splits(const ios_attn_desc &, int64_t) { return 1; }

hipError_t launch_attn_prompt(const ios_attn_desc &d, const ios_tokens &q, const ios_tokens &k, const ios_tokens &v,
                              const ios_tokens &out, float *lse, const int32_t *cu_q, const int32_t *cu_k, void *,
                              int, hipStream_t s) {
  if (d.dtype == IOS_F32) return launch_attn_prompt_float(d, q, k, v, out, lse, cu_q, cu_k, s);
  const PromptArgs a{d.heads, d.heads / d.kv_heads, d.head_dim, d.seqs, d.causal, d.scale, q, k, v, out, lse, cu_q, cu_k};
  return d.dtype == IOS_F16 ? for_dim<_Float16>(a, s) : for_dim<__bf16>(a, s);
}

}  // namespace ios
