// Joining the parts of attention rows whose keys were spread over workgroups.
//
// Part s of a row leaves in the workspace sum_j p_j v_j ([row][part][dim] floats), or half of that divided by sum_j p_j
// (`kMeans`: values may reach to float32's largest, and sums of them not), and behind all of those its reference m and the sum of
// p_j = 2^(score_j - m) ([row][part][2]).
#pragma once

#include <type_traits>

#include "decoder.h"

namespace ios {

typedef float floatx4 __attribute__((ext_vector_type(4)));
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxParts = 128;

// x times a weight f that may have come to 0: an infinity or NaN that a row sees stays one, however little it weighs.
__device__ __forceinline__ float weighed(float x, float f) { return __builtin_fabsf(x) < INFINITY || f != 0.f ? x * f : x; }

// x f + y g, and the same, to the bit, where infinities and NaN have to be expected.
__device__ __forceinline__ float joined(float x, float f, float y, float g) { return fmaf(x, f, y * g); }
__device__ __forceinline__ float joined_odd(float x, float f, float y, float g) {
  const bool finite = fmaxf(__builtin_fabsf(x), __builtin_fabsf(y)) < INFINITY && x == x && y == y;
  return finite ? joined(x, f, y, g) : weighed(x, f) + weighed(y, g);
}

// Of half a mean of T's values, the mean.  It is never beyond T's largest number: where rounded weights say so, it is that.
template <class T>
__device__ __forceinline__ T doubled(float half) {
  constexpr float most = std::is_same_v<T, _Float16> ? 65504.f : std::is_same_v<T, float> ? 0x1.fffffep127f : 0x1.fep127f;
  return (T)(2.f * (__builtin_fabsf(half) > 0.5f * most ? __builtin_copysignf(0.5f * most, half) : half));
}
template <class T>
__device__ __forceinline__ T doubled_odd(float half) {
  return __builtin_fabsf(half) < INFINITY ? doubled<T>(half) : (T)half;
}

// One workgroup of 256 threads joins row `row` of `rows`: weights of the parts first (a thread each), then four values
// a thread, the parts spread over the threads; every sum in a fixed order.  The first loads do not wait for the number
// of parts that hold anything (count()); the others' values are left out.
template <class T, bool kMeans, class F>
__device__ __forceinline__ void join_parts(int64_t row, int64_t rows, int dim, int splits, const float *part, F count,
                                           T *out, float *lse) {
  static_assert(kMaxParts <= 256, "a thread per part");
  __shared__ float weight[kMaxParts], red[2][4];
  __shared__ floatx4 sum[256];
  const int Q = dim / 4, W = 256 / Q;                             // W threads share four values
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, d4 = tid % Q, w = tid / Q;
  const floatx4 *src = (const floatx4 *)(part + row * splits * dim) + d4;
  floatx4 x[8];
  auto load = [&](int s0) {
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = src[(int64_t)min(s0 + u * W, splits - 1) * Q];
  };
  load(w);
  const float *ml = part + rows * splits * dim + row * splits * 2;
  const float m0 = ml[2 * min(tid, splits - 1)], l0 = ml[2 * min(tid, splits - 1) + 1];
  const int n = count();
  float mm = tid < n ? m0 : -INFINITY;
#pragma unroll
  for (int y = 1; y < 64; y <<= 1) mm = fmaxf(mm, __shfl_xor(mm, y));
  if (lane == 0) red[0][wave] = mm;
  __syncthreads();
  mm = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  const float mu = mm == -INFINITY ? 0.f : mm, f = tid < n ? __builtin_amdgcn_exp2f(m0 - mu) : 0.f;
  float ll = tid < n ? f * l0 : 0.f;
  if (!kMeans && tid < kMaxParts) weight[tid] = f;
  const float fl = ll;
#pragma unroll
  for (int y = 1; y < 64; y <<= 1) ll += __shfl_xor(ll, y);
  if (lane == 0) red[1][wave] = ll;
  __syncthreads();
  ll = red[1][0] + red[1][1] + red[1][2] + red[1][3];
  if constexpr (kMeans) {                                         // the parts' shares: they sum to 1
    if (tid < kMaxParts) weight[tid] = ll == 0.f ? 0.f : fl / ll;
    __syncthreads();
  }
  floatx4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = w; s0 < n; s0 += 8 * W) {
    if (s0 != w) load(s0);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (s0 + u * W < n) {
        const float f = weight[s0 + u * W];
        if constexpr (kMeans) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] += weighed(x[u][e], f);
        } else {
          v += f * x[u];
        }
      }
  }
  sum[tid] = v;
  __syncthreads();
  if (tid < Q) {
    for (int y = 1; y < W; ++y) v += sum[tid + y * Q];
    struct alignas(4 * sizeof(T)) { T v[4]; } r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (kMeans) r.v[e] = doubled_odd<T>(v[e]);
      else r.v[e] = (T)(ll == 0.f ? 0.f : v[e] / ll);
    }
    *(decltype(r) *)(out + 4 * tid) = r;
  }
  if (lse && tid == 0) *lse = (mm + __builtin_log2f(ll)) * kLn2;
}

}  // namespace ios
