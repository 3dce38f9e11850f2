// Queries and keys turned by their positions (ios_rotate).
//
// Every value is read and written once: bound by memory where there are many tokens, by a launch and one chain of loads
// where there are few.  A workgroup takes a few tokens and first fills a table of their cosines and sines, which all
// heads share, so the 64-bit work is a small part of what the values cost.
#include "rotary.h"

namespace ios {

namespace {

constexpr int kUnroll = 4;               // units of a thread on their way at once

template <class T>
__global__ __launch_bounds__(256) void rotate_kernel(ios_rotary r, int head_dim, int per, ios_tokens q, ios_tokens qo,
                                                     int heads, ios_tokens k, ios_tokens ko, int kv_heads,
                                                     const int32_t *pos) {
  extern __shared__ float2 table[];      // [per][half]
  const RotaryUnits u(r, head_dim);
  const int64_t t0 = (int64_t)blockIdx.x * per;
  const int tokens = (int)min((int64_t)per, q.tokens - t0), all = heads + kv_heads;
  // heads of this workgroup
  const int h0 = (int)((int64_t)all * blockIdx.y / gridDim.y), h1 = (int)((int64_t)all * (blockIdx.y + 1) / gridDim.y);
  const int units = tokens * (h1 - h0) * u.all;
  auto place = [&](int x, int *at, int *t, const ios_tokens &a, const ios_tokens &b) {
    const int row = x / u.all, tok = row / (h1 - h0), h = h0 + row - tok * (h1 - h0);
    *at = x - row * u.all;
    *t = tok;
    return h < heads ? (T *)a.data + (t0 + tok) * a.token_stride + h * a.head_stride
                     : (T *)b.data + (t0 + tok) * b.token_stride + (h - heads) * b.head_stride;
  };
  RotaryUnit<T> unit[kUnroll];
  int at, t;
  auto load = [&](int x0) {
#pragma unroll
    for (int e = 0; e < kUnroll; ++e)
      if (x0 + 256 * e < units) {
        const T *row = place(x0 + 256 * e, &at, &t, q, k);
        unit[e].load(u, row, at);
      }
  };
  load(threadIdx.x);
  for (int x = threadIdx.x; x < tokens * u.half; x += 256)
    table[x] = turn_of(pos[t0 + x / u.half], r.freq[x % u.half], r.amplitude);
  __syncthreads();
  for (int x0 = threadIdx.x; x0 < units; x0 += 256 * kUnroll) {
    if (x0 != (int)threadIdx.x) load(x0);
#pragma unroll
    for (int e = 0; e < kUnroll; ++e)
      if (x0 + 256 * e < units) {
        T *row = place(x0 + 256 * e, &at, &t, qo, ko);
        unit[e].turn_by(u, table + t * u.half, at);
        unit[e].store(u, row, at);
      }
  }
}

template <class T>
hipError_t run(const ios_rotary &r, int head_dim, const ios_tokens &q, const ios_tokens &qo, int heads,
               const ios_tokens &k, const ios_tokens &ko, int kv_heads, const int32_t *pos, hipStream_t s) {
  const int per = q.tokens >= 2048 ? 4 : 1;
  const int64_t blocks = (q.tokens + per - 1) / per;
  const int groups = 1;
  hipLaunchKernelGGL((rotate_kernel<T>), dim3((unsigned)blocks, groups), dim3(256), per * (r.dim / 2) * sizeof(float2), s, r,
                     head_dim, per, q, qo, heads, k, ko, kv_heads, pos);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const ios_rotary &r, int dtype, int head_dim, const ios_tokens &q, const ios_tokens &qo, int heads,
                         const ios_tokens &k, const ios_tokens &ko, int kv_heads, const int32_t *pos, hipStream_t s) {
  if (dtype == IOS_F32) return run<float>(r, head_dim, q, qo, heads, k, ko, kv_heads, pos, s);
  if (dtype == IOS_F16) return run<_Float16>(r, head_dim, q, qo, heads, k, ko, kv_heads, pos, s);
  return run<__bf16>(r, head_dim, q, qo, heads, k, ko, kv_heads, pos, s);
}

}  // namespace ios
