// Queries and keys turned by their positions (ios_rotate).
//
// Every value is read and written once: bound by memory where there are many tokens, by a launch and one chain of loads
// where there are few.  A workgroup takes a few tokens and first fills a table of their cosines and sines, which all
// heads share, so the 64-bit work is a small part of what the values cost; its units are all on their way before the table
// is, as many tokens as make four a thread.  17609 tokens of 40 heads of 128, bf16: 76 us, 4.75 TB/s (a large copy 4.9), in
// float32 139; 16 tokens of 10 heads of 64: 3.4.
#include "rotary.h"

namespace ios {

namespace {

constexpr int kUnroll = 4;               // units of a thread on their way at once

// x / d by a product with ceil(2^32 / d), right where x d < 2^32.
struct Divisor {
  uint32_t d, m;
  explicit Divisor(uint32_t d) : d(d), m((uint32_t)((((uint64_t)1 << 32) + d - 1) / d)) {}
  __device__ __forceinline__ int of(int x) const { return d == 1 ? x : (int)__umulhi((uint32_t)x, m); }
};

template <class T>
__global__ __launch_bounds__(256) void rotate_kernel(ios_rotary r, int head_dim, int per, Divisor by_unit, Divisor by_head,
                                                     ios_tokens q, ios_tokens qo, int heads, ios_tokens k, ios_tokens ko,
                                                     const int32_t *pos) {
  extern __shared__ float2 table[];      // [per][half]
  const RotaryUnits u(r, head_dim);
  const int64_t t0 = (int64_t)blockIdx.x * per;
  const int tokens = (int)min((int64_t)per, q.tokens - t0), all = by_head.d, units = tokens * all * u.all;
  RotaryUnit<T> unit[kUnroll];
  int at[kUnroll], tok[kUnroll], head[kUnroll];
  auto row = [&](int e, const ios_tokens &a, const ios_tokens &b) {
    const bool is_k = head[e] >= heads;
    const int64_t ts = is_k ? b.token_stride : a.token_stride, hs = is_k ? b.head_stride : a.head_stride;
    return (T *)(is_k ? b.data : a.data) + (t0 + tok[e]) * ts + (head[e] - (is_k ? heads : 0)) * hs;
  };
  auto load = [&](int x0) {
#pragma unroll
    for (int e = 0; e < kUnroll; ++e) {
      const int x = min(x0 + 256 * e, units - 1), y = by_unit.of(x);
      at[e] = x - y * u.all;
      tok[e] = by_head.of(y);
      head[e] = y - tok[e] * all;
      unit[e].load(u, row(e, q, k), at[e]);
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
        unit[e].turn_by(u, table + tok[e] * u.half, at[e]);
        unit[e].store(u, row(e, qo, ko), at[e]);
      }
  }
}

template <class T>
hipError_t run(const ios_rotary &r, int head_dim, const ios_tokens &q, const ios_tokens &qo, int heads,
               const ios_tokens &k, const ios_tokens &ko, int kv_heads, const int32_t *pos, hipStream_t s) {
  // tokens of a workgroup: up to kUnroll units and 8 pairs of the table a thread, but every CU has four workgroups first
  const RotaryUnits u(r, head_dim);
  const int all = heads + kv_heads, most = std::min(256 * kUnroll / (all * u.all), 256 * 8 / u.half);
  // (a grid has less than 2^32 threads)
  const int per = (int)std::max<int64_t>((q.tokens >> 23) + 1, std::min<int64_t>(most, q.tokens / 1024));
  hipLaunchKernelGGL((rotate_kernel<T>), dim3((unsigned)((q.tokens + per - 1) / per)), dim3(256),
                     per * u.half * sizeof(float2), s, r, head_dim, per, Divisor(u.all), Divisor(all), q, qo, heads, k, ko, pos);
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
