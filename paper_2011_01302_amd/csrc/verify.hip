// Drafted tokens against the model's probabilities (ios_verify).
//
// With p the model's and q the draft's probabilities in the node's row, the k-th rejection leaves
// max(p_k - q, 0) / its sum of what p_k was left before.  Written out that is max(p - C q, 0) / S, where C starts at 0 and
// grows by the S before, and S = sum max(p - C q, 0) starts at 1: max(max(p - C q, 0) / S - q, 0) = max(p - (C + S) q, 0) / S
// as q >= 0.  So a walk through the tree carries two numbers, a draft's test reads one p and one q, and a whole row is
// read only where a rejected draft has a sibling left to try, and at the end for the next token.
//
// A workgroup walks a sequence's tree.  With a small vocabulary it also draws the next token; with a large one a second
// launch sums that row over several workgroups, the last of which draws.
//
// A chain of loads and sums, each of a few hundred nanoseconds: the walk (offsets, tree, probabilities), the row, its sum
// across the card, the share that holds the mark.  32 chains over 131072 tokens, float32: 21 us (4 for the walk, 17 for 34 MB
// of rows, which memory alone would take 7 for); one tree over 32003 tokens 10.  A row that is read during the walk is read by
// the walk's one workgroup: where three drafts behind the root fall one after the other, two such rows, 1, 8 and 32 sequences of
// 131072 tokens take 58, 59 and 67 us in float32 (71, 71 and 78 in bf16) against 13, 14 and 19 where one falls.
#include <type_traits>

#include "decoder.h"

namespace ios {

namespace {

constexpr int kThreadsV = 1024, kThreadsD = 512, kUnrollV = 2;   // of a walk, and of a share of a row
constexpr int kMaxShares = 64;

// Where a walk stopped.
struct Stop {
  double c;
  int64_t row;                           // the last node's, -1: a sequence without rows
  int32_t out_n, done;                   // tokens that are left out, workgroups that have summed their share
  int32_t out[kMaxDrafts];
  double sums[kMaxShares];
};

// A value that is the same in every lane, in scalar registers: what the walk branches on is decided for the wave.
__device__ __forceinline__ double uniform(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b), hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ bool uniform(bool x) { return __builtin_amdgcn_readfirstlane((int)x) != 0; }
// Lane j's value, j the same in every lane.
__device__ __forceinline__ int of_lane(int x, int j) { return __builtin_amdgcn_readlane(x, j); }
__device__ __forceinline__ double of_lane(double x, int j) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, j), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), j);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// A probability: what is negative, infinite or NaN counts as 0.
template <class T>
__device__ __forceinline__ double prob(T x) {
  const float f = fmaxf((float)x, 0.f);                           // 0 for a NaN
  return (double)(f < INFINITY ? f : 0.f);
}

// 8 values of a row.  Rows start at any element; the loads need no more alignment than that.
template <class T>
struct __attribute__((packed, aligned(alignof(T)))) Raw8 {
  T v[8];
};
template <class T>
__device__ __forceinline__ Raw8<T> raw8(const T *row, int64_t t, int64_t end) {
  if (t + 8 <= end) return *(const Raw8<T> *)(row + t);
  Raw8<T> r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.v[e] = t + e < end ? row[t + e] : (T)0;
  return r;
}

// What the threads of a workgroup tell each other; two of each, so that one can be written while the other is read.
template <int TH>
struct Scratch {
  static constexpr int kWaves = TH / 64;
  double sums[2][kWaves];
  int32_t hit[2][kWaves], heavy[2][kWaves];
};

// What is left of a row: max(p - c q, 0), or p without some tokens.  For a workgroup of TH threads.
template <class T, bool GIVEN, int TH>
struct Rest {
  static constexpr int kWaves = TH / 64, kStep = TH * 8;
  const T *p, *q;
  double c;
  const int32_t *out;
  int out_n;

  __device__ __forceinline__ void weights(const Raw8<T> &a, const Raw8<T> &b, int64_t t, double (&w)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (GIVEN) w[e] = fmax(fma(-c, prob(b.v[e]), prob(a.v[e])), 0.0);
      else w[e] = prob(a.v[e]);
    }
    if constexpr (!GIVEN)
      for (int z = 0; z < out_n; ++z) {
        const int64_t at = out[z] - t;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = at == e ? 0.0 : w[e];
      }
  }

  // The sum over tokens from .. end - 1, the same in every thread; `sums` is not read any more by the time that the
  // call after the next one writes it.
  __device__ __forceinline__ double sum(int64_t from, int64_t end, double *sums) const {
    const int tid = threadIdx.x;
    double s = 0.0;
    for (int64_t t0 = from + tid * 8; t0 < end; t0 += kStep * kUnrollV) {
      Raw8<T> a[kUnrollV], b[kUnrollV];
#pragma unroll
      for (int u = 0; u < kUnrollV; ++u) {
        const int64_t t = t0 + u * kStep;
        if (t < end) {
          a[u] = raw8(p, t, end);
          if (GIVEN) b[u] = raw8(q, t, end);
        }
      }
#pragma unroll
      for (int u = 0; u < kUnrollV; ++u) {
        const int64_t t = t0 + u * kStep;
        if (t < end) {
          double w[8];
          weights(a[u], b[u], t, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) s += w[e];
        }
      }
    }
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) s += __shfl_xor(s, y);
    if ((tid & 63) == 0) sums[tid >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += sums[w];
    return uniform(s);
  }

  // The first token of from .. end - 1 with any weight whose running sum, `before` ahead of them, passes the mark; where
  // none does (a mark at the very end), the last with any weight.  In every thread.
  __device__ __forceinline__ int32_t find(int64_t from, int64_t end, double before, double mark, Scratch<TH> &lds) const {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int turn = 0, last = -1;
    for (int64_t t1 = from; t1 < end; t1 += kStep, turn ^= 1) {
      const int64_t t = t1 + tid * 8;
      double w[8] = {}, s = 0.0;
      if (t < end) {
        Raw8<T> a = raw8(p, t, end), b{};
        if (GIVEN) b = raw8(q, t, end);
        weights(a, b, t, w);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s += w[e];
      double incl = s;
#pragma unroll
      for (int y = 1; y < 64; y <<= 1) {
        const double z = __shfl_up(incl, y);
        incl += lane >= y ? z : 0.0;
      }
      if (lane == 63) lds.sums[turn][wave] = incl;
      __syncthreads();
      double run = before + (incl - s);
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        run += x < wave ? lds.sums[turn][x] : 0.0;
        before += lds.sums[turn][x];
      }
      int hit = INT32_MAX, heavy = -1;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        run += w[e];
        if (w[e] > 0.0) heavy = (int)(t + e);
        if (hit == INT32_MAX && w[e] > 0.0 && run > mark) hit = (int)(t + e);
      }
#pragma unroll
      for (int y = 1; y < 64; y <<= 1) {
        hit = min(hit, __shfl_xor(hit, y));
        heavy = max(heavy, __shfl_xor(heavy, y));
      }
      if (lane == 0) lds.hit[turn][wave] = hit, lds.heavy[turn][wave] = heavy;
      __syncthreads();
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        hit = min(hit, lds.hit[turn][x]);
        last = max(last, lds.heavy[turn][x]);
      }
      hit = __builtin_amdgcn_readfirstlane(hit);
      if (hit != INT32_MAX) return hit;
    }
    return last;
  }
};

// The next token of a row: the sum of its share x is lane x's, `share` tokens each.
template <class T, bool GIVEN, int TH>
__device__ __forceinline__ int32_t pick(Rest<T, GIVEN, TH> rest, int64_t vocab, int64_t share, int shares, double sums,
                                        float sample, Scratch<TH> &lds) {
  double whole = 0.0;
  for (int x = 0; x < shares; ++x) whole += of_lane(sums, x);
  double mark = fmax((double)sample, 0.0) * whole, before = 0.0;
  int64_t from = 0, end = vocab;
  if (!uniform(whole > 0.0)) {                                    // nothing is left: from p itself
    rest.c = 0.0;
    rest.out_n = 0;
    whole = rest.sum(0, vocab, lds.sums[0]);
    mark = fmax((double)sample, 0.0) * whole;
    __syncthreads();
  } else {
    int at = -1, last = 0;
    double upto = 0.0;
    for (int x = 0; x < shares; ++x) {
      const double s = of_lane(sums, x);
      if (at < 0 && uniform(upto + s > mark)) at = x, before = upto;
      if (uniform(s > 0.0)) last = x;
      upto += s;
    }
    if (at < 0) at = last, mark = INFINITY;
    from = at * share;
    end = min(from + share, vocab);
  }
  return rest.find(from, end, before, mark, lds);
}

// ONE: the whole check; otherwise the walk, whose end is left in `stop`.
template <class T, bool GIVEN, bool ONE>
__global__ __launch_bounds__(kThreadsV) void verify_kernel(int vocab, int most, ios_rows p, ios_rows q,
                                                           const int32_t *tokens, const int32_t *parent,
                                                           const int32_t *cu, const float *accept, const float *sample,
                                                           int32_t *path, int32_t *count, int32_t *next, Stop *stop) {
  __shared__ Scratch<kThreadsV> lds;
  __shared__ int32_t left_out[kMaxDrafts];
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t a = clip(cu[i], p.rows), b = clip(cu[i + 1], p.rows);
  const int m = __builtin_amdgcn_readfirstlane((int)min(max(b - a, (int64_t)0), (int64_t)most));
  int32_t *list = path + (int64_t)i * most;
  if (m == 0) {
    if (tid < most) list[tid] = -1;
    if (tid == 0) {
      count[i] = 0;
      next[i] = -1;
      if (!ONE) stop[i].row = -1;
    }
    return;
  }
  // every wave walks, draft j in lane j: the numbers that its test needs are read side by side
  const int up = lane > 0 && lane < m ? parent[a + lane] : -1, x = lane < m ? tokens[a + lane] : -1;
  const bool sound = up >= 0 && up < lane && x >= 0 && x < vocab;
  const double u = lane < m ? (double)accept[a + lane] : 0.0;
  const int64_t from = a + (sound ? up : 0);
  const int col = sound ? x : 0;
  const double px = prob(((const T *)p.data)[from * p.row_stride + col]);
  const double qx = GIVEN ? prob(((const T *)q.data)[from * q.row_stride + col]) : 1.0;
  int node = 0, n = 1, turn = 0;
  int mine = 0;                                                   // lane j: place j of the path
  double C = 0.0, S = 1.0, left_sum = 0.0;
  bool summed = false;                                            // left_sum is what is left of the node's row
  auto rest = [&](int out_n) {
    const int64_t row = a + node;
    return Rest<T, GIVEN, kThreadsV>{(const T *)p.data + row * p.row_stride, (const T *)q.data + row * q.row_stride, C, left_out, out_n};
  };
  uint64_t gone = 0, children = __ballot(sound && up == 0);
  while (children) {
    const int j = __builtin_ctzll(children);
    const double pj = of_lane(px, j), qj = of_lane(qx, j);
    const int xj = of_lane(x, j);
    const double left = GIVEN ? fmax(fma(-C, qj, pj), 0.0) : __ballot(x == xj) & gone ? 0.0 : pj;
    children &= children - 1;
    if (uniform(of_lane(u, j) * S * qj < left)) {
      node = j;
      mine = lane == n ? j : mine;
      ++n;
      C = 0.0;
      S = 1.0;
      summed = false;
      gone = 0;
      children = __ballot(sound && up == node);
    } else if (GIVEN) {
      if (uniform(S > 0.0)) {
        C += S;
        summed = children != 0;
        if (summed) {                                             // another child to try
          S = left_sum = rest(0).sum(0, vocab, lds.sums[turn]);
          turn ^= 1;
        }
      }
    } else {
      S -= left;
      gone |= 1ull << j;
    }
  }
  const int out_n = GIVEN ? 0 : __builtin_popcountll(gone);       // tokens that are left out of the draw
  if (wave == 0) {
    if (!GIVEN && (gone >> lane & 1)) {
      const int at = __builtin_popcountll(gone & ((1ull << lane) - 1));
      if (ONE) left_out[at] = x;
      else stop[i].out[at] = x;
    }
    if (lane < most) list[lane] = lane < n ? (int32_t)(a + mine) : -1;
    if (lane == 0) {
      count[i] = n;
      if (!ONE) {
        stop[i].c = C;
        stop[i].row = a + node;
        stop[i].out_n = out_n;
        stop[i].done = 0;
      }
    }
  }
  if (!ONE) return;
  __syncthreads();                                                // left_out
  const Rest<T, GIVEN, kThreadsV> r = rest(out_n);
  if (!summed) {
    left_sum = r.sum(0, vocab, lds.sums[turn]);
    __syncthreads();
  }
  const int32_t t = pick(r, (int64_t)vocab, (int64_t)vocab, 1, left_sum, sample[i], lds);
  if (tid == 0) next[i] = t;
}

template <class T, bool GIVEN>
__global__ __launch_bounds__(kThreadsD) void verify_draw_kernel(int vocab, int share, ios_rows p, ios_rows q,
                                                                const float *sample, int32_t *next, Stop *stop) {
  __shared__ Scratch<kThreadsD> lds;
  __shared__ int32_t left_out[kMaxDrafts], last;
  const int i = blockIdx.y, tid = threadIdx.x, shares = gridDim.x;
  Stop &st = stop[i];
  const int64_t row = st.row;
  if (row < 0) return;
  const int out_n = GIVEN ? 0 : st.out_n;
  if (tid < out_n) left_out[tid] = st.out[tid];
  __syncthreads();
  const Rest<T, GIVEN, kThreadsD> r{(const T *)p.data + row * p.row_stride, (const T *)q.data + row * q.row_stride, st.c, left_out, out_n};
  const int64_t from = (int64_t)blockIdx.x * share;
  const double s = r.sum(from, min(from + share, (int64_t)vocab), lds.sums[0]);
  if (tid == 0) {
    // the sum before the count, and no more than that: an exchange has happened for the whole device once its old value is
    // back (a release would write back all that the L2s hold, for every share)
    const double old = __hip_atomic_exchange(&st.sums[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::"v"(old) : "memory");
    last = __hip_atomic_fetch_add(&st.done, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == shares - 1;
  }
  __syncthreads();
  if (!last) return;
  static_assert(kMaxShares <= 64, "a lane for each share");
  const double sums = __hip_atomic_load(&st.sums[min(tid & 63, shares - 1)], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int32_t t = pick(r, (int64_t)vocab, (int64_t)share, shares, sums, sample[i], lds);
  if (tid == 0) next[i] = t;
}

// Workgroups that sum a row: one (and no second launch) for a small vocabulary.
int shares_of(const ios_verify_desc &d) {
  if (d.vocab < 2 * kThreadsV * 8) return 1;
  const int64_t want = (512 + d.seqs - 1) / d.seqs;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, kMaxShares), d.vocab / (kThreadsD * 8)));
}

}  // namespace

int64_t verify_bytes(const ios_verify_desc &d) { return shares_of(d) > 1 ? (int64_t)sizeof(Stop) * d.seqs : 0; }

hipError_t launch_verify(const ios_verify_desc &d, const ios_rows &p, const ios_rows *q, const int32_t *tokens,
                         const int32_t *parent, const int32_t *cu, const float *accept, const float *sample,
                         int32_t *path, int32_t *count, int32_t *next, void *work, hipStream_t s) {
  const int shares = shares_of(d);
  const ios_rows none{};
  auto run = [&](auto t, auto given) {
    using T = decltype(t);
    constexpr bool GIVEN = decltype(given)::value;
    Stop *stop = (Stop *)work;
    const ios_rows &qq = q ? *q : none;
    if (shares == 1) {
      hipLaunchKernelGGL((verify_kernel<T, GIVEN, true>), dim3(d.seqs), dim3(kThreadsV), 0, s, d.vocab, d.max_drafts, p, qq,
                         tokens, parent, cu, accept, sample, path, count, next, stop);
      return hipGetLastError();
    }
    hipLaunchKernelGGL((verify_kernel<T, GIVEN, false>), dim3(d.seqs), dim3(kThreadsV), 0, s, d.vocab, d.max_drafts, p, qq,
                       tokens, parent, cu, accept, sample, path, count, next, stop);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int share = (int)((((int64_t)d.vocab + shares - 1) / shares + 7) / 8 * 8);
    hipLaunchKernelGGL((verify_draw_kernel<T, GIVEN>), dim3(shares, d.seqs), dim3(kThreadsD), 0, s, d.vocab, share, p, qq,
                       sample, next, stop);
    return hipGetLastError();
  };
  auto go = [&](auto t) { return q ? run(t, std::true_type{}) : run(t, std::false_type{}); };
  if (d.dtype == IOS_F32) return go(float{});
  if (d.dtype == IOS_F16) return go(_Float16{});
  return go(__bf16{});
}

}  // namespace ios
