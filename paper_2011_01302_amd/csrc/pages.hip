// The pages of the key-value cache: taking, sharing, freeing, compacting and
// copying them (ios_cache_reserve, _fork, _free, _compact, _copy), on the
// device, so that a decoder's steps need no host.
//
// The bookkeeping is integers whose result does not depend on the order in
// which threads run: ids are handed out by prefix sums, counts are added to
// atomically.  Reserve and compact need the whole of refs (4 bytes a page):
// one workgroup reads it once.  Page contents move in a second launch over
// the list that the first one leaves, bound by memory.  16 sequences over 512
// pages: reserve 7.5 us, fork 2.8, free 3.1; compacting 512 pages of 8 layers and
// 8 heads of 128: 5 us for the lists, 32 for the contents (72 MB read and written;
// 23 if the pool stays in the 256 MB cache).
#include "decoder.h"

namespace ios {

namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
constexpr int kScanThreads = 1024;
constexpr int kCopyBytes = 16384;        // of one piece of a page, by one workgroup
constexpr int kCopyGrid = 2048;

// Exclusive prefix sum over the workgroup's 1024 threads; *total receives the
// sum.  red: 16 ints of LDS.
__device__ __forceinline__ int block_scan(int v, int *red, int *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = v;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(s, m);
    if (lane >= m) s += o;
  }
  __syncthreads();                       // red may still be read from the scan before
  if (lane == 63) red[wave] = s;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kScanThreads / 64; ++w) {
    const int r = red[w];
    before += w < wave ? r : 0;
    all += r;
  }
  *total = all;
  return before + s - v;
}

struct PageWork {
  int32_t *flags, *copies, *live, *count, *last, *src, *dst, *offs;
  __device__ PageWork(const ios_cache &c) {
    int32_t *w = (int32_t *)c.work;
    flags = w + CW_FLAGS;
    copies = w + CW_COPIES;
    live = w + CW_LIVE;
    count = w + CW_HEAD;                 // also: new id of a page that moves
    last = count + c.pages;              // also: list of free pages
    src = last + c.pages;
    dst = src + c.pages;
    offs = dst + c.pages;                // [slots] offset into the free list, [slots] of copies
  }
};

// What ios_cache_reserve does for one sequence, from the state before it.
struct Need {
  int slot, len, add, shared;            // shared: its last page, partly filled and shared, else -1
  int old_pages, new_pages;
};
__device__ __forceinline__ Need need_of(const ios_cache &c, int lg, const int32_t *seqs, const int32_t *add, int i) {
  Need d{seqs[i], 0, add[i], -1, 0, 0};
  if ((unsigned)d.slot >= (unsigned)c.slots || d.add <= 0) {
    d.slot = -1;
    return d;
  }
  d.len = (int)clip(c.lens[d.slot], (int64_t)c.row << lg);
  const int64_t end = (int64_t)d.len + d.add, t = (1 << lg) - 1;
  d.old_pages = (int)(((int64_t)d.len + t) >> lg);
  d.new_pages = (int)((end + t) >> lg);
  if (d.len & t) {
    const int p = c.table[(int64_t)d.slot * c.row + d.old_pages - 1];
    if ((unsigned)p < (unsigned)c.pages && c.refs[p] > 1) d.shared = p;
  }
  return d;
}

// One workgroup.  Sequences are taken kScanThreads at a time, in the order of
// the call; the free pages are found by a count per thread over a run of
// pages and a prefix sum.
__global__ __launch_bounds__(kScanThreads) void cache_reserve_kernel(ios_cache c, int lg, int n, const int32_t *seqs,
                                                                     const int32_t *add) {
  __shared__ int red[kScanThreads / 64];
  const int tid = threadIdx.x;
  const PageWork w(c);
  // nothing that it reads changes before the last step; each thread keeps its first sequence's
  const Need own = tid < n ? need_of(c, lg, seqs, add, tid) : Need{-1, 0, 0, -1, 0, 0};
  auto of = [&](int i) { return i == tid ? own : need_of(c, lg, seqs, add, i); };
  // which sequences share their last page, and which of them comes last
  for (int i = tid; i < n; i += kScanThreads) {
    const Need d = of(i);
    if (d.shared >= 0) {
      w.count[d.shared] = 0;
      w.last[d.shared] = -1;
    }
  }
  __syncthreads();
  for (int i = tid; i < n; i += kScanThreads) {
    const Need d = of(i);
    if (d.shared >= 0) {
      atomicAdd(&w.count[d.shared], 1);
      atomicMax(&w.last[d.shared], i);
    }
  }
  __syncthreads();
  // atomics are carried out in L2, past this workgroup's L1
  auto copies = [&](const Need &d, int i) {
    if (d.shared < 0) return 0;
    const int cnt = __hip_atomic_load(&w.count[d.shared], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int lst = __hip_atomic_load(&w.last[d.shared], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return cnt == c.refs[d.shared] && lst == i ? 0 : 1;
  };
  int total = 0, n_copies = 0, over = 0;
  for (int i0 = 0; i0 < n; i0 += kScanThreads) {
    const int i = i0 + tid;
    int need = 0, cp = 0;
    if (i < n) {
      const Need d = of(i);
      if (d.slot >= 0) {
        cp = copies(d, i);
        over |= d.new_pages > c.row;
        need = d.new_pages > c.row ? 0 : d.new_pages - d.old_pages + cp;
      }
    }
    int sum, csum;
    const int off = block_scan(need, red, &sum), coff = block_scan(cp, red, &csum);
    if (i < n) {
      w.offs[i] = total + off;
      w.offs[c.slots + i] = n_copies + coff;
    }
    total += sum;
    n_copies += csum;
  }
  over = __syncthreads_or(over);
  // free pages of this thread's run
  const int run = ((c.pages + kScanThreads - 1) / kScanThreads + 3) & ~3;
  const int p0 = min(tid * run, c.pages), p1 = min(p0 + run, c.pages);
  int mine = 0;
  for (int p = p0; p < p1; ++p) mine += c.refs[p] == 0;
  int avail;
  const int rank = block_scan(mine, red, &avail);
  const bool ok = !over && total <= avail;
  if (tid == 0) {
    *w.copies = ok ? n_copies : 0;
    if (!ok) atomicOr(w.flags, (over ? CACHE_NO_ENTRIES : 0) | (total > avail ? CACHE_NO_PAGES : 0));
  }
  if (!ok) return;
  int32_t *list = w.last;                                    // free, the scans have passed since it was read
  for (int p = p0, r = rank; p < p1 && r < total; ++p)
    if (c.refs[p] == 0) list[r++] = p;
  __syncthreads();
  for (int i = tid; i < n; i += kScanThreads) {
    // lens, table and refs of this sequence are still as they were: distinct slots, and a shared page's
    // count was compared above
    const Need d = of(i);
    if (d.slot < 0) continue;
    int at = w.offs[i];
    const int next = i + 1 < n ? w.offs[i + 1] : total;
    const bool copy = next - at > d.new_pages - d.old_pages;
    int32_t *row = c.table + (int64_t)d.slot * c.row;
    if (copy) {
      const int p = list[at++], k = w.offs[c.slots + i];
      w.src[k] = row[d.old_pages - 1];
      w.dst[k] = p;
      row[d.old_pages - 1] = p;
      c.refs[p] = 1;
    }
    for (int j = d.old_pages; j < d.new_pages; ++j) {
      const int p = list[at++];
      row[j] = p;
      c.refs[p] = 1;
    }
    c.lens[d.slot] = d.len + d.add;
  }
  __syncthreads();
  for (int k = tid; k < n_copies; k += kScanThreads) atomicSub(&c.refs[w.src[k]], 1);
}

// refs is only counted up, so the order of the pairs does not matter.
__global__ __launch_bounds__(256) void cache_fork_kernel(ios_cache c, int lg, const int32_t *parents,
                                                         const int32_t *children) {
  const int parent = parents[blockIdx.x], child = children[blockIdx.x];
  if ((unsigned)parent >= (unsigned)c.slots || (unsigned)child >= (unsigned)c.slots || parent == child) return;
  if (c.lens[child] != 0) {
    if (threadIdx.x == 0) atomicOr((int32_t *)c.work + CW_FLAGS, (int)CACHE_CHILD_USED);
    return;
  }
  const int len = (int)clip(c.lens[parent], (int64_t)c.row << lg);
  const int used = (int)(((int64_t)len + (1 << lg) - 1) >> lg);
  const int32_t *from = c.table + (int64_t)parent * c.row;
  int32_t *to = c.table + (int64_t)child * c.row;
  for (int j = threadIdx.x; j < used; j += 256) {
    const int p = from[j];
    to[j] = p;
    if ((unsigned)p < (unsigned)c.pages) atomicAdd(&c.refs[p], 1);
  }
  __syncthreads();                                           // every thread has seen that the child was empty
  if (threadIdx.x == 0) c.lens[child] = len;
}

__global__ __launch_bounds__(256) void cache_free_kernel(ios_cache c, int lg, const int32_t *seqs) {
  __shared__ int len_s;
  const int slot = seqs[blockIdx.x];
  if ((unsigned)slot >= (unsigned)c.slots) return;
  if (threadIdx.x == 0) len_s = atomicExch(&c.lens[slot], 0);  // a slot named twice is freed once
  __syncthreads();
  const int len = (int)clip(len_s, (int64_t)c.row << lg);
  const int used = (int)(((int64_t)len + (1 << lg) - 1) >> lg);
  int32_t *row = c.table + (int64_t)slot * c.row;
  for (int j = threadIdx.x; j < used; j += 256) {
    const int p = row[j];
    row[j] = -1;
    if ((unsigned)p < (unsigned)c.pages) atomicSub(&c.refs[p], 1);
  }
}

// One workgroup: the lists of pages that move and of the holes they move to,
// and each mover's new id (count[]).
__global__ __launch_bounds__(kScanThreads) void cache_compact_kernel(ios_cache c, int32_t *live) {
  __shared__ int red[kScanThreads / 64];
  const int tid = threadIdx.x;
  const PageWork w(c);
  const int run = ((c.pages + kScanThreads - 1) / kScanThreads + 3) & ~3;
  const int p0 = min(tid * run, c.pages), p1 = min(p0 + run, c.pages);
  int used = 0, n_live, holes, movers;
  for (int p = p0; p < p1; ++p) used += c.refs[p] != 0;
  block_scan(used, red, &n_live);
  int h = 0, m = 0;
  for (int p = p0; p < p1; ++p) {
    const bool u = c.refs[p] != 0;
    h += !u && p < n_live;
    m += u && p >= n_live;
  }
  int hr = block_scan(h, red, &holes), mr = block_scan(m, red, &movers);   // holes == movers
  for (int p = p0; p < p1; ++p) {
    const bool u = c.refs[p] != 0;
    if (!u && p < n_live) w.dst[hr++] = p;
    if (u && p >= n_live) w.src[mr++] = p;
  }
  __syncthreads();
  for (int k = tid; k < movers; k += kScanThreads) {
    const int a = w.src[k], b = w.dst[k];
    w.count[a] = b;
    c.refs[b] = c.refs[a];
    c.refs[a] = 0;
  }
  if (tid == 0) {
    *w.copies = movers;
    *w.live = n_live;
    if (live) *live = n_live;
  }
}

// Piece `item` of the contents of n pairs of pages in every layer.
__device__ __forceinline__ void copy_piece(const ios_cache &c, int64_t page_bytes, int pieces, int64_t item,
                                           const int32_t *src, const int32_t *dst) {
  const int piece = (int)(item % pieces);
  const int64_t rest = item / pieces;
  const int layer = (int)(rest % c.layers), k = (int)(rest / c.layers);
  const int a = src[k], b = dst[k];
  if ((unsigned)a >= (unsigned)c.pages || (unsigned)b >= (unsigned)c.pages) return;
  const int64_t base = (int64_t)layer * c.pages * page_bytes, off = (int64_t)piece * kCopyBytes;
  const uintx4 *from = (const uintx4 *)((unsigned char *)c.pool + base + a * page_bytes + off);
  uintx4 *to = (uintx4 *)((unsigned char *)c.pool + base + b * page_bytes + off);
  const int64_t left = page_bytes - off;
  const int words = (int)(left < kCopyBytes ? left : kCopyBytes) / 16;
#pragma unroll
  for (int i = 0; i < kCopyBytes / 16 / 256; ++i) {
    const int x = threadIdx.x + 256 * i;
    if (x < words) to[x] = from[x];
  }
}

// n < 0: the workspace's list and its count; entries of the table are moved too
// where `slots` > 0.
__global__ __launch_bounds__(256) void cache_copy_kernel(ios_cache c, int64_t page_bytes, int n, const int32_t *src,
                                                         const int32_t *dst, int64_t entries) {
  const PageWork w(c);
  if (n < 0) {
    n = *w.copies;
    src = w.src;
    dst = w.dst;
  }
  const int pieces = (int)((page_bytes + kCopyBytes - 1) / kCopyBytes);
  const int64_t items = (int64_t)n * c.layers * pieces;
  if (n > 0 && entries > 0) {
    const int live = *w.live;
    for (int64_t e = blockIdx.x * 256 + threadIdx.x; e < entries; e += (int64_t)gridDim.x * 256) {
      const int p = c.table[e];
      if (p >= live && p < c.pages) c.table[e] = w.count[p];
    }
  }
  for (int64_t i = blockIdx.x; i < items; i += gridDim.x) copy_piece(c, page_bytes, pieces, i, src, dst);
}

int page_lg(const ios_cache &c) {
  int lg = 5;
  while ((1 << lg) < c.page_tokens) ++lg;
  return lg;
}

}  // namespace

hipError_t launch_reserve(const ios_cache &c, int64_t page_bytes, int n, const int32_t *seqs, const int32_t *add,
                          hipStream_t s) {
  hipLaunchKernelGGL(cache_reserve_kernel, dim3(1), dim3(kScanThreads), 0, s, c, page_lg(c), n, seqs, add);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t items = (int64_t)n * c.layers * ((page_bytes + kCopyBytes - 1) / kCopyBytes);
  hipLaunchKernelGGL(cache_copy_kernel, dim3((unsigned)std::min<int64_t>(items, kCopyGrid)), dim3(256), 0, s, c,
                     page_bytes, -1, nullptr, nullptr, (int64_t)0);
  return hipGetLastError();
}

hipError_t launch_fork(const ios_cache &c, int n, const int32_t *parents, const int32_t *children, hipStream_t s) {
  hipLaunchKernelGGL(cache_fork_kernel, dim3(n), dim3(256), 0, s, c, page_lg(c), parents, children);
  return hipGetLastError();
}

hipError_t launch_free(const ios_cache &c, int n, const int32_t *seqs, hipStream_t s) {
  hipLaunchKernelGGL(cache_free_kernel, dim3(n), dim3(256), 0, s, c, page_lg(c), seqs);
  return hipGetLastError();
}

hipError_t launch_compact(const ios_cache &c, int64_t page_bytes, int32_t *live, hipStream_t s) {
  hipLaunchKernelGGL(cache_compact_kernel, dim3(1), dim3(kScanThreads), 0, s, c, live);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(cache_copy_kernel, dim3(kCopyGrid), dim3(256), 0, s, c, page_bytes, -1, nullptr, nullptr,
                     (int64_t)c.slots * c.row);
  return hipGetLastError();
}

hipError_t launch_copy(const ios_cache &c, int64_t page_bytes, int n, const int32_t *src, const int32_t *dst,
                       hipStream_t s) {
  const int64_t items = (int64_t)n * c.layers * ((page_bytes + kCopyBytes - 1) / kCopyBytes);
  hipLaunchKernelGGL(cache_copy_kernel, dim3((unsigned)std::min<int64_t>(items, kCopyGrid)), dim3(256), 0, s, c,
                     page_bytes, n, src, dst, (int64_t)0);
  return hipGetLastError();
}

}  // namespace ios
