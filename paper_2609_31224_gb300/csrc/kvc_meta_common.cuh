// What the bookkeeping kernels share: scans and maxima over a CTA, and the page allocator.
#pragma once

#include "kvc_launch.cuh"

namespace kvc {

namespace {

constexpr int META_THREADS = 1024;
constexpr unsigned FULL = 0xFFFFFFFFu;

__device__ inline unsigned lanemask_lt() {
  unsigned m;
  asm("mov.u32 %0, %%lanemask_lt;" : "=r"(m));
  return m;
}
__device__ inline unsigned lanemask_le() {
  unsigned m;
  asm("mov.u32 %0, %%lanemask_le;" : "=r"(m));
  return m;
}

// Block-wide exclusive scan of one int per thread (blockDim.x == 1024).
__device__ int block_exclusive_scan(int v, int* total, int* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    int y = __shfl_up_sync(FULL, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int w = s_warp[lane];
    int xs = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      int y = __shfl_up_sync(FULL, xs, o);
      if (lane >= o) xs += y;
    }
    s_warp[lane] = xs - w;  // exclusive warp offsets
    if (lane == 31) s_warp[32] = xs;
  }
  __syncthreads();
  int r = s_warp[warp] + x - v;
  *total = s_warp[32];
  __syncthreads();
  return r;
}

__device__ int block_max(int v, int* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(FULL, v, o));
  if (lane == 0) s_warp[warp] = v;
  __syncthreads();
  if (warp == 0) {
    int w = s_warp[lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) w = max(w, __shfl_xor_sync(FULL, w, o));
    if (lane == 0) s_warp[32] = w;
  }
  __syncthreads();
  int r = s_warp[32];
  __syncthreads();
  return r;
}

// Take the k lowest free page ids, mark them used and write them, ascending,
// to d.alloc_list[0..k).  Returns false (and marks nothing) if fewer than k
// pages are free.  Block-uniform result.  The search starts at the first bitmap word
// that can hold a free page: an allocation leaves none below its last one, freeing lowers
// the mark (free_page).
__device__ bool block_alloc_lowest(const Dev& d, int k, int* s_warp) {
  __shared__ int s_found;
  if (k == 0) return true;
  if (threadIdx.x == 0) s_found = 0;
  __syncthreads();
  for (int w0 = d.g->free_word; w0 < d.bitmap_words; w0 += META_THREADS) {
    const int w = w0 + threadIdx.x;
    uint32_t freebits = 0;
    if (w < d.bitmap_words) {
      freebits = ~d.bitmap[w];
      const int64_t first = (int64_t)w * 32;
      if (first + 32 > d.n_pages) {
        const int valid = (int)(d.n_pages - first);
        freebits &= (valid >= 32) ? 0xFFFFFFFFu : ((1u << valid) - 1u);
      }
    }
    int total;
    const int found = s_found;
    const int base = found + block_exclusive_scan(__popc(freebits), &total, s_warp);
    if (w < d.bitmap_words && base < k && freebits) {
      uint32_t take = 0;
      int idx = base;
      uint32_t fb = freebits;
      while (fb && idx < k) {
        const int bit = __ffs(fb) - 1;
        fb &= fb - 1;
        d.alloc_list[idx++] = w * 32 + bit;
        take |= 1u << bit;
      }
      d.bitmap[w] |= take;
    }
    __syncthreads();
    if (threadIdx.x == 0) s_found = min(k, found + total);
    __syncthreads();
    if (s_found >= k) {
      if (threadIdx.x == 0) d.g->free_word = d.alloc_list[k - 1] >> 5;
      return true;
    }
  }
  // Not enough pages: roll back what was marked.
  const int got = s_found;
  for (int i = threadIdx.x; i < got; i += META_THREADS) {
    const int p = d.alloc_list[i];
    atomicAnd(&d.bitmap[p >> 5], ~(1u << (p & 31)));
  }
  __syncthreads();
  return false;
}

__device__ inline void free_page(const Dev& d, int p) {
  atomicAnd(&d.bitmap[p >> 5], ~(1u << (p & 31)));
  atomicMin(&d.g->free_word, p >> 5);
}

}  // namespace

}  // namespace kvc
