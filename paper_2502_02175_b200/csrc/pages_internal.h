// Shared by the translation units of the paged K/V pool (pages.cu), of what appends to it (rotary.cu), of the attention that reads it
// (prefix_attention.cu) and of the trees of drafted tokens over it (tree.cu).
#pragma once
#include "vlac_internal.h"
#include <limits.h>
#include <atomic>

static inline int pages_shift(int page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}

// What every entry point checks of a caller's vlac_pages before anything is launched.
static inline int pages_check(const vlac_pages* p) {
  if (!p || !p->k || !p->v || !p->table || !p->len || !p->refs || !p->work) return VLAC_ERR_INVALID_ARG;
  if (((uintptr_t)p->k | (uintptr_t)p->v) & 15u) return VLAC_ERR_INVALID_ARG;
  if (((uintptr_t)p->table | (uintptr_t)p->len | (uintptr_t)p->refs) & 3u) return VLAC_ERR_INVALID_ARG;
  if ((uintptr_t)p->refs & 15u || (uintptr_t)p->work & 15u) return VLAC_ERR_INVALID_ARG;
  if (p->dtype != VLAC_BF16 && p->dtype != VLAC_FP16) return VLAC_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return VLAC_ERR_INVALID_ARG;
  if (p->n_layers < 1 || p->n_kv_heads < 1 || p->n_kv_heads > 1024 || p->n_pages < 1 || p->n_slots < 1 || p->max_pages < 1)
    return VLAC_ERR_INVALID_ARG;
  if (p->page_size < 8 || p->page_size > 256 || (p->page_size & (p->page_size - 1))) return VLAC_ERR_INVALID_ARG;
  if ((long long)p->n_pages * p->page_size > INT_MAX || (long long)p->max_pages * p->page_size > INT_MAX) return VLAC_ERR_INVALID_ARG;
  if (p->work_bytes < vlac_pages_work_bytes(p)) return VLAC_ERR_INVALID_ARG;
  return VLAC_OK;
}

static inline int list_check(int n) {
  if (n < 0) return VLAC_ERR_INVALID_ARG;
  return n > VLAC_PAGES_MAX_LIST ? VLAC_ERR_TOO_LARGE : VLAC_OK;
}

static inline int sm_count(int* out) {
  int dev = 0;
  VLAC_CUDA_CHECK(cudaGetDevice(&dev));
  VLAC_CUDA_CHECK(cudaDeviceGetAttribute(out, cudaDevAttrMultiProcessorCount, dev));
  return VLAC_OK;
}

// Dynamic shared memory beyond 48 KB is asked for once per device and kernel.
template <auto kernel> static inline int big_smem(int bytes) {
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  VLAC_CUDA_CHECK(cudaGetDevice(&dev));
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_acquire) & bit) return VLAC_OK;
  VLAC_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  done.fetch_or(bit, std::memory_order_release);
  return VLAC_OK;
}

// Whether a row of q (row r: wq bytes from q + r * qs on) and a row of out (wo bytes) share a byte: results are written while other rows are still read.
static inline bool rows_overlap(uintptr_t q, unsigned long long qs, uintptr_t out, unsigned long long os, unsigned long long wq, unsigned long long wo, int rows) {
  const unsigned long long last = (unsigned long long)(rows - 1);
  if (q + last * qs + wq <= out || out + last * os + wo <= q) return false;
  if (qs == os) {                                 // (columns of one buffer: q's rows begin d bytes behind out's, a number of rows on)
    const unsigned long long d = q >= out ? (q - out) % qs : (qs - (out - q) % qs) % qs;
    return d < wo || qs - d < wq;
  }
  for (unsigned long long i = 0, j = 0; i <= last && j <= last;) {
    if (q + i * qs + wq <= out + j * os) ++i;
    else if (out + j * os + wo <= q + i * qs) ++j;
    else return true;
  }
  return false;
}

// elements of one K (or V) row of the pool, and of one layer
static inline size_t pages_row(const vlac_pages* p) { return (size_t)p->n_kv_heads * p->head_dim; }
static inline size_t pages_layer(const vlac_pages* p) { return (size_t)p->n_pages * p->page_size * pages_row(p); }

// Whether a row of out (row r: w bytes from out + r * stride on, stride >= w) shares a byte with [a, a + bytes).
static inline bool rows_touch(const void* at, unsigned long long bytes, const void* out, unsigned long long stride, unsigned long long w, int rows) {
  const unsigned long long a = (uintptr_t)at, o = (uintptr_t)out;
  const unsigned long long r = o + w > a ? 0 : (a - o - w) / stride + 1;                  // the first row that ends behind a
  return r < (unsigned long long)rows && o + r * stride < a + bytes;
}
// The same for K and V of the pool, in any layer.
static inline bool rows_in_pool(const vlac_pages* p, const void* out, unsigned long long stride, unsigned long long w, int rows) {
  const unsigned long long bytes = 2ull * p->n_layers * pages_layer(p);
  return rows_touch(p->k, bytes, out, stride, w, rows) || rows_touch(p->v, bytes, out, stride, w, rows);
}

__device__ __forceinline__ void cluster_sync_all() {
  __syncwarp();                                 // (the aligned form wants whole warps, also after loops whose lanes ended apart)
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
