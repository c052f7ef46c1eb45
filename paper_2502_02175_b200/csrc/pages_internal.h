// Shared by the translation units of the paged K/V pool (pages.cu) and of the attention that reads it
// (prefix_attention.cu).
#pragma once
#include "vlac_internal.h"
#include <limits.h>

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

// elements of one K (or V) row of the pool, and of one layer
static inline size_t pages_row(const vlac_pages* p) { return (size_t)p->n_kv_heads * p->head_dim; }
static inline size_t pages_layer(const vlac_pages* p) { return (size_t)p->n_pages * p->page_size * pages_row(p); }

__device__ __forceinline__ void cluster_sync_all() {
  __syncwarp();                                 // (the aligned form wants whole warps, also after loops whose lanes ended apart)
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
