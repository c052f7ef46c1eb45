// Logits before a token is picked (vlac_logits_adjust): penalties for tokens that were there, biases, grammar masks, and the choice.
//
// A row is shared by a cluster of CTAs that take its vocabulary in chunks.  For a chunk, what is said of single tokens (history, drafted
// ancestors, biases) is first gathered into a table in shared memory with integer atomics, whose order changes nothing; then the chunk's
// logits, which were asked for before that, pass through it once.  Bound: HBM, the logits read once and written once.
#include "pages_internal.h"
#include "launch_util.h"
#include <cuda_fp16.h>

namespace {

constexpr int LG_THREADS = 512, LG_EACH = 8, LG_CHUNK = LG_THREADS * LG_EACH, LG_CTAS = 8;
constexpr unsigned LG_SEEN = 0x80000000u;       // of a token's entry in the table: it was in the prompt; the other bits: how often it was generated

struct LogitsArgs {
  int rows, vocab;
  const void* in; long long stride;
  void* out; long long out_stride;
  int *picked, *status;
  vlac_logits_rules r;
  const unsigned* mask; const int *entry, *q_ptr; int n, words;         // the tree's
  int allow_words;
};

template <typename T> __device__ __forceinline__ float lg_value(T x);
template <> __device__ __forceinline__ float lg_value<float>(float x) { return x; }
template <> __device__ __forceinline__ float lg_value<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float lg_value<__half>(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T lg_round(float x);
template <> __device__ __forceinline__ float lg_round<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 lg_round<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half lg_round<__half>(float x) { return __float2half_rn(x); }

// order-preserving: a larger value has a larger key, -0 and +0 the same one, a NaN the largest; never 0
__device__ __forceinline__ unsigned lg_key(float v) {
  if (v != v) return 0xffffffffu;
  const unsigned u = __float_as_uint(v + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// VEC: rows of whole, aligned 16-byte pieces; a thread's elements are then neighbours in pieces, else 512 apart.
template <typename T, bool VEC>
__global__ void __cluster_dims__(LG_CTAS, 1, 1) __launch_bounds__(LG_THREADS) logits_kernel(LogitsArgs a) {
  constexpr int PIECE = 16 / sizeof(T), PIECES = LG_EACH / PIECE;
  __shared__ unsigned s_made[LG_CHUNK];
  __shared__ int s_bias[LG_CHUNK];              // number of the token's last entry in the row's list of biases, from 1 on
  __shared__ unsigned s_key[LG_THREADS / 32], s_at[LG_THREADS / 32];
  __shared__ unsigned s_best[LG_CTAS][2];       // of CTA 0: what the others found
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.y, rank = (int)cluster_rank();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");                   // (CTA 0 runs before anything is put into its memory)
  pdl_trigger();
  pdl_wait();
  const vlac_logits_rules& u = a.r;
  int h0 = 0, h1 = 0, h2 = 0, b0 = 0, b1 = 0, allow_row = -1, first = -1, n_seen = 0;  // rows first .. first + n_seen may be seen
  bool ok = true;
  if (u.span) { h0 = u.span[3 * row]; h1 = u.span[3 * row + 1]; h2 = u.span[3 * row + 2]; ok = 0 <= h0 && h0 <= h1 && h1 <= h2 && h2 <= u.n_tokens; }
  if (u.bias_ptr) { b0 = u.bias_ptr[row]; b1 = u.bias_ptr[row + 1]; ok = ok && 0 <= b0 && b0 <= b1 && b1 <= u.n_bias; }
  if (u.allow) { allow_row = u.allow_row ? u.allow_row[row] : row; ok = ok && -1 <= allow_row && allow_row < u.n_allow; }
  const float rep = u.repetition ? u.repetition[row] : 1.f, freq = u.frequency ? u.frequency[row] : 0.f, pres = u.presence ? u.presence[row] : 0.f;
  if (a.mask) {
    const int e = a.entry[row];
    if ((unsigned)e < (unsigned)a.n) { first = a.q_ptr[e]; n_seen = min(a.q_ptr[e + 1], a.rows); }
    if (first < 0 || first > row || n_seen <= row) first = -1;
    n_seen = first < 0 ? 0 : min(n_seen - first, a.words * 32);
  }
  if (rank == 0 && tid == 0) a.status[row] = ok ? VLAC_OK : VLAC_ERR_INVALID_ARG;
  const bool made = ok && (h2 > h0 || first >= 0), biased = ok && b1 > b0;               // is there anything to gather (uniform)
  const unsigned* allow = u.allow && allow_row >= 0 ? u.allow + (size_t)allow_row * a.allow_words : nullptr;
  const T* in = (const T*)a.in + (size_t)row * a.stride;
  T* out = a.out ? (T*)a.out + (size_t)row * a.out_stride : nullptr;
  unsigned best = 0, best_at = 0;
  for (int c0 = rank * LG_CHUNK; ok && c0 < a.vocab; c0 += LG_CTAS * LG_CHUNK) {
    const int n = min(LG_CHUNK, a.vocab - c0);
    // ---- the logits, asked for before they are needed
    __align__(16) T x[LG_EACH];
    if (VEC) {
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        const int at = (q * LG_THREADS + tid) * PIECE;
        if (at < n) *reinterpret_cast<uint4*>(x + q * PIECE) = *reinterpret_cast<const uint4*>(in + c0 + at);
      }
    } else {
#pragma unroll
      for (int q = 0; q < LG_EACH; ++q) { const int at = q * LG_THREADS + tid; if (at < n) x[q] = in[c0 + at]; }
    }
    // ---- what is said of single tokens
    if (made || biased) {
      __syncthreads();                                                  // (the table of the chunk before is read)
#pragma unroll
      for (int q = 0; q < LG_EACH; ++q) { if (made) s_made[q * LG_THREADS + tid] = 0; if (biased) s_bias[q * LG_THREADS + tid] = 0; }
      __syncthreads();
      for (int i = h0 + tid; i < h2; i += LG_THREADS) {
        const unsigned t = (unsigned)u.tokens[i] - (unsigned)c0;
        if (t < (unsigned)n) { if (i >= h1) atomicAdd(&s_made[t], 1u); else atomicOr(&s_made[t], LG_SEEN); }
      }
      if (first >= 0)
        for (int j = tid; j < n_seen; j += LG_THREADS)
          if (a.mask[(size_t)row * a.words + (j >> 5)] >> (j & 31) & 1) {
            const unsigned t = (unsigned)u.drafted[first + j] - (unsigned)c0;
            if (t < (unsigned)n) atomicAdd(&s_made[t], 1u);
          }
      if (biased)
        for (int i = b0 + tid; i < b1; i += LG_THREADS) {
          const unsigned t = (unsigned)u.bias_token[i] - (unsigned)c0;
          if (t < (unsigned)n) atomicMax(&s_bias[t], i - b0 + 1);
        }
      __syncthreads();
    }
    // ---- through it
#pragma unroll
    for (int q = 0; q < LG_EACH; ++q) {
      const int at = VEC ? ((q / PIECE) * LG_THREADS + tid) * PIECE + q % PIECE : q * LG_THREADS + tid;
      if (at >= n) continue;
      float v = lg_value<T>(x[q]);
      if (made) {
        const unsigned m = s_made[at], c = m & ~LG_SEEN;
        if (m) v = v > 0.f ? __fdiv_rn(v, rep) : __fmul_rn(v, rep);
        if (c) { v = __fsub_rn(v, __fmul_rn(freq, (float)c)); v = __fsub_rn(v, pres); }
      }
      if (biased) { const int b = s_bias[at]; if (b) v = __fadd_rn(v, u.bias[b0 + b - 1]); }
      const bool may = !allow || (allow[(c0 + at) >> 5] >> (at & 31) & 1);               // (c0 is a multiple of 32)
      if (!may) v = -INFINITY;
      x[q] = lg_round<T>(v);
      const unsigned k = may ? lg_key(v) : 0;
      if (k > best || (k == best && k && (unsigned)(c0 + at) < best_at)) { best = k; best_at = c0 + at; }
    }
    if (!out) continue;
    if (VEC) {
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        const int at = (q * LG_THREADS + tid) * PIECE;
        if (at < n) *reinterpret_cast<uint4*>(out + c0 + at) = *reinterpret_cast<const uint4*>(x + q * PIECE);
      }
    } else {
#pragma unroll
      for (int q = 0; q < LG_EACH; ++q) { const int at = q * LG_THREADS + tid; if (at < n) out[c0 + at] = x[q]; }
    }
  }
  // ---- the largest, of equal ones the lowest: warp, CTA, cluster
  auto join = [&](unsigned k, unsigned at) {
    best = __reduce_max_sync(0xffffffffu, k);
    best_at = __reduce_min_sync(0xffffffffu, k == best ? at : 0xffffffffu);
  };
  join(best, best_at);
  if (lane == 0) { s_key[warp] = best; s_at[warp] = best_at; }
  __syncthreads();
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (warp == 0) {
    const bool in_use = lane < LG_THREADS / 32;
    join(in_use ? s_key[lane] : 0, in_use ? s_at[lane] : 0xffffffffu);
    if (lane == 0) {
      unsigned to;
      asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"((unsigned)__cvta_generic_to_shared(&s_best[rank][0])));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(best) : "memory");
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + 4), "r"(best_at) : "memory");
    }
  }
  cluster_sync_all();
  if (rank == 0 && warp == 0 && ok && a.picked) {
    join(lane < LG_CTAS ? s_best[lane][0] : 0, lane < LG_CTAS ? s_best[lane][1] : 0xffffffffu);
    if (lane == 0) a.picked[row] = best ? (int)best_at : -1;
  }
}

template <typename T>
int launch_logits(const LogitsArgs& a, cudaStream_t s) {
  const bool vec = a.vocab * (long long)sizeof(T) % 16 == 0 && a.stride * (long long)sizeof(T) % 16 == 0 && !((uintptr_t)a.in & 15u) &&
                   (!a.out || (a.out_stride * (long long)sizeof(T) % 16 == 0 && !((uintptr_t)a.out & 15u)));
  VLAC_CUDA_CHECK(launch_pdl(vec ? logits_kernel<T, true> : logits_kernel<T, false>, dim3(LG_CTAS, a.rows), dim3(LG_THREADS), 0, s, a));
  return VLAC_OK;
}

}  // namespace

extern "C" int vlac_logits_adjust(int rows, int vocab, int dtype, const void* logits, long long stride, const vlac_logits_rules* rules, void* out,
                                  long long out_stride, int* picked, int* status, void* stream) {
  if (rows < 0 || vocab < 1 || vocab > 1 << 30 || (dtype != VLAC_FP32 && dtype != VLAC_BF16 && dtype != VLAC_FP16) || !rules) return VLAC_ERR_INVALID_ARG;
  if (rows > 65535) return VLAC_ERR_TOO_LARGE;
  const vlac_logits_rules& u = *rules;
  if (u.n_tokens < 0 || u.n_bias < 0 || u.n_allow < 0 || (u.span && u.n_tokens > 0 && !u.tokens)) return VLAC_ERR_INVALID_ARG;
  if (u.bias_ptr && u.n_bias > 0 && (!u.bias_token || !u.bias)) return VLAC_ERR_INVALID_ARG;
  if (u.allow && !u.allow_row && u.n_allow < rows) return VLAC_ERR_INVALID_ARG;
  if ((u.tree == nullptr) != (u.drafted == nullptr)) return VLAC_ERR_INVALID_ARG;
  const uintptr_t ints = (uintptr_t)u.tokens | (uintptr_t)u.span | (uintptr_t)u.repetition | (uintptr_t)u.frequency | (uintptr_t)u.presence | (uintptr_t)u.bias_ptr |
                         (uintptr_t)u.bias_token | (uintptr_t)u.bias | (uintptr_t)u.allow | (uintptr_t)u.allow_row | (uintptr_t)u.drafted | (uintptr_t)picked | (uintptr_t)status;
  if (ints & 3u) return VLAC_ERR_INVALID_ARG;
  LogitsArgs a = {rows, vocab, logits, stride, out, out_stride, picked, status, u};
  if (u.tree) {
    const vlac_tree* t = u.tree;
    if (t->rows != rows || t->n < 0 || t->n > VLAC_PAGES_MAX_LIST || t->max_rows < 1 || t->max_rows > VLAC_TREE_MAX_ROWS) return VLAC_ERR_INVALID_ARG;
    if (rows > 0 && t->n > 0 && (!t->mask || !t->entry || !t->q_ptr || ((uintptr_t)t->mask | (uintptr_t)t->entry | (uintptr_t)t->q_ptr) & 3u)) return VLAC_ERR_INVALID_ARG;
    if (t->n > 0) { a.mask = t->mask; a.entry = t->entry; a.q_ptr = t->q_ptr; a.n = t->n; a.words = (t->max_rows + 31) / 32; }
  }
  if (rows == 0) return VLAC_OK;
  const int size = dtype == VLAC_FP32 ? 4 : 2;
  if (!logits || !status || stride < vocab || (uintptr_t)logits & (size - 1) || (uintptr_t)out & (size - 1)) return VLAC_ERR_INVALID_ARG;
  if (out) {
    const unsigned long long w = (unsigned long long)vocab * size;
    if (out_stride < vocab) return VLAC_ERR_INVALID_ARG;
    if (!(out == logits && out_stride == stride) && rows_overlap((uintptr_t)logits, (unsigned long long)stride * size, (uintptr_t)out, (unsigned long long)out_stride * size, w, w, rows))
      return VLAC_ERR_INVALID_ARG;
  }
  a.allow_words = (int)(((long long)vocab + 31) / 32);
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == VLAC_FP32 ? launch_logits<float>(a, s) : dtype == VLAC_BF16 ? launch_logits<__nv_bfloat16>(a, s) : launch_logits<__half>(a, s);
}
