// Logits before a token is picked (vlac_logits_adjust): penalties for tokens that were there, biases, grammar masks, and the choice.
//
// A row is shared by a cluster of CTAs, a run of the vocabulary each.  What is said of single tokens (history, drafted ancestors, biases) touches few of
// them: the CTA first goes through the row's lists, marks its tokens in a bit map and counts them in a small table; then it streams the run through once, 16
// bytes at a time with nothing but two masks to look at, and last it does the marked tokens one by one, whose logits are in L2 by then.  All gathering is
// by integer atomics, whose order changes nothing.  Bound: HBM, the logits read once and written once (512 rows of 128,000 in bf16: 51 us without lists and
// masks, 5.2 TB/s), and in front of and behind the stream the chains of a row's lists (histories of up to 2048 tokens +13 us, biases and drafted tokens
// +4 each, masks +6: 76 us).  A few rows are launch and chains: 25 of 32,000 8 us.
#include "pages_internal.h"
#include "launch_util.h"
#include <cuda_fp16.h>
#include <type_traits>

namespace {

constexpr int LG_RUN = 131072;                  // tokens whose marks a CTA holds at once
// Tokens whose counts a CTA holds: a run of at most as many by their place in it ("direct"), of a longer one the marked tokens by a hash.  Few rows: more, so
// that an eighth of 32,000 tokens is direct; many: fewer, so that four CTAs fit an SM.  A hash table that overflows, from 1000 to 1400 different tokens a CTA on, costs
// much: the rest of the CTA's share goes in direct runs, and the row's lists are gone through for each.  us, rows of 128,000 in bf16 by different tokens a row:
//   512 rows, a CTA each       1000 76    1400 248   2000 370   4000 583   8000 967
//   256 rows, two CTAs each    1000 40    2000 49    4000 287   8000 602
//   100 rows, four CTAs each   1000 20    2000 24    4000 33    8000 243
//    25 rows, eight CTAs each  1000 11    2000 12.5  4000 17    8000 25    32000 292
__host__ __device__ constexpr int lg_table(int ctas) { return ctas == 8 ? 4096 : 2048; }
constexpr int LG_TRIES = 64;                    // where a token finds no entry in as many tries, the run is cut into direct ones
constexpr int LG_LOOK = 4;                      // tokens of the history that a thread asks for at once
constexpr int LG_EACH = 2;                      // marked tokens that a thread has in flight
constexpr int LG_SMS = 148;
constexpr unsigned LG_SEEN = 0x80000000u;       // of a token's entry in the table: it was in the prompt; the other bits: how often it was generated
__host__ __device__ constexpr int lg_smem(int ctas) { return LG_RUN / 8 + lg_table(ctas) * 14; }

struct LogitsArgs {
  int rows, vocab;
  const void* in; long long stride;
  void* out; long long out_stride;
  int *picked, *status;
  vlac_logits_rules r;
  const unsigned* mask; const int *entry, *q_ptr; int n, words;         // the tree's
  int allow_words;
  int per;                                      // places of a CTA, a multiple of 64
};

// order-preserving: a larger value has a larger key, -0 and +0 the same one, a NaN the largest (an addition makes every NaN the same positive one).
// The smallest number stands for "none": no value has it.
constexpr int LG_NONE = INT_MIN;
__device__ __forceinline__ int lg_key(float v) {
  const int s = __float_as_int(v + 0.0f);
  return s ^ ((s >> 31) & 0x7fffffff);
}
__device__ __forceinline__ unsigned lg_hash(unsigned t, int table) { return __umulhi(t * 2654435769u, (unsigned)table); }      // (Knuth's multiplicative hash)
__device__ __forceinline__ float lg_max(float a, float b) { float d; asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b)); return d; }
// Bits b and b + 1 of the four lowest of x as masks of 16 bits side by side (b = 0 or 2): each bit to the top of a byte, and that spread out.
__device__ __forceinline__ unsigned lg_spread(unsigned x) { return (x * 0x00204081u & 0x01010101u) << 7; }
__device__ __forceinline__ unsigned lg_pair(unsigned spread, int b) {   // (a selector of 8 + i: the top bit of byte i, eight times)
  unsigned d;
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(d) : "r"(spread), "r"(b ? 0xbbaau : 0x9988u));
  return d;
}

template <typename T> struct Logit;             // one element, and two side by side
template <> struct Logit<float> {
  static __device__ __forceinline__ float value(float x) { return x; }
  static __device__ __forceinline__ float round(float x) { return x; }
};
template <> struct Logit<__nv_bfloat16> {
  static constexpr unsigned none = 0xff80ff80u; // -infinity
  static __device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 round(float x) { return __float2bfloat16_rn(x); }
  static __device__ __forceinline__ unsigned max2(unsigned a, unsigned b) { unsigned d; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
  static __device__ __forceinline__ float2 two(unsigned x) { return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
};
template <> struct Logit<__half> {
  static constexpr unsigned none = 0xfc00fc00u;
  static __device__ __forceinline__ float value(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half round(float x) { return __float2half_rn(x); }
  static __device__ __forceinline__ unsigned max2(unsigned a, unsigned b) { unsigned d; asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
  static __device__ __forceinline__ float2 two(unsigned x) { return __half22float2(*reinterpret_cast<__half2*>(&x)); }
};

// 16 bytes of logits, or one element where a row of the results is aligned otherwise than its logits
template <typename T, bool VEC> struct Piece {
  static constexpr int N = VEC ? 16 / sizeof(T) : 1;
  static constexpr unsigned ALL = (1u << N) - 1u;
  uint4 v;
  __device__ __forceinline__ void load(const T* p) {
    if (VEC) v = *reinterpret_cast<const uint4*>(p);
    else if (sizeof(T) == 4) v.x = *reinterpret_cast<const unsigned*>(p);
    else v.x = *reinterpret_cast<const unsigned short*>(p);
  }
  __device__ __forceinline__ void store(T* p) const {
    if (VEC) *reinterpret_cast<uint4*>(p) = v;
    else if (sizeof(T) == 4) *reinterpret_cast<unsigned*>(p) = v.x;
    else *reinterpret_cast<unsigned short*>(p) = (unsigned short)v.x;
  }
  __device__ __forceinline__ float value(int e) const {                 // (e is a constant where this is used)
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else { const float2 f = Logit<T>::two(w[e >> 1]); return e & 1 ? f.y : f.x; }
  }
  // -infinity in the elements outside `stay`; the largest of all so far, in two halves for 16-bit types
  using Max = std::conditional_t<sizeof(T) == 4, float, unsigned>;
  __device__ __forceinline__ void mask_and_max(unsigned stay, Max* m) {
    unsigned w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (!(stay >> e & 1)) w[e] = 0xff800000u;
        *m = lg_max(*m, __uint_as_float(w[e]));
      }
    } else {
      using L = Logit<T>;
      if (stay != ALL || !VEC) {
        const unsigned s[2] = {lg_spread(stay & 15), lg_spread(stay >> 4)};
#pragma unroll
        for (int i = 0; i < (VEC ? 4 : 1); ++i) { const unsigned k = lg_pair(s[i >> 1], i & 1); w[i] = (w[i] & k) | (L::none & ~k); }
      }
#pragma unroll
      for (int i = 0; i < (VEC ? 4 : 1); ++i) *m = L::max2(*m, w[i]);
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ Max none() { if constexpr (sizeof(T) == 4) return -INFINITY; else return Logit<T>::none; }
  static __device__ __forceinline__ float largest(Max m) {
    if constexpr (sizeof(T) == 4) return m;
    else { const float2 f = Logit<T>::two(m); return lg_max(f.x, f.y); }
  }
};

// LG_WHOLE: rows of whole, aligned 16-byte pieces.  LG_SHIFTED: a row may begin and end anywhere, its results like its logits.  Places are counted from the 16-byte boundary in front of the row, so that pieces are
// whole and aligned; token t has place t + off.  What lies in a piece that the row does not fill (at most 7 tokens at each end) is marked and done with
// the marked tokens (512 rows of 126,953 in bf16: 78 us, one element at a time 210).  LG_SINGLE: results that lie otherwise than their logits.
// CTAS share a row.  Few rows are shared by 8, so that there are enough CTAs; many by fewer, since every one of them goes through the row's lists.
enum { LG_SINGLE = 0, LG_WHOLE = 1, LG_SHIFTED = 2 };
template <typename T, int MODE, int CTAS, int LG_THREADS>
__global__ void __cluster_dims__(CTAS, 1, 1) __launch_bounds__(LG_THREADS, LG_THREADS > 256 ? 1 : CTAS == 8 ? 3 : 4) logits_kernel(LogitsArgs a) {
  constexpr bool VEC = MODE != LG_SINGLE, SHIFTED = MODE == LG_SHIFTED;
  using P = Piece<T, VEC>;
  using L = Logit<T>;
  constexpr int LG_TABLE = lg_table(CTAS), LG_WARPS = LG_THREADS / 32;
  constexpr int N = P::N, BATCH = VEC ? 2 : 8;  // pieces of a thread in flight
  extern __shared__ __align__(16) unsigned lg_raw[];
  unsigned* const s_mark = lg_raw;              // [LG_RUN / 32]
  unsigned* const s_made = s_mark + LG_RUN / 32;                        // [LG_TABLE]
  int* const s_bias = (int*)s_made + LG_TABLE;  // [LG_TABLE] number of the token's last entry in the row's list of biases, from 1 on
  int* const s_token = s_bias + LG_TABLE;       // [LG_TABLE] token + 1 of the hash's entry, 0: free
  unsigned short* const s_list = (unsigned short*)(s_token + LG_TABLE); // [LG_TABLE] the entries in use, each warp those of its share of the table
  __shared__ int s_key[LG_WARPS], s_full;
  __shared__ unsigned s_at[LG_WARPS];
  __shared__ int s_best[CTAS][2];               // of CTA 0: what the others found
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.y, rank = (int)cluster_rank();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");                   // (CTA 0 runs before anything is put into its memory)
  pdl_trigger();
  pdl_wait();
  const vlac_logits_rules& u = a.r;
  int h0 = 0, h1 = 0, h2 = 0, b0 = 0, b1 = 0, allow_row = -1, first = -1, n_seen = 0;     // rows first .. first + n_seen may be seen
  const int e = a.mask ? a.entry[row] : -1;
  bool ok = true;
  if (u.span) { h0 = u.span[3 * row]; h1 = u.span[3 * row + 1]; h2 = u.span[3 * row + 2]; ok = 0 <= h0 && h0 <= h1 && h1 <= h2 && h2 <= u.n_tokens; }
  if (u.bias_ptr) { b0 = u.bias_ptr[row]; b1 = u.bias_ptr[row + 1]; ok = ok && 0 <= b0 && b0 <= b1 && b1 <= u.n_bias; }
  if (u.allow) { allow_row = u.allow_row ? u.allow_row[row] : row; ok = ok && -1 <= allow_row && allow_row < u.n_allow; }
  const float rep = u.repetition ? u.repetition[row] : 1.f, freq = u.frequency ? u.frequency[row] : 0.f, pres = u.presence ? u.presence[row] : 0.f;
  // (the first of every list are asked for together: one after the other they would be the longest part of a call)
  int h[LG_LOOK], b = -1;
#pragma unroll
  for (int q = 0; q < LG_LOOK; ++q) { const int i = h0 + q * LG_THREADS + tid; h[q] = ok && i < h2 ? u.tokens[i] : -1; }
  if (ok && tid < b1 - b0) b = u.bias_token[b0 + tid];
  if ((unsigned)e < (unsigned)a.n) {            // (a.n is 0 without a tree)
    first = a.q_ptr[e]; n_seen = min(a.q_ptr[e + 1], a.rows);
    if (first < 0 || first > row || n_seen <= row) first = -1;
    n_seen = first < 0 ? 0 : min(n_seen - first, a.words * 32);
  }
  const int d = tid < n_seen ? u.drafted[first + tid] : -1;
  const unsigned seen = tid < n_seen ? a.mask[(size_t)row * a.words + (tid >> 5)] >> (tid & 31) & 1 : 0;
  if (rank == 0 && tid == 0) a.status[row] = ok ? VLAC_OK : VLAC_ERR_INVALID_ARG;
  const bool lists = ok && (h2 > h0 || first >= 0 || b1 > b0);                            // is anything said of single tokens (uniform)
  const unsigned char* allow = u.allow && allow_row >= 0 ? (const unsigned char*)(u.allow + (size_t)allow_row * a.allow_words) : nullptr;
  const T* const row_in = (const T*)a.in + (size_t)row * a.stride;
  const int off = SHIFTED ? (int)(((uintptr_t)row_in & 15u) / sizeof(T)) : 0, v_end = off + a.vocab;             // places of the row's tokens: off .. v_end
  const int v_lo = SHIFTED ? (off + N - 1) / N * N : 0, v_hi = SHIFTED ? v_end / N * N : v_end;              // of its whole pieces
  const T* const in = row_in - off;
  T* const out = a.out ? (T*)a.out + (size_t)row * a.out_stride - off : nullptr;
  auto allowed = [&](int place) { return !allow || (allow[(place - off) >> 3] >> ((place - off) & 7) & 1); };
  int best = LG_NONE, best1 = LG_NONE;          // largest key of the unmarked tokens, and of the marked ones
  unsigned best_at = 0, best_of = 0, best1_at = 0;                      // first place of the batch that has it, and which of the batch count; the place
  const int end = ok ? (int)min((long long)v_end, (long long)(rank + 1) * a.per) : 0;
  int most = LG_RUN;
  for (int c0 = rank * a.per, n; c0 < end; c0 += n) {
    n = min(most, end - c0);
    bool direct = n <= LG_TABLE;
    P x[BATCH];                                 // the first logits, asked for before they are needed
#pragma unroll
    for (int q = 0; q < BATCH; ++q) { const int at = c0 + (q * LG_THREADS + tid) * N; if ((!SHIFTED || at >= v_lo) && at < min(c0 + n, v_hi)) x[q].load(in + at); }
    // (the runs begin at multiples of 64: the ends' pieces lie in the row's first run and in its last)
    const bool head = SHIFTED && c0 < v_lo, any = lists || head || (SHIFTED && v_hi < v_end && c0 + n == v_end);
    // ---- what is said of which tokens
    for (bool again = any; again;) {            // (a cut run keeps `any`: its part without an end marks nothing)
      __syncthreads();                          // (what was there before is read)
      for (int i = tid * 4; i < (n + 31) >> 5; i += LG_THREADS * 4) *reinterpret_cast<uint4*>(s_mark + i) = make_uint4(0, 0, 0, 0);
      for (int i = tid * 4; i < (direct ? n : LG_TABLE); i += LG_THREADS * 4) {
        *reinterpret_cast<uint4*>(s_made + i) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(s_bias + i) = make_uint4(0, 0, 0, 0);
        if (!direct) *reinterpret_cast<uint4*>(s_token + i) = make_uint4(0, 0, 0, 0);
      }
      if (tid == 0) s_full = 0;
      __syncthreads();
      auto place = [&](unsigned t) -> int {     // the token's entry; -1: there are too many
        atomicOr(&s_mark[t >> 5], 1u << (t & 31));
        if (direct) return (int)t;
        unsigned i = lg_hash(t, LG_TABLE);
        for (int tries = 0; tries < LG_TRIES; ++tries, i = (i + 1) % LG_TABLE) {
          int had = *(volatile int*)&s_token[i];
          if (had == 0) had = atomicCAS(&s_token[i], 0, (int)t + 1);
          if (had == 0 || had == (int)t + 1) return (int)i;
        }
        s_full = 1;
        return -1;
      };
      auto count = [&](int token, bool made) {
        const unsigned t = (unsigned)token + (unsigned)off - (unsigned)c0;
        const int i = (unsigned)token < (unsigned)a.vocab && t < (unsigned)n ? place(t) : -1;
        if (i >= 0) { if (made) atomicAdd(&s_made[i], 1u); else atomicOr(&s_made[i], LG_SEEN); }
      };
      auto add = [&](int token, int number) {
        const unsigned t = (unsigned)token + (unsigned)off - (unsigned)c0;
        const int i = (unsigned)token < (unsigned)a.vocab && t < (unsigned)n ? place(t) : -1;
        if (i >= 0) atomicMax(&s_bias[i], number);
      };
#pragma unroll
      for (int q = 0; q < LG_LOOK; ++q) count(h[q], h0 + q * LG_THREADS + tid >= h1);
      for (int i0 = h0 + LG_LOOK * LG_THREADS; i0 < h2; i0 += LG_LOOK * LG_THREADS) {
        int g[LG_LOOK];
#pragma unroll
        for (int q = 0; q < LG_LOOK; ++q) { const int i = i0 + q * LG_THREADS + tid; g[q] = i < h2 ? u.tokens[i] : -1; }
#pragma unroll
        for (int q = 0; q < LG_LOOK; ++q) count(g[q], i0 + q * LG_THREADS + tid >= h1);
      }
      if (seen) count(d, true);
      for (int j = tid + LG_THREADS; j < n_seen; j += LG_THREADS)
        if (a.mask[(size_t)row * a.words + (j >> 5)] >> (j & 31) & 1) count(u.drafted[first + j], true);
      if (b >= 0) add(b, tid + 1);
      if (SHIFTED && tid < 2 * N) {                 // the ends
        const int v = tid < N ? off + tid : max(v_hi, v_lo) + tid - N;
        if (v < (tid < N ? min(v_lo, v_end) : v_end) && (unsigned)(v - c0) < (unsigned)n) place((unsigned)(v - c0));
      }
      for (int i = b0 + tid + LG_THREADS; i < b1; i += LG_THREADS) add(u.bias_token[i], i - b0 + 1);
      __syncthreads();
      again = s_full;                           // (never of a direct run)
      if (again) { most = n = LG_TABLE; direct = true; }                // (uniform; the first logits lie in the shorter run too, or are not looked at)
    }
    // ---- the run: BATCH pieces of a thread at a time, the next ones asked for in front of that.  Of a batch only the largest element is looked at; which
    // of its elements that is, is found out in the end.
    const unsigned char* mark_b = reinterpret_cast<const unsigned char*>(s_mark) + (tid * N >> 3);
    const T* from = in + c0 + tid * N;
    T* to = out ? out + c0 + tid * N : nullptr;
    constexpr int STEP = LG_THREADS * N, ALL_STEP = BATCH * STEP;       // tokens of a piece of every thread, of a batch
    const int n_vec = min(n, v_hi - c0);                                // whole pieces lie in front of this
    // bits of the mask: a piece's first token lies off behind a multiple of N, its bits in one byte or in two
    const int b_first = (c0 + tid * N - off) >> 3, b_shift = (c0 + tid * N - off) & 7, b_room = a.allow_words * 4 - 1 - b_first;
    const unsigned char* may_b = allow ? allow + b_first : nullptr;     // (of whole pieces no byte in front of the mask is read)
    auto batch = [&](int at0, auto whole) {                             // whole: every thread has BATCH whole pieces
      typename P::Max m = P::none();
      unsigned of = 0;
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const int at = at0 + q * STEP + tid * N;
        if (!decltype(whole)::value && (at >= n_vec || (SHIFTED && c0 + at < v_lo))) continue;
        unsigned stay = P::ALL;                                         // (c0 is a multiple of 32, a piece's first place one of N)
        if (may_b) {
          stay = may_b[(at0 + q * STEP) >> 3];
          if (SHIFTED) stay |= (unsigned)may_b[min(((at0 + q * STEP) >> 3) + 1, b_room)] << 8;
          if (N < 8 || SHIFTED) stay = stay >> b_shift & P::ALL;
        }
        unsigned mark = any ? mark_b[(at0 + q * STEP) >> 3] : 0;
        if (N < 8) mark = mark >> (tid * N & 7) & P::ALL;
        of |= (stay & ~mark) << q * N;
        P y = x[q];
        y.mask_and_max(stay & ~mark, &m);
        if (mark & stay) { typename P::Max none; y = x[q]; y.mask_and_max(stay, &none); }  // (a marked token stays as it is, where out is in)
        if (to) y.store(to + at0 + q * STEP);
      }
      const int k = lg_key(P::largest(m));
      if (k > best && of) { best = k; best_at = c0 + at0 + tid * N; best_of = of; }        // (ascending: of equal ones the first stays)
    };
    for (int at0 = 0; at0 < n_vec; at0 += ALL_STEP) {
      P y[BATCH];
      if (at0 + 2 * ALL_STEP <= n_vec && (at0 > 0 || !head)) {
#pragma unroll
        for (int q = 0; q < BATCH; ++q) y[q].load(from + at0 + ALL_STEP + q * STEP);
        batch(at0, std::true_type());
      } else {
#pragma unroll
        for (int q = 0; q < BATCH; ++q) if (at0 + ALL_STEP + q * STEP + tid * N < n_vec) y[q].load(from + at0 + ALL_STEP + q * STEP);
        batch(at0, std::false_type());
      }
#pragma unroll
      for (int q = 0; q < BATCH; ++q) x[q] = y[q];
    }
    // ---- the marked tokens: every warp collects those of its share of the table and does them, LG_EACH a lane at a time
    if (any) {
      constexpr int SHARE = LG_TABLE / LG_WARPS;
      unsigned short* const mine = s_list + warp * SHARE;
      int used = 0;
      for (int i0 = warp * SHARE; i0 < min((warp + 1) * SHARE, direct ? n : LG_TABLE); i0 += 32) {
        const bool in_use = direct ? s_mark[i0 >> 5] >> lane & 1 : s_token[i0 + lane] != 0;
        const unsigned b = __ballot_sync(0xffffffffu, in_use);
        if (in_use) mine[used + __popc(b & ((1u << lane) - 1))] = (unsigned short)(i0 + lane);
        used += __popc(b);
      }
      __syncthreads();                          // (the run is written: what comes now lies over it)
      for (int j0 = lane; j0 < used; j0 += 32 * LG_EACH) {
        int at[LG_EACH], number[LG_EACH];
        unsigned made[LG_EACH];
        float v[LG_EACH], add[LG_EACH];
        bool may[LG_EACH];
#pragma unroll
        for (int q = 0; q < LG_EACH; ++q) {
          const int j = j0 + q * 32, i = mine[min(j, used - 1)];
          at[q] = c0 + (direct ? i : s_token[i] - 1);
          made[q] = s_made[i]; number[q] = s_bias[i];
          v[q] = L::value(in[at[q]]);
          may[q] = allowed(at[q]);
          add[q] = number[q] ? u.bias[b0 + number[q] - 1] : 0.f;
        }
#pragma unroll
        for (int q = 0; q < LG_EACH; ++q) {
          if (j0 + q * 32 >= used || (!SHIFTED && !may[q])) continue;   // (in whole pieces what is not allowed is written already)
          const unsigned c = made[q] & ~LG_SEEN;
          float y = v[q];
          if (made[q]) y = y > 0.f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
          if (c) { y = __fsub_rn(y, __fmul_rn(freq, (float)c)); y = __fsub_rn(y, pres); }
          if (number[q]) y = __fadd_rn(y, add[q]);
          if (out) out[at[q]] = L::round(may[q] ? y : -INFINITY);
          const int k = may[q] ? lg_key(y) : LG_NONE;
          if (k > best1 || (k == best1 && (unsigned)at[q] < best1_at)) { best1 = k; best1_at = at[q]; }
        }
      }
    }
  }
  // ---- the largest, of equal ones the lowest: CTA, then cluster
  int top = __reduce_max_sync(0xffffffffu, max(best, best1));
  if (lane == 0) s_key[warp] = top;
  __syncthreads();
  top = LG_NONE;
#pragma unroll
  for (int w = 0; w < LG_WARPS; ++w) top = max(top, s_key[w]);
  unsigned at = best1 == top ? best1_at : 0xffffffffu;
  if (best == top && top != LG_NONE) {          // which of its batch (what counts was stored as it was)
    P z[BATCH];
#pragma unroll
    for (int q = 0; q < BATCH; ++q) if (best_of >> q * N & P::ALL) z[q].load(in + best_at + q * LG_THREADS * N);
#pragma unroll
    for (int q = BATCH - 1; q >= 0; --q)
#pragma unroll
      for (int e = N - 1; e >= 0; --e)
        if (best_of >> (q * N + e) & 1 && lg_key(z[q].value(e)) == top) at = min(at, best_at + q * LG_THREADS * N + e);
  }
  at = __reduce_min_sync(0xffffffffu, at);
  if (lane == 0) s_at[warp] = at;
  __syncthreads();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (warp == 0) {
    at = __reduce_min_sync(0xffffffffu, lane < LG_WARPS ? s_at[lane] : 0xffffffffu);
    if (lane == 0) {
      unsigned to;
      asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"((unsigned)__cvta_generic_to_shared(&s_best[rank][0])));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(top) : "memory");
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + 4), "r"(at) : "memory");
    }
  }
  cluster_sync_all();
  if (rank == 0 && warp == 0 && ok && a.picked) {
    const int k = lane < CTAS ? s_best[lane][0] : LG_NONE;
    top = __reduce_max_sync(0xffffffffu, k);
    at = __reduce_min_sync(0xffffffffu, k == top && lane < CTAS ? (unsigned)s_best[lane][1] : 0xffffffffu);
    if (lane == 0) a.picked[row] = top != LG_NONE ? (int)at - off : -1;
  }
}

template <typename T, int MODE, int CTAS, int THREADS>
int launch_logits(LogitsArgs a, cudaStream_t s) {
  a.per = (int)(((long long)a.vocab + (MODE == LG_SHIFTED ? 7 : 0) + CTAS * 64 - 1) / (CTAS * 64) * 64);  // (places: up to 7 more than tokens)
  const int rc = big_smem<logits_kernel<T, MODE, CTAS, THREADS>>(lg_smem(CTAS));
  if (rc != VLAC_OK) return rc;
  VLAC_CUDA_CHECK(launch_pdl(logits_kernel<T, MODE, CTAS, THREADS>, dim3(CTAS, a.rows), dim3(THREADS), lg_smem(CTAS), s, a));
  return VLAC_OK;
}
template <typename T, int CTAS, int THREADS>
int launch_logits(const LogitsArgs& a, cudaStream_t s) {
  const long long size = sizeof(T);
  const bool whole = a.vocab * size % 16 == 0 && a.stride * size % 16 == 0 && !((uintptr_t)a.in & 15u) &&
                     (!a.out || (a.out_stride * size % 16 == 0 && !((uintptr_t)a.out & 15u)));
  const bool alike = !a.out || (((uintptr_t)a.in - (uintptr_t)a.out) % 16 == 0 && (a.stride - a.out_stride) * size % 16 == 0);
  return whole ? launch_logits<T, LG_WHOLE, CTAS, THREADS>(a, s) : alike ? launch_logits<T, LG_SHIFTED, CTAS, THREADS>(a, s) : launch_logits<T, LG_SINGLE, CTAS, THREADS>(a, s);
}
template <typename T>
int launch_logits(const LogitsArgs& a, cudaStream_t s) {
  // The GPU holds 3 CTAs with the large table an SM, 4 of the others.  As few a row as fill three quarters of its places, since each goes through the row's
  // lists: 310 rows of 50,000 with histories of 3000, one / two a row 39 / 29 us; 512 of 128,000 81 / 81 (without lists 51 / 54); 140 of 50,000 in fp32,
  // two / four 31 / 25; 60 of them, eight (a second wave) / four 24 / 19.  Where not every SM has one, CTAs of 512 threads (one row of 260,000 11.6 -> 9.6).
  if (a.rows >= 3 * LG_SMS) return launch_logits<T, 1, 256>(a, s);
  if (a.rows >= 3 * LG_SMS / 2) return launch_logits<T, 2, 256>(a, s);
  if (a.rows > 3 * LG_SMS / 8) return launch_logits<T, 4, 256>(a, s);
  if (a.rows > LG_SMS / 8) return launch_logits<T, 8, 256>(a, s);
  return launch_logits<T, 8, 512>(a, s);
}

}  // namespace

extern "C" int vlac_logits_adjust(int rows, int vocab, int dtype, const void* logits, long long stride, const vlac_logits_rules* rules, void* out,
                                  long long out_stride, int* picked, int* status, void* stream) {
  if (rows < 0 || vocab < 1 || vocab > 1 << 30 || (dtype != VLAC_FP32 && dtype != VLAC_BF16 && dtype != VLAC_FP16) || !rules) return VLAC_ERR_INVALID_ARG;
  if (rows > 65535) return VLAC_ERR_TOO_LARGE;
  const vlac_logits_rules& u = *rules;
  if (u.n_tokens < 0 || u.n_tokens > 1 << 30 || u.n_bias < 0 || u.n_bias > 1 << 30 || u.n_allow < 0 || (u.span && u.n_tokens > 0 && !u.tokens)) return VLAC_ERR_INVALID_ARG;
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
