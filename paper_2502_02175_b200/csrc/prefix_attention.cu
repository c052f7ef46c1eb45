// Attention of new rows over paged sequences that share a prefix (vlac_prefix_plan, vlac_prefix_attention).
//
// Softmax attention over a union of disjoint key sets is a weighted sum of the attentions over the sets:
//     o = sum_i 2^(m_i - M) l_i o_i / sum_i 2^(m_i - M) l_i      (m_i, l_i: maximum and sum of 2^(s - m_i) of set i)
// so the pages that several sequences have in common are one problem with the query rows of all of them (and of all query
// heads of a K/V head) stacked, and each sequence's own rows are another with its rows alone.  These problems are "segments";
// a segment is cut into (K/V head, tile of stacked rows, block of keys) units, and the units of the whole call are dealt to a
// fixed number of warps or CTAs in equal contiguous runs, whatever the lengths: a run may begin and end inside a tile, every piece of a
// tile leaves (unnormalised o, m, l) in a slot of its own, and a second kernel adds a row's pieces in a fixed order.
#include "pages_internal.h"
#include "launch_util.h"
#include <cuda.h>
#include <cuda_fp16.h>
#include <math.h>
#include <stddef.h>
#include <algorithm>

namespace {

// Two kernels share the segments.  Wide: common pages with more than 16 stacked rows, which every row sees whole (tcgen05).  Narrow:
// the rest -- prefixes of few rows and every sequence's own rows, where the causal mask lies (warp-level tensor cores).
// The border is the narrow tile's height, and measured: four prompts, 32 heads of 128, narrow / wide in us: 4 rows a prompt behind 512 positions
// 18.2 / 22.9, behind 2048 35.4 / 39.2, behind 8192 99.7 / 99.1; 16 rows 22.2 / 24.2, 40.2 / 40.9, 103.1 / 100.8; 32 heads of 64, 16 rows: 16.2 / 21.1,
// 22.4 / 29.5, 65.2 / 63.9.  Behind 16 rows the narrow kernel would read every key again.
constexpr int NARROW = 0, WIDE = 1;
constexpr int PN_WARPS = 4, PN_CTAS = 2 * 148;  // narrow: two CTAs of four warps per SM, every warp works alone
constexpr int PW_CTAS = 148;                    // runs of the wide kernel: one CTA per SM
__host__ __device__ constexpr int pf_bm(int c) { return c == NARROW ? 16 : 256; }        // stacked rows of a tile
constexpr int WIDE_KEYS = 128;                  // keys of a unit
// Narrow: 64 (with fewer, a sequence's few own rows would count for less than they cost), or 32 while every unit has a warp of its own (8
// candidates, attention alone: 9.9 -> 8.7 us)
constexpr int NARROW_KEYS = 64, NARROW_FINE = 32;
__host__ __device__ constexpr int pf_runs(int c) { return c == NARROW ? PN_WARPS * PN_CTAS : PW_CTAS; }     // most runs

struct SeqRec { int slot /* -1: refused */, row0, nq, len, pre_seg, suf_seg, pad0, pad1; };          // segments: -1 none
struct __align__(16) SegRec {
  long long ustart, uend;                       // units of this segment in the call's order
  int slot;                                     // whose table holds the keys
  int row0, R;                                  // first q row; stacked rows per K/V head: (q rows) * (query heads per K/V head)
  int key0, key1;                               // positions [key0, key1)
  int pos0;                                     // position of q row row0; INT_MIN in a prefix: every row sees every key
  int cls, T, KB;                               // NARROW or WIDE, tiles, key blocks
  int rowbase;                                  // first slot row of this segment
  int keys;                                     // keys of a unit
};
// key: what the plan was made for (see plan_key).  An attention call for anything else would read beside its tables and records, and computes nothing.
struct __align__(16) PlanHead { long long units[2]; unsigned long long key; int n_act, error; };           // error: a wait gave up, or a call had another key

struct PlanMem {
  PlanHead* head;
  SeqRec* seq;                                  // [n] active sequences
  SegRec* seg;                                  // [2n]
  int* first[2];                                // segment of each run's first unit
  float2* ml;                                   // [slot rows] (m, l), m in units of log2
  float* po;                                    // [slot rows][head_dim]
  size_t bytes;
};
__host__ __device__ inline PlanMem plan_mem(void* mem, int n, int rows, int n_heads, int head_dim) {
  PlanMem p;
  unsigned char* b = (unsigned char*)mem;
  size_t o = 0;
  auto take = [&](size_t bytes) { unsigned char* r = b + o; o = (o + bytes + 255) & ~(size_t)255; return r; };
  p.head = (PlanHead*)take(sizeof(PlanHead));
  p.seq = (SeqRec*)take(sizeof(SeqRec) * n);
  p.seg = (SegRec*)take(sizeof(SegRec) * 2 * (size_t)n);
  for (int c = 0; c < 2; ++c) p.first[c] = (int*)take(sizeof(int) * pf_runs(c));
  const size_t slots = 2 * (size_t)rows * n_heads + (size_t)pf_runs(NARROW) * pf_bm(NARROW) + (size_t)pf_runs(WIDE) * pf_bm(WIDE);
  p.ml = (float2*)take(sizeof(float2) * slots);
  p.po = (float*)take(sizeof(float) * slots * head_dim);
  p.bytes = o;
  return p;
}

// The U units of a class are dealt to G = min(U, pf_runs) runs of equal length, so that none is empty: run c is [c*U/G, (c+1)*U/G).
// (Narrow, measured: three runs a warp, taken up as warps come free, gained nothing -- every run adds a partial sum per row -- although warps
// of some SMs get their bytes 1.4 times as fast as those of others.)
__device__ __forceinline__ long long runs(int cls, long long U) { return U < pf_runs(cls) ? U : pf_runs(cls); }
// The run of unit u:
__device__ __forceinline__ int run_of(int cls, long long u, long long U) {
  if (U < 1 << 20) return (int)(((unsigned)(u + 1) * (unsigned)runs(cls, U) - 1) / (unsigned)U);         // (a 64-bit division is five times as long)
  return (int)(((u + 1) * runs(cls, U) - 1) / U);
}

// ------------------------------------------------------------------------------------------------ plan
struct PlanArgs {
  const int *table, *len;
  int n_slots, max_pages, n_pages, page, shift, kv_heads, ratio, head_dim;
  int n, rows, n_heads, small;
  const int *seqs, *q_ptr;
  int* status;
  void* mem;
  unsigned long long key;
};
// One launch, bound by the chain of dependent reads and barriers, not by bytes: one CTA of 8 warps for few sequences with short tables, a cluster
// of eight CTAs that reads the tables together otherwise.  8 sequences of 19 pages 4.8 us; 32 of 4132 pages 9.5 us.  One CTA / the cluster: 8 sequences of
// 19 pages 4.8 / 6.7, 16 of 19 5.5 / 6.7, 16 of 256 7.2 / 7.4, one of 4096 5.8 / 7.2.  (Of the tables' width: 8 of 19 pages with 2048 columns 6.8 us.)
constexpr int PL_CTAS = 8;
constexpr int PL_MAX = VLAC_PAGES_MAX_LIST;
constexpr int PL_ONE = 4096;                    // table entries up to which one CTA is faster
struct Sums { long long u[3]; int r[2], g; };                           // units (narrow, wide, narrow if fine), slot rows of both classes, segments
__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y) { return {{x.u[0] + y.u[0], x.u[1] + y.u[1], x.u[2] + y.u[2]}, {x.r[0] + y.r[0], x.r[1] + y.r[1]}, x.g + y.g}; }
struct PlanShared {
  int i[PL_MAX], slot[PL_MAX], row0[PL_MAX], nq[PL_MAX], len[PL_MAX], lcp[PL_MAX], bad[PL_MAX];
  int c[PL_MAX], m[PL_MAX], last[PL_MAX], g[PL_MAX];                    // of a group, at its leader: common pages, members, last member; segment
  long long u0[2][PL_MAX];                                              // first unit of the sequence's segments, per class
  unsigned leads[PL_MAX / 32];
  int warps[32];
  Sums part[32];
};

// exclusive sums over the block's first n threads of five values (the barrier's cost is shared)
__device__ Sums plan_scan(Sums* part, const Sums& v, int n, Sums* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = (n + 31) >> 5;
  Sums before = {};
  if (warp < nw) {
    Sums x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Sums t = {{__shfl_up_sync(0xffffffffu, x.u[0], o), __shfl_up_sync(0xffffffffu, x.u[1], o), __shfl_up_sync(0xffffffffu, x.u[2], o)},
                      {__shfl_up_sync(0xffffffffu, x.r[0], o), __shfl_up_sync(0xffffffffu, x.r[1], o)}, __shfl_up_sync(0xffffffffu, x.g, o)};
      if (lane >= o) x = x + t;
    }
    if (lane == 31) part[warp] = x;
    before = {{x.u[0] - v.u[0], x.u[1] - v.u[1], x.u[2] - v.u[2]}, {x.r[0] - v.r[0], x.r[1] - v.r[1]}, x.g - v.g};
  }
  __syncthreads();
  Sums all = {};
  for (int w = 0; w < nw; ++w) {
    if (w == warp) before = before + all;
    all = all + part[w];
  }
  *total = all;
  return before;
}

// What an entry says, and its code as far as it does not depend on the pages or on other entries.
__device__ __forceinline__ int plan_entry(const PlanArgs& a, int i, int* slot, int* q0, int* q1, int* len) {
  *q0 = a.q_ptr[i]; *q1 = a.q_ptr[i + 1]; *slot = a.seqs[i];
  if (*q0 < 0 || *q1 > a.rows || (unsigned)*slot >= (unsigned)a.n_slots) return VLAC_ERR_INVALID_ARG;
  *len = a.len[*slot];
  return *len < 0 || *len > a.max_pages << a.shift ? VLAC_ERR_BAD_STATE : VLAC_OK;
}

// A plan without rows: the entries' codes are all there is to say.
__global__ void __launch_bounds__(PL_MAX, 1) prefix_status_kernel(PlanArgs a) {
  pdl_trigger();
  pdl_wait();
  const int i = threadIdx.x;
  int slot, q0 = 0, q1 = 0, len, status = VLAC_OK;
  if (i < a.n) status = plan_entry(a, i, &slot, &q0, &q1, &len);
  const int broken = __syncthreads_or(i < a.n && q1 < q0);
  if (i < a.n) a.status[i] = broken ? VLAC_ERR_INVALID_ARG : status;
}

template <int CTAS>
__global__ void __cluster_dims__(CTAS, 1, 1) __launch_bounds__(1024, 1) prefix_plan_kernel(PlanArgs a) {
  extern __shared__ __align__(16) unsigned char pl_raw[];
  PlanShared& s = *reinterpret_cast<PlanShared*>(pl_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = blockDim.x >> 5, rank = CTAS > 1 ? (int)cluster_rank() : 0;
  const PlanMem p = plan_mem(a.mem, a.n, a.rows, a.n_heads, a.head_dim);
  pdl_trigger();
  pdl_wait();
  // ---- the active sequences (rows to compute), in list order: every CTA for itself
  int slot = 0, q0 = 0, q1 = 0, len = 0, status = VLAC_OK;
  if (tid < a.n) status = plan_entry(a, tid, &slot, &q0, &q1, &len);
  const bool want = tid < a.n && status == VLAC_OK && q1 > q0;
  const unsigned ball = __ballot_sync(0xffffffffu, want);
  if (lane == 0) s.warps[warp] = __popc(ball);
  const int broken = __syncthreads_or(tid < a.n && q1 < q0);            // rows would overlap: nothing is computed
  if (broken && tid < a.n) status = VLAC_ERR_INVALID_ARG;
  int n_act = 0, k_of = __popc(ball & ((1u << lane) - 1));
  for (int w = 0; w < (a.n + 31) >> 5; ++w) { const int c = s.warps[w]; n_act += c; if (w < warp) k_of += c; }
  if (broken) n_act = 0;
  if (want && !broken) { s.i[k_of] = tid; s.slot[k_of] = slot; s.row0[k_of] = q0; s.nq[k_of] = q1 - q0; s.len[k_of] = len; }
  if (tid < PL_MAX / 32) s.leads[tid] = 0;
  for (int k = tid; k < n_act; k += blockDim.x) { s.lcp[k] = INT_MAX; s.bad[k] = 0; }
  if (rank == 0 && tid < a.n) a.status[tid] = status;
  __syncthreads();
  // (findings of the other CTAs go into CTA 0's memory only behind this: it has cleared its own, and every CTA runs)
  if (CTAS > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");

  // ---- tables: page numbers in range; leading pages in common with the previous active sequence.  CTA r has the sequences r, r + CTAS, ..
  const int n_mine = (n_act - rank + CTAS - 1) / CTAS;
  int team = 1;
  while (team < nw && team * 2 * n_mine <= nw) team *= 2;
  for (int x = warp / team; x < n_mine; x += nw / team) {
    const int k = x * CTAS + rank;
    const int *t = a.table + (size_t)s.slot[k] * a.max_pages, *tp = k ? a.table + (size_t)s.slot[k - 1] * a.max_pages : t;
    const int np = (s.len[k] + a.page - 1) >> a.shift;
    // only whole pages in front of every member's queries are shared: all rows of the group see all of them
    const int m = k ? min(max(0, s.len[k] - s.nq[k]), max(0, s.len[k - 1] - s.nq[k - 1])) >> a.shift : 0;
    int bad = 0, lcp = m;
#pragma unroll 8
    for (int j = (warp % team) * 32 + lane; j < np; j += team * 32) {
      const int y = t[j], z = j < m ? tp[j] : y;
      bad |= (unsigned)y >= (unsigned)a.n_pages;
      if (y != z) lcp = min(lcp, j);
    }
    lcp = __reduce_min_sync(0xffffffffu, lcp);
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) { atomicMin(&s.lcp[k], lcp); if (bad) atomicOr(&s.bad[k], 1); }
  }
  __syncthreads();
  if (CTAS > 1) {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    for (int x = tid; x < n_mine && rank; x += blockDim.x) {
      const int k = x * CTAS + rank;
      unsigned to;
      asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"((unsigned)__cvta_generic_to_shared(&s.lcp[k])));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(s.lcp[k]) : "memory");
      asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"((unsigned)__cvta_generic_to_shared(&s.bad[k])));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(s.bad[k]) : "memory");
    }
    cluster_sync_all();
    if (rank != 0) return;
  }

  // ---- neighbours into groups (one warp, 32 sequences at a time, from one change of the common length to the next)
  if (warp == 0) {
    int lead = 0, c = 0, m = 0;
    for (int k0 = 0; k0 < n_act; k0 += 32) {
      const int k = k0 + lane;
      int l = INT_MAX, vis = 0;                                         // lanes behind the last sequence never end a run
      if (k < n_act) {
        vis = max(0, s.len[k] - s.nq[k]) >> a.shift;
        const bool next = k > 0 && !s.bad[k] && !s.bad[k - 1] && s.row0[k] == s.row0[k - 1] + s.nq[k - 1];
        l = next ? s.lcp[k] : -1;                                       // -1: cannot follow its neighbour
      }
      unsigned flags = 0;
      const int count = min(32, n_act - k0);
      for (int pos = 0; pos < count;) {
        const unsigned stop = __ballot_sync(0xffffffffu, k < n_act && (l < c || c == 0 || m == 0)) & (0xffffffffu << pos);
        const int at = stop ? __ffs(stop) - 1 : count;                  // up to here all share at least the c pages
        m += at - pos;
        if (at == count) break;
        // joining spares the newcomer the reading of c2 common pages and costs the others the reading of c - c2 pages each
        const int c2 = min(c, __shfl_sync(0xffffffffu, l, at)), v = __shfl_sync(0xffffffffu, vis, at);
        if (m > 0 && c2 > 0 && (long long)c2 > (long long)(c - c2) * (m - 1)) { c = c2; ++m; }
        else {
          if (lane == 0 && m > 0) { s.c[lead] = c; s.m[lead] = m; s.last[lead] = k0 + at - 1; }
          lead = k0 + at; m = 1; c = v;
          flags |= 1u << at;
        }
        pos = at + 1;
      }
      if (lane == 0) s.leads[k0 >> 5] = flags;
    }
    if (lane == 0 && m > 0) { s.c[lead] = c; s.m[lead] = m; s.last[lead] = n_act - 1; }
  }
  __syncthreads();
  // ---- segments: thread k makes the prefix of a group that k leads, and k's own rows
  const bool mine = tid < n_act, bad = mine && s.bad[tid];
  int r_pre = 0, r_suf = 0, pre = 0, lead = tid, c_pre = NARROW, t_pre = 0, t_suf = 0, n_pre = 0, n_suf = 0;    // rows, tiles, keys
  if (bad) a.status[s.i[tid]] = VLAC_ERR_BAD_STATE;
  if (mine && !bad) {
    int w = tid >> 5;
    unsigned f = s.leads[w] & (0xffffffffu >> (31 - lane));
    while (!f) f = s.leads[--w];                                        // (sequence 0 leads)
    lead = w * 32 + 31 - __clz(f);
    const int last = s.last[lead], r_all = (s.row0[last] + s.nq[last] - s.row0[lead]) * a.ratio;
    // a sequence alone: its pages in front of many query rows are worth a segment of their own (no mask, wide tiles)
    if (s.m[lead] >= 2 || (r_all > pf_bm(NARROW) && !a.small)) pre = s.c[lead] << a.shift;
    if (lead == tid && pre > 0) {
      r_pre = r_all;
      c_pre = r_pre > pf_bm(NARROW) && !a.small ? WIDE : NARROW;
      t_pre = (r_pre + pf_bm(c_pre) - 1) / pf_bm(c_pre); n_pre = pre;
    }
    if (s.len[tid] > pre) {
      r_suf = s.nq[tid] * a.ratio;
      t_suf = (r_suf + pf_bm(NARROW) - 1) / pf_bm(NARROW); n_suf = s.len[tid] - pre;
    }
  }
  const bool wide = c_pre == WIDE;                                      // (then there is a prefix)
  auto units = [&](int t, int n, int keys) { return (long long)a.kv_heads * t * ((n + keys - 1) / keys); };
  const Sums own = {{(wide ? 0 : units(t_pre, n_pre, NARROW_KEYS)) + units(t_suf, n_suf, NARROW_KEYS), wide ? units(t_pre, n_pre, WIDE_KEYS) : 0,
                     (wide ? 0 : units(t_pre, n_pre, NARROW_FINE)) + units(t_suf, n_suf, NARROW_FINE)},
                    {((wide ? 0 : r_pre) + r_suf) * a.kv_heads, wide ? r_pre * a.kv_heads : 0}, (n_pre > 0) + (n_suf > 0)};
  Sums all;
  Sums at = plan_scan(s.part, own, n_act, &all);
  const bool fine = all.u[2] <= pf_runs(NARROW);
  if (fine) { at.u[0] = at.u[2]; all.u[0] = all.u[2]; }
  const int keys_n = fine ? NARROW_FINE : NARROW_KEYS, keys_pre = wide ? WIDE_KEYS : keys_n;
  const int kb_pre = (n_pre + keys_pre - 1) / keys_pre, kb_suf = (n_suf + keys_n - 1) / keys_n;
  const long long u_pre = units(t_pre, n_pre, keys_pre), u_suf = units(t_suf, n_suf, keys_n);
  const int g0 = at.g;
  if (mine) { s.g[tid] = g0; s.u0[NARROW][tid] = at.u[0]; s.u0[WIDE][tid] = at.u[1]; }
  if (tid == 0) { PlanHead h = {{all.u[0], all.u[1]}, a.key, n_act, 0}; *p.head = h; }
  __syncthreads();
  if (mine) {
    SeqRec q = {bad ? -1 : s.slot[tid], s.row0[tid], s.nq[tid], s.len[tid], pre > 0 ? s.g[lead] : -1, u_suf > 0 ? g0 + (u_pre > 0) : -1, 0, 0};
    p.seq[tid] = q;
    // slots: the narrow pieces' rows, then the wide ones' (each run sets itself off by a tile, see next_piece)
    const long long at_w = all.r[0] + (long long)pf_runs(NARROW) * pf_bm(NARROW);
    if (u_pre > 0) {
      const long long us = wide ? at.u[1] : at.u[0];
      SegRec r = {us, us + u_pre, s.slot[tid], s.row0[tid], r_pre, 0, pre, INT_MIN, c_pre, t_pre, kb_pre, (int)(wide ? at_w + at.r[1] : at.r[0]), keys_pre};
      p.seg[g0] = r;
    }
    if (u_suf > 0) {
      const long long us = at.u[0] + (wide ? 0 : u_pre);
      SegRec r = {us, us + u_suf, s.slot[tid], s.row0[tid], r_suf, pre, s.len[tid], s.len[tid] - s.nq[tid], NARROW, t_suf, kb_suf,
                  (int)(at.r[0] + (wide ? 0 : (long long)r_pre * a.kv_heads)), keys_n};
      p.seg[g0 + (u_pre > 0)] = r;
    }
  }
  // ---- the segment of each run's first unit: the last sequence whose units begin at or before it (its kernel walks on from there)
#pragma unroll
  for (int cls = 0; cls < 2; ++cls) {
    const long long U = all.u[cls];
    const int G = (int)runs(cls, U);
    for (int c = tid; c < G; c += blockDim.x) {
      const long long u = U < 1 << 20 ? (long long)((unsigned)c * (unsigned)U / (unsigned)G) : c * U / G;     // (a 64-bit division is five times as long)
      int lo = 0, hi = n_act - 1;
      while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (s.u0[cls][m] <= u) lo = m; else hi = m - 1; }
      p.first[cls][c] = s.g[lo];
    }
  }
}

// ------------------------------------------------------------------------------------------------ both kernels
struct AttnArgs {
  const void *k, *v;                            // this layer of the pool
  const int* table;
  int max_pages, n_pages, page, shift, kv_heads, ratio, n_heads, n, rows;
  const void* q; long long q_stride;
  void* out; long long out_stride;
  float* lse;
  float scale2;                                 // softmax scale * log2(e)
  void* mem;
  unsigned long long key;
  const unsigned* mask; int words;              // a tree's: which of its entry's newest rows each row of q sees, or NULL
};
// Weights are rounded to the 16-bit type for the product with V.  `shift`: the reference of the exponentials lies that many powers of two below the
// maximum that moved it, so that the weights use the upper part of the type's range; sums and outputs are scaled alike, and the division by the
// sum takes it out.  `growth`: the wide kernel moves its reference once the maximum has grown by that many.  bf16 has the exponents of fp32 and needs
// no shift.  fp16 ends at 2^16 and loses a bit with every power below 2^-14: with the maximum at 2^9 .. 2^15 (narrow: at 2^14) a weight keeps its 11
// bits down to 2^-23 (2^-28) of the maximum and is lost only below 2^-34 (2^-39), so that many keys far behind a single one count for what they are
// (65,600 keys 2^-25 behind one hold 0.2 % of the sum; with the maximum at 1 all of them were lost to the output).  The border between shift and
// growth, measured on 64 chunks of 7 in fp16, all kernels: growth 8 (no shift) 111 us, 6 115, 5 120, 4 127 (O is rescaled more often).
template <typename T> struct Half2;
template <> struct Half2<__nv_bfloat16> {
  static __device__ __forceinline__ unsigned pack(float lo, float hi) { __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi); return *reinterpret_cast<unsigned*>(&v); }
  static __device__ __forceinline__ void mma(float* c, const unsigned* a, unsigned b0, unsigned b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
  static constexpr unsigned exp_mask = 0x7f80u;
  static constexpr float shift_narrow = 0.f, shift_wide = 0.f, growth = 8.f;
  static __device__ __forceinline__ float value(unsigned short x) { return __uint_as_float((unsigned)x << 16); }
};
template <> struct Half2<__half> {
  static __device__ __forceinline__ unsigned pack(float lo, float hi) { __half2 v = __floats2half2_rn(lo, hi); return *reinterpret_cast<unsigned*>(&v); }
  static __device__ __forceinline__ void mma(float* c, const unsigned* a, unsigned b0, unsigned b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
  static constexpr unsigned exp_mask = 0x7c00u;
  static constexpr float shift_narrow = 14.f, shift_wide = 9.f, growth = 6.f;
  static __device__ __forceinline__ float value(unsigned short x) { return __half2float(__ushort_as_half(x)); }
};

__device__ __forceinline__ unsigned pf_smem(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float pf_ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
constexpr float PF_LN2 = 0.693147180559945f, PF_LOG2E = 1.44269504088896f;

// Piece of a tile that one run computes.
struct Piece {
  int slot, head, rt, nr;                       // table; K/V head; tile; valid stacked rows
  int row0, key0, key1, lim0;                   // q row of stacked row 0 of the segment; keys [key0, key1); see lim0 below (with a tree: its first position + 1)
  int n;                                        // key blocks (steps) of the piece
  int direct;
  size_t slot0;                                 // slot row of the tile's first row
};
// (through L2: the narrow kernel may start before the kernel in front of it has ended, and with it the life of what L1 holds)
__device__ __forceinline__ SegRec load_seg(const SegRec* p) {
  static_assert(sizeof(SegRec) % 16 == 0, "whole 16-byte pieces");
  union { SegRec s; int4 v[sizeof(SegRec) / 16]; } u;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(SegRec) / 16); ++i) u.v[i] = __ldcg(reinterpret_cast<const int4*>(p) + i);
  return u.s;
}

// Walks a run's pieces: one division to find the first, then tile after tile, segment after segment.
struct Cursor {
  long long u, u_end;                           // next unit, end of the run
  int cls, run, g;
  SegRec s;                                     // segment of the next unit
  int head, rt, kb;                             // its place in the segment
  __device__ __forceinline__ void begin(const PlanMem& pm, int c, int r, long long U, long long G, int first) {
    cls = c; run = r; g = first;
    if (U < 1 << 20) {                          // (a 64-bit division is five times as long)
      u = (unsigned)r * (unsigned)U / (unsigned)G; u_end = (unsigned)(r + 1) * (unsigned)U / (unsigned)G;
    } else { u = r * U / G; u_end = (r + 1) * U / G; }
    s = load_seg(pm.seg + g);
    while (u >= s.uend || s.cls != cls) s = load_seg(pm.seg + ++g);
    const long long local = u - s.ustart, per_head = (long long)s.T * s.KB;
    head = (int)(local / per_head);
    const long long rem = local - head * per_head;
    rt = (int)(rem / s.KB); kb = (int)(rem - (long long)rt * s.KB);
  }
  __device__ __forceinline__ bool more() const { return u < u_end; }
  __device__ __forceinline__ void next(const PlanMem& pm, Piece* p) {
    if (kb == s.KB) {                           // the last piece ended its tile
      kb = 0;
      if (++rt == s.T) { rt = 0; ++head; }
      if (u >= s.uend) {
        do s = load_seg(pm.seg + ++g); while (u >= s.uend || s.cls != cls);
        head = 0;
      }
    }
    const int bm = pf_bm(cls), n = (int)min((long long)(s.KB - kb), u_end - u);
    p->slot = s.slot; p->head = head; p->rt = rt; p->nr = min(bm, s.R - rt * bm); p->row0 = s.row0;
    p->key0 = s.key0 + kb * s.keys; p->key1 = min(s.key1, p->key0 + n * s.keys);
    // stacked row x of the tile sees the positions below lim0 + x / ratio (x counted from the segment's start)
    p->lim0 = s.pos0 == INT_MIN ? INT_MIN : s.pos0 + 1;
    p->n = n;
    p->direct = n == s.KB && s.pos0 != INT_MIN && s.key0 == 0;          // a whole tile, and all that its rows see: written as the result
    p->slot0 = (size_t)s.rowbase + (size_t)head * s.R + (size_t)rt * bm + (size_t)run * bm;
    kb += n; u += n;
  }
};

// ------------------------------------------------------------------------------------------------ narrow: warp-level tensor cores
// Every warp walks its own run of units in steps of 16 (head_dim 128) or 32 keys with 16 stacked rows, with a ring of three steps of K and V
// in shared memory filled by cp.async ahead of the products, across piece boundaries; nothing is synchronised beyond the warp.  Bound: HBM
// (K/V rows are read once; a lone query row fills one of the 16 rows of the products, which cost nothing next to the loads), and with
// head_dim 64 the latency of a step's dependent instructions, which is why its steps are twice as long (65 sequences of 32 heads, 211 MB: 16
// keys 43 % of the issue slots and 3.8 TB/s; 32 keys 34 % and 4.3 TB/s, 50 us).
constexpr int PN_STAGES = 3;
template <int D> struct Narrow {
  static constexpr int STEP = D == 128 ? 16 : 32;
  static constexpr int HALF = STEP * 128;                               // 64 elements of a step's rows
  static constexpr int TILE = STEP * D * 2;
  static constexpr int Q_HALF = 16 * 128, Q_TILE = 16 * D * 2;
  static constexpr int WARP = Q_TILE + TILE * 2 * PN_STAGES;            // Q, then the ring
  static constexpr int SMEM = WARP * PN_WARPS;
};
__device__ __forceinline__ void pf_ldsm4(unsigned addr, unsigned* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void pf_ldsm4t(unsigned addr, unsigned* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void pf_cp16(unsigned dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void pf_cp16(unsigned dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// byte offset of 16-byte piece c16 of a row in a [rows][64 elements] block whose pieces are XOR-swizzled by the row
__device__ __forceinline__ unsigned pf_swz(int row, int c16) { return (unsigned)(row * 128 + (((c16 ^ row) & 7) << 4)); }

template <typename T>
__device__ __forceinline__ bool any_nonfinite(uint4 x) {
  const unsigned w[4] = {x.x, x.y, x.z, x.w};
  bool r = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r |= (w[i] & Half2<T>::exp_mask) == Half2<T>::exp_mask;
    r |= ((w[i] >> 16) & Half2<T>::exp_mask) == Half2<T>::exp_mask;
  }
  return r;
}

// EARLY: behind the wide kernel of the same call, of which it reads nothing.  That kernel lets its successor start only once it has seen the plan
// complete, so the CTAs here begin as SMs come free and wait for its end before their own (what comes after reads both).
// TREE: a row sees all positions in front of its entry's newest rows and, of those, what its mask says.  The words are asked for before the scores are
// formed, in the steps that reach the newest rows alone.  The pages in front are the wide kernel's as ever, so that a tree costs what its rows cost as a
// chunk: 16 trees of up to 61 rows, 32 heads of 128, behind 8208 positions 254 us (6.2 TB/s) + 24 here; four of up to 64 rows with 8 K/V heads behind 65,600
// 178 us (its softmax chain) + 11.  Bound here: the chain of a step (16 rows by 16 keys: 340 instructions), two warps a scheduler.
template <typename T, int D, bool EARLY, bool TREE>
__global__ void __launch_bounds__(PN_WARPS * 32, 2) prefix_narrow_kernel(AttnArgs a) {
  using N = Narrow<D>;
  constexpr int STEP = N::STEP, NB = STEP / 16;                         // blocks of 16 keys in a step
  extern __shared__ __align__(1024) unsigned char pn_raw[];
  __shared__ Piece s_piece[PN_WARPS][4];
  const PlanMem pm = plan_mem(a.mem, a.n, a.rows, a.n_heads, D);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  if (!EARLY) pdl_wait();
  const int run = warp * PN_CTAS + blockIdx.x;                          // few runs: one per SM before two
  const unsigned long long key = __ldcg(&pm.head->key);
  const long long U = __ldcg(&pm.head->units[NARROW]), G = runs(NARROW, U);
  const int g = __ldcg(&pm.first[NARROW][run]);
  if (run >= G || key != a.key) { if (EARLY) pdl_wait(); return; }
  Cursor cur;                                                           // pieces not yet begun
  cur.begin(pm, NARROW, run, U, G, g);

  unsigned char* const base_p = pn_raw + warp * N::WARP;
  const unsigned q_s = pf_smem(base_p), ring = q_s + N::Q_TILE;
  constexpr int C16 = D / 8, RSTEP = 32 / C16, NROW = 16 / RSTEP;       // 16-byte pieces of a row; rows a warp copies at once; times for 16
  const int c16 = lane % C16, r_first = lane / C16;
  const unsigned q_off = (unsigned)(c16 >> 3) * N::Q_HALF, col_off = (unsigned)(c16 >> 3) * N::HALF;
  const size_t row_el = (size_t)a.kv_heads * D;

  // ---- load cursor.  Pieces may be a step or two long (a sequence's own rows), so that loads run up to three pieces ahead: three Q tiles
  // of up to 5 rows lie side by side in the 16 rows of the Q buffer; a larger one has it alone.
  constexpr int QN = 3, QR = 5;
  int l_begun = 0, l_step = 0, l_steps = 0, l_cnt = 0, pg = 0, pg_slot = -1, pg_key = -1, pg_end = -1;
  int c_begun = 0, c_cnt = 0;
  bool have = false, l_big = false;                                     // lp is prepared but not begun; the piece begun last has Q alone
  const T *kg = nullptr, *vg = nullptr;
  Piece lp;
  const int page_step = a.shift < 4 ? 3 : 4;                            // page numbers are fetched for blocks of 8 or 16 keys, one a lane
  auto issue = [&]() -> bool {                                          // one more step in flight
    if (l_step == l_steps) {
      if (!have) {
        if (!cur.more()) return false;
        cur.next(pm, &lp);
        have = true;
      }
      const bool big = lp.nr > QR;
      if (l_begun - c_begun >= (big || l_big ? 1 : QN) || (big && l_begun != c_begun)) return false;
      have = false; l_big = big;
      const int qs = big ? 0 : (l_begun % QN) * QR;                     // first row of its Q
      if (lane == 0) s_piece[warp][l_begun & 3] = lp;
      ++l_begun;
      l_step = 0; l_steps = (lp.key1 - lp.key0 + STEP - 1) / STEP;
      const size_t col = (size_t)r_first * row_el + (size_t)lp.head * D + c16 * 8;
      kg = (const T*)a.k + col; vg = (const T*)a.v + col;
      for (int r = r_first; r < lp.nr; r += RSTEP) {
        // stacked row x is q row row0 + x / ratio, query head head * ratio + x % ratio
        const int x = lp.rt * 16 + r, xq = x / a.ratio;
        const T* src = (const T*)a.q + (size_t)(lp.row0 + xq) * a.q_stride + (size_t)(lp.head * a.ratio + x - xq * a.ratio) * D + c16 * 8;
        pf_cp16(q_s + q_off + pf_swz(qs + r, c16 & 7), src);
      }
    }
    const int k0 = lp.key0 + l_step * STEP;
    const int per = STEP >> page_step, at = (l_step * per) & 31;        // page numbers of a step, and where the lanes hold them
    if (at == 0 && !(pg_slot == lp.slot && pg_key == k0 && pg_end == lp.key1)) {             // (the next head's piece begins where the last one did)
      const int k = k0 + (lane << page_step);
      pg_slot = lp.slot; pg_key = k0; pg_end = lp.key1;
      pg = k < lp.key1 ? __ldcg(&a.table[(size_t)lp.slot * a.max_pages + (k >> a.shift)]) : -1;
      if ((unsigned)pg >= (unsigned)a.n_pages) pg = -1;
    }
    const unsigned ks = ring + (unsigned)(l_cnt % PN_STAGES) * 2u * N::TILE + col_off;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int kb = k0 + 16 * b;
      const int lo = __shfl_sync(0xffffffffu, pg, at + (b << (4 - page_step)));
      const int hi = page_step == 4 ? lo : __shfl_sync(0xffffffffu, pg, at + 2 * b + 1);
      const size_t at_lo = (((size_t)lo << a.shift) + (kb & (a.page - 1))) * row_el;
      const size_t at_hi = page_step == 4 ? at_lo + 8 * row_el : ((size_t)hi << a.shift) * row_el;
      if (kb + 16 <= lp.key1 && lo >= 0 && hi >= 0) {
#pragma unroll
        for (int i = 0; i < NROW; ++i) {
          const size_t o = i < NROW / 2 ? at_lo + i * RSTEP * row_el : at_hi + (i - NROW / 2) * RSTEP * row_el;
          const unsigned off = ks + pf_swz(16 * b + r_first + i * RSTEP, c16 & 7);
          pf_cp16(off, kg + o);
          pf_cp16(off + N::TILE, vg + o);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NROW; ++i) {                                // zeros behind the segment
          const int r = r_first + i * RSTEP;
          const bool ok = kb + r < lp.key1 && (i < NROW / 2 ? lo : hi) >= 0;
          const size_t o = !ok ? 0 : i < NROW / 2 ? at_lo + i * RSTEP * row_el : at_hi + (i - NROW / 2) * RSTEP * row_el;
          const unsigned off = ks + pf_swz(16 * b + r, c16 & 7);
          pf_cp16(off, kg + o, ok);
          pf_cp16(off + N::TILE, vg + o, ok);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ++l_step; ++l_cnt;
    return true;
  };

  float o[D / 8][4], m[2], l[2];                                        // the lane's two rows: lane / 4 and lane / 4 + 8
  unsigned qf[D / 16][4];
  int c_left = 0, key_lo = 0, key1 = 0, lim[2] = {0, 0}, lim_min = 0;
  const unsigned* mrow[2] = {nullptr, nullptr};                         // TREE: the masks of the lane's two rows (NULL: sees all)
  int t0 = 0;                                                           // and the position of the entry's first newest row
  while (true) {
    while (l_cnt - c_cnt < PN_STAGES && issue()) {}
    if (l_cnt == c_cnt) break;
    const int younger = l_cnt - 1 - c_cnt;                              // steps in flight behind the one that is needed
    if (younger == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (younger == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 2;" ::: "memory");
    __syncwarp();
    if (c_left == 0) {                                                  // a piece begins
      const Piece& p = s_piece[warp][c_begun & 3];
      const int qs = p.nr > QR ? 0 : (c_begun % QN) * QR;
      key_lo = p.key0; key1 = p.key1;
      c_left = (key1 - key_lo + STEP - 1) / STEP;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int x = (lane >> 2) + 8 * r;
        if (TREE) {
          lim[r] = key1;
          mrow[r] = p.lim0 == INT_MIN || x >= p.nr ? nullptr : a.mask + (size_t)(p.row0 + (p.rt * 16 + x) / a.ratio) * a.words;
        } else
          lim[r] = p.lim0 == INT_MIN || x >= p.nr ? key1 : min(key1, p.lim0 + (p.rt * 16 + x) / a.ratio);
        m[r] = -INFINITY; l[r] = 0.f;
      }
      lim_min = p.lim0 == INT_MIN ? key1 : min(key1, TREE ? p.lim0 - 1 : p.lim0 + p.rt * 16 / a.ratio);
      if (TREE && p.lim0 != INT_MIN) t0 = p.lim0 - 1;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) { o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f; }
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        // (rows behind the last repeat it: nothing of them is kept)
        const int row = qs + min((lane & 7) + ((lane >> 3) & 1) * 8, p.nr - 1), c = ks * 2 + (lane >> 4);
        pf_ldsm4(q_s + (unsigned)(c >> 3) * N::Q_HALF + pf_swz(row, c & 7), qf[ks]);
      }
      ++c_begun;
      __syncwarp();
    }
    unsigned char* const k_p = base_p + N::Q_TILE + (c_cnt % PN_STAGES) * 2 * N::TILE;
    const unsigned k_s = pf_smem(k_p), v_s = k_s + N::TILE;
    const bool masked = key_lo + STEP > lim_min;                        // some row does not see the whole step
    unsigned mw[2][2] = {{~0u, ~0u}, {~0u, ~0u}};                       // TREE: the two words of each row's mask that the step's keys lie in
    if (TREE && masked) {
      const int w = (key_lo - t0) >> 5;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (mrow[r] && w + e >= 0) mw[r][e] = w + e < a.words ? __ldcg(mrow[r] + w + e) : 0u;
    }
    float s[2 * NB][4];
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const int c = ks * 2 + ((lane >> 3) & 1);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int key = 16 * b + (lane & 7) + ((lane >> 4) & 1) * 8;
        unsigned f[4];
        pf_ldsm4(k_s + (unsigned)(c >> 3) * N::HALF + pf_swz(key, c & 7), f);
        Half2<T>::mma(s[2 * b], qf[ks], f[0], f[1]);
        Half2<T>::mma(s[2 * b + 1], qf[ks], f[2], f[3]);
      }
    }
    unsigned seen[2] = {~0u, ~0u};                                      // TREE: the keys of the step that each row sees
    if (TREE && masked)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        seen[r] = __funnelshift_r(mw[r][0], mw[r][1], (key_lo - t0) & 31);
        if (key1 - key_lo < 32) seen[r] &= (1u << (key1 - key_lo)) - 1u;                  // (key1 > key_lo)
      }
    float bm[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = s[j][e] * a.scale2;
        const int key = j * 8 + 2 * (lane & 3) + (e & 1);
        if (masked && (TREE ? !(seen[e >> 1] >> key & 1) : key_lo + key >= lim[e >> 1])) x = -INFINITY;
        s[j][e] = x;
        bm[e >> 1] = fmaxf(bm[e >> 1], x);
      }
    float ref[2], al[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      bm[r] = fmaxf(bm[r], __shfl_xor_sync(0xffffffffu, bm[r], 1));
      bm[r] = fmaxf(bm[r], __shfl_xor_sync(0xffffffffu, bm[r], 2));
      const float mn = fmaxf(m[r], bm[r] - Half2<T>::shift_narrow);
      ref[r] = mn == -INFINITY ? 0.f : mn;                              // a row that has seen nothing yet: no inf - inf
      al[r] = pf_ex2(m[r] - ref[r]);
      m[r] = mn;
      l[r] *= al[r];
    }
    if (__any_sync(0xffffffffu, al[0] != 1.f || al[1] != 1.f)) {
#pragma unroll
      for (int j = 0; j < D / 8; ++j) { o[j][0] *= al[0]; o[j][1] *= al[0]; o[j][2] *= al[1]; o[j][3] *= al[1]; }
    }
    // P is rounded to the 16-bit type for the product with V (half a step: 2^-8 of each weight for bf16, 2^-11 for fp16 and at least 2^-39 of the largest
    // one, see Half2); the sum l takes the unrounded weights
    unsigned pf[NB][4];
#pragma unroll
    for (int j = 0; j < 2 * NB; ++j) {
      const float p0 = pf_ex2(s[j][0] - ref[0]), p1 = pf_ex2(s[j][1] - ref[0]), p2 = pf_ex2(s[j][2] - ref[1]), p3 = pf_ex2(s[j][3] - ref[1]);
      l[0] += p0 + p1; l[1] += p2 + p3;
      pf[j >> 1][(j & 1) * 2] = Half2<T>::pack(p0, p1);
      pf[j >> 1][(j & 1) * 2 + 1] = Half2<T>::pack(p2, p3);
    }
    if (masked && (TREE || lim_min < key1)) {
      // a row does not see some key of this step: infinities and NaN of such a V row must not reach it as 0 * inf
      bool bad = false;
      for (int i = lane; i < N::TILE / 16; i += 32) bad |= any_nonfinite<T>(*reinterpret_cast<const uint4*>(k_p + N::TILE + i * 16));
      if (__any_sync(0xffffffffu, bad)) {
        for (int key = 0; key < STEP; ++key)
#pragma unroll
          for (int j = 0; j < D / 8; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int col = j * 8 + 2 * (lane & 3) + e;
              const unsigned short x =
                  *reinterpret_cast<const unsigned short*>(k_p + N::TILE + (col >> 6) * N::HALF + pf_swz(key, (col & 63) >> 3) + (col & 7) * 2);
              if ((x & Half2<T>::exp_mask) == Half2<T>::exp_mask) {
                if (TREE ? seen[0] >> key & 1 : key_lo + key < lim[0]) o[j][e] += Half2<T>::value(x);
                if (TREE ? seen[1] >> key & 1 : key_lo + key < lim[1]) o[j][2 + e] += Half2<T>::value(x);
              }
            }
        __syncwarp();
        unsigned short* x = reinterpret_cast<unsigned short*>(k_p + N::TILE);
        for (int i = lane; i < STEP * D; i += 32)
          if ((x[i] & Half2<T>::exp_mask) == Half2<T>::exp_mask) x[i] = 0;
        __syncwarp();
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int np = 0; np < D / 16; ++np) {
        const int c = np * 2 + (lane >> 4), key = 16 * b + (lane & 7) + ((lane >> 3) & 1) * 8;
        unsigned f[4];
        pf_ldsm4t(v_s + (unsigned)(c >> 3) * N::HALF + pf_swz(key, c & 7), f);
        Half2<T>::mma(o[2 * np], pf[b], f[0], f[1]);
        Half2<T>::mma(o[2 * np + 1], pf[b], f[2], f[3]);
      }
    key_lo += STEP;
    ++c_cnt;
    if (--c_left == 0) {                                                // the piece ends
      const Piece& p = s_piece[warp][(c_begun - 1) & 3];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        const int x = (lane >> 2) + 8 * r;
        if (x >= p.nr) continue;
        if (p.direct) {
          const int xs = p.rt * 16 + x, xq = xs / a.ratio, row = p.row0 + xq, h = p.head * a.ratio + xs - xq * a.ratio;
          T* dst = (T*)a.out + (size_t)row * a.out_stride + (size_t)h * D;
          const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
#pragma unroll
          for (int j = 0; j < D / 8; ++j)
            *reinterpret_cast<unsigned*>(dst + j * 8 + 2 * (lane & 3)) = Half2<T>::pack(o[j][2 * r] * inv, o[j][2 * r + 1] * inv);
          if (a.lse && (lane & 3) == 0) a.lse[(size_t)row * a.n_heads + h] = (m[r] + log2f(l[r])) * PF_LN2;
        } else {
          float* dst = pm.po + (p.slot0 + x) * D;
#pragma unroll
          for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(dst + j * 8 + 2 * (lane & 3)) = make_float2(o[j][2 * r], o[j][2 * r + 1]);
          if ((lane & 3) == 0) pm.ml[p.slot0 + x] = make_float2(m[r], l[r]);
        }
      }
    }
    __syncwarp();                                                       // the step's tiles (and the piece record) may be refilled
  }
  if (EARLY) pdl_wait();
}

// ------------------------------------------------------------------------------------------------ wide: tcgen05
// One persistent CTA per SM walks its run of (K/V head, tile of 256 stacked rows, block of 128 keys) units:
//   warps 0, 2, 3  TMA: K and V blocks, one box per (page, 64 elements) into one ring of tiles in the order the products take them
//   warp 1         issues S = Q K^T (M 128, N 128) and O += P V, A = P from tensor memory
//   warps 4-7 and 8-11   softmax, a thread per row, in two sides with an S/P buffer and an O of their own:
//                  more than 128 rows (two): side b has rows 128 b .. and every key block; a K/V tile in shared memory serves both
//                  up to 128 rows: side b has all rows and every second key block, as if the keys were split in two; the sides' sums are
//                  added when the piece ends
// Either way the tensor cores work for one side while the other is in the softmax.  Every row sees every key of a common prefix: no mask
// but behind its last key, where zeros are loaded.
// Bound: the 16384 exponentials of 128 rows and keys (16 a cycle and SM: 1024 cycles, as long as their products at the dense peak) where the
// rows fill the tile, HBM (64 KB of K and V a block) where they do not.  Measured: 448 rows of 32 heads behind 8208 keys, 60 GFLOP, 71 us
// (0.85 PFLOP/s; 3240 cycles a unit: a side's softmax 1900, its PV, next S and three barriers 1300, while products and exponentials need 2048
// each); 128 rows of 8 heads behind 65,600 keys, 268 MB, 51 us (5.3 TB/s).
constexpr int PW_THREADS = 384;
constexpr int PW_SOFT = 256;                    // threads of the two softmax sides
constexpr unsigned long long PW_WAIT_LIMIT_NS = 400000000ull;
template <int D> struct Wide {
  static constexpr int HALVES = D / 64;
  static constexpr int HALF = 128 * 128;        // 64 elements of 128 rows
  static constexpr int TILE = HALVES * HALF;
  static constexpr int SLOTS = D == 128 ? 5 : 10;
  static constexpr int SMEM = TILE * (2 + SLOTS) + 2048;                // two tiles of Q, the ring of K and V tiles, the sides' (m, l)
};

__device__ __forceinline__ void pw_bar_init(unsigned long long* bar, unsigned count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(pf_smem(bar)), "r"(count));
}
__device__ __forceinline__ void pw_expect(unsigned long long* bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(pf_smem(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void pw_arrive(unsigned long long* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(pf_smem(bar)) : "memory");
}
__device__ __forceinline__ unsigned long long pw_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// (the hint: sleep in the barrier for up to 20 us a try)
__device__ __forceinline__ bool pw_try_at(unsigned bar, unsigned parity) {
  unsigned ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\nselp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Wait for a phase, at most `limit`; a wait that gives up (or finds that another has) returns false and marks the plan.  Its loop leaves lane by lane:
// where instructions of the whole warp follow, the caller brings the lanes together again.
__device__ __noinline__ bool pw_wait_slow(unsigned bar, unsigned parity, volatile int* abort_flag, int* error, unsigned long long limit) {
  const unsigned long long t0 = pw_ns();
  while (true) {
    for (int i = 0; i < 16; ++i)
      if (pw_try_at(bar, parity)) return true;
    if (*abort_flag) return false;
    if (pw_ns() - t0 > limit) break;
  }
  *abort_flag = 1;
  atomicExch(error, VLAC_ERR_TIMEOUT);
  return false;
}
__device__ __forceinline__ bool pw_wait(unsigned long long* bar, unsigned parity, volatile int* abort_flag, int* error, unsigned long long limit) {
  return pw_try_at(pf_smem(bar), parity) || pw_wait_slow(pf_smem(bar), parity, abort_flag, error, limit);
}
__device__ __forceinline__ void pw_tma(unsigned dst, const CUtensorMap* tm, int x, int y, unsigned long long* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(pf_smem(bar)) : "memory");
}
__device__ __forceinline__ void pw_tma3(unsigned dst, const CUtensorMap* tm, int x, int y, int z, unsigned long long* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(pf_smem(bar)) : "memory");
}
__device__ __forceinline__ unsigned long long pw_desc(unsigned addr, unsigned lbo, unsigned sbo) {
  unsigned long long d = 0;
  d |= (unsigned long long)((addr & 0x3FFFFu) >> 4);
  d |= (unsigned long long)((lbo >> 4) & 0x3FFFu) << 16;
  d |= (unsigned long long)((sbo >> 4) & 0x3FFFu) << 32;
  d |= (unsigned long long)1 << 46;             // descriptor version of this architecture
  d |= (unsigned long long)2 << 61;             // 128-byte swizzle
  return d;
}
// fp32 accumulate, A and B both bf16 or both fp16, M = 128; B K-major or (b_mn) MN-major
template <typename T> __device__ __forceinline__ unsigned pw_idesc(int n, bool b_mn) {
  const unsigned f = sizeof(T) == 2 && Half2<T>::exp_mask == 0x7f80u ? 1u : 0u;
  return (1u << 4) | (f << 7) | (f << 10) | (b_mn ? 1u << 16 : 0u) | ((unsigned)(n >> 3) << 17) | (8u << 24);
}
// The warp that issues products runs converged and one lane's predicate (`one`) lets the instruction through: operands then stay in
// uniform registers.  Issued from a branch that a single lane takes, every product paid the moves into them (about 70 cycles a product, as
// long as it executes, and twice that beside the softmax warps).
__device__ __forceinline__ void pw_mma_ss(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, bool acc, unsigned one) {
  asm volatile("{\n.reg .pred p, e;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 e, %5, 0;\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)acc), "r"(one) : "memory");
}
__device__ __forceinline__ void pw_mma_ts(unsigned d, unsigned a, unsigned long long b, unsigned idesc, bool acc, unsigned one) {
  asm volatile("{\n.reg .pred p, e;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 e, %5, 0;\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((unsigned)acc), "r"(one) : "memory");
}
__device__ __forceinline__ void pw_commit(unsigned long long* bar, unsigned one) {
  asm volatile("{\n.reg .pred e;\nsetp.ne.b32 e, %1, 0;\n@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n"
               ::"r"(pf_smem(bar)), "r"(one) : "memory");
}
#define PW_R32(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define PW_I32(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])
// 32 columns of the thread's row (no wait)
__device__ __forceinline__ void pw_ld32(unsigned addr, unsigned* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
               "%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : PW_R32(r, 0), PW_R32(r, 8), PW_R32(r, 16), PW_R32(r, 24) : "r"(addr));
}
// 16 rows (the warp's lanes 0-15 or 16-31 of tensor memory) x 64 columns: registers 4j + {0, 1} are row lane / 4, {2, 3} row lane / 4 + 8, columns
// 8j + 2 (lane % 4) + {0, 1} (no wait)
__device__ __forceinline__ void pw_ld_frag(unsigned addr, unsigned* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
               "%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : PW_R32(r, 0), PW_R32(r, 8), PW_R32(r, 16), PW_R32(r, 24) : "r"(addr));
}
__device__ __forceinline__ void pw_st32(unsigned addr, const unsigned* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
               "%25,%26,%27,%28,%29,%30,%31};"
               ::PW_I32(r, 0), PW_I32(r, 8), PW_I32(r, 16), PW_I32(r, 24), "r"(addr) : "memory");
}
__device__ __forceinline__ void pw_st16(unsigned addr, const unsigned* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               ::PW_I32(r, 0), PW_I32(r, 8), "r"(addr) : "memory");
}
#define PW_T32(r, o) "+r"(r[o]), "+r"(r[o + 1]), "+r"(r[o + 2]), "+r"(r[o + 3]), "+r"(r[o + 4]), "+r"(r[o + 5]), "+r"(r[o + 6]), "+r"(r[o + 7])
// the loads so far are done; the registers are named so that no use of them moves in front of the wait
__device__ __forceinline__ void pw_ld_wait(unsigned* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : PW_T32(r, 0), PW_T32(r, 8), PW_T32(r, 16), PW_T32(r, 24) :: "memory");
}
__device__ __forceinline__ void pw_ld_wait(unsigned* r, unsigned* r2) {
  pw_ld_wait(r);
  asm volatile("" : PW_T32(r2, 0), PW_T32(r2, 8), PW_T32(r2, 16), PW_T32(r2, 24) :: "memory");
}
__device__ __forceinline__ void pw_st1(unsigned addr, unsigned r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%1], {%0};" ::"r"(r), "r"(addr) : "memory");
}
// packed pairs of fp32: one instruction for two scores
__device__ __forceinline__ unsigned long long pw_pair(float lo, float hi) {
  unsigned long long d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void pw_unpair(unsigned long long d, float* lo, float* hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*lo), "=f"(*hi) : "l"(d)); }
__device__ __forceinline__ unsigned long long pw_fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ unsigned long long pw_add2(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float pw_max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void pw_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pw_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void pw_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// barrier of the softmax threads that also makes `ok` the same in all of them
__device__ __forceinline__ bool pw_all_ok(bool ok) {
  unsigned r;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbarrier.cta.red.and.pred p, 1, 256, q;\nselp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(r) : "r"((unsigned)ok) : "memory");
  return r != 0;
}

struct WideArgs {
  AttnArgs a;
  int flip;                                     // 1: the scale is negative (scale2 holds its magnitude; Q's signs are flipped)
  int box;                                      // rows of a TMA box: min(page, 128)
  unsigned delay_ns;                            // 0; the self-test holds the loads back
  unsigned long long limit_ns;                  // a wait gives up after it
};

// QTMA: Q comes by TMA, boxes of (64 elements, the query heads of a K/V head, rows), which lie in shared memory as the stacked rows do.  Needs a
// number of query heads per K/V head that divides 128 and a positive scale; otherwise the softmax warps copy it (through L2, behind the
// first K and V tiles: 5-8 us later).
template <typename T, int D, bool QTMA>
__global__ void __launch_bounds__(PW_THREADS, 1) prefix_wide_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                                                                    const __grid_constant__ CUtensorMap tm_q, WideArgs w) {
  using W = Wide<D>;
  extern __shared__ __align__(1024) unsigned char pw_raw[];
  __shared__ __align__(8) unsigned long long full[W::SLOTS], empty[W::SLOTS], s_full[2], p_full[2][2], q_full, o_full, o_free, drain;
  __shared__ unsigned tmem_slot;
  __shared__ int abort_flag;
  const AttnArgs& a = w.a;
  const PlanMem pm = plan_mem(a.mem, a.n, a.rows, a.n_heads, D);
  int* const error = &pm.head->error;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, run = blockIdx.x;
  unsigned char* const smem = pw_raw;
  const unsigned q_s = pf_smem(smem), ring = q_s + 2 * W::TILE;
  float* const red_m = reinterpret_cast<float*>(smem + W::TILE * (2 + W::SLOTS));            // [2][128] each
  float* const red_l = red_m + 256;
  if (tid == 0) {
    for (int i = 0; i < W::SLOTS; ++i) { pw_bar_init(&full[i], 1); pw_bar_init(&empty[i], 1); }
    for (int i = 0; i < 2; ++i) { pw_bar_init(&s_full[i], 1); pw_bar_init(&p_full[i][0], 128); pw_bar_init(&p_full[i][1], 128); }
    pw_bar_init(&q_full, QTMA ? 1 : PW_SOFT); pw_bar_init(&o_full, 1); pw_bar_init(&o_free, PW_SOFT); pw_bar_init(&drain, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  if (pf_smem(pw_raw) & 1023u) { if (tid == 0) atomicExch(error, VLAC_ERR_TIMEOUT); return; }        // (the swizzled tiles need it; uniform)
  const long long U = pm.head->units[WIDE], G = runs(WIDE, U);
  const int g_first = pm.first[WIDE][run];
  if (run >= G || pm.head->key != a.key) return;                        // uniform over the CTA
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(pf_smem(&tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pw_before();
  __syncthreads();
  pw_after();
  const unsigned tmem = tmem_slot;                                      // columns: S/P even 0, S/P odd 128, O even 256, O odd 384
  Cursor cur;
  cur.begin(pm, WIDE, run, U, G, g_first);
  Piece p;
  int sent = 0;                                                         // loads: tiles this warp has asked for; products: pieces' Q

  if (warp < 4 && warp != 1) {
    // ---------------------------------------------------------------- loads
    // Issuing a box takes a warp about 110 cycles whichever lane does it, and a tile of small pages has up to 32 of them (8 rows): the
    // boxes of a tile are shared out over three warps.  Each waits for the slot itself; one adds the byte count (a barrier's count of
    // bytes may run ahead of it: the phase ends only with the arrival).
    const int first = warp == 0 ? 0 : warp - 1;                         // 0, 1, 2
    const int n_box = 128 / w.box * W::HALVES, b = first + 3 * lane, chunk = b / W::HALVES, half = b % W::HALVES;
    const bool mine = b < n_box;
    const int none = a.n_pages << a.shift;                              // a row behind the pool: zeros
    bool ok = true;
    if (w.delay_ns) for (const unsigned long long t0 = pw_ns(); pw_ns() - t0 < w.delay_ns;) __nanosleep(500);
    auto put = [&](const CUtensorMap* tm, int y, int x0) {
      const int s = sent % W::SLOTS;
      if (sent >= W::SLOTS) ok = __all_sync(0xffffffffu, pw_wait(&empty[s], ((sent / W::SLOTS) & 1) ^ 1, &abort_flag, error, w.limit_ns));
      if (!ok) return;
      if (first == 0 && lane == 0) pw_expect(&full[s], W::TILE);
      if (mine) pw_tma(ring + (unsigned)s * W::TILE + (unsigned)half * W::HALF + (unsigned)chunk * w.box * 128u, tm, x0 + half * 64, y, &full[s]);
      __syncwarp();
      ++sent;
    };
    while (cur.more() && ok) {
      cur.next(pm, &p);
      const int* tab = a.table + (size_t)p.slot * a.max_pages;
      auto row = [&](int i) -> int {                                    // pool row of this lane's box of key block i
        const int key = p.key0 + i * 128 + chunk * w.box;
        if (!mine || key >= p.key1) return none;
        const int pg = tab[key >> a.shift];
        return (unsigned)pg < (unsigned)a.n_pages ? (pg << a.shift) + (key & (a.page - 1)) : none;
      };
      const bool two = p.nr > 128;
      int y = row(0), yp = 0;
      for (int i = 0; i < p.n && ok; ++i) {
        const int yn = i + 1 < p.n ? row(i + 1) : none;                 // fetched a block ahead of its use
        put(&tm_k, y, p.head * D);
        if (two) { if (ok) put(&tm_v, y, p.head * D); }
        else if (i > 0 && ok) put(&tm_v, yp, p.head * D);
        yp = y; y = yn;
      }
      if (ok && !two) put(&tm_v, yp, p.head * D);
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- products
    unsigned one;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(one));
    const unsigned tm = __shfl_sync(0xffffffffu, tmem, 0);
    const unsigned id_s = pw_idesc<T>(128, false), id_o = pw_idesc<T>(D, true);
    const unsigned long long q_d = pw_desc(q_s, 16, 1024), k_d = pw_desc(ring, 16, 1024), v_d = pw_desc(ring, W::HALF, 1024);
    // A wait on the way of every product has to be short (its dependent instructions are issued between those of the softmax warps): an
    // address and a parity at hand, and failures looked at once a block.
    const unsigned full_a = pf_smem(full), p_a = pf_smem(p_full);
    int slot = 0, pieces = 0, n_p[2] = {0, 0};
    unsigned phase = 0, failed = 0;
    bool ok = true;
    auto wait_at = [&](unsigned bar, unsigned parity) {
      if (!__all_sync(0xffffffffu, pw_try_at(bar, parity))) {            // (all lanes or none)
        failed |= !pw_wait_slow(bar, parity, &abort_flag, error, w.limit_ns);
        __syncwarp();
      }
    };
    auto still_ok = [&]() { return __all_sync(0xffffffffu, !failed); };
    auto same = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };    // tells the compiler that a value is the same in all lanes
    auto place = [&](int ahead) { const int sl = slot + ahead; return sl >= W::SLOTS ? sl - W::SLOTS : sl; };
    auto there = [&](int ahead) { wait_at(full_a + 8u * place(ahead), phase ^ (slot + ahead >= W::SLOTS)); };   // the ring's tile `ahead` places on
    auto next = [&]() { pw_commit(&empty[slot], one); if (++slot == W::SLOTS) { slot = 0; phase ^= 1; } };       // its first tile is done with
    auto s_mma = [&](int b, int q_tile, int sl) {                       // S of side b from the tile of Q and the K tile in slot sl
      const int bu = same(b);
      const unsigned long long d = k_d + (unsigned long long)(same(sl) * (W::TILE >> 4)), qd = q_d + (unsigned long long)(same(q_tile) * (W::TILE >> 4));
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const unsigned off = ((unsigned)(ks >> 2) * W::HALF + (unsigned)(ks & 3) * 32u) >> 4;
        pw_mma_ss(tm + 128u * bu, qd + off, d + off, id_s, ks > 0, one);
      }
      pw_commit(&s_full[b], one);
    };
    auto pv_mma = [&](int b, int sl, bool add) {                        // O of side b; the weights' halves arrive one after the other
      const int bu = same(b);
      const unsigned acc = same(add), par = n_p[b]++ & 1;
      const unsigned long long d = v_d + (unsigned long long)(same(sl) * (W::TILE >> 4));
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        wait_at(p_a + 16u * b + 8u * hf, par);
        pw_after();
#pragma unroll
        for (int j = 4 * hf; j < 4 * hf + 4; ++j)                       // 16 keys: 8 columns of packed P; 16 rows of V (MN-major)
          pw_mma_ts(tm + 256u + 128u * bu, tm + 128u * bu + 8u * j, d + 128u * j, id_o, acc || j > 0, one);
      }
    };
    // The weights come last, so everything else is waited for before them: O += P V and the side's next S, which takes the columns that P
    // leaves, then go out in one burst.
    while (cur.more() && ok) {
      cur.next(pm, &p);
      const int n = same(p.n), two = same(p.nr > 128);
      if (QTMA) {
        if (pieces > 0) wait_at(pf_smem(&o_full), (pieces - 1) & 1);    // the last piece's products are done: Q's memory is free
        if (one) {
          pw_expect(&q_full, (unsigned)(W::TILE << two));
          for (int t = 0; t <= two; ++t)
#pragma unroll
            for (int hf = 0; hf < W::HALVES; ++hf)
              pw_tma3(q_s + t * W::TILE + hf * W::HALF, &tm_q, hf * 64, p.head * a.ratio, p.row0 + (p.rt * 256 + t * 128) / a.ratio, &q_full);
        }
        ++sent;
        __syncwarp();
      }
      there(0);
      if (QTMA && pieces > 0) wait_at(pf_smem(&o_free), (pieces - 1) & 1);                     // and its O has been read
      wait_at(pf_smem(&q_full), pieces & 1);
      ok = still_ok();
      if (!ok) break;
      pw_after();
      s_mma(0, 0, slot);
      if (two) {                                                        // tiles K_0, V_0, K_1, V_1, ...
        s_mma(1, 1, slot);
        next();
        for (int i = 0; i < n; ++i) {
          const bool more = i + 1 < n;
          there(0);
          if (more) there(1);
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            pv_mma(b, slot, i > 0);
            if (more) s_mma(b, b, place(1));
          }
          next();
          if (more) next();
          ok = still_ok();
          if (!ok) break;
        }
      } else {                                                          // tiles K_0, K_1, V_0, K_2, V_1, ..., V_{n-1}
        next();
        if (n > 1) { there(0); s_mma(1, 0, slot); next(); }
        for (int i = 0; i < n; ++i) {
          there(0);
          if (i + 2 < n) there(1);
          pv_mma(i & 1, slot, i > 1);
          next();
          if (i + 2 < n) { s_mma(i & 1, 0, slot); next(); }
          ok = still_ok();
          if (!ok) break;
        }
      }
      if (ok) pw_commit(&o_full, one);
      ++pieces;
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ---------------------------------------------------------------- softmax
    const int st = tid - 128, side = st >> 7, q4 = warp & 3, r = 32 * q4 + lane;
    const unsigned trow = tmem + ((unsigned)(32 * q4) << 16), s_col = trow + 128u * side, o_col = trow + 256u + 128u * side;
    int n_s = 0, pieces = 0;
    bool ok = true;
    // Q of a piece: all loads first (a store between them would make each wait for the one before), and for the next piece before the
    // present one is written out
    constexpr int C16 = D / 8, NQ = 128 * C16 / 128;
    uint4 qv[NQ];
    // 16-byte pieces of Q: with two tiles each side copies its own (NQ a thread), otherwise both share one (NQ / 2)
    auto load_q = [&](const Piece& p) {
      // stacked row x is q row row0 + x / ratio, query head head * ratio + x % ratio; rows behind the last are zeros
      const bool two = p.nr > 128;
      const int x0 = p.rt * 256, q0 = x0 / a.ratio, h0 = x0 - q0 * a.ratio, c0 = two ? side * 128 * C16 + (st & 127) : st, dc = two ? 128 : 256;
      const T* src = (const T*)a.q + (size_t)(p.row0 + q0) * a.q_stride + (size_t)p.head * a.ratio * D;
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        if (i >= NQ / 2 && !two) break;
        const int c = c0 + i * dc, qr = c / C16, c16 = c % C16, x = h0 + qr, xq = x / a.ratio;
        qv[i] = make_uint4(0, 0, 0, 0);
        if (qr < p.nr) qv[i] = *reinterpret_cast<const uint4*>(src + (size_t)xq * a.q_stride + (x - xq * a.ratio) * D + c16 * 8);
      }
    };
    cur.next(pm, &p);
    if (!QTMA) load_q(p);
    while (true) {
      const bool two = p.nr > 128;
      const int c0 = two ? side * 128 * C16 + (st & 127) : st, dc = two ? 128 : 256;
#pragma unroll
      for (int i = 0; i < (QTMA ? 0 : NQ); ++i) {
        if (i >= NQ / 2 && !two) break;
        const int c = c0 + i * dc, qr = c / C16, c16 = c % C16;
        if (w.flip) { qv[i].x ^= 0x80008000u; qv[i].y ^= 0x80008000u; qv[i].z ^= 0x80008000u; qv[i].w ^= 0x80008000u; }
        *reinterpret_cast<uint4*>(smem + (qr >> 7) * W::TILE + (c16 >> 3) * W::HALF + pf_swz(qr & 127, c16 & 7)) = qv[i];
      }
      if (!QTMA) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        pw_before();
        pw_arrive(&q_full);
      }
      float m = -INFINITY, l = 0.f;
      const int row_t = (two ? 128 * side : 0) + r;                     // the thread's row in the tile
      const bool idle = row_t - lane >= p.nr;                           // a warp without rows: only its arrivals are needed
      const int step = two ? 1 : 2, first = two ? 0 : side;
      for (int i = first; i < p.n; i += step) {
        ok = __all_sync(0xffffffffu, pw_wait(&s_full[side], n_s++ & 1, &abort_flag, error, w.limit_ns));
        if (!ok) break;
        if (!idle) {
          pw_after();
          const int valid = p.key1 - p.key0 - i * 128;                  // keys of this block (fewer than 128 in the last)
          if (valid < 128) {
            for (int c = valid; c < 128; ++c) pw_st1(s_col + c, 0xff800000u);             // -inf behind them
            pw_st_wait();
          }
          // P is rounded to the 16-bit type for the product with V (half a step: 2^-8 of each weight for bf16, 2^-11 for fp16 and at least 2^-34 of the
          // largest one, see Half2); the sum takes the unrounded weights.  P lies over scores already read: 16 columns for 32.
          const unsigned long long sc = pw_pair(a.scale2, a.scale2);
          unsigned long long ls[2] = {0ull, 0ull};                      // two fp32 sums each
          auto weights = [&](const unsigned* v, unsigned long long nr, unsigned* pk) {
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              float x0, x1;
              pw_unpair(pw_fma2(pw_pair(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1])), sc, nr), &x0, &x1);
              x0 = pf_ex2(x0); x1 = pf_ex2(x1);
              ls[c & 1] = pw_add2(ls[c & 1], pw_pair(x0, x1));
              pk[c] = Half2<T>::pack(x0, x1);
            }
          };
          // The weights of the first half are formed with the reference of the block before while the maximum of all 128 scores is still being
          // found, and formed again in the rare block that moves the reference.  It moves when the maximum has grown by a factor of 2^8 (fp16: 2^6):
          // larger weights cost no precision (they are rounded relative to themselves, l is fp32), and O is seldom rescaled.
          unsigned pk[32], v[32], x[32];
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          {
            const float ref = m == -INFINITY ? 0.f : m;
            const unsigned long long nr = pw_pair(-ref, -ref);
            pw_ld32(s_col, v);
            pw_ld32(s_col + 64u, x);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              pw_ld_wait(v, x);
#pragma unroll
              for (int c = 0; c < 16; ++c) {
                mx[c & 3] = pw_max3(mx[c & 3], __uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1]));
                mx[c & 3] = pw_max3(mx[c & 3], __uint_as_float(x[2 * c]), __uint_as_float(x[2 * c + 1]));
              }
              if (q == 0) pw_ld32(s_col + 96u, x);
              weights(v, nr, pk + 16 * q);
              if (q == 0) pw_ld32(s_col + 32u, v);
            }
          }
          const float bm = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale2 - Half2<T>::shift_wide;
          const bool grow = bm > m + Half2<T>::growth || m == -INFINITY;
          if (__any_sync(0xffffffffu, grow)) {
            const float mn = grow ? fmaxf(m, bm) : m;
            const float al = mn == -INFINITY ? 1.f : pf_ex2(m - mn);    // (m = -inf: nothing summed yet, 0 * 0)
            m = mn;
            l *= al;
            if (i >= step) {
#pragma unroll 1
              for (int c = 0; c < D / 32; ++c) {
                pw_ld32(o_col + 32u * c, x);
                pw_ld_wait(x);
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * al);
                pw_st32(o_col + 32u * c, x);
              }
            }
            ls[0] = ls[1] = 0ull;
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              pw_ld32(s_col + 32u * q, v);
              pw_ld_wait(v);
              weights(v, pw_pair(-ref, -ref), pk + 16 * q);
            }
          }
          pw_ld32(s_col + 64u, v);
          pw_st32(s_col, pk);
          pw_st_wait();
          pw_before();
          pw_arrive(&p_full[side][0]);
          {
            const float ref = m == -INFINITY ? 0.f : m;
            const unsigned long long nr = pw_pair(-ref, -ref);
            pw_ld32(s_col + 96u, x);
            pw_ld_wait(v, x);
            weights(v, nr, pk);
            weights(x, nr, pk + 16);
            pw_st32(s_col + 32u, pk);
          }
          float l0, l1, l2, l3;
          pw_unpair(ls[0], &l0, &l1); pw_unpair(ls[1], &l2, &l3);
          l += (l0 + l1) + (l2 + l3);
          pw_st_wait();
        } else pw_arrive(&p_full[side][0]);
        pw_before();
        pw_arrive(&p_full[side][1]);
      }
      Piece pn;
      const bool more = cur.more();
      if (more) { cur.next(pm, &pn); if (!QTMA) load_q(pn); }
      if (ok) ok = pw_wait(&o_full, pieces & 1, &abort_flag, error, w.limit_ns);
      ++pieces;
      ok = pw_all_ok(ok);                                               // every product of the piece is done: Q's memory is free
      __syncwarp();
      if (!ok) break;
      if (!two) {
        red_m[side * 128 + r] = m; red_l[side * 128 + r] = l;
        pw_all_ok(true);
      }
      pw_after();
      if (!idle) {
        // O in the layout of fragments: four lanes hold 32 bytes of a row, which go out together
        if (two) {
          // every side its own rows
#pragma unroll 1
          for (int q = 0; q < 2 * (D / 64); ++q) {
            const int hf = q & 1, c0 = (q >> 1) * 64, row = row_t - lane + 16 * hf + (lane >> 2);
            unsigned x[32];
            pw_ld_frag(o_col + ((unsigned)(16 * hf) << 16) + c0, x);
            pw_ld_wait(x);
            float* dst = pm.po + (p.slot0 + row) * D + c0 + 2 * (lane & 3);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              if (row < p.nr) *reinterpret_cast<uint2*>(dst + 8 * j) = make_uint2(x[4 * j], x[4 * j + 1]);
              if (row + 8 < p.nr) *reinterpret_cast<uint2*>(dst + 8 * D + 8 * j) = make_uint2(x[4 * j + 2], x[4 * j + 3]);
            }
          }
          if (row_t < p.nr) pm.ml[p.slot0 + row_t] = make_float2(m, l);
        } else {
          // the two sides of a row: this side 16 of the warp's 32 rows
          const bool odd = p.n > 1;                                     // one block: the odd side holds nothing
          const int row = 32 * q4 + 16 * side + (lane >> 2);
          float f0[2], f1[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int rr = row + 8 * e;
            const float m0 = red_m[rr], m1 = red_m[128 + rr], M = fmaxf(m0, m1), ref = M == -INFINITY ? 0.f : M;
            f0[e] = pf_ex2(m0 - ref); f1[e] = pf_ex2(m1 - ref);
            if ((lane & 3) == 0 && rr < p.nr) pm.ml[p.slot0 + rr] = make_float2(M, f0[e] * red_l[rr] + (odd ? f1[e] * red_l[128 + rr] : 0.f));
          }
#pragma unroll 1
          for (int c0 = 0; c0 < D; c0 += 64) {
            unsigned x[32], y[32] = {};
            pw_ld_frag(trow + ((unsigned)(16 * side) << 16) + 256u + c0, x);
            if (odd) pw_ld_frag(trow + ((unsigned)(16 * side) << 16) + 384u + c0, y);
            pw_ld_wait(x, y);
            float* dst = pm.po + (p.slot0 + row) * D + c0 + 2 * (lane & 3);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float2 o = make_float2(f0[e] * __uint_as_float(x[4 * j + 2 * e]), f0[e] * __uint_as_float(x[4 * j + 2 * e + 1]));
                if (odd) { o.x += f1[e] * __uint_as_float(y[4 * j + 2 * e]); o.y += f1[e] * __uint_as_float(y[4 * j + 2 * e + 1]); }
                if (row + 8 * e < p.nr) *reinterpret_cast<float2*>(dst + e * 8 * D + 8 * j) = o;
              }
          }
        }
      }
      if (!more) break;
      if (QTMA) {
        pw_before();
        pw_arrive(&o_free);
      }
      p = pn;
    }
    pw_before();
  }
  __syncthreads();
  if (abort_flag) {                                                     // somebody gave up (uniform): what is in flight lands first, products and copies
    int alone = 0;
    if (warp == 1) {
      unsigned one;
      asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(one));        // (the lane that issued the products)
      pw_commit(&drain, one);
      pw_wait(&drain, 0, &alone, error, PW_WAIT_LIMIT_NS);
      if (QTMA && sent > 0) pw_wait(&q_full, (sent - 1) & 1, &alone, error, PW_WAIT_LIMIT_NS);
    } else if (warp < 4)
      for (int c = max(0, sent - W::SLOTS); c < sent; ++c) pw_wait(&full[c % W::SLOTS], (c / W::SLOTS) & 1, &alone, error, PW_WAIT_LIMIT_NS);
    __syncwarp();
  }
  if (warp == 1) {
    pw_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// Pieces to results: grid (sequences, shares); a warp takes (K/V head, stacked row) items of its sequence and adds the pieces of the row's
// prefix and of its own segment in order, B partial sums and their (m, l) in flight.  SHARE, for calls of few items, which may have hundreds
// of pieces each: a CTA takes an item, its warps every eighth piece, and their sums are added in order.
template <typename T, int D, bool SHARE, int B, int OCC>
__global__ void __launch_bounds__(256, OCC) prefix_join_kernel(AttnArgs a) {
  __shared__ float4 s_o[SHARE ? 8 : 1][D / 4];
  __shared__ float2 s_ml[8];
  const int warp = threadIdx.x >> 5;
  const PlanMem p = plan_mem(a.mem, a.n, a.rows, a.n_heads, D);
  const int lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  const PlanHead hd = *p.head;
  const SeqRec q = p.seq[blockIdx.x];
  if (hd.key != a.key) {                                                // (0: no plan yet)
    if (hd.key != 0 && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicExch(&p.head->error, VLAC_ERR_INVALID_ARG);
    return;
  }
  if ((int)blockIdx.x >= hd.n_act || q.slot < 0) return;                // (slot -1: refused)
  SegRec sg[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) sg[i] = p.seg[max(0, i ? q.suf_seg : q.pre_seg)];
  const int per = q.nq * a.ratio, items = per * a.kv_heads;
  const int c4 = lane < D / 4 ? lane : 0;
  for (int it = SHARE ? blockIdx.y : blockIdx.y * 8 + warp; it < items; it += SHARE ? gridDim.y : gridDim.y * 8) {
    const int kvh = it / per, xr = it - kvh * per, xq = xr / a.ratio, row = q.row0 + xq, h = kvh * a.ratio + xr - xq * a.ratio;
    int np[2] = {0, 0}, pad[2] = {0, 0};
    size_t base[2] = {0, 0};
    bool done = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if ((i ? q.suf_seg : q.pre_seg) < 0) continue;
      const SegRec& s = sg[i];
      const int bm = pf_bm(s.cls), x = (row - s.row0) * a.ratio + xr - xq * a.ratio, rt = x / bm;
      const long long U = hd.units[s.cls], u0 = s.ustart + ((long long)kvh * s.T + rt) * s.KB;
      const int c0 = run_of(s.cls, u0, U), c1 = run_of(s.cls, u0 + s.KB - 1, U);
      if (s.pos0 != INT_MIN && s.key0 == 0 && c0 == c1) done = true;    // written by its only piece
      np[i] = c1 - c0 + 1;
      pad[i] = bm;
      base[i] = (size_t)s.rowbase + (size_t)kvh * s.R + x + (size_t)c0 * bm;
    }
    if (done) continue;
    const int n = np[0] + np[1];
    float M = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    const int step = SHARE ? 8 : 1;
    for (int i0 = SHARE ? warp : 0; i0 < n; i0 += B * step) {
      float2 ml[B];
      float4 v[B];
#pragma unroll
      for (int e = 0; e < B; ++e) {
        const int i = i0 + e * step, first = i < np[0];
        ml[e] = make_float2(-INFINITY, 0.f);
        v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n) {
          const size_t sl = first ? base[0] + (size_t)i * pad[0] : base[1] + (size_t)(i - np[0]) * pad[1];
          ml[e] = p.ml[sl];
          v[e] = *reinterpret_cast<const float4*>(p.po + sl * D + c4 * 4);
        }
      }
      float m = M;
#pragma unroll
      for (int e = 0; e < B; ++e) m = fmaxf(m, ml[e].x);
      const float ref = m == -INFINITY ? 0.f : m, f = pf_ex2(M - ref);
      M = m;
      l *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
      for (int e = 0; e < B; ++e) {
        const float g = pf_ex2(ml[e].x - ref);
        l += g * ml[e].y;
        o.x += g * v[e].x; o.y += g * v[e].y; o.z += g * v[e].z; o.w += g * v[e].w;
      }
    }
    if (SHARE) {
      if (lane < D / 4) s_o[warp][lane] = o;
      if (lane == 0) s_ml[warp] = make_float2(M, l);
      __syncthreads();
      if (warp == 0) {
        M = -INFINITY; l = 0.f;
        o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) M = fmaxf(M, s_ml[e].x);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float g = pf_ex2(s_ml[e].x - ref);
          const float4 v = s_o[e][c4];
          l += g * s_ml[e].y;
          o.x += g * v.x; o.y += g * v.y; o.z += g * v.z; o.w += g * v.w;
        }
      }
      __syncthreads();
      if (warp != 0) continue;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (lane < D / 4)
      *reinterpret_cast<uint2*>((T*)a.out + (size_t)row * a.out_stride + (size_t)h * D + lane * 4) =
          make_uint2(Half2<T>::pack(o.x * inv, o.y * inv), Half2<T>::pack(o.z * inv, o.w * inv));
    if (a.lse && lane == 0) a.lse[(size_t)row * a.n_heads + h] = (M + log2f(l)) * PF_LN2;
  }
}

#define TRY(x) do { const int rc__ = (x); if (rc__ != VLAC_OK) return rc__; } while (0)

template <typename T, int D, bool QTMA>
int launch_wide(const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tq, const WideArgs& w, cudaStream_t s) {
  TRY((big_smem<prefix_wide_kernel<T, D, QTMA>>(Wide<D>::SMEM)));
  VLAC_CUDA_CHECK(launch_pdl(prefix_wide_kernel<T, D, QTMA>, dim3(PW_CTAS), dim3(PW_THREADS), Wide<D>::SMEM, s, tk, tv, tq, w));
  return VLAC_OK;
}

template <typename T, int D, bool EARLY, bool TREE>
int launch_narrow(const AttnArgs& a, cudaStream_t s) {
  TRY((big_smem<prefix_narrow_kernel<T, D, EARLY, TREE>>(Narrow<D>::SMEM)));
  VLAC_CUDA_CHECK(launch_pdl(prefix_narrow_kernel<T, D, EARLY, TREE>, dim3(PN_CTAS), dim3(PN_WARPS * 32), Narrow<D>::SMEM, s, a));
  return VLAC_OK;
}

template <typename T, int D>
int launch_attention(const AttnArgs& a, bool small, unsigned delay_ns, unsigned long long limit_ns, cudaStream_t s) {
  // more than 16 stacked rows, or the call cannot have a wide segment
  if ((long long)a.rows * a.ratio > pf_bm(NARROW) && !small) {
    WideArgs w = {a, a.scale2 < 0.f, a.page < 128 ? a.page : 128, delay_ns, limit_ns};
    w.a.scale2 = fmaxf(fabsf(a.scale2), 1e-30f);                        // not zero: -inf marks what is not there
    CUtensorMap tk, tv, tq;
    const int rows = a.n_pages << a.shift, cols = a.kv_heads * D;
    TRY(vlac_encode_map_2d(&tk, a.k, rows, cols, w.box));
    TRY(vlac_encode_map_2d(&tv, a.v, rows, cols, w.box));
    if (!w.flip && 128 % a.ratio == 0) {
      TRY(vlac_encode_map_heads(&tq, a.q, a.rows, a.n_heads, D, a.q_stride, a.ratio, 128 / a.ratio));
      TRY((launch_wide<T, D, true>(tk, tv, tq, w, s)));
    } else
      TRY((launch_wide<T, D, false>(tk, tv, tk, w, s)));
    TRY((a.mask ? launch_narrow<T, D, true, true>(a, s) : launch_narrow<T, D, true, false>(a, s)));
  } else
    TRY((a.mask ? launch_narrow<T, D, false, true>(a, s) : launch_narrow<T, D, false, false>(a, s)));
  // an item a CTA while the GPU holds them in two waves, else an item a warp (what an item costs is the chain of its reads): 32 rows behind
  // 32,768 positions of 8 heads 33 us against 46, but 1024 items behind 65,600 84 against 79
  const long long items = (long long)a.rows * a.n_heads, mean = (items + a.n - 1) / a.n;
  // (a row's pieces are about as many as runs per tile: more items, fewer pieces, and then more warps in flight count for more than loads)
  const dim3 grid(a.n, (unsigned)std::max(1ll, std::min({(mean + 7) / 8, 4096ll / a.n + 1, 65535ll})));
  if (items <= 592) VLAC_CUDA_CHECK(launch_pdl(prefix_join_kernel<T, D, true, 4, 2>, dim3(a.n, (unsigned)mean), dim3(256), 0, s, a));
  else if (items < 8192) VLAC_CUDA_CHECK(launch_pdl(prefix_join_kernel<T, D, false, 8, 2>, grid, dim3(256), 0, s, a));
  else VLAC_CUDA_CHECK(launch_pdl(prefix_join_kernel<T, D, false, 4, 4>, grid, dim3(256), 0, s, a));
  return VLAC_OK;
}

// Whether a call has no wide segments: not more than one narrow unit a warp, judged by what the host knows (the tables' width, not the lengths).
// The wide kernel is not launched then: 12 rows of 32 heads behind 288 positions of 8 K/V heads 15.1 -> 11.3 us, but 42 rows behind 1024
// (twice the units) would go from 15.4 to 18.4.
bool small_call(const vlac_pages* p, const vlac_prefix* plan) {
  const long long ratio = plan->n_heads / p->n_kv_heads, tiles = ((long long)plan->rows * ratio + 15) / 16 + plan->n;
  const long long blocks = (long long)p->max_pages * p->page_size / NARROW_KEYS + 2;
  return p->n_kv_heads * tiles * blocks <= pf_runs(NARROW);
}

// 64 bits of everything that the records of a plan and the tables' extent depend on, and of the tables' address (the steps of splitmix64 by
// Steele, Lea and Flood over one field after the other: two different calls agree by a chance of 2^-64); never 0.
unsigned long long plan_key(const vlac_pages* p, const vlac_prefix* plan) {
  const unsigned long long fields[] = {(unsigned long long)(uintptr_t)p->table, (unsigned)p->n_slots, (unsigned)p->max_pages, (unsigned)p->n_pages, (unsigned)p->page_size,
                                       (unsigned)p->n_kv_heads, (unsigned)p->head_dim, (unsigned)plan->n_heads, (unsigned)plan->n, (unsigned)plan->rows};
  unsigned long long h = 0;
  for (const unsigned long long f : fields) {
    h = (h ^ f) + 0x9e3779b97f4a7c15ull;
    h = (h ^ (h >> 30)) * 0xbf58476d1ce4e5b9ull;
    h = (h ^ (h >> 27)) * 0x94d049bb133111ebull;
    h ^= h >> 31;
  }
  return h ? h : 1;
}

int plan_check(const vlac_pages* p, const vlac_prefix* plan) {
  const int rc = pages_check(p);
  if (rc != VLAC_OK) return rc;
  if (!plan || plan->n < 0 || plan->rows < 0) return VLAC_ERR_INVALID_ARG;
  if (plan->n > VLAC_PAGES_MAX_LIST) return VLAC_ERR_TOO_LARGE;
  // positions behind a sequence's end, up to a unit of keys or the page numbers that a warp fetches at once (512), are formed in 32 bits
  if ((long long)p->max_pages * p->page_size > INT_MAX - 1024) return VLAC_ERR_INVALID_ARG;
  if (plan->n == 0 || plan->rows == 0) return VLAC_OK;
  const unsigned long long need = vlac_prefix_bytes(p, plan->n, plan->rows, plan->n_heads);
  if (need == 0 || !plan->mem || ((uintptr_t)plan->mem & 15u) || plan->bytes < need) return VLAC_ERR_INVALID_ARG;
  return VLAC_OK;
}

int attention(const vlac_pages* p, int layer, const vlac_prefix* plan, const vlac_tree* tree, const void* q, long long q_stride, float scale, void* out,
              long long out_stride, float* lse, unsigned delay_ns, unsigned long long limit_ns, cudaStream_t s) {
  const int rc = plan_check(p, plan);
  if (rc != VLAC_OK) return rc;
  if (tree && (tree->n != plan->n || tree->rows != plan->rows || tree->max_rows < 1 || tree->max_rows > VLAC_TREE_MAX_ROWS)) return VLAC_ERR_INVALID_ARG;
  if (layer < 0 || layer >= p->n_layers || !isfinite(scale * PF_LOG2E)) return VLAC_ERR_INVALID_ARG;
  if (plan->n == 0 || plan->rows == 0) return VLAC_OK;
  const long long w = (long long)plan->n_heads * p->head_dim;
  if (!q || !out || q_stride < w || out_stride < w || q_stride % 8 || out_stride % 8 || (((uintptr_t)q | (uintptr_t)out) & 15u) || ((uintptr_t)lse & 3u))
    return VLAC_ERR_INVALID_ARG;
  if (rows_overlap((uintptr_t)q, 2ull * q_stride, (uintptr_t)out, 2ull * out_stride, 2ull * w, 2ull * w, plan->rows)) return VLAC_ERR_INVALID_ARG;
  if (rows_in_pool(p, out, 2ull * out_stride, 2ull * w, plan->rows)) return VLAC_ERR_INVALID_ARG;
  if (lse && rows_touch(lse, 4ull * plan->rows * plan->n_heads, out, 2ull * out_stride, 2ull * w, plan->rows)) return VLAC_ERR_INVALID_ARG;
  if (tree && (!tree->mask || (uintptr_t)tree->mask & 3u)) return VLAC_ERR_INVALID_ARG;
  AttnArgs a = {};
  if (tree) { a.mask = tree->mask; a.words = (tree->max_rows + 31) / 32; }
  a.k = (const unsigned short*)p->k + (size_t)layer * pages_layer(p); a.v = (const unsigned short*)p->v + (size_t)layer * pages_layer(p);
  a.table = p->table; a.max_pages = p->max_pages; a.n_pages = p->n_pages; a.page = p->page_size; a.shift = pages_shift(p->page_size);
  a.kv_heads = p->n_kv_heads; a.ratio = plan->n_heads / p->n_kv_heads; a.n_heads = plan->n_heads; a.n = plan->n; a.rows = plan->rows;
  a.q = q; a.q_stride = q_stride; a.out = out; a.out_stride = out_stride; a.lse = lse;
  a.scale2 = scale * PF_LOG2E; a.mem = plan->mem; a.key = plan_key(p, plan);
  const bool small = small_call(p, plan);
  auto launch = p->dtype == VLAC_BF16 ? (p->head_dim == 128 ? launch_attention<__nv_bfloat16, 128> : launch_attention<__nv_bfloat16, 64>)
                                      : (p->head_dim == 128 ? launch_attention<__half, 128> : launch_attention<__half, 64>);
  return launch(a, small, delay_ns, limit_ns, s);
}

}  // namespace

extern "C" {

unsigned long long vlac_prefix_bytes(const vlac_pages* p, int n, int rows, int n_heads) {
  if (!p || n < 1 || n > VLAC_PAGES_MAX_LIST || rows < 1 || n_heads < 1 || p->n_kv_heads < 1 || n_heads % p->n_kv_heads) return 0;
  if ((p->head_dim != 64 && p->head_dim != 128) || (long long)n_heads * rows >= 1ll << 29) return 0;
  return plan_mem(nullptr, n, rows, n_heads, p->head_dim).bytes;
}

int vlac_prefix_plan(const vlac_pages* p, const vlac_prefix* plan, const int* seqs, const int* q_ptr, int* status, void* stream) {
  const int rc = plan_check(p, plan);
  if (rc != VLAC_OK || plan->n == 0) return rc;
  if (!seqs || !q_ptr || !status) return VLAC_ERR_INVALID_ARG;
  PlanArgs a = {};
  a.table = p->table; a.len = p->len; a.n_slots = p->n_slots; a.max_pages = p->max_pages; a.n_pages = p->n_pages; a.page = p->page_size;
  a.shift = pages_shift(p->page_size); a.kv_heads = p->n_kv_heads; a.ratio = plan->n_heads / p->n_kv_heads; a.head_dim = p->head_dim;
  a.n = plan->n; a.rows = plan->rows; a.n_heads = plan->n_heads; a.small = small_call(p, plan); a.seqs = seqs; a.q_ptr = q_ptr; a.status = status; a.mem = plan->mem;
  a.key = plan_key(p, plan);
  if (plan->rows == 0) {                          // nothing to compute, and no plan memory
    VLAC_CUDA_CHECK(launch_pdl(prefix_status_kernel, dim3(1), dim3(PL_MAX), 0, (cudaStream_t)stream, a));
    return VLAC_OK;
  }
  const size_t smem = sizeof(PlanShared);
  if (plan->n <= 16 && (long long)plan->n * p->max_pages <= PL_ONE) {
    TRY(big_smem<prefix_plan_kernel<1>>((int)smem));
    VLAC_CUDA_CHECK(launch_pdl(prefix_plan_kernel<1>, dim3(1), dim3(256), smem, (cudaStream_t)stream, a));
  } else {
    TRY(big_smem<prefix_plan_kernel<PL_CTAS>>((int)smem));
    VLAC_CUDA_CHECK(launch_pdl(prefix_plan_kernel<PL_CTAS>, dim3(PL_CTAS), dim3(1024), smem, (cudaStream_t)stream, a));
  }
  return VLAC_OK;
}

int vlac_prefix_error(const vlac_prefix* plan, void* stream) {
  if (!plan || plan->n < 0 || plan->rows < 0) return VLAC_ERR_INVALID_ARG;
  if (plan->n == 0 || plan->rows == 0) return VLAC_OK;
  if (!plan->mem || plan->bytes < sizeof(PlanHead)) return VLAC_ERR_INVALID_ARG;
  int v = 0;
  VLAC_CUDA_CHECK(cudaMemcpyAsync(&v, (const char*)plan->mem + offsetof(PlanHead, error), sizeof(int), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  VLAC_CUDA_CHECK(cudaStreamSynchronize((cudaStream_t)stream));
  return v == VLAC_ERR_INVALID_ARG ? VLAC_ERR_INVALID_ARG : v ? VLAC_ERR_TIMEOUT : VLAC_OK;
}

int vlac_prefix_attention(const vlac_pages* p, int layer, const vlac_prefix* plan, const void* q, long long q_stride, float scale,
                          void* out, long long out_stride, float* lse, void* stream) {
  return attention(p, layer, plan, nullptr, q, q_stride, scale, out, out_stride, lse, 0, PW_WAIT_LIMIT_NS, (cudaStream_t)stream);
}

int vlac_tree_attention(const vlac_pages* p, int layer, const vlac_prefix* plan, const vlac_tree* tree, const void* q, long long q_stride, float scale,
                        void* out, long long out_stride, float* lse, void* stream) {
  if (!tree) return VLAC_ERR_INVALID_ARG;
  return attention(p, layer, plan, tree, q, q_stride, scale, out, out_stride, lse, 0, PW_WAIT_LIMIT_NS, (cudaStream_t)stream);
}

int vlac_selftest_prefix_wait(const vlac_pages* p, int layer, const vlac_prefix* plan, const void* q, long long q_stride, float scale,
                              void* out, long long out_stride, float* lse, unsigned int delay_us, unsigned int limit_us, void* stream) {
  if (delay_us > 100000 || limit_us < 1 || limit_us > 100000) return VLAC_ERR_INVALID_ARG;
  return attention(p, layer, plan, nullptr, q, q_stride, scale, out, out_stride, lse, delay_us * 1000u, limit_us * 1000ull, (cudaStream_t)stream);
}

}  // extern "C"
