// Paged K/V pool: taking, sharing, copying, pruning and giving back pages, and writing rows into them.
//
// Every call that changes tables is one bookkeeping launch (pages_book_kernel: one cluster of 8 CTAs, phases separated by
// cluster barriers) and, where rows move, one copy launch (pages_copy_kernel) that reads the bookkeeping's result.
// Bookkeeping is integer work on a few hundred KB; what decides it is the chain of dependent phases, which is why it is one
// launch on one cluster and not a launch per phase (512 sequences of up to 256 pages given back or taken in a pool of 131,072: 15 us a
// call, of which the scattered atomics on the reference counts, through the eight SMs of the cluster, are a part that was not timed by itself).
// Copies are bound by HBM.
#include "pages_internal.h"
#include "launch_util.h"

namespace {

enum { OP_RESIZE = 0, OP_FORK = 1, OP_COMPACT = 2 };

constexpr int PB_CTAS = 8;                      // portable cluster size
constexpr int PB_THREADS = 1024;                // thread i of every CTA finalises entry i: VLAC_PAGES_MAX_LIST of them
constexpr int PB_WARPS = PB_CTAS * PB_THREADS / 32;
static_assert(PB_THREADS >= VLAC_PAGES_MAX_LIST, "one thread per list entry");

// Layout of vlac_pages.work (ints)
struct PagesWork {
  int *first, *read_by;                         // [n_slots] first entry naming the slot as target; 1: another entry reads it
  int *bad, *lead;                              // [1024] findings of the table / keep-list scans: code, first keep[t] != t
  int *ok, *src, *dst, *shared, *start, *rows;  // [1024] per entry: valid, slots, shared leading pages, first new page, rows
  int *taken;                                   // [4] new pages of this call
  int *count;                                   // [8] free pages seen by each CTA
  int *list;                                    // [n_pages] the free pages in ascending order (as many as are needed)
  int *old;                                     // [n_slots][max_pages] page lists of slots pruned in place
};
constexpr int PW_FIXED = 8 * VLAC_PAGES_MAX_LIST + 16;

__host__ __device__ inline PagesWork pages_work(int* w, int n_slots, int n_pages) {
  PagesWork r;
  const size_t m = VLAC_PAGES_MAX_LIST;
  r.bad = w; r.lead = w + m; r.ok = w + 2 * m; r.src = w + 3 * m; r.dst = w + 4 * m; r.shared = w + 5 * m; r.start = w + 6 * m;
  r.rows = w + 7 * m; r.taken = w + 8 * m; r.count = r.taken + 4;
  w += PW_FIXED;
  r.first = w; r.read_by = w + n_slots; r.list = r.read_by + n_slots; r.old = r.list + n_pages;
  return r;
}

struct BookArgs {
  int *table, *len, *refs, *work;
  int n_slots, max_pages, n_pages, page, shift;
  int op, n, deep, n_keep;
  const int *src, *dst;                         // dst only for OP_RESIZE
  const int* lens;                              // OP_RESIZE; NULL: 0
  const int *keep_ptr, *keep;                   // OP_COMPACT
  int* status;
};

// Value of entry i of a list that may be anything: -1 unless it is a slot.
__device__ __forceinline__ int slot_of(const int* list, int i, int n_slots) {
  const int s = list[i];
  return (unsigned)s < (unsigned)n_slots ? s : -1;
}

// exclusive sum of v over the block (blockDim = 1024), total in *total; the 64-bit form for needs of bad lists, which may be large
template <typename I>
__device__ I block_scan(I v, I* total) {
  __shared__ I part[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  I x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const I t = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += t; }
  __syncthreads();                              // part may still be read by the previous scan
  if (lane == 31) part[warp] = x;
  __syncthreads();
  I y = part[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const I t = __shfl_up_sync(0xffffffffu, y, o); if (lane >= o) y += t; }
  *total = __shfl_sync(0xffffffffu, y, 31);
  const I before = __shfl_sync(0xffffffffu, y, warp ? warp - 1 : 0);
  return x - v + (warp ? before : 0);
}

__global__ void __cluster_dims__(PB_CTAS, 1, 1) __launch_bounds__(PB_THREADS, 1) pages_book_kernel(BookArgs a) {
  __shared__ int s_dst[VLAC_PAGES_MAX_LIST];    // target slot, -1: refused
  __shared__ int s_src[VLAC_PAGES_MAX_LIST];
  __shared__ int s_shared[VLAC_PAGES_MAX_LIST], s_total[VLAC_PAGES_MAX_LIST], s_start[VLAC_PAGES_MAX_LIST], s_had[VLAC_PAGES_MAX_LIST];
  __shared__ int s_d[VLAC_PAGES_MAX_LIST], s_s[VLAC_PAGES_MAX_LIST], s_ls[VLAC_PAGES_MAX_LIST], s_ld[VLAC_PAGES_MAX_LIST];  // the lists, slots' lengths
  __shared__ int s_red;
  const int tid = threadIdx.x, lane = tid & 31, rank = (int)cluster_rank();
  const int gthread = rank * PB_THREADS + tid, gwarp = (tid >> 5) * PB_CTAS + rank;
  const PagesWork w = pages_work(a.work, a.n_slots, a.n_pages);
  pdl_trigger();
  pdl_wait();

  // teams of warps, one entry at a time: up to 32 warps each when there are few entries
  int team = 1;
  while (team < 32 && team * 2 * a.n <= PB_WARPS) team *= 2;
  const int n_teams = PB_WARPS / team, my_team = gwarp / team, step = team * 32, at0 = (gwarp % team) * 32 + lane;

  // ---- 0: the lists and lengths into every CTA's shared memory; clear the marks of the slots named as targets
  if (tid < a.n) {
    const int d = slot_of(a.dst, tid, a.n_slots), s = a.op == OP_RESIZE ? d : slot_of(a.src, tid, a.n_slots);
    s_d[tid] = d; s_s[tid] = s;
    s_ls[tid] = s >= 0 ? a.len[s] : 0; s_ld[tid] = d >= 0 ? a.len[d] : 0;
  }
  __syncthreads();
  if (gthread < a.n) {
    const int d = s_d[gthread];
    if (d >= 0) { w.first[d] = INT_MAX; w.read_by[d] = 0; }
    w.bad[gthread] = 0; w.lead[gthread] = INT_MAX;
  }
  cluster_sync_all();

  // ---- 1: who names which slot; scan the tables and keep lists
  if (gthread < a.n) {
    const int d = s_d[gthread], s = s_s[gthread];
    if (d >= 0) atomicMin(&w.first[d], gthread);
    if (a.op != OP_RESIZE && s >= 0 && !(a.op == OP_COMPACT && s == d)) w.read_by[s] = 1;
  }
  for (int i = my_team; i < a.n; i += n_teams) {
    const int d = s_d[i], s = s_s[i];
    if (d < 0 || s < 0) continue;
    int bad = 0;
    const int ls = s_ls[i], ld = s_ld[i];
    if (ls < 0 || ls > a.max_pages << a.shift || ld < 0 || ld > a.max_pages << a.shift) bad = 1;
    else {
      const int ps = (ls + a.page - 1) >> a.shift, pd = (ld + a.page - 1) >> a.shift;
      const int *ts = a.table + (size_t)s * a.max_pages, *td = a.table + (size_t)d * a.max_pages;
      for (int j0 = at0; j0 < max(ps, d == s ? 0 : pd); j0 += step * 4) {
        int x[4], y[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int j = j0 + q * step;
          x[q] = j < ps ? ts[j] : 0;
          y[q] = d != s && j < pd ? td[j] : 0;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) bad |= (unsigned)x[q] >= (unsigned)a.n_pages || (unsigned)y[q] >= (unsigned)a.n_pages;
      }
      if (a.op == OP_COMPACT) {
        const int k0 = a.keep_ptr[i], k1 = a.keep_ptr[i + 1];
        if (k0 >= 0 && k1 >= k0 && k1 <= a.n_keep) {
          int lead = INT_MAX;
#pragma unroll 4
          for (int t = at0; t < k1 - k0; t += step) {
            const int x = a.keep[k0 + t], y = t ? a.keep[k0 + t - 1] : -1;
            if (x < 0 || x >= ls || x <= y) bad |= 2;
            if (x != t) lead = min(lead, t);
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) lead = min(lead, __shfl_xor_sync(0xffffffffu, lead, o));
          if (lane == 0 && lead != INT_MAX) atomicMin(&w.lead[i], lead);
        } else bad |= 2;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) bad |= __shfl_xor_sync(0xffffffffu, bad, o);
    if (lane == 0 && bad) atomicOr(&w.bad[i], bad);
  }
  cluster_sync_all();

  // ---- 2: the entries' fates as far as they do not depend on free pages (every CTA for itself: thread i has entry i)
  int status = VLAC_OK, d = -1, s = -1, total = 0, shared = 0, had = 0, rows = 0;
  if (tid < a.n) {
    d = s_d[tid];
    s = s_s[tid];
    const int bad = d >= 0 && s >= 0 ? __ldcg(&w.bad[tid]) : 0;
    if (d < 0 || s < 0 || __ldcg(&w.first[d]) != tid || (a.op != OP_RESIZE && __ldcg(&w.read_by[d])) || (a.op == OP_FORK && s == d))
      status = VLAC_ERR_INVALID_ARG;
    else if (bad & 1) status = VLAC_ERR_BAD_STATE;
    else if (bad & 2) status = VLAC_ERR_INVALID_ARG;
    else {
      const int ls = s_ls[tid];
      had = (s_ld[tid] + a.page - 1) >> a.shift;
      if (a.op == OP_RESIZE) {
        rows = a.lens ? a.lens[tid] : 0;
        if (rows < 0 || rows > a.max_pages << a.shift) status = VLAC_ERR_INVALID_ARG;
        else {
          total = (rows + a.page - 1) >> a.shift;
          shared = min(total, had);                                   // pages that stay
          if (rows < ls && (rows & (a.page - 1)) && __ldcg(&a.refs[a.table[(size_t)d * a.max_pages + total - 1]]) > 1)
            status = VLAC_ERR_BAD_STATE;
        }
      } else {
        rows = a.op == OP_FORK ? ls : a.keep_ptr[tid + 1] - a.keep_ptr[tid];
        total = (rows + a.page - 1) >> a.shift;
        shared = (a.op == OP_FORK ? (a.deep ? 0 : rows) : min(rows, __ldcg(&w.lead[tid]))) >> a.shift;
      }
    }
  }
  if (status != VLAC_OK) total = shared = rows = 0;
  const int need = total - shared;
  long long need_all;
  const long long start = block_scan((long long)need, &need_all);
  if (tid < a.n) {
    s_dst[tid] = status == VLAC_OK ? d : -1;
    s_src[tid] = s; s_shared[tid] = shared; s_total[tid] = total; s_had[tid] = had;
  }
  cluster_sync_all();                                                // every CTA has read refs and len before any changes

  // ---- 3: give back.  A target that is not pruned in place loses all its pages, a shortened sequence its tail.
  for (int i = my_team; i < a.n; i += n_teams) {
    const int t = s_dst[i];
    if (t < 0 || (a.op == OP_COMPACT && s_src[i] == t)) continue;
    int* td = a.table + (size_t)t * a.max_pages;
    const int pd = (s_ld[i] + a.page - 1) >> a.shift;
    for (int j0 = (a.op == OP_RESIZE ? s_shared[i] : 0) + at0; j0 < pd; j0 += step * 8) {
      int page[8];                                                      // (loads first: each would wait for the write before it)
#pragma unroll
      for (int q = 0; q < 8; ++q) { const int j = j0 + q * step; page[q] = j < pd ? td[j] : -1; }
#pragma unroll
      for (int q = 0; q < 8; ++q) { const int j = j0 + q * step; if (j < pd) { atomicSub(&a.refs[page[q]], 1); td[j] = -1; } }
    }
  }

  // ---- 4: free pages in ascending order.  CTA r owns a run of pages, looked at 16384 at a time: 512 to a warp, 16 to a lane, 32 side by side
  // (so that pages and list entries are written side by side too); first the counts, then the ranks.
  constexpr int LOOK = PB_THREADS * 16;
  const int per = ((a.n_pages + PB_CTAS * 32 - 1) / (PB_CTAS * 32)) * 32;
  const int p0 = min(a.n_pages, rank * per), p1 = min(a.n_pages, p0 + per), mine = (tid >> 5) * 512 + lane;
  auto free16 = [&](int p) -> unsigned {                                 // bit g: page p + 32 g is free
    int r[16];
    unsigned m = 0;
#pragma unroll
    for (int g = 0; g < 16; ++g) r[g] = p + 32 * g < p1 ? __ldcg(a.refs + p + 32 * g) : 1;
#pragma unroll
    for (int g = 0; g < 16; ++g) m |= (r[g] == 0 ? 1u : 0u) << g;
    return m;
  };
  // (a call that takes no page goes on to the tables: what it gives back counts for nobody, and its threads write the entries that they gave
  // back)
  unsigned mask = 0;                                                     // of the first look
  long long n_free = 0, before = 0;
  if (tid == 0) s_red = 0;
  __syncthreads();
  if (need_all > 0) {
    cluster_sync_all();                                                  // every page is given back
    int c = 0;
    for (int p = p0; p < p1; p += LOOK) {
      const unsigned m = free16(p + mine);
      if (p == p0) mask = m;
      c += __popc(m);
    }
    c = __reduce_add_sync(0xffffffffu, c);
    if (lane == 0) atomicAdd(&s_red, c);
    __syncthreads();
    if (tid == 0) { w.count[rank] = s_red; s_red = 0; }
    cluster_sync_all();
#pragma unroll
    for (int r = 0; r < PB_CTAS; ++r) { const int x = __ldcg(&w.count[r]); n_free += x; before += r < rank ? x : 0; }
  }
  if (need > 0 && start + need > n_free) status = VLAC_ERR_OOM;           // and every later one that needs a page: start only grows
  if (tid < a.n && status == VLAC_OK && need > 0) atomicMax(&s_red, (int)(start + need));
  __syncthreads();
  const int taken = s_red;
  if (tid < a.n) {
    s_start[tid] = (int)start;
    if (status != VLAC_OK) s_dst[tid] = -1;
    if (rank == 0) {
      w.ok[tid] = status == VLAC_OK; w.src[tid] = s; w.dst[tid] = d; w.shared[tid] = shared; w.rows[tid] = rows;
      w.start[tid] = (int)min(start, (long long)INT_MAX);
      a.status[tid] = status;
      if (status == VLAC_OK || (status == VLAC_ERR_OOM && a.op != OP_RESIZE && !(a.op == OP_COMPACT && s == d)))
        a.len[d] = status == VLAC_OK ? rows : 0;
      if (tid == 0) w.taken[0] = taken;
    }
  }
  for (int p = p0; p < p1 && before < taken; p += LOOK) {                 // uniform over the CTA
    const unsigned m = p == p0 ? mask : free16(p + mine);
    const int count = __reduce_add_sync(0xffffffffu, __popc(m));
    int all;
    long long at = before + block_scan(lane == 31 ? count : 0, &all);    // (lane 31 holds its warp's count, every lane the sum before it)
    at = __shfl_sync(0xffffffffu, at, 0);
    for (int g = 0; g < 16 && at < taken; ++g) {
      const unsigned b = __ballot_sync(0xffffffffu, m >> g & 1);
      const long long i = at + __popc(b & ((1u << lane) - 1));
      if ((m >> g & 1) && i < taken) {
        const int page = p + mine + 32 * g;
        w.list[i] = page;
        a.refs[page] = 1;
      }
      at += __popc(b);
    }
    before += all;
  }
  if (need_all > 0) cluster_sync_all();

  // ---- 5: the new tables
  for (int i = my_team; i < a.n; i += n_teams) {
    const int t = s_dst[i];
    if (t < 0) continue;
    int* td = a.table + (size_t)t * a.max_pages;
    const int sh = s_shared[i], tot = s_total[i], st = s_start[i];
    if (a.op == OP_RESIZE) {
      for (int j = sh + at0; j < tot; j += step) td[j] = __ldcg(&w.list[st + j - sh]);
      continue;
    }
    const bool in_place = s_src[i] == t;
    const int* ts = a.table + (size_t)s_src[i] * a.max_pages;
    int* to = w.old + (size_t)t * a.max_pages;
    for (int j = at0; j < (in_place ? s_had[i] : tot); j += step) {
      const int p = in_place || j < sh ? ts[j] : 0;
      if (in_place) to[j] = p;
      if (j < sh) {
        if (!in_place) { td[j] = p; atomicAdd(&a.refs[p], 1); }
      } else {
        if (in_place) atomicSub(&a.refs[p], 1);
        td[j] = j < tot ? __ldcg(&w.list[st + j - sh]) : -1;
      }
    }
  }
}

// The same for few entries with short tables, which a chain of cluster barriers and reads through L2 would only hold up: one CTA, everything
// between its phases in shared memory, entries compared pair by pair, free pages searched from the lowest on until there are enough
// (8 sequences of 35 pages given back or taken: 3.6 us a call; bound: launch and dependent reads).  The borders are of table entries, not of pages in
// use, because the host knows no lengths.  One CTA / the cluster, us a call: 8 sequences of 35 pages 3.6 / 9.4, 64 of 16 6.0 / 10.4, 64 of 64 8.3 / 10.1,
// 64 of 128 (8192 entries) 11.8 / 10.7, 64 of 256 20.1 / 10.8; 16 of 128 4.2 / 10.0, 16 of 512 10.4 / 10.8.  Short sequences in wide tables pay the
// cluster's price: 8 of 30 pages with 2048 columns 9.5 us a call.
constexpr int PO_THREADS = 512;
constexpr int PO_LIST = 64;                     // entries
constexpr int PO_ENTRIES = 8192;                // table or keep-list entries of all together
constexpr int PO_POOL = 32768;                  // pages of the pool (2048 a look)
constexpr int PO_PAGES = 2048;                  // new pages remembered in shared memory

__global__ void __launch_bounds__(PO_THREADS, 1) pages_book_one_kernel(BookArgs a) {
  __shared__ int s_dst[PO_LIST], s_src[PO_LIST], s_ls[PO_LIST], s_ld[PO_LIST], s_bad[PO_LIST], s_lead[PO_LIST], s_shared[PO_LIST], s_total[PO_LIST], s_start[PO_LIST];
  __shared__ int s_keep0[PO_LIST], s_keeps[PO_LIST];                    // the part of the keep list that is looked at: first, number (0 of a refused entry)
  __shared__ int s_new[PO_PAGES], s_warp[PO_THREADS / 32], s_need, s_taken;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const PagesWork w = pages_work(a.work, a.n_slots, a.n_pages);
  pdl_trigger();
  pdl_wait();
  // ---- the lists
  int d = -1, s = -1, k0 = 0, k1 = 0, rows = 0;
  if (tid < a.n) {
    d = slot_of(a.dst, tid, a.n_slots);
    s = a.op == OP_RESIZE ? d : slot_of(a.src, tid, a.n_slots);
    if (a.op == OP_COMPACT) { k0 = a.keep_ptr[tid]; k1 = a.keep_ptr[tid + 1]; }
    if (a.op == OP_RESIZE) rows = a.lens ? a.lens[tid] : 0;
    s_dst[tid] = d; s_src[tid] = s; s_bad[tid] = 0; s_lead[tid] = INT_MAX;
  }
  __syncthreads();
  // ---- lengths; targets named before or read by another entry
  int status = VLAC_OK, ls = 0, ld = 0;
  if (tid < a.n) {
    if (d < 0 || s < 0 || (a.op == OP_FORK && s == d)) status = VLAC_ERR_INVALID_ARG;
    if (d >= 0 && s >= 0) {
      ls = a.len[s]; ld = a.len[d];
      for (int j = 0; j < a.n; ++j) {
        if (j < tid && s_dst[j] == d) status = VLAC_ERR_INVALID_ARG;
        if (a.op != OP_RESIZE && s_src[j] == d && !(a.op == OP_COMPACT && s_dst[j] == d)) status = VLAC_ERR_INVALID_ARG;
      }
      const int most = a.max_pages << a.shift;
      if (status == VLAC_OK && (ls < 0 || ls > most || ld < 0 || ld > most)) status = VLAC_ERR_BAD_STATE;
      if (status == VLAC_OK && a.op == OP_RESIZE && (rows < 0 || rows > most)) s_bad[tid] = 2;
    }
    if (a.op == OP_COMPACT && (status != VLAC_OK || k0 < 0 || k1 < k0 || k1 > a.n_keep)) { s_bad[tid] = 2; k0 = k1 = 0; }
    s_keep0[tid] = k0; s_keeps[tid] = k1 - k0;
    s_ls[tid] = status == VLAC_OK ? ls : 0; s_ld[tid] = status == VLAC_OK ? ld : 0;          // (nothing is read for a refused entry)
  }
  __syncthreads();
  // ---- tables in range, keep lists ascending: teams of warps, an entry each
  int team = 1;
  while (team < PO_THREADS / 32 && team * 2 * a.n <= PO_THREADS / 32) team *= 2;
  const int n_teams = PO_THREADS / 32 / team, my_team = warp / team, step = team * 32, at0 = (warp % team) * 32 + lane;
  for (int i = my_team; i < a.n; i += n_teams) {
    const int e_d = s_dst[i], e_s = s_src[i], e_ls = s_ls[i];
    const int ps = (e_ls + a.page - 1) >> a.shift, pd = e_d == e_s ? 0 : (s_ld[i] + a.page - 1) >> a.shift;
    int bad = 0;
    if (ps | pd) {
      const int *ts = a.table + (size_t)e_s * a.max_pages, *td = a.table + (size_t)e_d * a.max_pages;
#pragma unroll 4
      for (int j = at0; j < max(ps, pd); j += step) {
        if (j < ps) bad |= (unsigned)ts[j] >= (unsigned)a.n_pages;
        if (j < pd) bad |= (unsigned)td[j] >= (unsigned)a.n_pages;
      }
    }
    if (a.op == OP_COMPACT) {                                           // (uniform over the team: what it goes by was written before the barrier)
      const int* k = a.keep + s_keep0[i];
      const int n = s_keeps[i];
      int lead = INT_MAX;
#pragma unroll 4
      for (int t = at0; t < n; t += step) {
        const int x = k[t], y = t ? k[t - 1] : -1;
        if (x < 0 || x >= e_ls || x <= y) bad |= 2;
        if (x != t) lead = min(lead, t);
      }
      lead = __reduce_min_sync(0xffffffffu, lead);
      if (lane == 0) atomicMin(&s_lead[i], lead);
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
    if (lane == 0 && bad) atomicOr(&s_bad[i], bad);
  }
  __syncthreads();
  // ---- what each entry needs (two warps hold the entries)
  int total = 0, shared = 0, had = 0;
  if (tid < a.n && status == VLAC_OK) {
    if (s_bad[tid] & 1) status = VLAC_ERR_BAD_STATE;
    else if (s_bad[tid] & 2) status = VLAC_ERR_INVALID_ARG;
    else {
      had = (ld + a.page - 1) >> a.shift;
      if (a.op == OP_RESIZE) {
        total = (rows + a.page - 1) >> a.shift;
        shared = min(total, had);
        if (rows < ls && (rows & (a.page - 1)) && __ldcg(&a.refs[a.table[(size_t)d * a.max_pages + total - 1]]) > 1) status = VLAC_ERR_BAD_STATE;
      } else {
        rows = a.op == OP_FORK ? ls : k1 - k0;
        total = (rows + a.page - 1) >> a.shift;
        shared = (a.op == OP_FORK ? (a.deep ? 0 : rows) : min(rows, s_lead[tid])) >> a.shift;
      }
    }
  }
  if (status != VLAC_OK) total = shared = rows = 0;
  const int need = total - shared;
  int start = need;                                                     // (at most 64 x 8192)
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, start, o); if (lane >= o) start += t; }
  if (tid < PO_LIST && lane == 31) s_warp[warp] = start;
  __syncthreads();                                                      // (also: every reference count has been read before any changes)
  if (tid < PO_LIST && warp == 1) start += s_warp[0];
  start -= need;
  if (tid == PO_LIST - 1) s_need = start + need;
  if (tid < a.n) {
    if (status != VLAC_OK) s_dst[tid] = -1;
    s_shared[tid] = shared; s_total[tid] = total; s_start[tid] = start;
  }
  if (tid == 0) s_taken = 0;
  __syncthreads();
  // ---- give back
  for (int i = my_team; i < a.n; i += n_teams) {
    const int t = s_dst[i];
    if (t < 0 || (a.op == OP_COMPACT && s_src[i] == t)) continue;
    int* td = a.table + (size_t)t * a.max_pages;
    const int pd = (s_ld[i] + a.page - 1) >> a.shift;
#pragma unroll 4
    for (int j = (a.op == OP_RESIZE ? s_shared[i] : 0) + at0; j < pd; j += step) {
      atomicSub(&a.refs[td[j]], 1);
      td[j] = -1;
    }
  }
  __syncthreads();
  // ---- the lowest free pages, in order
  const int want = s_need;
  int found = 0;
  for (int p = 0; p < a.n_pages && found < want; p += PO_THREADS * 4) {
    const int q = p + tid * 4;
    int m = 0;
    if (q + 3 < a.n_pages) {
      const int4 r = __ldcg(reinterpret_cast<const int4*>(a.refs + q));
      m = (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
    } else
      for (int b = 0; b < 4; ++b) if (q + b < a.n_pages && __ldcg(a.refs + q + b) == 0) m |= 1 << b;
    const int c = __popc(m);
    int x = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += t; }
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    int at = found + x - c;
    for (int v = 0; v < PO_THREADS / 32; ++v) { const int y = s_warp[v]; found += y; if (v < warp) at += y; }
#pragma unroll
    for (int b = 0; b < 4; ++b)
      if (m >> b & 1) { if (at < want) { w.list[at] = q + b; if (at < PO_PAGES) s_new[at] = q + b; } ++at; }
    __syncthreads();
  }
  // ---- fates: when there are too few, an entry that needs more than is left and every later one that needs any
  if (need > 0 && start + need > found) status = VLAC_ERR_OOM;
  if (tid < a.n && status == VLAC_OK && need > 0) atomicMax(&s_taken, start + need);
  if (tid < a.n) {
    w.ok[tid] = status == VLAC_OK; w.src[tid] = s; w.dst[tid] = d; w.shared[tid] = shared; w.rows[tid] = rows; w.start[tid] = start;
    a.status[tid] = status;
    if (status == VLAC_OK || (status == VLAC_ERR_OOM && a.op != OP_RESIZE && !(a.op == OP_COMPACT && s == d)))
      a.len[d] = status == VLAC_OK ? rows : 0;
    if (status != VLAC_OK) s_dst[tid] = -1;
  }
  __syncthreads();
  const int taken = s_taken;
  if (tid == 0) w.taken[0] = taken;
  auto page_of = [&](int i) { return i < PO_PAGES ? s_new[i] : __ldcg(&w.list[i]); };
  for (int i = tid; i < taken; i += PO_THREADS) a.refs[page_of(i)] = 1;
  // ---- the new tables
  for (int i = my_team; i < a.n; i += n_teams) {
    const int t = s_dst[i];
    if (t < 0) continue;
    int* td = a.table + (size_t)t * a.max_pages;
    const int sh = s_shared[i], tot = s_total[i], st = s_start[i];
    if (a.op == OP_RESIZE) {
      for (int j = sh + at0; j < tot; j += step) td[j] = page_of(st + j - sh);
      continue;
    }
    const bool in_place = s_src[i] == t;
    const int* ts = a.table + (size_t)s_src[i] * a.max_pages;
    int* to = w.old + (size_t)t * a.max_pages;
    for (int j = at0; j < (in_place ? (s_ld[i] + a.page - 1) >> a.shift : tot); j += step) {
      const int p = in_place || j < sh ? ts[j] : 0;
      if (in_place) to[j] = p;
      if (j < sh) {
        if (!in_place) { td[j] = p; atomicAdd(&a.refs[p], 1); }
      } else {
        if (in_place) atomicSub(&a.refs[p], 1);
        td[j] = j < tot ? page_of(st + j - sh) : -1;
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Rows of the new pages of a fork / compaction: unit = (new page, layer, part of the page's rows, at most 32 KB of K and of V); a CTA of 256
// threads moves it with 16-byte accesses, four of K and four of V in flight per thread.  HBM-bound: read once, written once (8 sequences of 297 rows
// in 32 layers, 2.2 GB with the writes: 361 us with the bookkeeping, 6.2 TB/s; pruned in place it is as long as into another slot).
constexpr int PC_THREADS = 256;
struct Rows16 {                                 // rows of 16-byte pieces
  int n;                                        // pieces of a row
  int shift;                                    // log2(n), or -1
  __device__ __forceinline__ int row(int c) const { return shift >= 0 ? c >> shift : c / n; }
  __device__ __forceinline__ int col(int c, int r) const { return c - r * n; }
};
struct CopyArgs {
  uint4 *k, *v;
  const int *table;
  int* work;
  int n_slots, max_pages, n_pages, page, shift, n_layers, n;
  Rows16 row16;
  int part_rows, parts;                         // rows of a part, parts of a page
  const int *keep_ptr, *keep;                   // NULL: row at position x is row x of the source
};

__global__ void __launch_bounds__(PC_THREADS) pages_copy_kernel(CopyArgs a) {
  __shared__ int s_start[VLAC_PAGES_MAX_LIST];  // first new page of each entry (not decreasing)
  __shared__ long long s_from[256];             // source row of each row of the part
  __shared__ int s_rows;
  __shared__ long long s_to;
  const int tid = threadIdx.x;
  const PagesWork w = pages_work(a.work, a.n_slots, a.n_pages);
  pdl_wait();
  const int taken = w.taken[0];
  const long long per_layer = (long long)taken * a.parts, units = per_layer * a.n_layers;
  if ((long long)blockIdx.x >= units) return;
  for (int i = tid; i < a.n; i += PC_THREADS) s_start[i] = w.start[i];
  const size_t layer16 = ((size_t)a.n_pages << a.shift) * a.row16.n;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int layer = (int)(u / per_layer), in = (int)(u - layer * per_layer), np = in / a.parts, r0 = (in - np * a.parts) * a.part_rows;
    __syncthreads();
    // the entry that owns new page np: the last with start <= np (entries that take none share their successor's start)
    int lo = 0, hi = a.n - 1;
    while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (s_start[m] <= np) lo = m; else hi = m - 1; }
    const int e = lo, shared = w.shared[e], src = w.src[e], dst = w.dst[e];
    const int j = shared + np - s_start[e], first = (j << a.shift) + r0;
    const int rows = w.ok[e] ? min(a.part_rows, w.rows[e] - first) : 0;
    if (tid < rows) {
      const int x = first + tid, y = a.keep_ptr ? a.keep[a.keep_ptr[e] + x] : x;
      const int* from = (src == dst ? w.old : a.table) + (size_t)src * a.max_pages;
      s_from[tid] = ((long long)from[y >> a.shift] << a.shift) + (y & (a.page - 1));
    }
    if (tid == 0) { s_rows = rows; s_to = ((long long)w.list[np] << a.shift) + r0; }
    __syncthreads();
    const int n16 = max(0, s_rows) * a.row16.n;
    const size_t base = (size_t)layer * layer16;
    const uint4 *kl = a.k + base, *vl = a.v + base;
    uint4 *ko = a.k + base + (size_t)s_to * a.row16.n, *vo = a.v + base + (size_t)s_to * a.row16.n;
    for (int c0 = tid; c0 < n16; c0 += PC_THREADS * 4) {
      uint4 x[4], y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = c0 + q * PC_THREADS;
        if (c < n16) {
          const int r = a.row16.row(c);
          const size_t at = (size_t)s_from[r] * a.row16.n + a.row16.col(c, r);
          x[q] = kl[at]; y[q] = vl[at];
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = c0 + q * PC_THREADS;
        if (c < n16) { ko[c] = x[q]; vo[c] = y[q]; }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Rows into pages.  grid (x, entries, layers): the CTAs of an entry share its rows out in groups; each checks the whole entry for
// itself (its pages must exist and be the slot's own), so that an entry is written whole or not at all without a second launch.
// HBM-bound (8 prompts of up to 4096 rows, 0.9 GB with the writes: 152 us, 5.9 TB/s; a step's prompt of 290 rows in 32 layers, 0.3 GB: 52 us, 5.8 TB/s);
// one row each for 64 sequences: 3.6 us.
constexpr int PR_THREADS = 256;
constexpr int PR_ROWS = 8;                      // rows of K and of V per group
struct WriteArgs {
  uint4 *k, *v;
  const int *table, *len, *refs;
  int n_slots, max_pages, n_pages, page, shift, layer, n, rows;
  Rows16 row16;
  const int *seqs, *start, *row_ptr;            // NULL seqs: one entry, `slot`, rows 0 .. rows-1 at position 0
  int slot;
  const unsigned char* hidden;                  // with `slot`: 1 = the source holds no row at this position, or NULL
  const uint4 *kin, *vin;
  long long kstride16, vstride16, layer_stride16;
  int* status;
};

__global__ void __launch_bounds__(PR_THREADS) pages_write_kernel(WriteArgs a) {
  const int tid = threadIdx.x, i = blockIdx.y;
  pdl_trigger();
  pdl_wait();
  const int slot = a.seqs ? a.seqs[i] : a.slot;
  const int r0 = a.row_ptr ? a.row_ptr[i] : 0, r1 = a.row_ptr ? a.row_ptr[i + 1] : a.rows;
  int code = 0, pos = 0;
  if ((unsigned)slot >= (unsigned)a.n_slots || r0 < 0 || r1 < r0 || r1 > a.rows) code = VLAC_ERR_INVALID_ARG;
  else {
    const int len = a.len[slot];
    if (len < 0 || len > a.max_pages << a.shift) code = VLAC_ERR_BAD_STATE;
    else {
      pos = a.seqs ? (a.start ? a.start[i] : len - (r1 - r0)) : 0;
      if (pos < 0 || (long long)pos + (r1 - r0) > len) code = VLAC_ERR_INVALID_ARG;
    }
  }
  // (uniform so far) an earlier entry with the same slot stands; pages of the range must exist and belong to this slot alone
  int dup = 0, bad = 0;
  if (a.seqs) for (int j = tid; j < i; j += PR_THREADS) dup |= a.seqs[j] == slot;
  const int* t = a.table + (size_t)(code == 0 ? slot : 0) * a.max_pages;
  if (code == 0 && r1 > r0)
    for (int j = (pos >> a.shift) + tid; j <= (pos + r1 - r0 - 1) >> a.shift; j += PR_THREADS) {
      const int p = t[j];
      bad |= (unsigned)p >= (unsigned)a.n_pages || a.refs[p] != 1;
    }
  if (code == 0 && a.hidden) for (int j = tid; j < r1; j += PR_THREADS) bad |= a.hidden[j] != 0;
  if (__syncthreads_or(dup)) code = VLAC_ERR_INVALID_ARG;
  if (__syncthreads_or(bad) && code == 0) code = VLAC_ERR_BAD_STATE;
  if (tid == 0 && blockIdx.x == 0 && blockIdx.z == 0) a.status[i] = code;
  if (code != 0) return;
  const size_t base = (size_t)(a.layer + blockIdx.z) * ((size_t)a.n_pages << a.shift) * a.row16.n;
  const uint4 *kin = a.kin + blockIdx.z * a.layer_stride16, *vin = a.vin + blockIdx.z * a.layer_stride16;
  for (int g = r0 + blockIdx.x * PR_ROWS; g < r1; g += gridDim.x * PR_ROWS) {
    const int n16 = min(PR_ROWS, r1 - g) * a.row16.n;
    for (int c0 = tid; c0 < n16; c0 += PR_THREADS * 4) {
      uint4 x[4], y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = c0 + q * PR_THREADS;
        if (c < n16) {
          const int r = a.row16.row(c), o = a.row16.col(c, r);
          x[q] = kin[(size_t)(g + r) * a.kstride16 + o]; y[q] = vin[(size_t)(g + r) * a.vstride16 + o];
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = c0 + q * PR_THREADS;
        if (c < n16) {
          const int r = a.row16.row(c), at = pos + (g - r0) + r;
          const size_t to = base + (((size_t)t[at >> a.shift] << a.shift) + (at & (a.page - 1))) * a.row16.n + a.row16.col(c, r);
          a.k[to] = x[q]; a.v[to] = y[q];
        }
      }
    }
  }
}

Rows16 rows16(const vlac_pages* p) {
  const int n = (int)(pages_row(p) / 8);
  return {n, n & (n - 1) ? -1 : pages_shift(n)};
}

int book(const vlac_pages* p, int op, const int* src, const int* dst, const int* lens, int n, int deep, const int* keep_ptr,
         const int* keep, int n_keep, int* status, cudaStream_t s) {
  BookArgs b = {};
  b.table = p->table; b.len = p->len; b.refs = p->refs; b.work = (int*)p->work;
  b.n_slots = p->n_slots; b.max_pages = p->max_pages; b.n_pages = p->n_pages; b.page = p->page_size; b.shift = pages_shift(p->page_size);
  b.op = op; b.n = n; b.deep = deep; b.n_keep = n_keep; b.src = src; b.dst = dst; b.lens = lens; b.keep_ptr = keep_ptr; b.keep = keep;
  b.status = status;
  if (n <= PO_LIST && (long long)n * p->max_pages <= PO_ENTRIES && n_keep <= PO_ENTRIES && p->n_pages <= PO_POOL)
    VLAC_CUDA_CHECK(launch_pdl(pages_book_one_kernel, dim3(1), dim3(PO_THREADS), 0, s, b));
  else
    VLAC_CUDA_CHECK(launch_pdl(pages_book_kernel, dim3(PB_CTAS), dim3(PB_THREADS), 0, s, b));
  if (op == OP_RESIZE) return VLAC_OK;
  int n_sm = 0;
  const int rc = sm_count(&n_sm);
  if (rc != VLAC_OK) return rc;
  CopyArgs c = {};
  c.k = (uint4*)p->k; c.v = (uint4*)p->v; c.table = p->table; c.work = (int*)p->work;
  c.n_slots = p->n_slots; c.max_pages = p->max_pages; c.n_pages = p->n_pages; c.page = p->page_size; c.shift = b.shift;
  c.n_layers = p->n_layers; c.n = n; c.row16 = rows16(p);
  c.part_rows = p->page_size;
  while (c.part_rows > 1 && (long long)c.part_rows * c.row16.n > 2048) c.part_rows /= 2;
  c.parts = p->page_size / c.part_rows;
  c.keep_ptr = keep_ptr; c.keep = keep;
  VLAC_CUDA_CHECK(launch_pdl(pages_copy_kernel, dim3(n_sm * 8), dim3(PC_THREADS), 0, s, c));
  return VLAC_OK;
}

int write_rows(const vlac_pages* p, WriteArgs a, int n, int layers, cudaStream_t s) {
  int n_sm = 0;
  const int rc = sm_count(&n_sm);
  if (rc != VLAC_OK) return rc;
  a.k = (uint4*)p->k; a.v = (uint4*)p->v; a.table = p->table; a.len = p->len; a.refs = p->refs;
  a.n_slots = p->n_slots; a.max_pages = p->max_pages; a.n_pages = p->n_pages; a.page = p->page_size; a.shift = pages_shift(p->page_size);
  a.row16 = rows16(p); a.n = n;
  // enough CTAs for the whole GPU; no more per entry than one entry could use
  const int groups = (a.rows + PR_ROWS - 1) / PR_ROWS, spread = (n_sm * 8 + n * layers - 1) / (n * layers);
  const int x = groups < 1 ? 1 : groups < spread ? groups : spread;
  VLAC_CUDA_CHECK(launch_pdl(pages_write_kernel, dim3(x, n, layers), dim3(PR_THREADS), 0, s, a));
  return VLAC_OK;
}

}  // namespace

extern "C" {

unsigned long long vlac_pages_work_bytes(const vlac_pages* p) {
  if (!p || p->n_pages < 1 || p->n_slots < 1 || p->max_pages < 1) return 0;
  return 4ull * ((unsigned long long)PW_FIXED + 2ull * p->n_slots + p->n_pages + (unsigned long long)p->n_slots * p->max_pages);
}

int vlac_pages_resize(const vlac_pages* p, const int* seqs, const int* lens, int n, int* status, void* stream) {
  int rc = pages_check(p);
  if (rc == VLAC_OK) rc = list_check(n);
  if (rc != VLAC_OK || n == 0) return rc;
  if (!seqs || !lens || !status) return VLAC_ERR_INVALID_ARG;
  return book(p, OP_RESIZE, nullptr, seqs, lens, n, 0, nullptr, nullptr, 0, status, (cudaStream_t)stream);
}

int vlac_pages_free(const vlac_pages* p, const int* seqs, int n, int* status, void* stream) {
  int rc = pages_check(p);
  if (rc == VLAC_OK) rc = list_check(n);
  if (rc != VLAC_OK || n == 0) return rc;
  if (!seqs || !status) return VLAC_ERR_INVALID_ARG;
  return book(p, OP_RESIZE, nullptr, seqs, nullptr, n, 0, nullptr, nullptr, 0, status, (cudaStream_t)stream);
}

int vlac_pages_fork(const vlac_pages* p, const int* src, const int* dst, int n, int deep, int* status, void* stream) {
  int rc = pages_check(p);
  if (rc == VLAC_OK) rc = list_check(n);
  if (rc != VLAC_OK || n == 0) return rc;
  if (!src || !dst || !status || (deep != 0 && deep != 1)) return VLAC_ERR_INVALID_ARG;
  return book(p, OP_FORK, src, dst, nullptr, n, deep, nullptr, nullptr, 0, status, (cudaStream_t)stream);
}

int vlac_pages_compact(const vlac_pages* p, const int* src, const int* dst, int n, const int* keep_ptr, const int* keep, int n_keep,
                       int* status, void* stream) {
  int rc = pages_check(p);
  if (rc == VLAC_OK) rc = list_check(n);
  if (rc != VLAC_OK || n == 0) return rc;
  if (!src || !dst || !keep_ptr || !status || n_keep < 0 || (n_keep > 0 && !keep)) return VLAC_ERR_INVALID_ARG;
  return book(p, OP_COMPACT, src, dst, nullptr, n, 0, keep_ptr, keep, n_keep, status, (cudaStream_t)stream);
}

int vlac_pages_write(const vlac_pages* p, int layer, const int* seqs, const int* start, const int* row_ptr, int n, int rows,
                     const void* k_rows, long long k_stride, const void* v_rows, long long v_stride, int* status, void* stream) {
  int rc = pages_check(p);
  if (rc == VLAC_OK) rc = list_check(n);
  if (rc != VLAC_OK) return rc;
  if (layer < 0 || layer >= p->n_layers || rows < 0) return VLAC_ERR_INVALID_ARG;
  if (n == 0) return VLAC_OK;
  if (!seqs || !row_ptr || !status || (rows > 0 && (!k_rows || !v_rows))) return VLAC_ERR_INVALID_ARG;
  const long long w = (long long)pages_row(p);
  if (k_stride < w || v_stride < w || k_stride % 8 || v_stride % 8 || (((uintptr_t)k_rows | (uintptr_t)v_rows) & 15u)) return VLAC_ERR_INVALID_ARG;
  WriteArgs a = {};
  a.layer = layer; a.rows = rows; a.seqs = seqs; a.start = start; a.row_ptr = row_ptr;
  a.kin = (const uint4*)k_rows; a.vin = (const uint4*)v_rows; a.kstride16 = k_stride / 8; a.vstride16 = v_stride / 8; a.status = status;
  return write_rows(p, a, n, 1, (cudaStream_t)stream);
}

int vlac_pages_from_cache(const vlac_pages* p, vlac_cache* cache, int seq, int slot, int n_rows, int* status, void* stream) {
  const int rc = pages_check(p);
  if (rc != VLAC_OK) return rc;
  if (!cache || !status || seq < 0 || seq >= cache->batch || slot < 0 || slot >= p->n_slots) return VLAC_ERR_INVALID_ARG;
  const vlac_ctx* ctx = cache->ctx;
  const vlac_config& g = ctx->cfg;
  if (p->dtype != VLAC_BF16 || p->n_layers != g.n_layers || p->n_kv_heads != g.n_kv_heads || p->head_dim != g.head_dim ||
      n_rows < 0 || n_rows > ctx->max_seq || g.n_layers > 65535)
    return VLAC_ERR_INVALID_ARG;
  const size_t kv = kv_layer_elems(ctx), off = (size_t)seq * kv;
  WriteArgs a = {};
  a.layer = 0; a.rows = n_rows; a.slot = slot; a.hidden = cache->hidden_keys + (size_t)seq * ctx->max_seq;
  a.kin = (const uint4*)(cache->k + off); a.vin = (const uint4*)(cache->v + off);
  a.kstride16 = a.vstride16 = (long long)(pages_row(p) / 8); a.layer_stride16 = (long long)(cache->batch * kv / 8);
  a.status = status;
  return write_rows(p, a, 1, g.n_layers, (cudaStream_t)stream);
}

}  // extern "C"
