// Trees of drafted tokens: which rows a row sees and where it is rotated to (vlac_tree_plan), and the path that the decoder
// confirms (vlac_tree_accept).  Integer work on a few KB; what decides it is the chain of dependent reads.
#include "pages_internal.h"
#include "launch_util.h"
#include <algorithm>
#include <atomic>

namespace {

constexpr int TP_THREADS = 128;

struct TreeArgs {
  const int *len;                               // NULL: no pool, positions are depths
  int n_slots, most, n, rows, max_rows, words;  // most: positions of a slot
  const int *seqs, *q_ptr, *parent;
  unsigned* mask;
  int *pos, *entry, *status;
};

// What an entry says.  Its rows can be read as soon as q0 and q1 are known to be sound, before the slot's length is there: one chain of reads less.
struct TreeEntry {
  int q0, q1, slot, nq;                         // nq: 0 where the rows cannot be read
  __device__ __forceinline__ TreeEntry(const TreeArgs& a, int i) {
    q0 = a.q_ptr[i]; q1 = a.q_ptr[i + 1]; slot = a.len ? a.seqs[i] : 0;
    nq = q0 >= 0 && q1 >= q0 && q1 <= a.rows && q1 - q0 <= a.max_rows ? q1 - q0 : 0;
  }
  // The code as far as it does not depend on the rows or on other entries; the slot's length, -1 where there is none.
  __device__ __forceinline__ int code(const TreeArgs& a, int* len) const {
    *len = INT_MAX;
    if (a.len) {
      *len = (unsigned)slot < (unsigned)a.n_slots ? a.len[slot] : -1;
      if ((unsigned)slot >= (unsigned)a.n_slots) return VLAC_ERR_INVALID_ARG;
      if (*len < 0 || *len > a.most) { *len = -1; return VLAC_ERR_BAD_STATE; }
    }
    if (q0 < 0 || q1 > a.rows || q1 < q0 || q1 - q0 > *len) return VLAC_ERR_INVALID_ARG;
    return q1 - q0 > a.max_rows ? VLAC_ERR_TOO_LARGE : VLAC_OK;
  }
};

__device__ __forceinline__ void tree_blank(const TreeArgs& a, int from, int to) {
  for (int r = from + threadIdx.x; r < to; r += TP_THREADS) { a.pos[r] = -1; a.entry[r] = -1; }
  for (long long w = (long long)from * a.words + threadIdx.x; w < (long long)to * a.words; w += TP_THREADS) a.mask[w] = 0;
}

// A CTA an entry, and one for the rows of none.  A row's ancestors are found by walking up; their indices fall, so that its mask is filled word
// by word from the last on.  Bound: launch and two dependent reads (trees of tens of rows, about 3 us in a captured step); in large deep trees the walk, a
// dependent read a step and thread (1024 rows, one tree or 16 of them: all children of the first 21 to 25 us, random parents 31, each behind one of the four rows
// in front of it 300, a chain 749).
__global__ void __launch_bounds__(TP_THREADS) tree_plan_kernel(TreeArgs a) {
  __shared__ int s_parent[VLAC_TREE_MAX_ROWS];
  const int tid = threadIdx.x, i = blockIdx.x;
  pdl_trigger();
  pdl_wait();
  int broken = 0;
  for (int j = tid; j < a.n; j += TP_THREADS) broken |= a.q_ptr[j + 1] < a.q_ptr[j];      // rows would overlap: all are refused
  if (i == a.n) {
    const int q_first = a.q_ptr[0], q_last = a.q_ptr[a.n];
    broken = __syncthreads_or(broken);
    const int first = broken ? a.rows : min(max(q_first, 0), a.rows), last = broken ? a.rows : min(max(q_last, 0), a.rows);
    tree_blank(a, 0, first);
    tree_blank(a, last, a.rows);
    return;
  }
  const TreeEntry e(a, i);
  const int q0 = e.q0, nq = e.nq;
  int bad = 0, len;
  for (int j = tid; j < nq; j += TP_THREADS) {
    const int p = a.parent[q0 + j];
    s_parent[j] = p;
    bad |= p < -1 || p >= j;
  }
  int code = e.code(a, &len);
  broken = __syncthreads_or(broken);
  if (__syncthreads_or(bad) && code == VLAC_OK) code = VLAC_ERR_INVALID_ARG;
  if (broken) code = VLAC_ERR_INVALID_ARG;
  if (tid == 0) a.status[i] = code;
  if (code != VLAC_OK) {
    if (!broken) tree_blank(a, min(max(q0, 0), a.rows), min(max(e.q1, 0), a.rows));
    return;
  }
  for (int j = tid; j < nq; j += TP_THREADS) {
    unsigned* to = a.mask + (size_t)(q0 + j) * a.words;
    unsigned bits = 0;
    int w = a.words - 1, depth = -1;
    for (int k = j; k >= 0; k = s_parent[k]) {
      for (; w > k >> 5; --w) { to[w] = bits; bits = 0; }
      bits |= 1u << (k & 31);
      ++depth;
    }
    for (; w >= 0; --w) { to[w] = bits; bits = 0; }
    a.pos[q0 + j] = (a.len ? len - nq : 0) + depth;
    a.entry[q0 + j] = i;
  }
}

// ------------------------------------------------------------------------------------------------ accept
struct AcceptArgs {
  TreeArgs t;
  const int *drafted, *chosen;
  int *count, *path, *tokens, *keep_ptr, *keep;
  int n_keep;
};
constexpr int TA_CTAS = 8, TA_THREADS = 1024, TA_WARPS = TA_THREADS / 32;
// One CTA / the cluster, us a call: 8 entries of 25 rows behind 300 positions 4.8 / 5.5, behind 4000 6.9 / 6.2; 32 of 61 behind 500 6.9 / 6.3; one behind 65,000
// 11.0 / 6.2; 100 of 250 behind 300 22.6 / 9.5.
constexpr int TA_ONE = 16, TA_SHORT = 8192;     // entries, positions that stay
static_assert(TA_THREADS >= VLAC_PAGES_MAX_LIST, "one thread per list entry");

// One launch.  A warp an entry: every row that its parent's choice fits bids for being the parent's successor, the lowest wins, and the path follows the
// successors.  Then the lists of all entries, behind a cluster barrier: where each begins depends on the counts in front of it.  Bound: the chain of
// dependent reads and barriers (one tree of 25 rows 4.8 us, 64 of up to 61 rows behind up to 4100 positions 8.2).
template <int CTAS>
__global__ void __cluster_dims__(CTAS, 1, 1) __launch_bounds__(TA_THREADS, 1) tree_accept_kernel(AcceptArgs a) {
  extern __shared__ int ta_next[];              // [warps][max_rows]
  __shared__ long long s_part[32];
  __shared__ int s_at[VLAC_PAGES_MAX_LIST], s_before[VLAC_PAGES_MAX_LIST], s_kept[VLAC_PAGES_MAX_LIST];
  const TreeArgs& t = a.t;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = CTAS > 1 ? (int)cluster_rank() : 0;
  pdl_trigger();
  pdl_wait();
  const int broken = __syncthreads_or(tid < t.n && t.q_ptr[min(tid, t.n - 1) + 1] < t.q_ptr[min(tid, t.n - 1)]);
  int* const next = ta_next + warp * t.max_rows;
  for (int i = warp * CTAS + rank; i < t.n; i += TA_WARPS * CTAS) {
    const TreeEntry e(t, i);
    const int q0 = e.q0, q1 = e.q1, nq = e.nq;
    for (int j = lane; j < nq; j += 32) next[j] = INT_MAX;
    __syncwarp();
    bool bad = false;
    for (int j = lane; j < nq; j += 32) {
      const int p = t.parent[q0 + j], d = a.drafted[q0 + j];
      bad |= p < -1 || p >= j;
      if (p >= 0 && p < j && d >= 0 && d == a.chosen[q0 + p]) atomicMin(&next[p], j);
    }
    int len, code = e.code(t, &len);
    if (broken) code = VLAC_ERR_INVALID_ARG;
    if (__any_sync(0xffffffffu, bad) && code == VLAC_OK) code = VLAC_ERR_INVALID_ARG;
    __syncwarp();
    int count = 0;
    if (code == VLAC_OK) {
      int cur = nq > 0 ? 0 : INT_MAX;
      for (int base = 0; base < nq; base += 32) {                       // 32 rows of the path at a time, -1 behind its end
        int mine = -1;
        for (int j = 0; j < 32 && cur < nq; ++j) {
          if (lane == j) mine = cur;
          cur = next[cur];
          ++count;
        }
        if (base + lane < nq) {
          a.path[q0 + base + lane] = mine;
          a.tokens[q0 + base + lane] = mine < 0 ? -1 : a.chosen[q0 + mine];
        }
      }
    } else if (!broken)
      for (int r = max(q0, 0) + lane; r < min(q1, t.rows); r += 32) { a.path[r] = -1; a.tokens[r] = -1; }
    if (lane == 0) {
      a.count[i] = count;
      t.status[i] = code;
      a.keep_ptr[i + 1] = code == VLAC_OK ? len - nq + count : max(len, 0);               // rows that stay; where they begin comes below
    }
    __syncwarp();                                                       // (the successors are read until here)
  }
  if (CTAS > 1) cluster_sync_all(); else __syncthreads();
  // ---- where each entry's list begins (every CTA for itself: thread i has entry i)
  int kept = 0, before = 0;
  if (tid < t.n) {
    kept = __ldcg(&a.keep_ptr[tid + 1]);
    const int c = __ldcg(&a.count[tid]);
    before = __ldcg(&t.status[tid]) == VLAC_OK ? kept - c : kept;
  }
  long long x = kept;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
  if (lane == 31) s_part[warp] = x;
  __syncthreads();
  for (int w = 0; w < warp; ++w) x += s_part[w];
  if (CTAS > 1) cluster_sync_all();                                     // every CTA has read what is overwritten now
  if (tid < t.n) {
    const bool fits = x <= a.n_keep;
    s_at[tid] = (int)min(x - kept, (long long)INT_MAX);
    s_before[tid] = before;
    s_kept[tid] = fits ? kept : 0;
    if (rank == 0) {
      a.keep_ptr[tid + 1] = (int)min(x, (long long)INT_MAX);
      if (tid == 0) a.keep_ptr[0] = 0;
      if (!fits && t.status[tid] == VLAC_OK) t.status[tid] = VLAC_ERR_TOO_LARGE;
    }
  }
  __syncthreads();
  // ---- the lists: teams of warps, an entry each
  int team = 1;
  while (team < TA_WARPS * CTAS && team * 2 * t.n <= TA_WARPS * CTAS) team *= 2;
  const int g = warp * CTAS + rank, n_teams = TA_WARPS * CTAS / team, step = team * 32;
  for (int i = g / team; i < t.n; i += n_teams) {
    const int n = s_kept[i], b = s_before[i];
    int* to = a.keep + s_at[i];
    const int q0 = n > b ? t.q_ptr[i] : 0;
    for (int j = (g % team) * 32 + lane; j < n; j += step) to[j] = j < b ? j : b + __ldcg(&a.path[q0 + j - b]);
  }
}

int tree_check(const vlac_tree* t) {
  if (!t || t->n < 0 || t->rows < 0 || t->max_rows < 1 || t->max_rows > VLAC_TREE_MAX_ROWS) return VLAC_ERR_INVALID_ARG;
  const int rc = list_check(t->n);
  if (rc != VLAC_OK) return rc;
  if (t->n > 0 && (!t->q_ptr || (t->rows > 0 && !t->parent))) return VLAC_ERR_INVALID_ARG;
  return ((uintptr_t)t->q_ptr | (uintptr_t)t->parent) & 3u ? VLAC_ERR_INVALID_ARG : VLAC_OK;
}

TreeArgs tree_args(const vlac_pages* p, const vlac_tree* t, const int* seqs, int* status) {
  TreeArgs a = {};
  if (p) { a.len = p->len; a.n_slots = p->n_slots; a.most = p->max_pages * p->page_size; }
  a.n = t->n; a.rows = t->rows; a.max_rows = t->max_rows; a.words = (t->max_rows + 31) / 32;
  a.seqs = seqs; a.q_ptr = t->q_ptr; a.parent = t->parent; a.mask = t->mask; a.pos = t->pos; a.entry = t->entry; a.status = status;
  return a;
}

}  // namespace

extern "C" {

int vlac_tree_plan(const vlac_pages* p, const vlac_tree* tree, const int* seqs, int* status, void* stream) {
  int rc = p ? pages_check(p) : VLAC_OK;
  if (rc == VLAC_OK) rc = tree_check(tree);
  if (rc != VLAC_OK) return rc;
  if ((p == nullptr) != (seqs == nullptr) && tree->n > 0) return VLAC_ERR_INVALID_ARG;
  if (tree->rows > 0 && (!tree->mask || !tree->pos || !tree->entry || ((uintptr_t)tree->mask | (uintptr_t)tree->pos | (uintptr_t)tree->entry) & 3u))
    return VLAC_ERR_INVALID_ARG;
  if (tree->n == 0) return VLAC_OK;
  if (!status || ((uintptr_t)seqs | (uintptr_t)status) & 3u) return VLAC_ERR_INVALID_ARG;
  VLAC_CUDA_CHECK(launch_pdl(tree_plan_kernel, dim3(tree->n + 1), dim3(TP_THREADS), 0, (cudaStream_t)stream, tree_args(p, tree, seqs, status)));
  return VLAC_OK;
}

int vlac_tree_accept(const vlac_pages* p, const vlac_tree* tree, const int* seqs, const int* drafted, const int* chosen, int* count, int* path, int* tokens,
                     int* keep_ptr, int* keep, int n_keep, int* status, void* stream) {
  int rc = pages_check(p);
  if (rc == VLAC_OK) rc = tree_check(tree);
  if (rc != VLAC_OK) return rc;
  if (n_keep < 0 || n_keep == INT_MAX) return VLAC_ERR_INVALID_ARG;
  if (tree->n == 0) return VLAC_OK;
  if (!seqs || !count || !keep_ptr || !status || (n_keep > 0 && !keep) || (tree->rows > 0 && (!drafted || !chosen || !path || !tokens))) return VLAC_ERR_INVALID_ARG;
  if (((uintptr_t)seqs | (uintptr_t)drafted | (uintptr_t)chosen | (uintptr_t)count | (uintptr_t)path | (uintptr_t)tokens | (uintptr_t)keep_ptr | (uintptr_t)keep |
       (uintptr_t)status) & 3u)
    return VLAC_ERR_INVALID_ARG;
  AcceptArgs a = {tree_args(p, tree, seqs, status), drafted, chosen, count, path, tokens, keep_ptr, keep, n_keep};
  const int smem = TA_WARPS * tree->max_rows * 4;                       // at most 128 KB
  if (tree->n <= TA_ONE && n_keep <= TA_SHORT) {
    if (smem > 32768) { rc = big_smem<tree_accept_kernel<1>>(TA_WARPS * VLAC_TREE_MAX_ROWS * 4); if (rc != VLAC_OK) return rc; }
    VLAC_CUDA_CHECK(launch_pdl(tree_accept_kernel<1>, dim3(1), dim3(TA_THREADS), smem, (cudaStream_t)stream, a));
  } else {
    if (smem > 32768) { rc = big_smem<tree_accept_kernel<TA_CTAS>>(TA_WARPS * VLAC_TREE_MAX_ROWS * 4); if (rc != VLAC_OK) return rc; }
    VLAC_CUDA_CHECK(launch_pdl(tree_accept_kernel<TA_CTAS>, dim3(TA_CTAS), dim3(TA_THREADS), smem, (cudaStream_t)stream, a));
  }
  return VLAC_OK;
}

}  // extern "C"
