// Attention of new rows over paged sequences that share a prefix (vlac_prefix_plan, vlac_prefix_attention).
//
// Softmax attention over a union of disjoint key sets is a weighted sum of the attentions over the sets:
//     o = sum_i 2^(m_i - M) l_i o_i / sum_i 2^(m_i - M) l_i      (m_i, l_i: maximum and sum of 2^(s - m_i) of set i)
// so the pages that several sequences have in common are one problem with the query rows of all of them (and of all query
// heads of a K/V head) stacked, and each sequence's own rows are another with its rows alone.  These problems are "segments";
// a segment is cut into (K/V head, tile of stacked rows, block of 64 keys) units, and the units of the whole call are dealt to a
// fixed number of CTAs in equal contiguous runs, whatever the lengths: a run may begin and end inside a tile, every piece of a
// tile leaves (unnormalised o, m, l) in a slot of its own, and a second kernel adds a row's pieces in a fixed order.
#include "pages_internal.h"
#include "launch_util.h"
#include <cuda_fp16.h>
#include <math.h>

namespace {

constexpr int PF_GRID_A = 2 * 148;              // CTAs of the warp-MMA kernel: two per SM
constexpr int PF_KB = 64;                       // keys per unit
constexpr int PF_BM = 64;                       // stacked rows of a tile (16 in segments that have no more)
constexpr int PF_STAGES = 3;
constexpr int PF_THREADS = 128;

struct SeqRec { int slot, row0, nq, len, pre_seg, suf_seg, pad0, pad1; };          // segments: -1 none
struct SegRec {
  long long ustart, uend;                       // units of this segment in the call's order
  int slot;                                     // whose table holds the keys
  int row0, R;                                  // first q row; stacked rows per K/V head: (q rows) * (query heads per K/V head)
  int key0, key1;                               // positions [key0, key1)
  int pos0;                                     // position of q row row0; INT_MIN in a prefix: every row sees every key
  int bm, T, KB;                                // rows per tile, tiles, key blocks
  int rowbase;                                  // first slot row of this segment
};
struct PlanHead { long long units; int n_seg; int n_act; };

struct PlanMem {
  PlanHead* head;
  int *lcp, *bad;                               // [n] common pages with the previous active sequence; findings
  SeqRec* seq;                                  // [n] active sequences
  SegRec* seg;                                  // [2n]
  int* first;                                   // [PF_GRID_A] segment of each CTA's first unit
  int* row_k;                                   // [rows] active sequence of each row, -1: none
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
  p.lcp = (int*)take(sizeof(int) * n);
  p.bad = (int*)take(sizeof(int) * n);
  p.seq = (SeqRec*)take(sizeof(SeqRec) * n);
  p.seg = (SegRec*)take(sizeof(SegRec) * 2 * (size_t)n);
  p.first = (int*)take(sizeof(int) * PF_GRID_A);
  p.row_k = (int*)take(sizeof(int) * (size_t)(rows > 0 ? rows : 1));
  const size_t slots = 2 * (size_t)rows * n_heads + (size_t)PF_GRID_A * PF_BM;
  p.ml = (float2*)take(sizeof(float2) * slots);
  p.po = (float*)take(sizeof(float) * slots * head_dim);
  p.bytes = o;
  return p;
}

// U units are dealt to G = min(U, PF_GRID_A) CTAs, so that no run is empty: run c is [c*U/G, (c+1)*U/G).  The CTA whose run holds u:
__device__ __forceinline__ long long runs(long long U) { return U < PF_GRID_A ? U : PF_GRID_A; }
__device__ __forceinline__ int run_of(long long u, long long U) { return (int)(((u + 1) * runs(U) - 1) / U); }

// ------------------------------------------------------------------------------------------------ plan
struct PlanArgs {
  const int *table, *len;
  int n_slots, max_pages, n_pages, page, shift, kv_heads, ratio, head_dim;
  int n, rows, n_heads;
  const int *seqs, *q_ptr;
  int* status;
  void* mem;
};
constexpr int PL_CTAS = 8;
constexpr int PL_THREADS = 1024;
constexpr int PL_WARPS = PL_CTAS * PL_THREADS / 32;

// exclusive sum over the block of 1024 threads
__device__ long long plan_scan(long long v, long long* total) {
  __shared__ long long part[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += t; }
  __syncthreads();
  if (lane == 31) part[warp] = x;
  __syncthreads();
  if (warp == 0) {
    long long y = part[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, y, o); if (lane >= o) y += t; }
    part[lane] = y;
  }
  __syncthreads();
  *total = part[31];
  return x - v + (warp ? part[warp - 1] : 0);
}

__global__ void __cluster_dims__(PL_CTAS, 1, 1) __launch_bounds__(PL_THREADS, 1) prefix_plan_kernel(PlanArgs a) {
  __shared__ int s_i[1024], s_slot[1024], s_row0[1024], s_nq[1024], s_len[1024], s_lcp[1024], s_lead[1024], s_c[1024], s_m[1024], s_end[1024];
  const int tid = threadIdx.x, lane = tid & 31, rank = (int)cluster_rank();
  const int gwarp = (tid >> 5) * PL_CTAS + rank;
  const PlanMem p = plan_mem(a.mem, a.n, a.rows, a.n_heads, a.head_dim);
  pdl_trigger();
  pdl_wait();
  // ---- the active sequences (rows to compute), in list order: every CTA for itself
  int status = VLAC_OK, slot = 0, q0 = 0, q1 = 0, len = 0;
  if (tid < a.n) { q0 = a.q_ptr[tid]; q1 = a.q_ptr[tid + 1]; }
  const int broken = __syncthreads_or(tid < a.n && q1 < q0);            // rows would overlap: nothing is computed
  if (tid < a.n) {
    slot = a.seqs[tid];
    if (broken || q0 < 0 || q1 > a.rows || (unsigned)slot >= (unsigned)a.n_slots) status = VLAC_ERR_INVALID_ARG;
    else {
      len = a.len[slot];
      if (len < 0 || len > a.max_pages << a.shift) status = VLAC_ERR_BAD_STATE;
    }
  }
  const bool act = tid < a.n && status == VLAC_OK && q1 > q0;
  long long tot;
  const int k_of = (int)plan_scan(act ? 1 : 0, &tot);
  const int n_act = (int)tot;
  if (act) { s_i[k_of] = tid; s_slot[k_of] = slot; s_row0[k_of] = q0; s_nq[k_of] = q1 - q0; s_len[k_of] = len; }
  if (rank == 0 && tid < a.n) { p.lcp[tid] = INT_MAX; p.bad[tid] = 0; a.status[tid] = status; }
  cluster_sync_all();

  // ---- tables: page numbers in range; leading pages in common with the previous active sequence
  int team = 1;
  while (team < 32 && team * 2 * n_act <= PL_WARPS) team *= 2;
  const int n_teams = PL_WARPS / team;
  for (int k = gwarp / team; k < n_act; k += n_teams) {
    const int *t = a.table + (size_t)s_slot[k] * a.max_pages, *tp = k ? a.table + (size_t)s_slot[k - 1] * a.max_pages : t;
    const int np = (s_len[k] + a.page - 1) >> a.shift;
    // only whole pages in front of every member's queries are shared: all rows of the group see all of them
    const int m = k ? min(max(0, s_len[k] - s_nq[k]), max(0, s_len[k - 1] - s_nq[k - 1])) >> a.shift : 0;
    int bad = 0, lcp = m;
#pragma unroll 4
    for (int j = (gwarp % team) * 32 + lane; j < np; j += team * 32) {
      const int x = t[j];
      bad |= (unsigned)x >= (unsigned)a.n_pages;
      if (j < m && x != tp[j]) lcp = min(lcp, j);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { bad |= __shfl_xor_sync(0xffffffffu, bad, o); lcp = min(lcp, __shfl_xor_sync(0xffffffffu, lcp, o)); }
    if (lane == 0) { atomicMin(&p.lcp[k], lcp); if (bad) atomicOr(&p.bad[k], 1); }
  }
  cluster_sync_all();
  const bool mine = tid < n_act, bad = mine && __ldcg(&p.bad[tid]);
  // which sequence each row belongs to
  for (int r = rank * PL_THREADS + tid; r < a.rows; r += PL_CTAS * PL_THREADS) {
    int lo = 0, hi = n_act - 1;
    while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (s_row0[m] <= r) lo = m; else hi = m - 1; }
    const bool in = n_act > 0 && r >= s_row0[lo] && r < s_row0[lo] + s_nq[lo] && !__ldcg(&p.bad[lo]);
    p.row_k[r] = in ? lo : -1;
  }
  if (rank != 0) return;

  // ---- neighbours into groups
  if (mine) s_lcp[tid] = bad ? -1 : __ldcg(&p.lcp[tid]);
  if (bad) a.status[s_i[tid]] = VLAC_ERR_BAD_STATE;
  __syncthreads();
  if (tid == 0) {
    int lead = 0, c = 0, m = 0;
    for (int k = 0; k < n_act; ++k) {
      // joining spares the newcomer the reading of c2 common pages and costs the others the reading of c - c2 pages each
      const int c2 = min(c, s_lcp[k]);
      const bool join = m > 0 && s_lcp[k] >= 0 && s_lcp[lead] >= 0 && s_row0[k] == s_end[lead] && (long long)c2 > (long long)(c - c2) * (m - 1);
      if (join) { c = c2; ++m; }
      else { lead = k; m = 1; c = max(0, s_len[k] - s_nq[k]) >> a.shift; }
      s_lead[k] = lead; s_c[lead] = c; s_m[lead] = m; s_end[lead] = s_row0[k] + s_nq[k];
    }
  }
  __syncthreads();
  // ---- segments: thread k makes the prefix of a group that k leads, and k's own rows
  long long u_pre = 0, u_suf = 0;
  int r_pre = 0, r_suf = 0, pre = 0, lead = 0, t_pre = 0, t_suf = 0, kb_pre = 0, kb_suf = 0;
  if (mine && !bad) {
    lead = s_lead[tid];
    if (s_m[lead] >= 2) pre = s_c[lead] << a.shift;
    if (lead == tid && pre > 0) {
      r_pre = (s_end[tid] - s_row0[tid]) * a.ratio;
      const int bm = r_pre <= 16 ? 16 : PF_BM;
      t_pre = (r_pre + bm - 1) / bm; kb_pre = (pre + PF_KB - 1) / PF_KB;
      u_pre = (long long)a.kv_heads * t_pre * kb_pre;
    }
    if (s_len[tid] > pre) {
      r_suf = s_nq[tid] * a.ratio;
      const int bm = r_suf <= 16 ? 16 : PF_BM;
      t_suf = (r_suf + bm - 1) / bm; kb_suf = (s_len[tid] - pre + PF_KB - 1) / PF_KB;
      u_suf = (long long)a.kv_heads * t_suf * kb_suf;
    }
  }
  long long units, slots, segs;
  const long long u0 = plan_scan(u_pre + u_suf, &units);
  const long long b0 = plan_scan((long long)(r_pre + r_suf) * a.kv_heads, &slots);
  const int g0 = (int)plan_scan((u_pre > 0) + (u_suf > 0), &segs);
  s_c[tid] = g0;                                                        // (s_c was read above, before the scans' barriers)
  __syncthreads();
  if (mine) {
    SeqRec q = {s_slot[tid], s_row0[tid], s_nq[tid], s_len[tid], pre > 0 ? s_c[lead] : -1, u_suf > 0 ? g0 + (u_pre > 0) : -1, 0, 0};
    p.seq[tid] = q;
    const long long G = runs(units);
    auto put = [&](int g, long long us, long long n, int R, int k0, int k1, int pos0, int T, int KB, long long base) {
      SegRec s = {us, us + n, s_slot[tid], s_row0[tid], R, k0, k1, pos0, R <= 16 ? 16 : PF_BM, T, KB, (int)base};
      p.seg[g] = s;
      for (long long c = (us * G + units - 1) / units, e = ((us + n) * G + units - 1) / units; c < e; ++c) p.first[c] = g;
    };
    if (u_pre > 0) put(g0, u0, u_pre, r_pre, 0, pre, INT_MIN, t_pre, kb_pre, b0);
    if (u_suf > 0) put(g0 + (u_pre > 0), u0 + u_pre, u_suf, r_suf, pre, s_len[tid], s_len[tid] - s_nq[tid], t_suf, kb_suf, b0 + (long long)r_pre * a.kv_heads);
  }
  if (tid == 0) { PlanHead h = {units, (int)segs, n_act}; *p.head = h; }
}

// ------------------------------------------------------------------------------------------------ attention, warp-level tensor cores
struct AttnArgs {
  const void *k, *v;                            // this layer of the pool
  const int* table;
  int max_pages, n_pages, page, shift, kv_heads, ratio, n_heads, n, rows;
  const void* q; long long q_stride;
  void* out; long long out_stride;
  float* lse;
  float scale2;                                 // softmax scale * log2(e)
  void* mem;
};

template <typename T> struct Half2;
template <> struct Half2<__nv_bfloat16> {
  static __device__ __forceinline__ unsigned pack(float lo, float hi) { __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi); return *reinterpret_cast<unsigned*>(&v); }
  static __device__ __forceinline__ void mma(float* c, const unsigned* a, unsigned b0, unsigned b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
  static constexpr unsigned exp_mask = 0x7f80u;
  static __device__ __forceinline__ float value(unsigned short x) { return __uint_as_float((unsigned)x << 16); }
};
template <> struct Half2<__half> {
  static __device__ __forceinline__ unsigned pack(float lo, float hi) { __half2 v = __floats2half2_rn(lo, hi); return *reinterpret_cast<unsigned*>(&v); }
  static __device__ __forceinline__ void mma(float* c, const unsigned* a, unsigned b0, unsigned b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
  static constexpr unsigned exp_mask = 0x7c00u;
  static __device__ __forceinline__ float value(unsigned short x) { return __half2float(__ushort_as_half(x)); }
};

__device__ __forceinline__ unsigned pf_smem(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ float pf_ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ void pf_ldsm4(unsigned addr, unsigned* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void pf_ldsm4t(unsigned addr, unsigned* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void pf_cp16(unsigned dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
// byte offset of 16-byte piece `col16` of row `row` in a [64 rows][64 elements] block whose pieces are XOR-swizzled by the row
__device__ __forceinline__ unsigned pf_swz(int row, int col16) { return (unsigned)(row * 128 + (((col16 ^ row) & 7) << 4)); }

// A tile is [halves of 64 elements][64 rows][128 bytes].  Shared memory of a CTA: Q tile, then PF_STAGES x (K tile, V tile).
template <int D> __host__ __device__ constexpr int pf_tile() { return 64 * D * 2; }
template <int D> constexpr int pf_smem_bytes() { return pf_tile<D>() * (1 + 2 * PF_STAGES); }

// One 64-key block.  WIDE: 64 rows, warp w holds rows 16w..16w+15 and all keys.  Otherwise 16 rows and warp w holds keys 16w..16w+15.
template <typename T, int D, bool WIDE>
struct Block {
  static constexpr int NK = WIDE ? 8 : 2;       // 8-key column groups of S per warp
  float o[D / 8][4];
  float m[2], l[2];                             // of the thread's two rows (lane/4 and lane/4 + 8)
  unsigned qf[D / 16][4];

  __device__ __forceinline__ void begin(unsigned q_s, int warp, int lane) {
#pragma unroll
    for (int j = 0; j < D / 8; ++j) { o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f; }
    m[0] = m[1] = -INFINITY; l[0] = l[1] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const int row = (WIDE ? warp * 16 : 0) + (lane & 7) + ((lane >> 3) & 1) * 8, c16 = ks * 2 + (lane >> 4);
      pf_ldsm4(q_s + (unsigned)(c16 >> 3) * 8192u + pf_swz(row, c16 & 7), qf[ks]);
    }
  }
  // key_lo: position of the block's first key; lim[r]: first position row r does not see (masked blocks only)
  __device__ __forceinline__ void step(unsigned k_s, unsigned v_s, const unsigned char* v_p, int warp, int lane, float scale2, bool masked,
                                       int key_lo, const int* lim, bool dirty) {
    const int kw = WIDE ? 0 : warp * 16;
    float s[NK][4];
#pragma unroll
    for (int j = 0; j < NK; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const int c16 = ks * 2 + ((lane >> 3) & 1);
#pragma unroll
      for (int jp = 0; jp < NK / 2; ++jp) {
        const int key = kw + jp * 16 + (lane & 7) + ((lane >> 4) & 1) * 8;
        unsigned b[4];
        pf_ldsm4(k_s + (unsigned)(c16 >> 3) * 8192u + pf_swz(key, c16 & 7), b);
        Half2<T>::mma(s[2 * jp], qf[ks], b[0], b[1]);
        Half2<T>::mma(s[2 * jp + 1], qf[ks], b[2], b[3]);
      }
    }
    float bm[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < NK; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = key_lo + kw + j * 8 + 2 * (lane & 3) + (e & 1);
        float x = s[j][e] * scale2;
        if (masked && key >= lim[e >> 1]) x = -INFINITY;
        s[j][e] = x;
        bm[e >> 1] = fmaxf(bm[e >> 1], x);
      }
    float ref[2], al[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      bm[r] = fmaxf(bm[r], __shfl_xor_sync(0xffffffffu, bm[r], 1));
      bm[r] = fmaxf(bm[r], __shfl_xor_sync(0xffffffffu, bm[r], 2));
      const float mn = fmaxf(m[r], bm[r]);
      ref[r] = mn == -INFINITY ? 0.f : mn;                              // a row that has seen nothing yet: no inf - inf
      al[r] = pf_ex2(m[r] - ref[r]);
      m[r] = mn;
      l[r] *= al[r];
    }
#pragma unroll
    for (int j = 0; j < D / 8; ++j) { o[j][0] *= al[0]; o[j][1] *= al[0]; o[j][2] *= al[1]; o[j][3] *= al[1]; }
    unsigned pf[NK / 2][4];
    // P is rounded to the 16-bit type for the product with V (half a step: 2^-9 bf16, 2^-12 fp16 of each weight); the sum l takes the
    // unrounded weights
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      const float p0 = pf_ex2(s[j][0] - ref[0]), p1 = pf_ex2(s[j][1] - ref[0]), p2 = pf_ex2(s[j][2] - ref[1]), p3 = pf_ex2(s[j][3] - ref[1]);
      l[0] += p0 + p1; l[1] += p2 + p3;
      pf[j >> 1][(j & 1) * 2] = Half2<T>::pack(p0, p1);
      pf[j >> 1][(j & 1) * 2 + 1] = Half2<T>::pack(p2, p3);
    }
    if (dirty) {
      // a masked block with infinities or NaN in V: they reach the rows that see them, and no other (0 * inf would)
      for (int key = kw; key < kw + NK * 8; ++key)
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int col = j * 8 + 2 * (lane & 3) + e;
            const unsigned short x = *reinterpret_cast<const unsigned short*>(v_p + (col >> 6) * 8192 + pf_swz(key, (col & 63) >> 3) + (col & 7) * 2);
            if ((x & Half2<T>::exp_mask) == Half2<T>::exp_mask) {
              if (key_lo + key < lim[0]) o[j][e] += Half2<T>::value(x);
              if (key_lo + key < lim[1]) o[j][2 + e] += Half2<T>::value(x);
            }
          }
    }
    if (!dirty) pv(v_s, pf, kw, lane);
    else {
      clean(v_p);
      pv(v_s, pf, kw, lane);
    }
  }
  __device__ __forceinline__ void pv(unsigned v_s, const unsigned (*pf)[4], int kw, int lane) {
#pragma unroll
    for (int ks = 0; ks < NK / 2; ++ks) {
      const int key = kw + ks * 16 + (lane & 7) + ((lane >> 3) & 1) * 8;
#pragma unroll
      for (int np = 0; np < D / 16; ++np) {
        const int c16 = np * 2 + (lane >> 4);
        unsigned b[4];
        pf_ldsm4t(v_s + (unsigned)(c16 >> 3) * 8192u + pf_swz(key, c16 & 7), b);
        Half2<T>::mma(o[2 * np], pf[ks], b[0], b[1]);
        Half2<T>::mma(o[2 * np + 1], pf[ks], b[2], b[3]);
      }
    }
  }
  // all threads: zeros in the place of infinities and NaN of the V tile
  static __device__ __noinline__ void clean(const unsigned char* v_p) {
    __syncthreads();
    unsigned short* x = reinterpret_cast<unsigned short*>(const_cast<unsigned char*>(v_p));
    for (int i = threadIdx.x; i < 64 * D; i += PF_THREADS)
      if ((x[i] & Half2<T>::exp_mask) == Half2<T>::exp_mask) x[i] = 0;
    __syncthreads();
  }
};

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

template <typename T, int D, bool WIDE>
__device__ __forceinline__ void piece(const AttnArgs& a, const PlanMem& p, const SegRec& sg, int head, int rt, int kb0, int nkb, int cta, bool direct,
                                      unsigned char* sm) {
  constexpr int BM = WIDE ? 64 : 16, C16 = D / 8, RSTEP = PF_THREADS / C16, TILE = pf_tile<D>();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const unsigned q_s = pf_smem(sm), ring = q_s + TILE;
  const int nr = min(BM, sg.R - rt * BM);
  const int c16 = tid % C16, r_first = tid / C16;
  const size_t row_el = (size_t)a.kv_heads * D;
  const T *kg = (const T*)a.k + head * D + c16 * 8, *vg = (const T*)a.v + head * D + c16 * 8;
  const int* tab = a.table + (size_t)sg.slot * a.max_pages;
  const unsigned col_off = (unsigned)(c16 >> 3) * 8192u;
  auto load = [&](int i) {                                              // key block kb0 + i into stage i % PF_STAGES
    const unsigned ks = ring + (unsigned)(i % PF_STAGES) * 2u * TILE, vs = ks + TILE;
    const int k0 = sg.key0 + (kb0 + i) * PF_KB;
    int pg[64 / RSTEP];
#pragma unroll
    for (int x = 0; x < 64 / RSTEP; ++x) {
      const int key = k0 + r_first + x * RSTEP;
      pg[x] = key < sg.key1 ? tab[key >> a.shift] : -1;
    }
#pragma unroll
    for (int x = 0; x < 64 / RSTEP; ++x) {
      const int r = r_first + x * RSTEP, key = k0 + r;
      const bool ok = (unsigned)pg[x] < (unsigned)a.n_pages;            // beyond the segment: zeros
      const size_t at = (((size_t)(ok ? pg[x] : 0) << a.shift) + (key & (a.page - 1))) * row_el;
      const unsigned off = col_off + pf_swz(r, c16 & 7);
      pf_cp16(ks + off, kg + at, ok);
      pf_cp16(vs + off, vg + at, ok);
    }
  };
  // Q tile: stacked row x is q row row0 + x / ratio, query head head * ratio + x % ratio
  for (int r = r_first; r < BM; r += RSTEP) {
    const int x = rt * BM + min(r, nr - 1);
    const T* src = (const T*)a.q + (size_t)(sg.row0 + x / a.ratio) * a.q_stride + (size_t)(head * a.ratio + x % a.ratio) * D + c16 * 8;
    pf_cp16(q_s + col_off + pf_swz(r, c16 & 7), src, r < nr);
  }
#pragma unroll
  for (int i = 0; i < PF_STAGES - 1; ++i) {
    if (i < nkb) load(i);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // the thread's two rows
  const int rl[2] = {(WIDE ? warp * 16 : 0) + (lane >> 2), (WIDE ? warp * 16 : 0) + (lane >> 2) + 8};
  int lim[2] = {sg.key1, sg.key1};
#pragma unroll
  for (int r = 0; r < 2; ++r)
    if (rl[r] < nr && sg.pos0 != INT_MIN) lim[r] = min(sg.key1, sg.pos0 + (rt * BM + rl[r]) / a.ratio + 1);
  const int lim_min = sg.pos0 == INT_MIN ? sg.key1 : min(sg.key1, sg.pos0 + (rt * BM) / a.ratio + 1);
  Block<T, D, WIDE> blk;
  for (int i = 0; i < nkb; ++i) {
    asm volatile("cp.async.wait_group %0;" ::"n"(PF_STAGES - 2) : "memory");
    __syncthreads();
    if (i == 0) blk.begin(q_s, warp, lane);
    if (i + PF_STAGES - 1 < nkb) load(i + PF_STAGES - 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const unsigned st = (unsigned)(i % PF_STAGES) * 2u * TILE;
    const int key_lo = sg.key0 + (kb0 + i) * PF_KB;
    const bool masked = key_lo + PF_KB > lim_min;                       // some row does not see the whole block
    bool dirty = false;
    if (masked && lim_min < sg.key1) {
      bool bad = false;
      const uint4* vt = reinterpret_cast<const uint4*>(sm + TILE + st + TILE);
      for (int x = tid; x < TILE / 16; x += PF_THREADS) bad |= any_nonfinite<T>(vt[x]);
      dirty = __syncthreads_or(bad);
    }
    blk.step(ring + st, ring + st + TILE, sm + TILE + st + TILE, warp, lane, a.scale2, masked, key_lo, lim, dirty);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    blk.l[r] += __shfl_xor_sync(0xffffffffu, blk.l[r], 1);
    blk.l[r] += __shfl_xor_sync(0xffffffffu, blk.l[r], 2);
  }
  const size_t slot0 = (size_t)sg.rowbase + (size_t)head * sg.R + (size_t)rt * BM + (size_t)cta * PF_BM;
  auto where = [&](int r, T** dst, float** lse) {                       // final place of stacked row r
    const int x = rt * BM + r, row = sg.row0 + x / a.ratio, h = head * a.ratio + x % a.ratio;
    *dst = (T*)a.out + (size_t)row * a.out_stride + (size_t)h * D;
    *lse = a.lse ? a.lse + (size_t)row * a.n_heads + h : nullptr;
  };
  if (WIDE) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      if (rl[r] >= nr) continue;
      if (direct) {
        T* dst; float* ls;
        where(rl[r], &dst, &ls);
        const float inv = blk.l[r] == 0.f ? 0.f : 1.f / blk.l[r];
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
          *reinterpret_cast<unsigned*>(dst + j * 8 + 2 * (lane & 3)) = Half2<T>::pack(blk.o[j][2 * r] * inv, blk.o[j][2 * r + 1] * inv);
        if (ls && (lane & 3) == 0) *ls = (blk.m[r] + log2f(blk.l[r])) * 0.693147180559945f;
      } else {
        float* dst = p.po + (slot0 + rl[r]) * D;
#pragma unroll
        for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(dst + j * 8 + 2 * (lane & 3)) = make_float2(blk.o[j][2 * r], blk.o[j][2 * r + 1]);
        if ((lane & 3) == 0) p.ml[slot0 + rl[r]] = make_float2(blk.m[r], blk.l[r]);
      }
    }
    __syncthreads();                                                    // the next piece refills the tiles
  } else {
    // the four warps hold the same rows over different keys: add them up in warp order through the ring
    float* ox = reinterpret_cast<float*>(sm + TILE);                    // [4][16][D + 4]
    float2* mx = reinterpret_cast<float2*>(ox + 4 * 16 * (D + 4));      // [4][16]
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
      for (int j = 0; j < D / 8; ++j)
        *reinterpret_cast<float2*>(ox + (warp * 16 + rl[r]) * (D + 4) + j * 8 + 2 * (lane & 3)) = make_float2(blk.o[j][2 * r], blk.o[j][2 * r + 1]);
      if ((lane & 3) == 0) mx[warp * 16 + rl[r]] = make_float2(blk.m[r], blk.l[r]);
    }
    __syncthreads();
    for (int x = tid; x < nr * (D / 4); x += PF_THREADS) {
      const int r = x / (D / 4), c = (x % (D / 4)) * 4;
      float M = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) M = fmaxf(M, mx[w * 16 + r].x);
      const float ref = M == -INFINITY ? 0.f : M;
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float2 ml = mx[w * 16 + r];
        const float f = pf_ex2(ml.x - ref);
        const float4 o4 = *reinterpret_cast<const float4*>(ox + (w * 16 + r) * (D + 4) + c);
        l += f * ml.y;
        s.x += f * o4.x; s.y += f * o4.y; s.z += f * o4.z; s.w += f * o4.w;
      }
      if (direct) {
        T* dst; float* ls;
        where(r, &dst, &ls);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        *reinterpret_cast<uint2*>(dst + c) = make_uint2(Half2<T>::pack(s.x * inv, s.y * inv), Half2<T>::pack(s.z * inv, s.w * inv));
        if (ls && c == 0) *ls = (M + log2f(l)) * 0.693147180559945f;
      } else {
        *reinterpret_cast<float4*>(p.po + (slot0 + r) * D + c) = s;
        if (c == 0) p.ml[slot0 + r] = make_float2(M, l);
      }
    }
    __syncthreads();
  }
}

// Whether a tile of a segment is one piece and holds everything its rows see: then the piece writes the result itself.
__device__ __forceinline__ bool tile_direct(const SegRec& s, long long u_tile, long long U) {
  return s.pos0 != INT_MIN && s.key0 == 0 && run_of(u_tile, U) == run_of(u_tile + s.KB - 1, U);
}

template <typename T, int D>
__global__ void __launch_bounds__(PF_THREADS, 2) prefix_mma_kernel(AttnArgs a) {
  extern __shared__ __align__(1024) unsigned char pf_raw[];
  const PlanMem p = plan_mem(a.mem, a.n, a.rows, a.n_heads, D);
  pdl_trigger();
  pdl_wait();
  const long long U = p.head->units;
  const int cta = blockIdx.x;
  const long long G = runs(U);
  if (cta >= G) return;
  long long u = cta * U / G;
  const long long u_end = (cta + 1) * U / G;
  int g = p.first[cta];
  SegRec s = p.seg[g];
  while (u < u_end) {
    while (u >= s.uend) s = p.seg[++g];
    const long long local = u - s.ustart;
    const int per_head = s.T * s.KB, head = (int)(local / per_head), rem = (int)(local % per_head), rt = rem / s.KB, kb = rem % s.KB;
    const int n = (int)min((long long)(s.KB - kb), u_end - u);
    const bool direct = tile_direct(s, u - kb, U);
    if (s.bm == 16) piece<T, D, false>(a, p, s, head, rt, kb, n, cta, direct, pf_raw);
    else piece<T, D, true>(a, p, s, head, rt, kb, n, cta, direct, pf_raw);
    u += n;
  }
}

// One warp per (row, query head): the pieces of its prefix and of its own segment, added in order.
template <typename T, int D>
__global__ void __launch_bounds__(256) prefix_join_kernel(AttnArgs a) {
  constexpr int E = D / 32;                                             // outputs per lane
  const PlanMem p = plan_mem(a.mem, a.n, a.rows, a.n_heads, D);
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_trigger();
  pdl_wait();
  if (w >= (long long)a.rows * a.n_heads) return;
  const int row = (int)(w / a.n_heads), h = (int)(w % a.n_heads), kvh = h / a.ratio;
  const int k = p.row_k[row];
  if (k < 0) return;
  const long long U = p.head->units;
  const SeqRec q = p.seq[k];
  int np[2] = {0, 0};
  size_t base[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int g = i ? q.suf_seg : q.pre_seg;
    if (g < 0) continue;
    const SegRec s = p.seg[g];
    const int x = (row - s.row0) * a.ratio + h % a.ratio, rt = x / s.bm;
    const long long u0 = s.ustart + ((long long)kvh * s.T + rt) * s.KB;
    if (tile_direct(s, u0, U)) return;                                  // written by its only piece
    const int c0 = run_of(u0, U);
    np[i] = run_of(u0 + s.KB - 1, U) - c0 + 1;
    base[i] = (size_t)s.rowbase + (size_t)kvh * s.R + x + (size_t)c0 * PF_BM;
  }
  const int n = np[0] + np[1];
  auto slot = [&](int i) { return i < np[0] ? base[0] + (size_t)i * PF_BM : base[1] + (size_t)(i - np[0]) * PF_BM; };
  float M = -INFINITY;
  for (int i = lane; i < n; i += 32) M = fmaxf(M, p.ml[slot(i)].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  const float ref = M == -INFINITY ? 0.f : M;
  float l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const size_t sl = slot(i);
    const float2 ml = p.ml[sl];
    const float f = pf_ex2(ml.x - ref);
    l += f * ml.y;
    const float* src = p.po + sl * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 v = *reinterpret_cast<const float2*>(src + e);
      o[e] += f * v.x; o[e + 1] += f * v.y;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* dst = (T*)a.out + (size_t)row * a.out_stride + (size_t)h * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; e += 2) *reinterpret_cast<unsigned*>(dst + e) = Half2<T>::pack(o[e] * inv, o[e + 1] * inv);
  if (a.lse && lane == 0) a.lse[(size_t)row * a.n_heads + h] = (M + log2f(l)) * 0.693147180559945f;
}

template <typename T, int D>
int launch_attention(const AttnArgs& a, cudaStream_t s) {
  VLAC_CUDA_CHECK(cudaFuncSetAttribute(prefix_mma_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, pf_smem_bytes<D>()));
  VLAC_CUDA_CHECK(launch_pdl(prefix_mma_kernel<T, D>, dim3(PF_GRID_A), dim3(PF_THREADS), pf_smem_bytes<D>(), s, a));
  const long long warps = (long long)a.rows * a.n_heads;
  VLAC_CUDA_CHECK(launch_pdl(prefix_join_kernel<T, D>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, s, a));
  return VLAC_OK;
}

int plan_check(const vlac_pages* p, const vlac_prefix* plan) {
  const int rc = pages_check(p);
  if (rc != VLAC_OK) return rc;
  if (!plan || plan->n < 0 || plan->rows < 0) return VLAC_ERR_INVALID_ARG;
  if (plan->n > VLAC_PAGES_MAX_LIST) return VLAC_ERR_TOO_LARGE;
  if (plan->n == 0 || plan->rows == 0) return VLAC_OK;
  const unsigned long long need = vlac_prefix_bytes(p, plan->n, plan->rows, plan->n_heads);
  if (need == 0 || !plan->mem || ((uintptr_t)plan->mem & 15u) || plan->bytes < need) return VLAC_ERR_INVALID_ARG;
  return VLAC_OK;
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
  if (plan->rows == 0) {                          // nothing to compute; every entry is fine
    VLAC_CUDA_CHECK(cudaMemsetAsync(status, 0, sizeof(int) * plan->n, (cudaStream_t)stream));
    return VLAC_OK;
  }
  PlanArgs a = {};
  a.table = p->table; a.len = p->len; a.n_slots = p->n_slots; a.max_pages = p->max_pages; a.n_pages = p->n_pages; a.page = p->page_size;
  a.shift = pages_shift(p->page_size); a.kv_heads = p->n_kv_heads; a.ratio = plan->n_heads / p->n_kv_heads; a.head_dim = p->head_dim;
  a.n = plan->n; a.rows = plan->rows; a.n_heads = plan->n_heads; a.seqs = seqs; a.q_ptr = q_ptr; a.status = status; a.mem = plan->mem;
  VLAC_CUDA_CHECK(launch_pdl(prefix_plan_kernel, dim3(PL_CTAS), dim3(PL_THREADS), 0, (cudaStream_t)stream, a));
  return VLAC_OK;
}

int vlac_prefix_attention(const vlac_pages* p, int layer, const vlac_prefix* plan, const void* q, long long q_stride, float scale,
                          void* out, long long out_stride, float* lse, void* stream) {
  const int rc = plan_check(p, plan);
  if (rc != VLAC_OK) return rc;
  if (layer < 0 || layer >= p->n_layers || !isfinite(scale)) return VLAC_ERR_INVALID_ARG;
  if (plan->n == 0 || plan->rows == 0) return VLAC_OK;
  const long long w = (long long)plan->n_heads * p->head_dim;
  if (!q || !out || q_stride < w || out_stride < w || q_stride % 8 || out_stride % 8 || (((uintptr_t)q | (uintptr_t)out) & 15u) || ((uintptr_t)lse & 3u))
    return VLAC_ERR_INVALID_ARG;
  AttnArgs a = {};
  a.k = (const unsigned short*)p->k + (size_t)layer * pages_layer(p); a.v = (const unsigned short*)p->v + (size_t)layer * pages_layer(p);
  a.table = p->table; a.max_pages = p->max_pages; a.n_pages = p->n_pages; a.page = p->page_size; a.shift = pages_shift(p->page_size);
  a.kv_heads = p->n_kv_heads; a.ratio = plan->n_heads / p->n_kv_heads; a.n_heads = plan->n_heads; a.n = plan->n; a.rows = plan->rows;
  a.q = q; a.q_stride = q_stride; a.out = out; a.out_stride = out_stride; a.lse = lse;
  a.scale2 = scale * 1.44269504088896f; a.mem = plan->mem;
  cudaStream_t s = (cudaStream_t)stream;
  if (p->dtype == VLAC_BF16) return p->head_dim == 128 ? launch_attention<__nv_bfloat16, 128>(a, s) : launch_attention<__nv_bfloat16, 64>(a, s);
  return p->head_dim == 128 ? launch_attention<__half, 128>(a, s) : launch_attention<__half, 64>(a, s);
}

}  // extern "C"
