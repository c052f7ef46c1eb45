// Rotary tables, and new rows on their way into the paged pool: norm of each head's queries and keys, rotation, append.
#include "pages_internal.h"
#include "launch_util.h"
#include <cuda_fp16.h>
#include <math.h>

namespace {

// ------------------------------------------------------------------------------------------------ tables
// Angles are kept as turns (angle / 2 pi): the whole turns of a far position fall away exactly before a sine is taken.  Turns per position come
// from the host as a pair of doubles (from its extended type); a thread takes one frequency and a run of positions: one sine and cosine in
// 64 bits for the first, then a rotation by the angle of one position each (four products in 64 bits; the error grows by about 2^-53 a step).
// Bound: the stores (262,144 positions of 128 dimensions, 134 MB: 21.6 us, 6.2 TB/s); a table of 2048 positions is a launch (2.8 us).
constexpr int RT_MAX = 256, RT_THREADS = 256;
struct TableArgs {
  double turns[RT_MAX / 2], rest[RT_MAX / 2];   // per position; what the double leaves of it
  double amplitude;
  int half, first, n_pos, run;
  float *cos, *sin;
};

__device__ __forceinline__ void turn_sincos(double pos, double t, double rest, double* s, double* c) {
  const double whole = pos * t, low = fma(pos, t, -whole) + pos * rest;
  sincospi(2.0 * ((whole - rint(whole)) + low), s, c);
}

__global__ void __launch_bounds__(RT_THREADS) rope_tables_kernel(const __grid_constant__ TableArgs a) {
  pdl_trigger();
  pdl_wait();
  const long long u = (long long)blockIdx.x * RT_THREADS + threadIdx.x;
  const long long at = u < 1ll << 32 ? (unsigned)u / (unsigned)a.half : u / a.half;       // (a 64-bit division is five times as long)
  const int i = (int)(u - at * a.half);
  const long long p0 = at * a.run;
  if (p0 >= a.n_pos) return;
  double s, c, ds, dc;
  turn_sincos((double)(a.first + p0), a.turns[i], a.rest[i], &s, &c);
  turn_sincos(1.0, a.turns[i], a.rest[i], &ds, &dc);
  const int n = (int)min((long long)a.run, a.n_pos - p0);
  float *co = a.cos + (size_t)p0 * a.half + i, *so = a.sin + (size_t)p0 * a.half + i;
  for (int p = 0; p < n; ++p) {
    co[(size_t)p * a.half] = (float)(a.amplitude * c);
    so[(size_t)p * a.half] = (float)(a.amplitude * s);
    const double t = c * dc - s * ds;
    s = s * dc + c * ds;
    c = t;
  }
}

// ------------------------------------------------------------------------------------------------ append
constexpr int AP_THREADS = 256, AP_WARPS = AP_THREADS / 32, AP_BATCH = 6, AP_CTAS = 24;
struct AppendArgs {
  void *k, *v;                                  // the layer
  const int *table, *len, *refs;
  int n_slots, max_pages, n_pages, page, shift, n, rows;
  const int *seqs, *start, *row_ptr, *pos;
  int heads, kv_heads;
  const float *cos, *sin;
  int n_pos, rot;
  const void *q_gain, *k_gain;
  float eps;
  const void *q, *kin, *vin; void* qout;
  long long q_stride, qout_stride, k_stride, v_stride;
  int* status;
  int split;                                    // warps that share a row: 1, 2, 4 or 8
};

// pairs of fp32: one instruction for two elements
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float lo, float hi) { F2 d; asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi)); return d; }
__device__ __forceinline__ float2 f2_parts(F2 d) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(d)); return r; }
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) { F2 d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) { F2 d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }

template <typename T> struct Pair16;
template <> struct Pair16<__nv_bfloat16> {
  static __device__ __forceinline__ F2 two(unsigned x) { return f2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
  static __device__ __forceinline__ unsigned pack(F2 x) { const float2 p = f2_parts(x); __nv_bfloat162 v = __floats2bfloat162_rn(p.x, p.y); return *reinterpret_cast<unsigned*>(&v); }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};
template <> struct Pair16<__half> {
  static __device__ __forceinline__ F2 two(unsigned x) { const float2 p = __half22float2(*reinterpret_cast<__half2*>(&x)); return f2(p.x, p.y); }
  static __device__ __forceinline__ unsigned pack(F2 x) { const float2 p = f2_parts(x); __half2 v = __floats2half2_rn(p.x, p.y); return *reinterpret_cast<unsigned*>(&v); }
  static __device__ __forceinline__ float one(const __half* p) { return __half2float(*p); }
};

// two pieces of 4 elements, which may be neighbours
template <bool ONE> __device__ __forceinline__ void load8(uint2* x, const void* p0, const void* p1) {
  if (ONE) { const uint4 v = *reinterpret_cast<const uint4*>(p0); x[0] = make_uint2(v.x, v.y); x[1] = make_uint2(v.z, v.w); }
  else { x[0] = *reinterpret_cast<const uint2*>(p0); x[1] = *reinterpret_cast<const uint2*>(p1); }
}
template <bool ONE> __device__ __forceinline__ void store8(const uint2* x, void* p0, void* p1) {
  if (ONE) *reinterpret_cast<uint4*>(p0) = make_uint4(x[0].x, x[0].y, x[1].x, x[1].y);
  else { *reinterpret_cast<uint2*>(p0) = x[0]; *reinterpret_cast<uint2*>(p1) = x[1]; }
}

// grid (x, entries).  A lane holds 8 elements of a head in two pieces of 4, a warp two heads of 128 or four of 64 at a time, all of one row, so that a lane's
// cosines and sines stay in registers for the whole row.  The pieces are the two that are rotated with one another (half layout: rot/2 apart;
// interleaved, and behind the rotated part: neighbours), so that nothing is exchanged between lanes but the sum of a norm.  (With pieces of 8 neighbours and
// the partner's values by shuffles 96 heads of 128 took 260 us a 1.45 GB call against 201, 48 of 64 111 against 66.)  Each CTA checks the whole entry for
// itself, so that an entry is written whole or not at all without a second launch.  Bound: HBM where heads are 128 wide and only rotated (201 us, 7.2 TB/s of
// algorithmic bytes, part of the writes still in L2), the instructions beside it with norms (fp16, interleaved quarter, 0.63 GB: 113 us, 5.6 TB/s, 72 % of the
// issue slots); one row each for 64 sequences 4.8 us, launch and dependent reads.
template <typename T, int D, bool INTER, bool NORM>
__global__ void __launch_bounds__(AP_THREADS, 4) pages_append_kernel(AppendArgs a) {
  constexpr int LANES = D / 8, PER = 32 / LANES;                        // lanes of a head; heads of a warp
  __shared__ __align__(16) float s_gain[NORM ? 2 : 1][D];
  const int tid = threadIdx.x, i = blockIdx.y, warp = tid >> 5, lane = tid & 31;
  pdl_trigger();
  pdl_wait();
  const int slot = a.seqs[i], r0 = a.row_ptr[i], r1 = a.row_ptr[i + 1];
  int code = 0, at0 = 0;
  if ((unsigned)slot >= (unsigned)a.n_slots || r0 < 0 || r1 < r0 || r1 > a.rows) code = VLAC_ERR_INVALID_ARG;
  else {
    const int len = a.len[slot];
    if (len < 0 || len > a.max_pages << a.shift) code = VLAC_ERR_BAD_STATE;
    else {
      at0 = a.start ? a.start[i] : len - (r1 - r0);
      if (at0 < 0 || (long long)at0 + (r1 - r0) > len) code = VLAC_ERR_INVALID_ARG;
      else if (a.rot && !a.pos && r1 > r0 && at0 + (r1 - r0) > a.n_pos) code = VLAC_ERR_INVALID_ARG;
    }
  }
  // (uniform so far) an earlier entry with the same slot stands; positions have a row in the tables; pages exist and are the slot's own
  int wrong = 0, bad = 0, falls = 0;
  for (int j = tid; j < i; j += AP_THREADS) wrong |= a.seqs[j] == slot;
  for (int j = tid; j < a.n; j += AP_THREADS) falls |= a.row_ptr[j + 1] < a.row_ptr[j];    // entries would share rows of q: all are refused
  const int* t = a.table + (size_t)(code == 0 ? slot : 0) * a.max_pages;
  if (code == 0 && r1 > r0) {
    for (int j = (at0 >> a.shift) + tid; j <= (at0 + r1 - r0 - 1) >> a.shift; j += AP_THREADS) {
      const int p = t[j];
      bad |= (unsigned)p >= (unsigned)a.n_pages || a.refs[p] != 1;
    }
    if (a.pos && a.rot) for (int j = r0 + tid; j < r1; j += AP_THREADS) wrong |= (unsigned)a.pos[j] >= (unsigned)a.n_pos;
  }
  if (__syncthreads_or(wrong)) code = VLAC_ERR_INVALID_ARG;
  if (__syncthreads_or(bad) && code == 0) code = VLAC_ERR_BAD_STATE;
  if (__syncthreads_or(falls)) code = VLAC_ERR_INVALID_ARG;
  if (tid == 0 && blockIdx.x == 0) a.status[i] = code;
  if (code != 0) return;

  if (NORM) {
    for (int e = tid; e < D; e += AP_THREADS) {
      s_gain[0][e] = a.q_gain ? Pair16<T>::one((const T*)a.q_gain + e) : 1.f;
      s_gain[1][e] = a.k_gain ? Pair16<T>::one((const T*)a.k_gain + e) : 1.f;
    }
    __syncthreads();
  }
  const int c = lane % LANES, pairs = a.rot / 8;                        // lanes whose pieces are rotated
  const bool turned = c < pairs;
  const int el0 = INTER || !turned ? 8 * c : 4 * c, el1 = INTER || !turned ? 8 * c + 4 : 4 * c + a.rot / 2;      // first element of each piece
  const size_t lane0 = (size_t)(lane / LANES) * D + el0, lane1 = (size_t)(lane / LANES) * D + el1;
  // A warp's share of a row: slots of PER heads, those of q, of k, of v, the same for all its lanes (the compiler is told)
  const int w = __shfl_sync(0xffffffffu, warp, 0), per_cta = AP_WARPS / a.split;
  const int nq = (a.heads + PER - 1) / PER, nk = (a.kv_heads + PER - 1) / PER, slots = nq + 2 * nk;
  for (int r = r0 + blockIdx.x * per_cta + w / a.split; r < r1; r += gridDim.x * per_cta) {
    const int at = at0 + (r - r0);
    const size_t pool = (((size_t)t[at >> a.shift] << a.shift) + (at & (a.page - 1))) * ((size_t)a.kv_heads * D);
    float4 cs = make_float4(1.f, 1.f, 1.f, 1.f), sn = make_float4(0.f, 0.f, 0.f, 0.f);  // of the lane's four pairs
    if (turned) {
      const size_t row = (size_t)(a.pos ? a.pos[r] : at) * (a.rot / 2) + 4 * c;
      cs = *reinterpret_cast<const float4*>(a.cos + row);
      sn = *reinterpret_cast<const float4*>(a.sin + row);
    }
    const T *qi = (const T*)a.q + (size_t)r * a.q_stride, *ki = (const T*)a.kin + (size_t)r * a.k_stride, *vi = (const T*)a.vin + (size_t)r * a.v_stride;
    T *qo = (T*)a.qout + (size_t)r * a.qout_stride, *ko = (T*)a.k + pool, *vo = (T*)a.v + pool;
    for (int s0 = w % a.split; s0 < slots; s0 += a.split * AP_BATCH) {
      uint2 x[AP_BATCH][2];
#pragma unroll
      for (int b = 0; b < AP_BATCH; ++b) {
        const int s = s0 + b * a.split, kind = s < nq ? 0 : s < nq + nk ? 1 : 2, h = (kind == 0 ? s : kind == 1 ? s - nq : s - nq - nk) * PER;
        const T* from = (kind == 0 ? qi : kind == 1 ? ki : vi) + (size_t)h * D;
        if (s < slots && h + lane / LANES < (kind == 0 ? a.heads : a.kv_heads)) load8<INTER>(x[b], from + lane0, from + lane1);
        else x[b][0] = x[b][1] = make_uint2(0, 0);
      }
#pragma unroll
      for (int b = 0; b < AP_BATCH; ++b) {
        const int s = s0 + b * a.split, kind = s < nq ? 0 : s < nq + nk ? 1 : 2, h = (kind == 0 ? s : kind == 1 ? s - nq : s - nq - nk) * PER;
        if (s >= slots) break;
        if (kind < 2) {
          F2 f[4] = {Pair16<T>::two(x[b][0].x), Pair16<T>::two(x[b][0].y), Pair16<T>::two(x[b][1].x), Pair16<T>::two(x[b][1].y)};
          if (NORM && (kind == 0 ? a.q_gain : a.k_gain) != nullptr) {
            F2 s2 = f2_mul(f[0], f[0]);
#pragma unroll
            for (int e = 1; e < 4; ++e) s2 = f2_fma(f[e], f[e], s2);
            const float2 p = f2_parts(s2);
            float ss = p.x + p.y;
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            const float inv = rsqrtf(ss * (1.f / D) + a.eps);
            const float4 g0 = *reinterpret_cast<const float4*>(&s_gain[kind][el0]), g1 = *reinterpret_cast<const float4*>(&s_gain[kind][el1]);
            const F2 g[4] = {f2(g0.x, g0.y), f2(g0.z, g0.w), f2(g1.x, g1.y), f2(g1.z, g1.w)}, i2 = f2(inv, inv);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = f2_mul(f2_mul(f[e], i2), g[e]);
          }
          if (turned) {                                                 // (without rotation infinities pass as they are)
            if (INTER) {
              const float cc[4] = {cs.x, cs.y, cs.z, cs.w}, ss[4] = {sn.x, sn.y, sn.z, sn.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 y = f2_parts(f[e]);
                f[e] = f2(y.x * cc[e] - y.y * ss[e], y.x * ss[e] + y.y * cc[e]);
              }
            } else {
              const F2 cc[2] = {f2(cs.x, cs.y), f2(cs.z, cs.w)}, ss[2] = {f2(sn.x, sn.y), f2(sn.z, sn.w)}, ns[2] = {f2(-sn.x, -sn.y), f2(-sn.z, -sn.w)};
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const F2 u = f[e], v = f[2 + e];
                f[e] = f2_fma(v, ns[e], f2_mul(u, cc[e]));
                f[2 + e] = f2_fma(u, ss[e], f2_mul(v, cc[e]));
              }
            }
          }
          x[b][0] = make_uint2(Pair16<T>::pack(f[0]), Pair16<T>::pack(f[1]));
          x[b][1] = make_uint2(Pair16<T>::pack(f[2]), Pair16<T>::pack(f[3]));
        }
        T* to = (kind == 0 ? qo : kind == 1 ? ko : vo) + (size_t)h * D;
        if (h + lane / LANES < (kind == 0 ? a.heads : a.kv_heads)) store8<INTER>(x[b], to + lane0, to + lane1);
      }
    }
  }
}

template <typename T, int D>
int launch_append(const AppendArgs& a, bool inter, bool norm, dim3 grid, cudaStream_t s) {
  auto kernel = inter ? (norm ? pages_append_kernel<T, D, true, true> : pages_append_kernel<T, D, true, false>)
                      : (norm ? pages_append_kernel<T, D, false, true> : pages_append_kernel<T, D, false, false>);
  VLAC_CUDA_CHECK(launch_pdl(kernel, grid, dim3(AP_THREADS), 0, s, a));
  return VLAC_OK;
}

}  // namespace

extern "C" {

int vlac_rope_tables(const vlac_rope_scaling* r, int first, int n_pos, float* cos, float* sin, void* stream) {
  if (!r || r->rot_dim < 2 || r->rot_dim > RT_MAX || r->rot_dim % 2 || first < 0 || n_pos < 0 || (long long)first + n_pos > INT_MAX) return VLAC_ERR_INVALID_ARG;
  if (!(r->theta > 0) || !isfinite(r->theta) || !(r->factor > 0) || !isfinite(r->factor) || !(r->original_len >= 0) || !isfinite(r->original_len) ||
      !isfinite(r->amplitude))
    return VLAC_ERR_INVALID_ARG;
  if (r->original_len > 0 && !(r->turns_low < r->turns_high)) return VLAC_ERR_INVALID_ARG;
  if (n_pos == 0) return VLAC_OK;
  if (!cos || !sin || ((uintptr_t)cos | (uintptr_t)sin) & 3u) return VLAC_ERR_INVALID_ARG;
  TableArgs a = {};
  a.half = r->rot_dim / 2; a.first = first; a.n_pos = n_pos; a.cos = cos; a.sin = sin; a.amplitude = r->amplitude;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  // f_i = theta^(-i/half) as the product of the theta^(-2^b/half) for the bits b of i: the highest by powl, its exponent in a short and a rest so that nothing of it is
  // rounded, the others as roots of one another, which halve its error.  With powl right to 2^-63 the factors are right to 2^-63 times 2.5, 1.75, 1.38, .., 1.02, and a
  // frequency, with its products and what follows here, to 2^-59 (2^-61.7 the worst of some 2,000).  128 products in a row left 2^-57 (theta far from one: 2^-55).
  long double f[RT_MAX / 2];
  const long double shrink = 1.0L / r->factor;
  int top = 1;
  while (top * 2 < a.half) top *= 2;
  const long double high = (float)((long double)-top / a.half), low = (-top - high * a.half) / a.half;
  long double part = powl((long double)r->theta, high) * powl((long double)r->theta, low);
  f[0] = 1.0L;
  for (int n = top; n > 0; n /= 2, part = sqrtl(part))
    for (int i = 0; i + n < a.half; i += 2 * n) f[i + n] = f[i] * part;
  for (int i = 0; i < a.half; ++i) {
    const long double turns = r->original_len * f[i] / two_pi;
    long double g = 0.0L;
    if (r->original_len > 0) {
      g = (turns - r->turns_low) / ((long double)r->turns_high - r->turns_low);
      g = g < 0.0L ? 0.0L : g > 1.0L ? 1.0L : g;
    }
    const long double per = f[i] * (g + (1.0L - g) * shrink) * (1.0L / two_pi);
    if (!(per < 65536.0L)) return VLAC_ERR_INVALID_ARG;
    a.turns[i] = (double)per;
    a.rest[i] = (double)(per - a.turns[i]);
  }
  // longer runs spare sines, shorter ones fill the GPU: 262,144 positions of 128 dimensions, runs of 8 / 16 / 32 / 64 41.0 / 24.2 / 21.6 / 22.6 us (the
  // stores take 20.5); of 32 dimensions 9.6 / 7.3 / 8.2 / 8.2
  a.run = (long long)n_pos * a.half >= 1 << 23 ? 32 : 16;
  const long long units = (long long)a.half * ((n_pos + a.run - 1LL) / a.run), ctas = (units + RT_THREADS - 1) / RT_THREADS;
  VLAC_CUDA_CHECK(launch_pdl(rope_tables_kernel, dim3((unsigned)ctas), dim3(RT_THREADS), 0, (cudaStream_t)stream, a));
  return VLAC_OK;
}

int vlac_pages_append(const vlac_pages* p, int layer, const int* seqs, const int* start, const int* row_ptr, int n, int rows, const vlac_rope* rope,
                      const int* pos, int n_heads, const void* q, long long q_stride, void* q_out, long long q_out_stride, const void* k_rows,
                      long long k_stride, const void* v_rows, long long v_stride, int* status, void* stream) {
  int rc = pages_check(p);
  if (rc == VLAC_OK) rc = list_check(n);
  if (rc != VLAC_OK) return rc;
  if (layer < 0 || layer >= p->n_layers || rows < 0 || n_heads < 0 || n_heads > 65536 || !rope) return VLAC_ERR_INVALID_ARG;
  if (rope->rot_dim < 0 || rope->rot_dim > p->head_dim || rope->rot_dim % 16 || (rope->interleaved != 0 && rope->interleaved != 1) || rope->n_pos < 0)
    return VLAC_ERR_INVALID_ARG;
  if (rope->rot_dim && (!rope->cos || !rope->sin || ((uintptr_t)rope->cos | (uintptr_t)rope->sin) & 15u)) return VLAC_ERR_INVALID_ARG;
  if (((uintptr_t)rope->q_gain | (uintptr_t)rope->k_gain) & 15u) return VLAC_ERR_INVALID_ARG;
  if ((rope->q_gain || rope->k_gain) && !(rope->eps >= 0.f && isfinite(rope->eps))) return VLAC_ERR_INVALID_ARG;
  if (n == 0) return VLAC_OK;
  if (!seqs || !row_ptr || !status || (rows > 0 && (!k_rows || !v_rows))) return VLAC_ERR_INVALID_ARG;
  if (((uintptr_t)seqs | (uintptr_t)start | (uintptr_t)row_ptr | (uintptr_t)pos | (uintptr_t)status) & 3u) return VLAC_ERR_INVALID_ARG;
  const long long w = (long long)pages_row(p), wq = (long long)n_heads * p->head_dim;
  if (k_stride < w || v_stride < w || k_stride % 8 || v_stride % 8 || (((uintptr_t)k_rows | (uintptr_t)v_rows) & 15u)) return VLAC_ERR_INVALID_ARG;
  if (n_heads > 0 && rows > 0) {
    if (!q || !q_out || q_stride < wq || q_out_stride < wq || q_stride % 8 || q_out_stride % 8 || (((uintptr_t)q | (uintptr_t)q_out) & 15u))
      return VLAC_ERR_INVALID_ARG;
    if (!(q == q_out && q_stride == q_out_stride) && rows_overlap((uintptr_t)q, 2ull * q_stride, (uintptr_t)q_out, 2ull * q_out_stride, 2ull * wq, 2ull * wq, rows))
      return VLAC_ERR_INVALID_ARG;
    if (rows_overlap((uintptr_t)k_rows, 2ull * k_stride, (uintptr_t)q_out, 2ull * q_out_stride, 2ull * w, 2ull * wq, rows) ||
        rows_overlap((uintptr_t)v_rows, 2ull * v_stride, (uintptr_t)q_out, 2ull * q_out_stride, 2ull * w, 2ull * wq, rows))
      return VLAC_ERR_INVALID_ARG;
    if (rows_in_pool(p, q_out, 2ull * q_out_stride, 2ull * wq, rows)) return VLAC_ERR_INVALID_ARG;
  }
  int n_sm = 0;
  rc = sm_count(&n_sm);
  if (rc != VLAC_OK) return rc;
  AppendArgs a = {};
  a.k = (unsigned short*)p->k + (size_t)layer * pages_layer(p); a.v = (unsigned short*)p->v + (size_t)layer * pages_layer(p);
  a.table = p->table; a.len = p->len; a.refs = p->refs; a.n_slots = p->n_slots; a.max_pages = p->max_pages; a.n_pages = p->n_pages; a.page = p->page_size;
  a.shift = pages_shift(p->page_size); a.n = n; a.rows = rows; a.seqs = seqs; a.start = start; a.row_ptr = row_ptr; a.pos = pos; a.heads = n_heads; a.kv_heads = p->n_kv_heads;
  a.cos = rope->cos; a.sin = rope->sin; a.n_pos = rope->n_pos; a.rot = rope->rot_dim; a.q_gain = rope->q_gain; a.k_gain = rope->k_gain; a.eps = rope->eps;
  a.q = q; a.kin = k_rows; a.vin = v_rows; a.qout = q_out; a.q_stride = q_stride; a.qout_stride = q_out_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.status = status;
  a.split = 1;
  while (a.split < AP_WARPS && (long long)rows * a.split < n_sm * 64ll) a.split *= 2;
  // CTAs: no more per entry than an entry of up to twice the mean length can use; what fits the GPU at once is not given a second wave (16 entries of 17 to 33
  // rows, 49 / 37 CTAs each: 8.2 / 6.9 us); larger calls get many short CTAs, which even out (8, 24, 48 an SM: 131 / 124 / 127 us for 8 prompts)
  const int per = AP_WARPS / a.split, mean = (int)((2ll * rows - n + (long long)n * per - 1) / ((long long)n * per));
  const int most = n_sm * ((long long)rows * a.split <= n_sm * 4ll * AP_WARPS ? 4 : AP_CTAS), spread = (most + n - 1) / n;
  const dim3 grid(mean < 1 ? 1 : mean < spread ? mean : spread, n);
  const bool norm = rope->q_gain || rope->k_gain;
  auto launch = p->dtype == VLAC_BF16 ? (p->head_dim == 128 ? launch_append<__nv_bfloat16, 128> : launch_append<__nv_bfloat16, 64>)
                                      : (p->head_dim == 128 ? launch_append<__half, 128> : launch_append<__half, 64>);
  return launch(a, rope->interleaved, norm, grid, (cudaStream_t)stream);
}

}  // extern "C"
