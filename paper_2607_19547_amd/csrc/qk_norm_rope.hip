// Per-head RMS norm and three-axis rotation (Eq. 2) of a step's queries and
// keys, with the keys and values put into their pages, in one pass.
//
//   y = x / sqrt(mean x^2 + eps) * weight
//   (y_i, y_{i+D/2}) -> (y_i c_i - y_{i+D/2} s_i,  y_i s_i + y_{i+D/2} c_i)
// with c, s of coords[axis(i)] * theta_i.  A row's D/2 angles serve all of its
// heads, so a workgroup takes a few whole rows: its threads make the rows'
// cos/sin tables in LDS, then groups of lanes take one head each.  Bound by
// memory: a head is read once and written once (the launch, 32,762 rows of 16 + 2 x 2
// heads of 128 in bf16: 61 us, 5.5 TB/s, with or without a norm; 5,172 rows in
// float32: 18.9 us, part of them cached; one row: 3.1 us).  Four rows a workgroup
// make one table entry per thread.
#include <algorithm>

#include "batch.h"

namespace cs {

constexpr int kAppendThreads = 256;

struct AppendArgs {
  const void *q, *k, *v;
  void* q_out;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;  // strides in elements
  const void *wq, *wk;
  const int32_t* n_used;  // row_start[B]
  const int32_t* slot;
  const int32_t* coords;
  PoolView pool;
  int64_t slots;  // n_pages x P
  FastDiv page;
  int n_rows, Hq, Hkv, D, layer, rows_per_wg;
  int sec0, sec01;
  float eps;
  double theta[256];
};

template <typename E>
__device__ __forceinline__ float to_f32(E x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<uint16_t>(uint16_t x) { return bf16_to_f32(x); }
template <typename E>
__device__ __forceinline__ E from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ uint16_t from_f32<uint16_t>(float x) { return f32_to_bf16(x); }

// cos/sin tables of the workgroup's rows [r0, r0 + rows) into LDS.
__device__ __forceinline__ void append_tables(const AppendArgs& a, int r0, int rows, float2* tab) {
  const int half = a.D >> 1;
  for (int x = threadIdx.x; x < rows * half; x += kAppendThreads) {
    const int r = x / half, i = x - r * half;
    tab[x] = cos_sin_of((double)a.coords[3 * (int64_t)(r0 + r) + axis_of(i, a.sec0, a.sec01)] * a.theta[i]);
  }
}

// Where unit (row r, head h of Hq + 2 Hkv) reads and writes; dst is null for a
// key or value row without a slot in the pool.
template <typename E>
struct AppendUnit {
  const E* src;
  E* dst;
  int kind;  // 0 query, 1 key, 2 value
};
template <typename E>
__device__ __forceinline__ AppendUnit<E> append_unit(const AppendArgs& a, int r, int h) {
  AppendUnit<E> u;
  if (h < a.Hq) {
    u.kind = 0;
    u.src = (const E*)a.q + r * a.q_row + h * a.q_head;
    u.dst = (E*)a.q_out + r * a.o_row + h * a.o_head;
    return u;
  }
  h -= a.Hq;
  u.kind = h < a.Hkv ? 1 : 2;
  if (u.kind == 2) h -= a.Hkv;
  u.src = u.kind == 1 ? (const E*)a.k + r * a.k_row + h * a.k_head : (const E*)a.v + r * a.v_row + h * a.v_head;
  const int s = a.slot[r];
  if (s < 0 || s >= a.slots) {
    u.dst = nullptr;
    return u;
  }
  const int pg = a.page.div(s), off = s - pg * a.page.d;
  u.dst = (E*)((u.kind == 1 ? a.pool.k : a.pool.v) + pg * a.pool.page_bytes +
               (((int64_t)a.layer * a.Hkv + h) * a.page.d + off) * a.pool.row_bytes);
  return u;
}

// PV rotary pairs per lane and LH = D / 2 / PV lanes per head: a lane holds
// elements [PV j, PV j + PV) of both halves of the head, 16 bytes each, so a
// pair's two elements meet in one lane.  ONCE: with the non-temporal hint, for
// steps whose rows would not stay in the 256 MB cache until they are read (32,762
// rows of 20 heads, 335 MB, the whole call: 66.5 -> 62.7 us; 4,000 rows, 41 MB, cached
// by the calls around it: 10.6 -> 12.8).
template <typename T, bool ONCE>
__device__ __forceinline__ T get(const T* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool ONCE, typename T>
__device__ __forceinline__ void put(T* p, T v) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <typename E, int PV, int LH, bool ONCE>
__global__ __launch_bounds__(kAppendThreads) void qk_norm_rope(const AppendArgs a) {
  typedef E vec __attribute__((ext_vector_type(PV)));
  extern __shared__ float2 tab[];
  constexpr int kHalf = PV * LH, kUnits = kAppendThreads / LH;
  const int r0 = blockIdx.x * a.rows_per_wg;
  const int rows = min(a.rows_per_wg, min(*a.n_used, a.n_rows) - r0);
  if (rows <= 0) return;
  const int heads = a.Hq + 2 * a.Hkv, units = rows * heads;
  const int j = threadIdx.x % LH;
  append_tables(a, r0, rows, tab);
  __syncthreads();
  for (int x = threadIdx.x / LH; x < units; x += kUnits) {
    const int r = x / heads;
    const AppendUnit<E> u = append_unit<E>(a, r0 + r, x - r * heads);
    vec lo = get<vec, ONCE>((const vec*)(u.src + PV * j)), hi = get<vec, ONCE>((const vec*)(u.src + kHalf + PV * j));
    if (u.kind < 2) {
      float f[PV], g[PV], ss = 0.f;
#pragma unroll
      for (int e = 0; e < PV; ++e) {
        f[e] = to_f32<E>(lo[e]);
        g[e] = to_f32<E>(hi[e]);
        ss = fmaf(f[e], f[e], fmaf(g[e], g[e], ss));
      }
      const E* w = (const E*)(u.kind == 0 ? a.wq : a.wk);
      if (w) {
#pragma unroll
        for (int o = 1; o < LH; o <<= 1) ss += __shfl_xor(ss, o);
        const float inv = 1.f / sqrtf(fmaf(ss, 1.f / (2 * kHalf), a.eps));
        const vec wl = *(const vec*)(w + PV * j), wh = *(const vec*)(w + kHalf + PV * j);
#pragma unroll
        for (int e = 0; e < PV; ++e) {
          f[e] = f[e] * inv * to_f32<E>(wl[e]);
          g[e] = g[e] * inv * to_f32<E>(wh[e]);
        }
      }
      const float2* t = tab + r * kHalf + PV * j;
#pragma unroll
      for (int e = 0; e < PV; ++e) {
        const float2 cs = t[e];
        lo[e] = from_f32<E>(fmaf(f[e], cs.x, -(g[e] * cs.y)));
        hi[e] = from_f32<E>(fmaf(f[e], cs.y, g[e] * cs.x));
      }
    }
    if (u.dst) {
      put<ONCE>((vec*)(u.dst + PV * j), lo);
      put<ONCE>((vec*)(u.dst + kHalf + PV * j), hi);
    }
  }
}

// Any even D up to 512, any alignment: one wavefront per head, element by element
// (32,762 rows of 20 heads of 80 in bf16: 197 us, 1.1 TB/s; one row: 8.1 us).
template <typename E>
__global__ __launch_bounds__(kAppendThreads) void qk_norm_rope_any(const AppendArgs a) {
  extern __shared__ float2 tab[];
  const int r0 = blockIdx.x * a.rows_per_wg, half = a.D >> 1;
  const int rows = min(a.rows_per_wg, min(*a.n_used, a.n_rows) - r0);
  if (rows <= 0) return;
  const int heads = a.Hq + 2 * a.Hkv, units = rows * heads, lane = threadIdx.x & 63;
  append_tables(a, r0, rows, tab);
  __syncthreads();
  for (int x = threadIdx.x >> 6; x < units; x += kAppendThreads / 64) {
    const int r = x / heads;
    const AppendUnit<E> u = append_unit<E>(a, r0 + r, x - r * heads);
    E lo[4], hi[4];
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = lane + 64 * e;
      if (i >= half) break;
      lo[e] = u.src[i];
      hi[e] = u.src[half + i];
      ss = fmaf(to_f32<E>(lo[e]), to_f32<E>(lo[e]), fmaf(to_f32<E>(hi[e]), to_f32<E>(hi[e]), ss));
    }
    if (!u.dst) continue;  // (the whole wavefront)
    const E* w = u.kind == 0 ? (const E*)a.wq : u.kind == 1 ? (const E*)a.wk : nullptr;
    float inv = 1.f;
    if (w) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) ss += __shfl_xor(ss, o);
      inv = 1.f / sqrtf(ss / (float)a.D + a.eps);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = lane + 64 * e;
      if (i >= half) break;
      if (u.kind < 2) {
        const float f = to_f32<E>(lo[e]) * (w ? inv * to_f32<E>(w[i]) : 1.f);
        const float g = to_f32<E>(hi[e]) * (w ? inv * to_f32<E>(w[half + i]) : 1.f);
        const float2 cs = tab[r * half + i];
        lo[e] = from_f32<E>(fmaf(f, cs.x, -(g * cs.y)));
        hi[e] = from_f32<E>(fmaf(f, cs.y, g * cs.x));
      }
      u.dst[i] = lo[e];
      u.dst[half + i] = hi[e];
    }
  }
}

constexpr double kOnceBytes = 128e6;
template <typename E, int LH>
static void run_vec(const AppendArgs& a, dim3 grid, size_t lds, TraceScope& tr, hipStream_t s) {
  constexpr int PV = 16 / sizeof(E);
  const double bytes = 2. * a.n_rows * (a.Hq + 2. * a.Hkv) * a.D * sizeof(E);
  if (bytes >= kOnceBytes) CS_LAUNCH(tr, (qk_norm_rope<E, PV, LH, true>), grid, dim3(kAppendThreads), lds, s, a);
  else CS_LAUNCH(tr, (qk_norm_rope<E, PV, LH, false>), grid, dim3(kAppendThreads), lds, s, a);
}
template <typename E>
static void run_append(const AppendArgs& a, bool vec_ok, unsigned blocks, hipStream_t s) {
  const size_t lds = (size_t)a.rows_per_wg * (a.D / 2) * sizeof(float2);
  TraceScope tr(vec_ok ? "qk_norm_rope" : "qk_norm_rope_any", s);
  switch (vec_ok ? a.D / 2 * (int)sizeof(E) / 16 : 0) {
    case 1: return run_vec<E, 1>(a, dim3(blocks), lds, tr, s);
    case 2: return run_vec<E, 2>(a, dim3(blocks), lds, tr, s);
    case 4: return run_vec<E, 4>(a, dim3(blocks), lds, tr, s);
    case 8: return run_vec<E, 8>(a, dim3(blocks), lds, tr, s);
    case 16: return run_vec<E, 16>(a, dim3(blocks), lds, tr, s);
    case 32: return run_vec<E, 32>(a, dim3(blocks), lds, tr, s);
    case 64: return run_vec<E, 64>(a, dim3(blocks), lds, tr, s);
    default: CS_LAUNCH(tr, (qk_norm_rope_any<E>), dim3(blocks), dim3(kAppendThreads), lds, s, a);
  }
}

cs_status launch_append(const Geo& g, const cs_page_pool& pool, int layer, const cs_batch& b, const AppendJob& job,
                        const double* theta, hipStream_t s, bool check_only) {
  AppendArgs a;
  a.rows_per_wg = 4;
  const int64_t blocks = ((int64_t)b.n_rows + a.rows_per_wg - 1) / a.rows_per_wg;
  const cs_status st = check_grid(blocks, 1, 1, kAppendThreads, "norm and rotation");
  if (st || check_only) return st;
  a.q = job.q.data;
  a.k = job.k.data;
  a.v = job.v.data;
  a.q_out = job.q_out.data;
  a.q_row = job.q.row_stride;
  a.q_head = job.q.head_stride;
  a.k_row = job.k.row_stride;
  a.k_head = job.k.head_stride;
  a.v_row = job.v.row_stride;
  a.v_head = job.v.head_stride;
  a.o_row = job.q_out.row_stride;
  a.o_head = job.q_out.head_stride;
  a.wq = job.wq;
  a.wk = job.wk;
  a.n_used = b.row_start + b.n_requests;
  a.slot = b.slot;
  a.coords = b.coords;
  a.pool = pool_view(g, pool);
  a.slots = pool.n_pages * g.T;
  a.page = fast_div((int)g.T);
  a.n_rows = b.n_rows;
  a.Hq = g.Hq;
  a.Hkv = g.Hkv;
  a.D = g.D;
  a.layer = layer;
  a.sec0 = g.sec[0];
  a.sec01 = g.sec[0] + g.sec[1];
  a.eps = job.eps;
  for (int i = 0; i < g.P; ++i) a.theta[i] = theta[i];
  // 16-byte accesses: a power of two of them to each half of a head, every
  // head at a multiple of 16 bytes
  const int pv = 16 / g.esize, lanes = g.P / pv;
  uint64_t low = (uint64_t)a.q | (uint64_t)a.k | (uint64_t)a.v | (uint64_t)a.q_out | (uint64_t)a.wq | (uint64_t)a.wk;
  low |= (uint64_t)((a.q_row | a.q_head | a.k_row | a.k_head | a.v_row | a.v_head | a.o_row | a.o_head) * g.esize);
  const bool vec_ok = g.P % pv == 0 && (lanes & (lanes - 1)) == 0 && low % 16 == 0;
  if (g.dtype == CS_BF16) run_append<uint16_t>(a, vec_ok, (unsigned)blocks, s);
  else run_append<float>(a, vec_ok, (unsigned)blocks, s);
  return check_launch("norm and rotation launch");
}

}  // namespace cs
