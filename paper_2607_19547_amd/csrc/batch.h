// Internal helpers of the batch calls (requests over a pool of pages).
#pragma once

#include "cs_common.h"

namespace cs {

constexpr int kMaxRequests = 4096;

// The pool's layout as the kernels see it: page p's plane (layer, KV head) is
// P consecutive rows of row_bytes at p * page_bytes + plane * P * row_bytes.
struct PoolView {
  char* k;
  char* v;
  int64_t page_bytes;
  int n_pages, P, row_bytes;
};

// One request's place in the step, bounded so that no contents of the arrays
// lead outside them: rows [r0, r0 + n), the first `cached` keys of `len`.
struct Request {
  int r0, n, cached, len;
};
__device__ __forceinline__ Request request_of(int start, int end, int cached_len, int n_rows, int64_t table_tokens) {
  Request q;
  q.r0 = min(max(start, 0), n_rows);
  q.n = min(max(end, q.r0), n_rows) - q.r0;
  q.cached = max(cached_len, 0);
  q.len = (int)min(min((int64_t)q.cached + q.n, table_tokens), (int64_t)0x7fffffff);
  return q;
}

// Division of 0 <= x < 2^31 by d >= 1 through a multiplication: with
// s = ceil(log2 d) and m = ceil(2^(31 + s) / d), x * m >> (31 + s) is exact
// for x < 2^31 (m < 2^32; Granlund and Montgomery, 1994).
struct FastDiv {
  uint32_t m;
  int s, d;
  __device__ __forceinline__ int div(int x) const { return (int)(((uint64_t)(uint32_t)x * m) >> (31 + s)); }
};
inline FastDiv fast_div(int d) {
  FastDiv f;
  f.d = d;
  f.s = 0;
  while ((int64_t(1) << f.s) < d) ++f.s;
  f.m = (uint32_t)(((uint64_t(1) << (31 + f.s)) + d - 1) / d);
  return f;
}

// Sum over the lanes before this one and itself (64-bit).
__device__ __forceinline__ int64_t wave_scan64(int64_t x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o);
    if ((int)(threadIdx.x & 63) >= o) x += y;
  }
  return x;
}

PoolView pool_view(const Geo& g, const cs_page_pool& p);

// ------------------------------------------------------------------ launches (per source file)
// With check_only set a launcher validates its launch sizes and enqueues nothing.
cs_status launch_batch_plan(const Geo& g, int64_t n_pages, const cs_batch& b, const cs_page_plan& p, hipStream_t s,
                            bool check_only);
cs_status launch_tree_commit(const Geo& g, const cs_page_pool& pool, int lb, int le, const cs_batch& b,
                             const int32_t* accepted, int max_accept, const int32_t* n_accepted, int32_t* cached_out,
                             hipStream_t s, bool check_only);
struct AppendJob {
  cs_rows q, k, v, q_out;
  const void *wq, *wk;
  float eps;
};
cs_status launch_append(const Geo& g, const cs_page_pool& pool, int layer, const cs_batch& b, const AppendJob& job,
                        const double* theta, hipStream_t s, bool check_only);
size_t tree_attend_workspace(const Geo& g);
cs_status launch_tree_attend(const Geo& g, const cs_page_pool& pool, int layer, const cs_batch& b, const cs_rows& q,
                             const cs_rows& out, float* lse, void* ws, hipStream_t s, bool check_only);

}  // namespace cs
