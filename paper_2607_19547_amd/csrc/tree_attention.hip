// Attention of a batch's rows over their requests' pages (Eq. 1): a single
// token, a tree of drafted tokens or a question's tokens per request.
#include <math.h>

#include <algorithm>

#include "batch.h"

namespace cs {

struct TreeArgs {
  const void* q;
  void* out;
  float* lse;
  int64_t q_row, q_head, o_row, o_head;  // strides in elements
  const int32_t* cached;
  const int32_t* row_start;
  const int32_t* table;
  const unsigned long long* mask;
  PoolView pool;
  FastDiv page;
  int B, n_rows, max_blocks, words, layer, Hq, Hkv, G, D;
  float scale;  // 1 / sqrt(D)
};

__device__ __forceinline__ Request load_request(const TreeArgs& a, int b) {
  return request_of(a.row_start[b], a.row_start[b + 1], a.cached[b], a.n_rows, (int64_t)a.max_blocks * a.page.d);
}

// Whether row i of a request sees its new row w (w >= 0).
__device__ __forceinline__ bool sees(const TreeArgs& a, const Request& q, int i, int w) {
  if (!a.mask) return w <= i;
  if (w >> 6 >= a.words) return false;
  return (a.mask[(int64_t)(q.r0 + i) * a.words + (w >> 6)] >> (w & 63)) & 1;
}

// ============================================================== any geometry
// One workgroup per (row, query head), keys in blocks of 256: a thread scores
// one key, then the threads take the head's elements and add up the block's
// visible values.  Slow (every head reads its keys for itself), right for any
// even head_dim up to 512, page size and stride.
constexpr int kAnyThreads = 256;

template <typename E>
__device__ __forceinline__ float elem(const E* p);
template <>
__device__ __forceinline__ float elem<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float elem<uint16_t>(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void put_elem(float* p, float x) { *p = x; }
__device__ __forceinline__ void put_elem(uint16_t* p, float x) { *p = f32_to_bf16(x); }

template <typename E>
__global__ __launch_bounds__(kAnyThreads) void tree_attend_any(const TreeArgs a) {
  __shared__ float s_q[512], s_p[kAnyThreads], s_red[kAnyThreads / 64];
  __shared__ int64_t s_at[kAnyThreads];  // byte offset of the key's row, -1 where the row does not see it
  const int r = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, P = a.page.d;
  if (r >= a.row_start[a.B]) return;
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.row_start[mid] <= r) lo = mid;
    else hi = mid;
  }
  const Request q = load_request(a, lo);
  const int i = r - q.r0;
  if (i < 0 || i >= q.n) return;  // (arrays that are no plan's)
  const int32_t* table = a.table + (int64_t)lo * a.max_blocks;
  const int64_t plane = ((int64_t)a.layer * a.Hkv + h / a.G) * P * a.pool.row_bytes;
  const E* qp = (const E*)a.q + r * a.q_row + h * a.q_head;
  for (int d = tid; d < a.D; d += kAnyThreads) s_q[d] = elem(qp + d);
  float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
  bool any = false;
  for (int k0 = 0; k0 < q.len; k0 += kAnyThreads) {
    __syncthreads();
    const int key = k0 + tid;
    int64_t at = -1;
    float s = -INFINITY;
    if (key < q.len && (key < q.cached || sees(a, q, i, key - q.cached))) {
      const int blk = a.page.div(key), pg = table[blk];
      if (pg >= 0 && pg < a.pool.n_pages) {
        at = pg * a.pool.page_bytes + plane + (int64_t)(key - blk * P) * a.pool.row_bytes;
        const E* kp = (const E*)(a.pool.k + at);
        s = 0.f;
        for (int d = 0; d < a.D; ++d) s = fmaf(s_q[d], elem(kp + d), s);
        s *= a.scale;
      }
    }
    float mx = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    if ((tid & 63) == 0) s_red[tid >> 6] = mx;
    __syncthreads();
    for (int w = 0; w < kAnyThreads / 64; ++w) mx = fmaxf(mx, s_red[w]);
    const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = expf(m - ref);  // (0 where nothing was seen yet)
    s_p[tid] = at >= 0 ? expf(s - ref) : 0.f;
    s_at[tid] = at;
    __syncthreads();
    l *= alpha;
    acc[0] *= alpha;
    acc[1] *= alpha;
    const int cnt = min(kAnyThreads, q.len - k0);
    for (int x = 0; x < cnt; ++x) {
      if (s_at[x] < 0) continue;  // an unseen value is not read
      const float p = s_p[x];
      const E* vp = (const E*)(a.pool.v + s_at[x]);
      any = true;
      l += p;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (tid + kAnyThreads * e < a.D) acc[e] = fmaf(p, elem(vp + tid + kAnyThreads * e), acc[e]);
    }
    m = m_new;
  }
  E* op = (E*)a.out + r * a.o_row + h * a.o_head;
  const float inv = any ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (tid + kAnyThreads * e < a.D) put_elem(op + tid + kAnyThreads * e, any ? acc[e] * inv : 0.f);
  if (a.lse && tid == 0) a.lse[(int64_t)r * a.Hq + h] = any ? m + logf(l) : -INFINITY;
}

size_t tree_attend_workspace(const Geo&, const cs_batch&) { return 0; }

cs_status launch_tree_attend(const Geo& g, const cs_page_pool& pool, int layer, const cs_batch& b, const cs_rows& q,
                             const cs_rows& out, float* lse, void*, hipStream_t s, bool check_only) {
  const cs_status st = check_grid(b.n_rows, g.Hq, 1, kAnyThreads, "tree attention");
  if (st || check_only) return st;
  TreeArgs a;
  a.q = q.data;
  a.out = out.data;
  a.lse = lse;
  a.q_row = q.row_stride;
  a.q_head = q.head_stride;
  a.o_row = out.row_stride;
  a.o_head = out.head_stride;
  a.cached = b.cached_len;
  a.row_start = b.row_start;
  a.table = b.block_table;
  a.mask = (const unsigned long long*)b.tree_mask;
  a.pool = pool_view(g, pool);
  a.page = fast_div((int)g.T);
  a.B = b.n_requests;
  a.n_rows = b.n_rows;
  a.max_blocks = b.max_blocks;
  a.words = b.mask_words;
  a.layer = layer;
  a.Hq = g.Hq;
  a.Hkv = g.Hkv;
  a.G = g.G;
  a.D = g.D;
  a.scale = 1.f / sqrtf((float)g.D);
  TraceScope tr("tree_attend_any", s);
  const dim3 grid(b.n_rows, g.Hq);
  if (g.dtype == CS_BF16) CS_LAUNCH(tr, tree_attend_any<uint16_t>, grid, dim3(kAnyThreads), 0, s, a);
  else CS_LAUNCH(tr, tree_attend_any<float>, grid, dim3(kAnyThreads), 0, s, a);
  return check_launch("tree attention launch");
}

}  // namespace cs
