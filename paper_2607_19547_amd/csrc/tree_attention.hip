// Attention of a batch's rows over their requests' pages (Eq. 1): a single
// token, a tree of drafted tokens or a question's tokens per request.
#include <math.h>

#include <algorithm>

#include "tree_attention_few.h"

namespace cs {

// ============================================================== any geometry
// One workgroup per (row, query head), keys in blocks of 256: a thread scores
// one key, then the threads take the head's elements and add up the block's
// visible values.  Slow (every head reads its keys for itself, and a thread its
// whole key: 16 / 2 heads of 80 in bf16, one row over 8,211 tokens 2.6 ms, over
// 1,025 0.18 ms), right for any even head_dim up to 512, page size and stride.
constexpr int kAnyThreads = 256;

template <typename E>
__device__ __forceinline__ float elem(const E* p);
template <>
__device__ __forceinline__ float elem<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float elem<uint16_t>(const uint16_t* p) { return bf16_to_f32(*p); }

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
  if (a.lse && tid == 0) a.lse[(int64_t)r * a.Hq + h] = !any ? -INFINITY : l == 0.f ? __builtin_nanf("") : m + logf(l);  // (0: only scores of -inf)
}

// ============================================================== launch
constexpr int kRunBits = 9, kRuns = 1 << kRunBits;  // workgroups of the attention launch: two for each CU

// Whether the matrix-instruction path has an instance: bf16 rows of 64 to 256
// bytes, or 512; float32 rows of 64, 128, 256 or 512 bytes.
static bool has_instance(const Geo& g) {
  if (g.T % 16) return false;
  if (g.dtype == CS_BF16) return g.D == 32 || g.D == 64 || g.D == 96 || g.D == 128 || g.D == 256;
  return g.D == 16 || g.D == 32 || g.D == 64 || g.D == 128;
}
static bool wide_type(const Geo& g) { return g.dtype == CS_BF16 && g.D == 128; }
// Row tiles of 16, 32 or 64 query vectors.  A larger one reads the keys fewer times, in
// fewer and longer pieces of work; with rows of more than 128 bytes 64 do not fit the
// registers (float32 x 128 with 32 spills 12 of them, bf16 x 256 with 16 spills 56).
// bf16 x 128 has 32 for outputs alone that are not aligned to 16 bytes: the kernel for
// many rows takes the rest.  Row tiles of 16 win where they read little in all:
// measured (us with 16 / 32, 8 query heads a KV head, 6 and 17 rows, 4,000 to 32,000
// tokens), the two meet near 200 MB for float32 x 128 (147 MB: 23 / 28, 295 MB: 47 /
// 38), 130 MB for float32 x 64 (74: 16 / 20, 295: 46 / 34) and 90 MB for bf16 x 64 (37:
// 12 / 14, 147: 24 / 21).  The host knows only the block tables' room, which is seldom
// filled: the border is put at 1.6 times that.
static int64_t query_vectors(const Geo& g, const cs_batch& b) { return (int64_t)(b.max_rows > 0 ? b.max_rows : b.n_rows) * g.G; }
static double room_bytes(const Geo& g, const cs_batch& b) {  // of the keys and values the block tables have room for
  return (double)b.n_requests * b.max_blocks * g.T * g.Hkv * g.D * g.esize * 2;
}
static int most_row_groups(const Geo& g) { return g.D > 128 ? 1 : g.D * g.esize > 128 ? 2 : 4; }
static int row_groups(const Geo& g, const cs_batch& b) {
  const int64_t qv = query_vectors(g, b);
  if (qv <= 16) return 1;
  const double row_bytes = g.D * g.esize;
  if (room_bytes(g, b) * ((qv + 15) / 16) < 1.6 * (50e6 + 0.3e6 * row_bytes)) return 1;
  return std::min(most_row_groups(g), qv <= 256 ? 2 : 4);
}

// Whether the kernel for many rows takes the batch (where its pointers are
// aligned): it reads the keys and values once for 256 query vectors and has more to
// do before its first tile.  Measured (us, row tiles of 16 query vectors / that
// kernel), by what the row tiles of 16 read in all: 35 MB (4,000 tokens, 3 rows, 8
// query heads for each of 8 KV heads) 16 / 23; 69 MB (4,000 tokens, 32 rows, 8 for
// each of 2) 20 / 27; 119 MB (8 requests of 1,000 tokens, 5 rows, 8 for each of 8)
// 27 / 23; 134 MB (65,000 tokens, 3 rows, 8 for each of 2) 30 / 29; 277 MB (8
// requests of 4,000 tokens, 4 rows, 8 for each of 8) 50 / 37; 1.1 GB (32 of them) 160
// / 103.  (The room is seldom filled.)
static bool wide(const Geo& g, const cs_batch& b) {
  const int64_t row_tiles = (query_vectors(g, b) + 15) / 16;
  return wide_type(g) && row_tiles > 1 && room_bytes(g, b) * row_tiles >= 150e6;
}

// The most that any instance of the geometry uses: which one a call takes depends
// on the batch's sizes and hints, the workspace does not.
size_t tree_attend_workspace(const Geo& g) {
  if (!has_instance(g)) return 0;
  const size_t rows = 16 * (size_t)most_row_groups(g);
  const size_t few = 2 * (size_t)kRuns * rows * (g.D + 2) * sizeof(float) + 512;
  return wide_type(g) ? std::max(few, tree_wide_workspace()) : few;
}

template <typename E, int D, int NR, bool ONCE = false>
static void run_split(const SplitArgs& a, hipStream_t s) {
  const int runs = most_runs(a);
  {
    TraceScope tr("tree_attend", s);
    CS_LAUNCH(tr, (tree_attend<E, D, NR, ONCE>), dim3(NR > 1 ? (runs + 7) / 8 * 8 : runs), dim3(kThreads), 0, s, a);
  }
  if (runs == 1) return;
  TraceScope tr("tree_combine", s);
  CS_LAUNCH(tr, (tree_combine<E, D, (NR > 1)>), dim3(runs - 1, 2 * NR), dim3(kThreads), 0, s, a);
}
template <typename E, int D>
static void run_split(const SplitArgs& a, int nr, bool once, hipStream_t s) {
  if constexpr (D * sizeof(E) <= 128)
    if (nr == 4) return run_split<E, D, 4>(a, s);
  if constexpr (D <= 128)
    if (nr == 2) return run_split<E, D, 2>(a, s);
  if (once) return run_split<E, D, 1, true>(a, s);
  run_split<E, D, 1>(a, s);
}

cs_status launch_tree_attend(const Geo& g, const cs_page_pool& pool, int layer, const cs_batch& b, const cs_rows& q,
                             const cs_rows& out, float* lse, void* ws, hipStream_t s, bool check_only) {
  SplitArgs a;
  TreeArgs& t = a.t;
  t = tree_args(g, pool, layer, b, q, out, lse);
  // 16-byte accesses of queries, 4-byte ones of outputs
  const uint64_t low = (uint64_t)t.q | (uint64_t)((t.q_row | t.q_head) * g.esize);
  const uint64_t low_o = (uint64_t)t.out | (uint64_t)((t.o_row | t.o_head) * g.esize);
  if (!has_instance(g) || low % 16 || low_o % 4) {
    const cs_status st = check_grid(b.n_rows, g.Hq, 1, kAnyThreads, "tree attention");
    if (st || check_only) return st;
    TraceScope tr("tree_attend_any", s);
    const dim3 grid(b.n_rows, g.Hq);
    if (g.dtype == CS_BF16) CS_LAUNCH(tr, tree_attend_any<uint16_t>, grid, dim3(kAnyThreads), 0, s, t);
    else CS_LAUNCH(tr, tree_attend_any<float>, grid, dim3(kAnyThreads), 0, s, t);
    return check_launch("tree attention launch");
  }
  if (check_only) return CS_OK;
  a.group = fast_div(g.G);
  if (wide(g, b) && low_o % 16 == 0) {
    launch_tree_wide(a, ws, query_vectors(g, b) <= 256 && room_bytes(g, b) >= kWideOnceBytes, s);
    return check_launch("tree attention launch");
  }
  const int nr = row_groups(g, b);
  const bool once = query_vectors(g, b) <= 16 && room_bytes(g, b) >= kOnceBytes;
  a.row_bits = nr == 1 ? 4 : nr == 2 ? 5 : 6;
  a.tile_bits = g.dtype == CS_BF16 ? 5 : 4;
  a.min_tiles = 2 * kWaves;
  a.run_bits = kRunBits;
  a.units = fast_div(even_units(a));
  a.by_xcd = nr > 1 && room_bytes(g, b) >= 16e6;  // (half of what the L2 caches hold together)
  a.part = (float*)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  a.part_ml = a.part + 2 * ((size_t)kRuns << a.row_bits) * g.D;
  if (g.dtype == CS_BF16) {
    switch (g.D) {
      case 32: run_split<uint16_t, 32>(a, nr, once, s); break;
      case 64: run_split<uint16_t, 64>(a, nr, once, s); break;
      case 96: run_split<uint16_t, 96>(a, nr, once, s); break;
      case 128: run_split<uint16_t, 128>(a, nr, once, s); break;
      default: run_split<uint16_t, 256>(a, nr, once, s);
    }
  } else {
    switch (g.D) {
      case 16: run_split<float, 16>(a, nr, once, s); break;
      case 32: run_split<float, 32>(a, nr, once, s); break;
      case 64: run_split<float, 64>(a, nr, once, s); break;
      default: run_split<float, 128>(a, nr, once, s);
    }
  }
  return check_launch("tree attention launch");
}

}  // namespace cs
