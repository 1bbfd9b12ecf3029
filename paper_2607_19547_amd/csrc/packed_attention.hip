// Attention of a batch's rows over memories whose first pages are packed, or of
// which rows see a span (the first `sinks` tokens and the last `window`).
//
// The kernel is tree_attend's (tree_attention_few.h) with a loop of its own over
// the packed tiles before the one over ordinary pages.  A window makes a row
// tile's work shorter, not its tiles emptier: what lies between the sinks and the
// first row's window is left out of its count, so runs stay even.
//
// Few rows are bound by memory: 64 requests of up to 32,768 packed tokens, one row, 16 / 2
// heads of 128 (234 MB) 51 us and 6 for the merge, 4.6 TB/s.  One row over 8,192 tokens takes
// 7.1 us and 4.2 (two launches' chains of loads).  What many rows are bound by is told
// in tree_attention_wide.hip.
#include <math.h>

#include <algorithm>

#include "packed_attention.h"
#include "tree_attention_few.h"

namespace cs {

// ============================================================== any geometry
// As tree_attend_any: one workgroup per (row, query head), keys in blocks of 256.
// A packed key's scores and values are decoded one by one.  Slow, right for any
// even head_dim up to 512, page size and stride.
constexpr int kAnyThreads = 256;

template <typename E>
__device__ __forceinline__ float elem(const E* p);
template <>
__device__ __forceinline__ float elem<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float elem<uint16_t>(const uint16_t* p) { return bf16_to_f32(*p); }

template <typename E>
__global__ __launch_bounds__(kAnyThreads) void packed_attend_any(const MemoryArgs a) {
  __shared__ float s_q[512], s_p[kAnyThreads], s_red[kAnyThreads / 64];
  __shared__ int64_t s_at[kAnyThreads];  // where the key lies (packed: its plane), -1 where the row does not see it
  __shared__ int s_row[kAnyThreads];     // a packed key's row in its page, -1: an ordinary page
  const TreeArgs& t = a.t;
  const int r = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, P = t.page.d, D = t.D;
  if (r >= t.row_start[t.B]) return;
  int lo = 0, hi = t.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.row_start[mid] <= r) lo = mid;
    else hi = mid;
  }
  const Request q = load_request(t, lo);
  const int i = r - q.r0;
  if (i < 0 || i >= q.n) return;  // (arrays that are no plan's)
  const int32_t* table = t.table + (int64_t)lo * t.max_blocks;
  const int64_t lh = (int64_t)t.layer * t.Hkv + h / t.G, plane = lh * P * t.pool.row_bytes;
  const int packed = a.blocks ? min(max(a.blocks[lo], 0), t.page.div(q.cached)) : 0;
  const Hidden gone = hidden_keys(a, q, i);
  const E* qp = (const E*)t.q + r * t.q_row + h * t.q_head;
  for (int d = tid; d < D; d += kAnyThreads) s_q[d] = elem(qp + d);
  float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
  bool any = false;
  for (int k0 = 0; k0 < q.len; k0 += kAnyThreads) {
    if (k0 >= gone.lo && gone.hi - k0 >= kAnyThreads) continue;  // (the whole workgroup)
    __syncthreads();
    const int key = k0 + tid;
    int64_t at = -1;
    int row = -1;
    float s = -INFINITY;
    if (key < q.len && (key < q.cached || sees(t, q, i, key - q.cached)) && !(key >= gone.lo && key < gone.hi)) {
      const int blk = t.page.div(key), pg = table[blk], off = key - blk * P;
      if (blk < packed) {
        if (pg >= 0 && pg < a.packed.n_pages) {
          at = pg * a.packed.page_bytes + lh * a.packed.plane_bytes();
          row = off;
          const unsigned char* p = (const unsigned char*)a.packed.base + at;
          const unsigned char* sc = p + a.packed.k_scales() + (off >> 5) * D + (off & 31);
          s = 0.f;
          for (int d = 0; d < D; ++d)
            s = fmaf(s_q[d], decode1(p[((int64_t)off * D + d) >> 1] >> (4 * (d & 1)), sc[(d >> 5) * kBlock]), s);
          s *= t.scale;
        }
      } else if (pg >= 0 && pg < t.pool.n_pages) {
        at = pg * t.pool.page_bytes + plane + (int64_t)off * t.pool.row_bytes;
        const E* kp = (const E*)(t.pool.k + at);
        s = 0.f;
        for (int d = 0; d < D; ++d) s = fmaf(s_q[d], elem(kp + d), s);
        s *= t.scale;
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
    s_row[tid] = row;
    __syncthreads();
    l *= alpha;
    acc[0] *= alpha;
    acc[1] *= alpha;
    const int cnt = min(kAnyThreads, q.len - k0);
    for (int x = 0; x < cnt; ++x) {
      if (s_at[x] < 0) continue;  // an unseen value is not read
      const float p = s_p[x];
      const int off = s_row[x];
      any = true;
      l += p;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int d = tid + kAnyThreads * e;
        if (d >= D) break;
        if (off < 0) {
          acc[e] = fmaf(p, elem((const E*)(t.pool.v + s_at[x]) + d), acc[e]);
        } else {
          const unsigned char* vp = (const unsigned char*)a.packed.base + s_at[x];
          const uint32_t code = vp[a.packed.v_codes() + ((int64_t)(off >> 3) * D + d) * 4 + ((off & 7) >> 1)] >> (4 * (off & 1));
          acc[e] = fmaf(p, decode1(code, vp[a.packed.v_scales() + (off >> 5) * D + d]), acc[e]);
        }
      }
    }
    m = m_new;
  }
  E* op = (E*)t.out + r * t.o_row + h * t.o_head;
  const float inv = any ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (tid + kAnyThreads * e < D) put_elem(op + tid + kAnyThreads * e, any ? acc[e] * inv : 0.f);
  if (t.lse && tid == 0) t.lse[(int64_t)r * t.Hq + h] = !any ? -INFINITY : l == 0.f ? __builtin_nanf("") : m + logf(l);  // (0: only scores of -inf)
}

// ============================================================== launch
constexpr int kRunBits = 9, kRuns = 1 << kRunBits;  // workgroups of the attention launch: two for each CU

static bool has_instance(const Geo& g) {
  if (g.T % 16) return false;
  if (g.dtype == CS_BF16) return g.D == 32 || g.D == 64 || g.D == 96 || g.D == 128 || g.D == 256;
  return g.D == 16 || g.D == 32 || g.D == 64 || g.D == 128;
}

// Which kernel and row tile takes a batch, by the key tiles (of 32, over all requests
// and KV heads) that a row tile of each may see, the row tiles of 16 query vectors that
// each of them meets, and the units (row tiles of all requests and KV heads), whose
// starts and ends count where they are short.  The host does not know the lengths, and
// tables are seldom filled: keys are taken to fill 1 / 1.6 of their room.  What a window
// leaves is known, and taken as it is.
constexpr double kRoom = 1.6;
struct Work {
  double tiles, row_tiles, row_tiles_wide;  // (of 256)
  double units, units_wide;
  bool window;                              // that bounds the tiles
};
static Work work_of(const Geo& g, const cs_batch& b, int sinks, int window) {
  const double rows = b.max_rows > 0 ? b.max_rows : b.n_rows, vectors = rows * g.G;
  const double row_tiles = ceil(vectors / 16), heads = (double)b.n_requests * g.Hkv;
  const double keys = (double)b.max_blocks * g.T / kRoom;
  const double seen = window ? (double)sinks + window + std::min(rows, 32.) : keys;  // (with a row tile's rows, about)
  return {heads * std::min(keys, seen) / 32, row_tiles, ceil(vectors / 256), heads * row_tiles, heads * ceil(vectors / 256),
          seen < keys};
}
// Row tiles of 32 or 64 convert a packed tile half or a quarter as often, in fewer and
// longer pieces of work.  Measured, tiles x row tiles of 16 and us with row tiles of 16 /
// 32 / 64: bf16 x 64 33,000 23.7 / 27.1 / 32.8, 67,000 39.8 / 37.6 / 43.3, 131,000 59.7 /
// 51.4 / 52.4, 809,000 337 / 219 / 191; x 32 33,000 21.3 / 25.3 / 27.3, 131,000 50.0 / 46.0 / 43.7;
// x 96 9,000 21.8 / 22.4, 19,000 33.0 / 30.3, 131,000 121 / 77; float32 x 64 67,000 51.6 / 51.5,
// 131,000 78.7 / 76.2; x 32 66,000 43.9 / 41.2 / 47.9, 131,000 66.3 / 60.6 / 63.8.  Row tiles of 32
// spill registers with bf16 x 128 (which has the kernel for many rows), x 256 and float32 x 128.
// With windows the start and end of a unit, beyond the two that a request and KV head have in any
// case, weigh as 25 tiles.  Bf16 x 64, x 96, float32 x 64: 1,000 rows that see 1,024 keys each 44.4 /
// 38.5, 52.7 / 45.9, 72.3 / 66.4; 250 rows that see 4,096 27.8 / 27.8, 43.7 / 35.9, 33.8 / 35.8; 512 requests of
// 8 rows that see 128 89 / 87, 106 / 97, 100 / 101, of 3 rows 61 / 67, 70 / 72, 66 / 73.  32 query vectors
// fill half of a row tile of 64: 64 requests of 65,536 tokens, 3 rows, x 64 164 / 226, x 32 171 / 225 (32 / 64).
static int most_row_groups(const Geo& g) {
  if (g.dtype == CS_F32) return g.D <= 64 ? 2 : 1;
  return g.D <= 64 ? 4 : g.D <= 96 ? 2 : 1;
}
static int row_groups(const Geo& g, const Work& w) {
  const double n = w.tiles * w.row_tiles, ends = w.window ? 25 * w.units * (1 - 2 / w.row_tiles) : 0;
  if (w.row_tiles <= 1 || n + ends < (g.D == 96 ? 12e3 : 55e3)) return 1;
  return std::min(most_row_groups(g), n < 200e3 || w.row_tiles <= 2 ? 2 : 4);
}
// Two packed tiles a step, with row tiles of 16, in place of one: more in flight where
// much is read.  Measured (us, tiles x row tiles of memories that the cache does not hold, one / two):
// bf16 x 128 16,400 24.8 / 25.2, 33,000 38.8 / 39.3, 66,000 60.6 / 56.8, 131,000 105 / 96; x 64 33,000
// 25.7 / 24.5, 66,000 46.4 / 40.5, 131,000 80.5 / 67.6; float32 x 64 33,000 28.8 / 28.8, 66,000 49.5 / 45.6;
// windows of 8,192 keys, 64 requests, 33,000 (bf16 x 128, x 64, float32 x 64) 43.7 / 43.4, 30.6 / 30.2, 33.1 /
// 34.2; x 32 no change; bf16 x 96 66,000 67.4 / 75.3, 131,000 121 / 134: there always one.
constexpr double kDeepTiles = 30e3;
constexpr bool has_deep(bool bf16, int d) { return d == 64 || (bf16 && d == 128); }
// The kernel for many rows (bf16 x 128) starts and ends 11 us later than row tiles of 16.  A
// key tile of 32 takes it 2.7 ns for 256 query vectors, on the whole GPU, and a unit 50 ns; row
// tiles of 16 take 0.55 ns a tile, of ordinary pages 1.2 (whether there are other than ordinary ones
// is known, how many is not), and 15 ns a unit: fitted to 238 batches of 1 to 48 requests and 2 to
// 2,000 rows, of which the rule takes the faster side, or one within 5% of it, in all but 6, the worst
// 16% off; of 41 others, of 64 to 4,096 requests, in all but 4 (11%).
// Measured (us, row tiles of 16 / many rows; 16 / 2 heads): 65,536 tokens, 17 rows 36.4 / 42.8, 64 rows 77 /
// 58; 16,384, 64 rows 32.0 / 32.5; 8,192, 250 rows 49.8 / 40.5; 1,024, 250 rows 22.5 / 25.3; 8 requests of
// 4,096, 64 rows 45 / 43; 32 of 8,192, 4 rows 35 / 66; 39 of 768, 27 rows 43.6 / 32.0.  Rows that see
// 1,024 keys each, ordinary and packed: 250 rows 28.9 / 28.7 and 25.2 / 30.5, 500 39.7 / 29.5 and 34.2 / 31.2, 1,950
// 106 / 47.5 and 110 / 51.8; 256 keys: 250 rows 18.8 / 28.8 and 19.9 / 30.5, 1,000 36.7 / 30.5 and 39.1 / 31.9; 4,096
// keys: 64 rows 27.9 / 26.3 and 20.6 / 28.1, 1,000 169 / 59 and 106 / 63; 48 requests of 16 rows 246 / 71 and 84 / 65.
static bool wide(const Geo& g, const Work& w, bool all_paged) {
  const double few = (all_paged ? 1.2 : 0.55) * w.tiles * w.row_tiles + 15 * w.units;  // ns
  const double many = 2.7 * w.tiles * w.row_tiles_wide + 50 * w.units_wide;
  return g.dtype == CS_BF16 && g.D == 128 && few - many > 11e3;
}

size_t packed_attend_workspace(const Geo& g) {
  const size_t rows = 16 * (size_t)most_row_groups(g);
  const size_t few = has_instance(g) ? 2 * (size_t)kRuns * rows * (g.D + 2) * sizeof(float) + 512 : 0;
  return std::max(few, tree_attend_workspace(g));  // (a call without packed pages and window is that one)
}

template <typename E, int D, int NR, int PT = 1>
static void run_split(const MemoryArgs& a, hipStream_t s) {
  const int runs = most_runs(a);
  {
    TraceScope tr("packed_attend", s);
    CS_LAUNCH(tr, (tree_attend<E, D, NR, false, MemoryArgs, PT>), dim3(NR > 1 ? (runs + 7) / 8 * 8 : runs), dim3(kThreads), 0, s, a);
  }
  if (runs == 1) return;
  TraceScope tr("packed_combine", s);
  CS_LAUNCH(tr, (tree_combine<E, D, (NR > 1), MemoryArgs>), dim3(runs - 1, 2 * NR), dim3(kThreads), 0, s, a);
}
template <typename E, int D>
static void run_split(const MemoryArgs& a, int nr, bool deep, hipStream_t s) {
  constexpr bool kBf16 = sizeof(E) == 2;
  if constexpr (kBf16 && D <= 64)
    if (nr == 4) return run_split<E, D, 4>(a, s);
  if constexpr (D <= (kBf16 ? 96 : 64))
    if (nr == 2) return run_split<E, D, 2>(a, s);
  if constexpr (has_deep(kBf16, D))
    if (deep) return run_split<E, D, 1, 2>(a, s);
  run_split<E, D, 1>(a, s);
}

cs_status launch_packed_attend(const Geo& g, const cs_page_pool& pool, const cs_packed_pool* packed, int layer,
                               const cs_batch& b, const SpanJob& job, const cs_rows& q, const cs_rows& out, float* lse,
                               void* ws, hipStream_t s, bool check_only) {
  MemoryArgs a;
  TreeArgs& t = a.t;
  t = tree_args(g, pool, layer, b, q, out, lse);
  a.packed = packed ? packed_view(g, *packed) : PackedView{};
  a.blocks = job.blocks;
  a.sinks = job.sinks;
  a.window = job.window;
  a.group = fast_div(g.G);
  // 16-byte accesses of queries, 4-byte ones of outputs
  const uint64_t low = (uint64_t)t.q | (uint64_t)((t.q_row | t.q_head) * g.esize);
  const uint64_t low_o = (uint64_t)t.out | (uint64_t)((t.o_row | t.o_head) * g.esize);
  if (!has_instance(g) || low % 16 || low_o % 4) {
    const cs_status st = check_grid(b.n_rows, g.Hq, 1, kAnyThreads, "packed attention");
    if (st || check_only) return st;
    TraceScope tr("packed_attend_any", s);
    const dim3 grid(b.n_rows, g.Hq);
    if (g.dtype == CS_BF16) CS_LAUNCH(tr, packed_attend_any<uint16_t>, grid, dim3(kAnyThreads), 0, s, a);
    else CS_LAUNCH(tr, packed_attend_any<float>, grid, dim3(kAnyThreads), 0, s, a);
    return check_launch("packed attention launch");
  }
  if (check_only) return CS_OK;
  // (without: a tree of 61 rows over 65,408 tokens 61 -> 68 us, 8 trees of 64 over 4,096 45 -> 51)
  a.paged_bits = 0;
  a.unit_tiles = 5;
  const Work w = work_of(g, b, job.sinks, job.window);
  if (wide(g, w, !job.blocks) && low_o % 16 == 0) {
    launch_packed_wide(a, ws, s);
    return check_launch("packed attention launch");
  }
  const int nr = row_groups(g, w);
  const bool deep = w.tiles * w.row_tiles >= kDeepTiles;
  a.row_bits = nr == 1 ? 4 : nr == 2 ? 5 : 6;
  a.tile_bits = kFewTileBits;
  // (tiles of ordinary pages by their bytes; with 1 and 0: 64 requests 49.5 -> 56 us, one row
  // over 1,024 tokens 10.3 -> 13.9, over 8,192 11.9 -> 14.6)
  a.paged_bits = 2;
  a.unit_tiles = 8;
  a.min_tiles = 2 * kWaves;
  a.run_bits = kRunBits;
  a.units = fast_div(even_units(a));
  a.by_xcd = nr > 1;
  a.part = (float*)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  a.part_ml = a.part + 2 * ((size_t)kRuns << a.row_bits) * g.D;
  if (g.dtype == CS_BF16) {
    switch (g.D) {
      case 32: run_split<uint16_t, 32>(a, nr, deep, s); break;
      case 64: run_split<uint16_t, 64>(a, nr, deep, s); break;
      case 96: run_split<uint16_t, 96>(a, nr, deep, s); break;
      case 128: run_split<uint16_t, 128>(a, nr, deep, s); break;
      default: run_split<uint16_t, 256>(a, nr, deep, s);
    }
  } else {
    switch (g.D) {
      case 16: run_split<float, 16>(a, nr, deep, s); break;
      case 32: run_split<float, 32>(a, nr, deep, s); break;
      case 64: run_split<float, 64>(a, nr, deep, s); break;
      default: run_split<float, 128>(a, nr, deep, s);
    }
  }
  return check_launch("packed attention launch");
}

}  // namespace cs
