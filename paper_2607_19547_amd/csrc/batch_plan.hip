// The plan of a batch's step (block tables, slots, coordinates, tree masks
// from the requests' lengths) and the commit of accepted paths.
#include <algorithm>

#include "batch.h"

namespace cs {

// ============================================================== plan
// With need_b = ceil((cached_b + new_b) / P) and grow_b = max(0, need_b -
// held_b), request b's rows start at the sum of the new lengths before it and
// its new pages at the sum of the growths before it: two prefix sums over the
// requests.  Everything else is a lookup per row.
//
// The arrays are small (a few KB to a MB) and the step waits for them, so the
// launch is bound by its latency: one launch, in which every workgroup makes
// both prefix sums for itself (the lengths come from the L2) and then writes
// its own 256 rows and its own share of the requests.  Nothing passes between
// workgroups, since no array is read that the launch writes: a row's page is
// the table's where the request held it before, the free list's otherwise.
constexpr int kPlanThreads = 256;
constexpr int kParentWindow = 2048;  // parents kept in LDS: the workgroup's rows and the tree before them

struct BatchPlanArgs {
  const int32_t* cached;
  const int32_t* new_len;
  const int32_t* held;
  const int32_t* free_pages;
  const int32_t* free_head;
  const int32_t* parent;
  const int32_t* base;
  int32_t* row_start;
  int32_t* table;
  int32_t* slot;
  int32_t* coords;
  unsigned long long* mask;
  int32_t* held_out;
  int32_t* free_head_out;
  int32_t* status;
  int B, n_rows, max_blocks, words, n_free, n_pages;
  FastDiv page;
};

// Sums of x over the workgroup's threads before this one; *total gets the sum.
__device__ __forceinline__ int64_t block_scan64(int64_t x, int64_t* red, int64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t inc = wave_scan64(x);
  if (lane == 63) red[wave] = inc;
  __syncthreads();
  int64_t before = 0, sum = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    before += w < wave ? red[w] : 0;
    sum += red[w];
  }
  __syncthreads();  // red is used again
  *total = sum;
  return before + inc - x;
}

__global__ __launch_bounds__(kPlanThreads) void batch_plan(const BatchPlanArgs a) {
  extern __shared__ int lds[];
  int* s_row = lds;                // [B + 1] first row of request b
  int* s_take = lds + a.B + 1;     // [B] first entry of the free list that request b takes
  int* s_par = s_take + a.B;       // [kParentWindow]
  __shared__ int64_t red[kPlanThreads / 64];
  __shared__ int s_flags;
  const int tid = threadIdx.x, P = a.page.d;
  if (tid == 0) s_flags = 0;
  __syncthreads();
  const int head = *a.free_head;
  // each thread takes `per` consecutive requests
  const int per = (a.B + kPlanThreads - 1) / kPlanThreads;
  int64_t rows = 0, grow = 0;
  int flags = head < 0 ? CS_PLAN_BAD_LENGTH : 0;
  for (int j = 0; j < per; ++j) {
    const int b = tid * per + j;
    if (b >= a.B) break;
    const int c = a.cached[b], n = a.new_len[b], h = a.held[b];
    if (c < 0 || n < 0 || h < 0 || (int64_t)c + n > 0x7fffffff || (int64_t)h * P < c) flags |= CS_PLAN_BAD_LENGTH;
    if (n > a.n_rows) flags |= CS_PLAN_TOO_MANY_ROWS;
    if (a.mask && n > 64 * (int64_t)a.words) flags |= CS_PLAN_MASK_TOO_SMALL;
    const int64_t need = ((int64_t)c + n + P - 1) / P;
    if (need > a.max_blocks || h > a.max_blocks) flags |= CS_PLAN_TABLE_FULL;
    rows += max(n, 0);
    grow += max(need - h, (int64_t)0);
  }
  int64_t n_total, n_grow;
  const int64_t row0 = block_scan64(rows, red, &n_total);
  const int64_t take0 = block_scan64(grow, red, &n_grow);
  if (n_total > a.n_rows) flags |= CS_PLAN_TOO_MANY_ROWS;
  if (head + n_grow > a.n_free) flags |= CS_PLAN_POOL_FULL;
  if (flags) atomicOr(&s_flags, flags);
  __syncthreads();
  flags = s_flags;
  const bool ok = flags == 0;
  if (!ok) {
    n_total = 0;
    n_grow = 0;
  }
  {
    int r = ok ? (int)row0 : 0, t = head + (ok ? (int)take0 : 0);
    for (int j = 0; j < per; ++j) {
      const int b = tid * per + j;
      if (b >= a.B) break;
      s_row[b] = r;
      s_take[b] = t;
      if (ok) {
        const int n = a.new_len[b];
        r += n;
        t += max((int)(((int64_t)a.cached[b] + n + P - 1) / P) - a.held[b], 0);
      }
    }
    if (tid == 0) s_row[a.B] = (int)n_total;
  }
  __syncthreads();

  // the workgroup's share of the requests: what the step leaves of them
  const int share = (a.B + gridDim.x - 1) / gridDim.x;
  const int b_end = min((int)(blockIdx.x + 1) * share, a.B);
  for (int b = blockIdx.x * share + (tid >> 4); b < b_end; b += kPlanThreads / 16) {  // 16 threads a request
    const int h = a.held[b];
    const int need = ok ? (int)(((int64_t)a.cached[b] + a.new_len[b] + P - 1) / P) : h;
    for (int x = h + (tid & 15); x < need; x += 16) {
      const int page = a.free_pages[s_take[b] + x - h];
      a.table[(int64_t)b * a.max_blocks + x] = page;
      if (page < 0 || page >= a.n_pages) atomicOr(a.status, CS_PLAN_BAD_PAGE);
    }
    if ((tid & 15) == 0) {
      a.held_out[b] = max(need, h);
      a.row_start[b] = s_row[b];
    }
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.row_start[a.B] = (int)n_total;
    *a.free_head_out = head + (int)n_grow;
    if (flags) atomicOr(a.status, flags);
  }

  // the workgroup's rows
  const int r = blockIdx.x * kPlanThreads + tid;
  const int r_first = blockIdx.x * kPlanThreads;
  auto request_at = [&](int row) {  // the last request that starts at or before the row
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_row[mid] <= row) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  int w0 = 0, w1 = 0;  // rows whose parents are in LDS
  if (a.parent && r_first < n_total) {
    w1 = min(r_first + kPlanThreads, (int)n_total);
    w0 = max(s_row[request_at(r_first)], w1 - kParentWindow);
    for (int x = w0 + tid; x < w1; x += kPlanThreads) s_par[x - w0] = a.parent[x];
    __syncthreads();
  }
  if (r >= a.n_rows) return;
  if (r >= n_total) {
    a.slot[r] = -1;
    return;
  }
  const int b = request_at(r), r0 = s_row[b], i = r - r0;
  const int pos = a.cached[b] + i, blk = a.page.div(pos), h = a.held[b];
  const int page = blk < h ? a.table[(int64_t)b * a.max_blocks + blk] : a.free_pages[s_take[b] + blk - h];
  a.slot[r] = page >= 0 && page < a.n_pages ? page * P + (pos - blk * P) : -1;
  int depth = i;
  if (a.parent) {
    // ancestors come in descending order, so a mask word is complete when
    // the walk leaves it
    unsigned long long* m = a.mask + (int64_t)r * a.words;
    int w = a.words - 1, j = i;
    unsigned long long bits = 0;
    bool bad = false;
    depth = -1;
    while (j >= 0) {
      ++depth;
      while (w > j >> 6) {
        m[w--] = bits;
        bits = 0;
      }
      bits |= 1ull << (j & 63);
      const int x = r0 + j;
      int p = x >= w0 ? s_par[x - w0] : a.parent[x];
      if (p < -1 || p >= j) {
        bad = true;
        p = -1;
      }
      j = p;
    }
    for (; w >= 0; --w) {
      m[w] = bits;
      bits = 0;
    }
    if (bad) atomicOr(a.status, CS_PLAN_BAD_PARENT);
  } else if (a.mask) {
    unsigned long long* m = a.mask + (int64_t)r * a.words;
    for (int w = 0; w < a.words; ++w)
      m[w] = i >= 64 * w + 63 ? ~0ull : i >= 64 * w ? (2ull << (i & 63)) - 1 : 0ull;
  }
  const int at = (int)((unsigned)(a.base ? a.base[b] : a.cached[b]) + (unsigned)depth);
  a.coords[3 * (int64_t)r] = at;
  a.coords[3 * (int64_t)r + 1] = at;
  a.coords[3 * (int64_t)r + 2] = at;
}

cs_status launch_batch_plan(const Geo& g, int64_t n_pages, const cs_batch& b, const cs_page_plan& p, hipStream_t s,
                            bool check_only) {
  const int64_t blocks = std::max<int64_t>(1, ((int64_t)b.n_rows + kPlanThreads - 1) / kPlanThreads);
  const cs_status st = check_grid(blocks, 1, 1, kPlanThreads, "batch plan");
  if (st || check_only) return st;
  BatchPlanArgs a;
  a.cached = b.cached_len;
  a.new_len = p.new_len;
  a.held = p.n_blocks;
  a.free_pages = p.free_pages;
  a.free_head = p.free_head;
  a.parent = p.parent;
  a.base = p.coord_base;
  a.row_start = b.row_start;
  a.table = b.block_table;
  a.slot = b.slot;
  a.coords = b.coords;
  a.mask = (unsigned long long*)b.tree_mask;
  a.held_out = p.n_blocks_out;
  a.free_head_out = p.free_head_out;
  a.status = p.status;
  a.B = b.n_requests;
  a.n_rows = b.n_rows;
  a.max_blocks = b.max_blocks;
  a.words = b.mask_words;
  a.n_free = p.n_free;
  a.n_pages = (int)n_pages;
  a.page = fast_div((int)g.T);
  TraceScope tr("batch_plan", s);
  const size_t lds = (2 * (size_t)a.B + 1 + (p.parent ? kParentWindow : 0)) * sizeof(int);
  CS_LAUNCH(tr, batch_plan, dim3((unsigned)blocks), dim3(kPlanThreads), lds, s, a);
  return check_launch("batch plan launch");
}

// ============================================================== commit
// Row accepted[i] -> row i of the request's new rows, i ascending.  Since the
// path ascends, accepted[i] >= i: a destination is never the source of a later
// entry, so copying the entries in order is a move in place.  A thread owns one
// 16-byte column of one (layer, KV head, K or V) plane and copies it for all
// entries, kBatchRows loads in flight before their stores, so nothing passes
// between threads; the rows' places are found once per workgroup, in LDS.
constexpr int kCommitThreads = 256;
constexpr int kPathChunk = 64;
constexpr int kBatchRows = 8;

struct CommitArgs {
  PoolView pool;
  const int32_t* cached;
  const int32_t* row_start;
  const int32_t* table;
  const int32_t* accepted;
  const int32_t* n_accepted;
  int32_t* cached_out;
  int n_rows, max_blocks, max_accept, Hkv, lb, columns, words;  // columns: planes x 2 x words of a row
  FastDiv page;
};

template <typename W>
__global__ __launch_bounds__(kCommitThreads) void tree_commit(const CommitArgs a) {
  __shared__ int64_t s_src[kPathChunk], s_dst[kPathChunk];
  __shared__ int s_bad;
  const int b = blockIdx.y, tid = threadIdx.x, P = a.page.d;
  const Request q = request_of(a.row_start[b], a.row_start[b + 1], a.cached[b], a.n_rows, (int64_t)a.max_blocks * P);
  const int n = min(max(a.n_accepted[b], 0), a.max_accept);
  const int u = blockIdx.x * kCommitThreads + tid;
  const bool mine = u < a.columns;
  const int w = u % a.words, pl = u / a.words;  // plane of the call: layer, head, K or V
  char* base = (pl & 1 ? a.pool.v : a.pool.k) +
               ((int64_t)a.lb * a.Hkv + (pl >> 1)) * P * a.pool.row_bytes + (int64_t)w * (int)sizeof(W);
  int done = 0;
  for (int i0 = 0; i0 < n; i0 += kPathChunk) {
    if (tid == 0) s_bad = kPathChunk;
    __syncthreads();
    const int cnt = min(n - i0, kPathChunk);
    if (tid < cnt) {
      const int i = i0 + tid;
      const int j = a.accepted[(int64_t)b * a.max_accept + i];
      const int before = i > 0 ? a.accepted[(int64_t)b * a.max_accept + i - 1] : -1;
      if (j <= before || j >= q.n) atomicMin(&s_bad, tid);
      int64_t from = -1, to = -1;
      if (j > before && j < q.n && j != i) {
        const int64_t ts = (int64_t)q.cached + j, td = (int64_t)q.cached + i;
        if (ts < q.len && td < q.len) {
          const int bs = a.page.div((int)ts), bd = a.page.div((int)td);
          const int ps = a.table[(int64_t)b * a.max_blocks + bs], pd = a.table[(int64_t)b * a.max_blocks + bd];
          if (ps >= 0 && ps < a.pool.n_pages && pd >= 0 && pd < a.pool.n_pages) {
            from = ps * a.pool.page_bytes + (ts - (int64_t)bs * P) * a.pool.row_bytes;
            to = pd * a.pool.page_bytes + (td - (int64_t)bd * P) * a.pool.row_bytes;
          }
        }
      }
      s_src[tid] = from;
      s_dst[tid] = to;
    }
    __syncthreads();
    const int good = min(cnt, s_bad);
    if (mine)
      for (int x = 0; x < good; x += kBatchRows) {
        W v[kBatchRows];
#pragma unroll
        for (int y = 0; y < kBatchRows; ++y)
          if (x + y < good && s_src[x + y] >= 0) v[y] = *(const W*)(base + s_src[x + y]);
#pragma unroll
        for (int y = 0; y < kBatchRows; ++y)
          if (x + y < good && s_src[x + y] >= 0) *(W*)(base + s_dst[x + y]) = v[y];
      }
    done += good;
    if (good < cnt) break;
    __syncthreads();  // the lists are written again
  }
  if (a.cached_out && blockIdx.x == 0 && tid == 0) a.cached_out[b] = a.cached[b] + done;
}

cs_status launch_tree_commit(const Geo& g, const cs_page_pool& pool, int lb, int le, const cs_batch& b,
                             const int32_t* accepted, int max_accept, const int32_t* n_accepted, int32_t* cached_out,
                             hipStream_t s, bool check_only) {
  CommitArgs a;
  a.pool = pool_view(g, pool);
  const int wide = a.pool.row_bytes % 16 == 0 ? 16 : 4;
  a.words = a.pool.row_bytes / wide;
  const int64_t columns = (int64_t)(le - lb) * g.Hkv * 2 * a.words;
  const int64_t blocks = std::max<int64_t>(1, (columns + kCommitThreads - 1) / kCommitThreads);
  if (columns >= (int64_t(1) << 31) - kCommitThreads)
    return fail(CS_ERR_UNSUPPORTED, "tree commit: too many layers and heads for one launch");
  const cs_status st = check_grid(blocks, b.n_requests, 1, kCommitThreads, "tree commit");
  if (st || check_only) return st;
  a.cached = b.cached_len;
  a.row_start = b.row_start;
  a.table = b.block_table;
  a.accepted = accepted;
  a.n_accepted = n_accepted;
  a.cached_out = cached_out;
  a.n_rows = b.n_rows;
  a.max_blocks = b.max_blocks;
  a.max_accept = max_accept;
  a.Hkv = g.Hkv;
  a.lb = lb;
  a.columns = (int)columns;
  a.page = fast_div((int)g.T);
  TraceScope tr("tree_commit", s);
  const dim3 grid((unsigned)blocks, b.n_requests);
  if (wide == 16) CS_LAUNCH(tr, tree_commit<u32x4>, grid, dim3(kCommitThreads), 0, s, a);
  else CS_LAUNCH(tr, tree_commit<uint32_t>, grid, dim3(kCommitThreads), 0, s, a);
  return check_launch("tree commit launch");
}

}  // namespace cs
