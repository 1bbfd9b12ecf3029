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
// its own 256 rows or its own 64 requests.  Nothing passes between workgroups,
// since no array is read that the launch writes: a row's page is the table's
// where the request held it before, the free list's otherwise.  (512 requests,
// 25,000 rows in trees of up to 64: 6.5 us; one request, one row: 2.5.)
constexpr int kPlanThreads = 256;
constexpr int kPlanRequests = 64;    // requests of a workgroup
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
  unsigned row_blocks;  // workgroups for rows; the others take requests
  FastDiv page;
};

// Prefix sums over the wavefront that stay at 2^32 - 1 once they get there, so
// that a sum beyond the arrays' sizes is seen as one.
__device__ __forceinline__ unsigned wave_scan_sat(unsigned x) {
  auto add = [](unsigned u, int v) { return __builtin_elementwise_add_sat(u, (unsigned)v); };
  x = add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));  // row_shr 1, 2, 4, 8
  x = add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  x = add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  x = add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  x = add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));  // lane 15 to rows 1 and 3
  x = add(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));  // lane 31 to rows 2 and 3
  return x;
}

__global__ __launch_bounds__(kPlanThreads) void batch_plan(const BatchPlanArgs a) {
  extern __shared__ int lds[];
  int* s_row = lds;                // [B + 1] first row of request b
  int* s_take = lds + a.B + 1;     // [B + 1] first entry of the free list that request b takes
  int* s_par = s_take + a.B + 1;   // [kParentWindow]
  __shared__ unsigned s_rows[kPlanThreads / 64], s_grow[kPlanThreads / 64];
  __shared__ int s_flags[kPlanThreads / 64];
  const int tid = threadIdx.x, P = a.page.d, lane = tid & 63, wave = tid >> 6;
  const int head = *a.free_head;
  // each thread takes `per` consecutive requests
  const int per = (a.B + kPlanThreads - 1) / kPlanThreads;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  unsigned rows = 0, grow = 0;
  int flags = head < 0 ? CS_PLAN_BAD_LENGTH : 0;
  for (int b = b0; b < b1; ++b) {
    const int c = a.cached[b], n = a.new_len[b], h = a.held[b];
    if (c < 0 || n < 0 || h < 0 || (int64_t)c + n > 0x7fffffff || (int64_t)h * P < c) flags |= CS_PLAN_BAD_LENGTH;
    if (n > a.n_rows) flags |= CS_PLAN_TOO_MANY_ROWS;
    if (a.mask && n > 64 * (int64_t)a.words) flags |= CS_PLAN_MASK_TOO_SMALL;
    const int last = (int)min((unsigned)max(c, 0) + (unsigned)max(n, 0), 0x7fffffffu) - 1;
    const int need = last < 0 ? 0 : a.page.div(last) + 1, more = max(need - max(h, 0), 0);
    if (need > a.max_blocks || h > a.max_blocks) flags |= CS_PLAN_TABLE_FULL;
    rows = __builtin_elementwise_add_sat(rows, (unsigned)max(n, 0));
    grow = __builtin_elementwise_add_sat(grow, (unsigned)more);
    s_row[b] = n;
    s_take[b] = more;
  }
  const unsigned up_rows = wave_scan_sat(rows), up_grow = wave_scan_sat(grow);
  if (__ballot(flags))
    for (int o = 1; o < 64; o <<= 1) flags |= __shfl_xor(flags, o);
  if (lane == 63) {
    s_rows[wave] = up_rows;
    s_grow[wave] = up_grow;
    s_flags[wave] = flags;
  }
  __syncthreads();
  unsigned n_total = 0, n_grow = 0, row0 = up_rows - rows, take0 = up_grow - grow;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    row0 += w < wave ? s_rows[w] : 0;
    take0 += w < wave ? s_grow[w] : 0;
    n_total = __builtin_elementwise_add_sat(n_total, s_rows[w]);
    n_grow = __builtin_elementwise_add_sat(n_grow, s_grow[w]);
    flags |= s_flags[w];
  }
  if (n_total > (unsigned)a.n_rows) flags |= CS_PLAN_TOO_MANY_ROWS;
  if ((int64_t)head + n_grow > a.n_free) flags |= CS_PLAN_POOL_FULL;
  const bool ok = flags == 0;
  if (!ok) n_total = n_grow = row0 = take0 = 0;
  take0 += head;
  for (int b = b0; b < b1; ++b) {
    const int n = s_row[b], more = s_take[b];
    s_row[b] = row0;
    s_take[b] = take0;
    row0 += ok ? n : 0;
    take0 += ok ? more : 0;
  }
  if (tid == 0) {
    s_row[a.B] = n_total;
    s_take[a.B] = head + n_grow;
  }
  __syncthreads();

  if (blockIdx.x >= a.row_blocks) {  // requests: what the step leaves of them
    const int first = (blockIdx.x - a.row_blocks) * kPlanRequests;
    for (int b = first + (tid >> 2); b < min(first + kPlanRequests, a.B); b += kPlanThreads / 4) {  // 4 threads each
      const int h = a.held[b], take = s_take[b], more = s_take[b + 1] - take;
      for (int x = tid & 3; x < more; x += 4) {
        const int page = a.free_pages[take + x];
        a.table[(int64_t)b * a.max_blocks + h + x] = page;
        if (page < 0 || page >= a.n_pages) atomicOr(a.status, CS_PLAN_BAD_PAGE);
      }
      if ((tid & 3) == 0) {
        a.held_out[b] = h + more;
        a.row_start[b] = s_row[b];
      }
    }
    if (first == 0 && tid == 0) {
      a.row_start[a.B] = n_total;
      *a.free_head_out = head + n_grow;
      if (flags) atomicOr(a.status, flags);
    }
    return;
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
  if (a.parent && r_first < (int)n_total) {
    w1 = min(r_first + kPlanThreads, (int)n_total);
    w0 = max(s_row[request_at(r_first)], w1 - kParentWindow);
    for (int x = w0 + tid; x < w1; x += kPlanThreads) s_par[x - w0] = a.parent[x];
    __syncthreads();
  }
  if (r >= a.n_rows) return;
  if (r >= (int)n_total) {
    a.slot[r] = -1;
    return;
  }
  const int b = request_at(r), r0 = s_row[b], i = r - r0;
  const int pos = a.cached[b] + i, blk = a.page.div(pos), h = a.held[b];
  const int page = blk < h ? a.table[(int64_t)b * a.max_blocks + blk] : a.free_pages[s_take[b] + blk - h];
  const bool in_pool = page >= 0 && page < a.n_pages;
  a.slot[r] = in_pool ? page * P + (pos - blk * P) : -1;
  if (!in_pool) atomicOr(a.status, CS_PLAN_BAD_PAGE);
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
  const int64_t row_blocks = ((int64_t)b.n_rows + kPlanThreads - 1) / kPlanThreads;
  const int64_t blocks = row_blocks + std::max(1, (b.n_requests + kPlanRequests - 1) / kPlanRequests);
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
  a.row_blocks = (unsigned)row_blocks;
  TraceScope tr("batch_plan", s);
  const size_t lds = (2 * (size_t)a.B + 2 + (p.parent ? kParentWindow : 0)) * sizeof(int);
  CS_LAUNCH(tr, batch_plan, dim3((unsigned)blocks), dim3(kPlanThreads), lds, s, a);
  return check_launch("batch plan launch");
}

// ============================================================== commit
// Row accepted[i] -> row i of the request's new rows, i ascending.  Since the
// path ascends, accepted[i] >= i: a destination is never the source of a later
// entry, so copying the entries in order is a move in place.  A thread owns one
// 16-byte column of one (layer, KV head, K or V) plane and copies it for all
// entries, kBatchRows loads in flight before their stores, so nothing passes
// between threads; the rows' places are found once per workgroup, in LDS.  Bound by
// its chain of loads (lengths, path, table, rows): 3.9 us for one path in 36
// layers, 5.5 for 48 paths of about four rows (11 MB).
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
