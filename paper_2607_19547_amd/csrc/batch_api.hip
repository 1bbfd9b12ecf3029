// C-ABI entry points of the batch calls: argument validation, then the launches.
#include <math.h>

#include <string>
#include <vector>

#include "batch.h"

namespace cs {

PoolView pool_view(const Geo& g, const cs_page_pool& p) {
  PoolView v;
  v.k = (char*)p.k_pages;
  v.v = (char*)p.v_pages;
  v.P = (int)g.T;
  v.row_bytes = g.D * g.esize;
  v.page_bytes = (int64_t)g.L * g.Hkv * g.T * v.row_bytes;
  v.n_pages = (int)p.n_pages;
  return v;
}

namespace {

cs_status check_n_pages(const Geo& g, int64_t n_pages) {
  if (n_pages < 1) return fail(CS_ERR_INVALID_ARGUMENT, "n_pages must be >= 1");
  if (n_pages >= (int64_t(1) << 31) || n_pages * g.T >= (int64_t(1) << 31))
    return fail(CS_ERR_INVALID_ARGUMENT, "n_pages x the page's tokens must be below 2^31");
  return CS_OK;
}

cs_status check_pool(const Geo& g, const cs_page_pool* p) {
  if (!p) return fail(CS_ERR_INVALID_ARGUMENT, "pool is NULL");
  cs_status st = check_n_pages(g, p->n_pages);
  if (st) return st;
  if (!p->k_pages || !p->v_pages) return fail(CS_ERR_INVALID_ARGUMENT, "k_pages or v_pages is NULL");
  if (((uintptr_t)p->k_pages | (uintptr_t)p->v_pages) & 15)
    return fail(CS_ERR_INVALID_ARGUMENT, "k_pages and v_pages must be aligned to 16 bytes");
  return CS_OK;
}

// The batch's sizes and the arrays every call uses.
cs_status check_batch(const cs_batch* b) {
  if (!b) return fail(CS_ERR_INVALID_ARGUMENT, "batch is NULL");
  if (b->n_requests < 0 || b->n_rows < 0 || b->max_blocks < 0 || b->mask_words < 0 || b->max_rows < 0)
    return fail(CS_ERR_INVALID_ARGUMENT, "a size of the batch is negative");
  if (b->n_requests > kMaxRequests)
    return fail(CS_ERR_UNSUPPORTED, "a batch holds at most " + std::to_string(kMaxRequests) + " requests");
  if (!b->row_start) return fail(CS_ERR_INVALID_ARGUMENT, "row_start is NULL");
  if (b->n_requests > 0 && (!b->cached_len || (b->max_blocks > 0 && !b->block_table)))
    return fail(CS_ERR_INVALID_ARGUMENT, "cached_len or block_table is NULL");
  if (b->tree_mask && b->mask_words == 0)
    return fail(CS_ERR_INVALID_ARGUMENT, "mask_words must be >= 1 with a tree mask");
  return CS_OK;
}

cs_status check_rows(const cs_rows* r, const char* what) {
  if (!r || !r->data) return fail(CS_ERR_INVALID_ARGUMENT, std::string(what) + " is NULL");
  if (r->row_stride < 0 || r->head_stride < 0)
    return fail(CS_ERR_INVALID_ARGUMENT, std::string(what) + " has a negative stride");
  return CS_OK;
}

bool same_rows(const cs_rows& x, const cs_rows& y) {
  return x.row_stride == y.row_stride && x.head_stride == y.head_stride;
}

// Rows that are written: no two heads of them may share an element.
cs_status check_written(const Geo& g, const cs_rows* r, int n_rows, int heads, const char* what) {
  const int64_t rs = r->row_stride, hs = r->head_stride;
  const bool heads_apart = heads <= 1 || hs >= g.D, rows_apart = n_rows <= 1 || rs >= g.D;
  // heads within rows, or rows within heads
  const bool nested = heads <= 1 || n_rows <= 1 || rs >= (heads - 1) * hs + g.D || hs >= (n_rows - 1) * rs + g.D;
  if (!heads_apart || !rows_apart || !nested)
    return fail(CS_ERR_INVALID_ARGUMENT, std::string(what) + " has strides that make its heads overlap");
  return CS_OK;
}

// Rows x heads are counted in 32 bits.
cs_status check_row_count(const Geo& g, const cs_batch& b) {
  if ((int64_t)b.n_rows * (g.Hq + 2 * (int64_t)g.Hkv) >= (int64_t(1) << 31))
    return fail(CS_ERR_UNSUPPORTED, "rows x heads must be below 2^31");
  return CS_OK;
}

// Keys are counted in 32 bits: the attention kernels step over a request's keys
// in tiles and look up pages a few tiles ahead, so the room of a block table
// (no length goes beyond it) stays that far below 2^31.
constexpr int64_t kMaxTableTokens = (int64_t(1) << 31) - 65536;
cs_status check_table(const Geo& g, const cs_batch& b) {
  if (b.max_blocks > 0 && g.T > kMaxTableTokens / b.max_blocks)
    return fail(CS_ERR_UNSUPPORTED, "max_blocks x the page's tokens must be at most 2^31 - 65536");
  return CS_OK;
}

cs_status check_layer(const Geo& g, int32_t layer) {
  if (layer < 0 || layer >= g.L) return fail(CS_ERR_INVALID_ARGUMENT, "layer out of range");
  return CS_OK;
}

// theta_i in float64: inv_freq, or the powers of rope_base.
cs_status thetas(const cs_geometry* gp, const Geo& g, double* theta) {
  for (int i = 0; i < g.P; ++i) {
    theta[i] = gp->inv_freq ? gp->inv_freq[i] : pow(gp->rope_base, -2.0 * i / (double)g.D);
    if (!isfinite(theta[i])) return fail(CS_ERR_INVALID_ARGUMENT, "inv_freq holds a non-finite value");
  }
  return CS_OK;
}

}  // namespace
}  // namespace cs

using namespace cs;

extern "C" {

cs_status batch_plan_pages(const cs_geometry* page, int64_t n_pages, const cs_batch* batch, const cs_page_plan* plan,
                           void* stream) {
  Geo g;
  cs_status st = check_geometry(page, &g);
  if (!st) st = check_n_pages(g, n_pages);
  if (!st) st = check_batch(batch);
  if (st) return st;
  if (!plan) return fail(CS_ERR_INVALID_ARGUMENT, "plan is NULL");
  if (plan->n_free < 0) return fail(CS_ERR_INVALID_ARGUMENT, "n_free must be >= 0");
  if (!plan->free_head || !plan->free_head_out || !plan->status || (plan->n_free > 0 && !plan->free_pages) ||
      (batch->n_requests > 0 && (!plan->new_len || !plan->n_blocks || !plan->n_blocks_out)) ||
      (batch->n_rows > 0 && (!batch->slot || !batch->coords)))
    return fail(CS_ERR_INVALID_ARGUMENT, "a required device pointer is NULL");
  if (plan->n_blocks_out == plan->n_blocks && batch->n_requests > 0)
    return fail(CS_ERR_INVALID_ARGUMENT, "n_blocks_out must not be n_blocks");
  if (plan->free_head_out == plan->free_head)
    return fail(CS_ERR_INVALID_ARGUMENT, "free_head_out must not be free_head");
  if (plan->parent && !batch->tree_mask)
    return fail(CS_ERR_INVALID_ARGUMENT, "parent needs a tree mask");
  return launch_batch_plan(g, n_pages, *batch, *plan, (hipStream_t)stream, false);
}

cs_status qk_norm_rope_append(const cs_geometry* page, const cs_page_pool* pool, int32_t layer, const cs_batch* batch,
                              const cs_rows* q, const cs_rows* k, const cs_rows* v, const void* q_weight,
                              const void* k_weight, float eps, const cs_rows* q_out, void* stream) {
  Geo g;
  cs_status st = check_geometry(page, &g);
  if (!st) st = check_pool(g, pool);
  if (!st) st = check_layer(g, layer);
  if (!st) st = check_batch(batch);
  if (st) return st;
  if (!(eps >= 0.f && isfinite(eps))) return fail(CS_ERR_INVALID_ARGUMENT, "eps must be finite and >= 0");
  if (batch->n_requests == 0 || batch->n_rows == 0) return CS_OK;
  if (!batch->slot || !batch->coords) return fail(CS_ERR_INVALID_ARGUMENT, "slot or coords is NULL");
  st = check_row_count(g, *batch);
  if (!st) st = check_rows(q, "q");
  if (!st) st = check_rows(k, "k");
  if (!st) st = check_rows(v, "v");
  if (!st) st = check_rows(q_out, "q_out");
  if (!st) st = check_written(g, q_out, batch->n_rows, g.Hq, "q_out");
  if (st) return st;
  if (q_out->data == q->data && !same_rows(*q, *q_out))
    return fail(CS_ERR_INVALID_ARGUMENT, "q_out in place of q must have q's strides");
  AppendJob job{*q, *k, *v, *q_out, q_weight, k_weight, eps};
  double theta[256];
  st = thetas(page, g, theta);
  if (st) return st;
  return launch_append(g, *pool, layer, *batch, job, theta, (hipStream_t)stream, false);
}

cs_status tree_attend_paged_workspace(const cs_geometry* page, const cs_batch* batch, size_t* bytes) {
  Geo g;
  cs_status st = check_geometry(page, &g);
  if (!st) st = check_batch(batch);
  if (st) return st;
  if (!bytes) return fail(CS_ERR_INVALID_ARGUMENT, "bytes is NULL");
  st = check_table(g, *batch);
  if (st) return st;
  *bytes = batch->n_requests == 0 || batch->n_rows == 0 ? 0 : tree_attend_workspace(g);
  return CS_OK;
}

cs_status tree_attend_paged(const cs_geometry* page, const cs_page_pool* pool, int32_t layer, const cs_batch* batch,
                            const cs_rows* q, const cs_rows* out, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream) {
  Geo g;
  cs_status st = check_geometry(page, &g);
  if (!st) st = check_pool(g, pool);
  if (!st) st = check_layer(g, layer);
  if (!st) st = check_batch(batch);
  if (st) return st;
  if (batch->n_requests == 0 || batch->n_rows == 0) return CS_OK;
  st = check_row_count(g, *batch);
  if (!st) st = check_table(g, *batch);
  if (!st) st = check_rows(q, "q");
  if (!st) st = check_rows(out, "out");
  if (!st) st = check_written(g, out, batch->n_rows, g.Hq, "out");
  if (st) return st;
  if (out->data == q->data && !same_rows(*q, *out))
    return fail(CS_ERR_INVALID_ARGUMENT, "out in place of q must have q's strides");
  const size_t need = tree_attend_workspace(g);
  if (need && (!workspace || workspace_bytes < need))
    return fail(CS_ERR_WORKSPACE_TOO_SMALL,
                "workspace smaller than tree_attend_paged_workspace() (" + std::to_string(need) + " bytes)");
  return launch_tree_attend(g, *pool, layer, *batch, *q, *out, lse, workspace, (hipStream_t)stream, false);
}

cs_status tree_commit_paged(const cs_geometry* page, const cs_page_pool* pool, int32_t layer_begin, int32_t layer_end,
                            const cs_batch* batch, const int32_t* accepted, int32_t max_accept,
                            const int32_t* n_accepted, int32_t* cached_len_out, void* stream) {
  Geo g;
  cs_status st = check_geometry(page, &g);
  if (!st) st = check_pool(g, pool);
  if (!st) st = check_batch(batch);
  if (st) return st;
  if (layer_begin < 0 || layer_end < layer_begin || layer_end > g.L)
    return fail(CS_ERR_INVALID_ARGUMENT, "need 0 <= layer_begin <= layer_end <= n_layers");
  if (max_accept < 0) return fail(CS_ERR_INVALID_ARGUMENT, "max_accept must be >= 0");
  if (batch->n_requests == 0) return CS_OK;
  if (!n_accepted || (max_accept > 0 && !accepted))
    return fail(CS_ERR_INVALID_ARGUMENT, "accepted or n_accepted is NULL");
  if (cached_len_out == batch->cached_len)
    return fail(CS_ERR_INVALID_ARGUMENT, "cached_len_out must not be cached_len");
  return launch_tree_commit(g, *pool, layer_begin, layer_end, *batch, accepted, max_accept, n_accepted, cached_len_out,
                            (hipStream_t)stream, false);
}

}  // extern "C"
