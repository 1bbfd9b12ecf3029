/*
 * chronostitch.h -- C ABI of the ChronoStitch KV-composition hot path for
 * AMD Instinct MI355X (gfx950).
 *
 * The method (ChronoStitch, Section 2) composes independently prefilled
 * visual KV caches: stored post-rotary keys are moved from local chunk
 * coordinates to a global three-axis (t, h, w) mRoPE timeline by a delta
 * rotation (Eq. 3); later-chunk tokens are ranked by the deviation of their
 * recomputed scoring-layer key (Eq. 5); the top rho fraction is recomputed,
 * attending causally over the composed cache (Eq. 1), and their fresh keys
 * and values are scattered back.
 *
 * Conventions shared by every entry point
 *  - All functions are extern "C", take plain pointers and sizes, and never
 *    throw.  They return CS_OK or an error code; cs_last_error() then gives
 *    a human-readable message (thread-local, valid until the next call on
 *    the same thread).
 *  - Argument errors are detected before anything is enqueued and before any
 *    HIP runtime call, so a rejected call leaves device memory untouched.
 *    The same holds for a call whose kernel launches would exceed the GPU's
 *    grid limits (caches of tens of millions of tokens per call): every launch
 *    of the call is sized first, and such a call returns CS_ERR_UNSUPPORTED.
 *  - DEVICE pointers are device memory of the current HIP device; HOST
 *    pointers are read (or written) before the call returns, except the host
 *    chunk data of compose_load_rebase_k_paged, which its enqueued copies
 *    read (the pointer arrays themselves are read before it returns).  The caller
 *    owns every buffer; the library allocates no device memory.  Scratch
 *    memory is a caller-provided workspace sized by the *_workspace query.
 *  - Device work is asynchronous on `stream` (a hipStream_t; NULL = the null
 *    stream).  Outputs in device memory are valid once the stream has
 *    reached the enqueued work.  Host outputs are written synchronously.
 *  - Calls are re-entrant for distinct buffers and streams.  Inputs must not
 *    alias outputs except for the documented in-place caches.
 *  - Tensor layouts are dense, row-major, with the last index contiguous:
 *      caches      [L][H_kv][T][D]   chunks are contiguous token ranges, so
 *                                    the concatenation of the chunk caches is
 *                                    the layout itself (the *_paged calls
 *                                    take one buffer per chunk instead)
 *      fresh Q     [L][H_q][n][D]    row r <-> token chunk_start[1] + r
 *      fresh K, V  [L][H_kv][n][D]   row r <-> token chunk_start[1] + r
 *    where n = T - chunk_start[1] is the number of later-chunk tokens.
 *  - Element type of every K/V/Q/O tensor is geometry.dtype; bf16 values are
 *    rounded to nearest even.
 */
#ifndef CHRONOSTITCH_H
#define CHRONOSTITCH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CS_OK = 0,
  CS_ERR_INVALID_ARGUMENT = 1,   /* a pointer, size or value is out of its documented range */
  CS_ERR_UNSUPPORTED = 2,        /* a valid request this library does not implement           */
  CS_ERR_WORKSPACE_TOO_SMALL = 3,/* workspace_bytes is below the *_workspace query's answer    */
  CS_ERR_HIP = 4                 /* a HIP runtime call or kernel launch failed                 */
} cs_status;

typedef enum { CS_F32 = 0, CS_BF16 = 1 } cs_dtype;

/* Geometry of a composed cache (Section 3 gives the model's: 36 layers,
 * 16 query heads, 2 KV heads, head dim 128, mRoPE sections 16/24/24).
 *   n_q_heads % n_kv_heads == 0; query head h reads KV head h / (n_q_heads/n_kv_heads).
 *   head_dim even, 2 <= head_dim <= 512.
 *   sections: rotary pairs on the t, h, w axes, in that order; they sum to
 *     head_dim/2.  Pair i is the element pair (i, i + head_dim/2) and rotates
 *     with axis t for i < s_t, h for i < s_t + s_h, w otherwise (Eq. 2).
 *   rope_base: theta_i = rope_base^(-2i/head_dim) when inv_freq is NULL.
 *   inv_freq: HOST [head_dim/2] float64 theta_i overriding rope_base, or NULL.
 *   chunk_start: HOST [n_chunks + 1], 0 = s_0 < s_1 < ... < s_N = n_tokens;
 *     chunk c owns tokens [s_c, s_{c+1}).  n_tokens < 2^31.             */
typedef struct {
  int32_t n_layers;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t sections[3];
  int32_t dtype;               /* cs_dtype */
  double rope_base;
  const double* inv_freq;
  int64_t n_tokens;
  int32_t n_chunks;
  const int64_t* chunk_start;
} cs_geometry;

/* ---------------------------------------------------------------------------
 * compose_rebase_k -- Section 2, Eq. 3 (three-axis delta rotation).
 *
 * Gives chunk c the global coordinates p' = p + Delta_c and rotates every
 * stored post-rotary key of the chunk, in place, by R(Delta): pair i turns by
 * Delta_c[sigma(i)] * theta_i, so a key stored as f(x, p) becomes f(x, p').
 * Angles are formed in float64 and reduced modulo 2*pi before the cos/sin
 * table is rounded to float32, so offsets of 1e5 and beyond stay accurate.
 * Chunks with Delta_c = (0,0,0) are not touched (bit-identical).  Values are
 * never rotated, so there is no V argument.
 *
 *   g             geometry (HOST)
 *   k_cache       DEVICE [L][H_kv][T][D] keys, post-rotary at local
 *                 coordinates on entry and at global coordinates on return
 *   chunk_offsets HOST int32 [n_chunks][3]: (dt, dh, dw) = p' - p of chunk c
 *   local_coords  HOST int32 [T][3] token coordinates (t, h, w), or NULL
 *   global_coords HOST int32 [T][3] output p' = p + Delta_c, or NULL; needs
 *                 local_coords.  Written before the call returns.
 *   stream        hipStream_t or NULL
 * Errors: CS_ERR_INVALID_ARGUMENT for a bad geometry, a NULL k_cache or
 * chunk_offsets, or global_coords without local_coords.                    */
cs_status compose_rebase_k(const cs_geometry* g, void* k_cache,
                           const int32_t* chunk_offsets,
                           const int32_t* local_coords, int32_t* global_coords,
                           void* stream);

/* ---------------------------------------------------------------------------
 * compose_rebase_k_tokens -- Eq. 3 with one offset per token (the position
 * policies compared in Section 3 and Table 1).
 *
 * Rotates every stored post-rotary key, in place, by its own token's offset:
 * pair i of token t turns by Delta_t[sigma(i)] * theta_i, so f(x, p_t) becomes
 * f(x, p_t + Delta_t).  With Delta_t equal to the chunk offset for every token
 * of a chunk this is compose_rebase_k; a per-token offset expresses policies
 * such as scalar re-basing, which moves token j of the composed cache to
 * (j, j, j).  Angles are formed in float64 and reduced modulo 2*pi as in
 * compose_rebase_k.  Tokens with Delta_t = (0,0,0) are not touched.
 *
 *   g              geometry (HOST)
 *   k_cache        DEVICE [L][H_kv][T][D] keys, rotated in place
 *   token_offsets  DEVICE int32 [T][3]: (dt, dh, dw) = p' - p of every token
 *                  (read on the device; contents are not checked)
 *   stream         hipStream_t or NULL
 * Errors: CS_ERR_INVALID_ARGUMENT for a bad geometry or a NULL pointer,
 * CS_ERR_HIP for a launch failure.                                          */
cs_status compose_rebase_k_tokens(const cs_geometry* g, void* k_cache,
                                  const int32_t* token_offsets, void* stream);

/* ---------------------------------------------------------------------------
 * score_deviation_topk -- Section 2, Eq. 5 and the top-rho selection after it.
 *
 * For every later-chunk token t in [s_1, T):
 *   delta_t = || k_fresh[:, t - s_1, :] - k_cache[score_layer][:, t, :] ||_2
 * over all H_kv x D elements, accumulated in float64 and rounded once to
 * float32.  Then selects the k = n_select(rho, n) largest float32 scores,
 * lower token index first among equal scores, and writes their token indices
 * in ascending order.  n_select(rho, n) = 0 if rho == 0, else
 * min(n, ceil(rho * n - 1e-9)).
 *
 *   g             geometry (HOST)
 *   k_cache       DEVICE [L][H_kv][T][D] keys, already re-based
 *   score_layer   layer whose keys are compared, 0 <= score_layer < L (the
 *                 paper scores layer 1)
 *   k_fresh       DEVICE [H_kv][n][D] recomputed keys at score_layer,
 *                 post-rotary at global coordinates
 *   rho           repair fraction in [0, 1]
 *   scores        DEVICE float32 [n] output delta_t, or NULL (then the
 *                 workspace holds them)
 *   sel_idx       DEVICE int32 [k] output, ascending token indices in [s_1, T);
 *                 may be NULL when k == 0
 *   n_sel         HOST int64 output k (computed on the host; no device sync)
 *   workspace     DEVICE scratch of workspace_bytes, >= the query's answer
 * Errors: CS_ERR_INVALID_ARGUMENT (bad geometry, rho outside [0,1] or NaN,
 * score_layer out of range, NULL required pointer), CS_ERR_WORKSPACE_TOO_SMALL.
 * Scores must be finite (NaN ranking is undefined).                       */
cs_status score_deviation_topk_workspace(const cs_geometry* g, size_t* bytes);
cs_status score_deviation_topk(const cs_geometry* g, const void* k_cache,
                               int32_t score_layer, const void* k_fresh,
                               double rho, float* scores, int32_t* sel_idx,
                               int64_t* n_sel, void* workspace,
                               size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * selective_attend_scatter_rope -- selective_attend_scatter with the rotary
 * embedding of the recomputed rows fused in (Eq. 2 at the global coordinates
 * p' of Section 2).
 *
 * The recompute of a selected token applies RoPE at its global coordinate;
 * here the caller hands over the PRE-rotary fresh queries and keys and the
 * global coordinates, and only the selected rows are rotated: for each layer,
 *   1. K row of selected token t (every KV head): f(k_pre, p'_t), rounded to
 *      the storage dtype, scattered into the cache; V rows are scattered as in
 *      selective_attend_scatter;
 *   2. Q row (every query head): f(q_pre, p'_t), rounded to the storage
 *      dtype;
 *   3. attention exactly as in selective_attend_scatter.
 * For bf16 with head_dim 128 the rotations run inside the attention's own
 * launches (the keys while they are scattered, the queries as the attention
 * loads them) from a cos/sin table of the selected tokens kept in the
 * workspace; otherwise the rotated queries pass through the workspace.
 * The result equals selective_attend_scatter on q_fresh = f(q_pre, p') and
 * k_fresh = f(k_pre, p') rounded the same way.  Angles are formed in float64
 * and reduced modulo 2*pi (float32 cos/sin), as in compose_rebase_k.
 *
 *   q_pre          DEVICE [L][H_q][n][D] pre-rotary fresh queries
 *   k_pre          DEVICE [L][H_kv][n][D] pre-rotary fresh keys
 *   v_fresh        DEVICE [L][H_kv][n][D] fresh values
 *   coords         DEVICE int32 [T][3] global coordinates p' of every token
 *                  (compose_rebase_k's global_coords, copied to the device)
 *   workspace      DEVICE, >= selective_attend_scatter_rope_workspace() for
 *                  the same n_sel and n_layers_per_call >= layer_end -
 *                  layer_begin: the attention's partials plus, for bf16 with
 *                  head_dim 128, the cos/sin table (n_sel x D/2 x 8 bytes),
 *                  otherwise the rotated queries (n_layers x H_q x n_sel x D
 *                  elements); the work plan is kept from call to call as in
 *                  selective_attend_scatter's workspace
 *   other arguments as for selective_attend_scatter.
 * Errors: CS_ERR_INVALID_ARGUMENT, CS_ERR_WORKSPACE_TOO_SMALL, CS_ERR_HIP. */
cs_status selective_attend_scatter_rope_workspace(const cs_geometry* g, int64_t n_sel,
                                                  int32_t n_layers_per_call,
                                                  size_t* bytes);
cs_status selective_attend_scatter_rope(const cs_geometry* g, void* k_cache,
                                        void* v_cache, int32_t layer_begin,
                                        int32_t layer_end, const int32_t* sel_idx,
                                        int64_t n_sel, const void* q_pre,
                                        const void* k_pre, const void* v_fresh,
                                        const int32_t* coords, void* out,
                                        float* lse, void* workspace,
                                        size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * selective_attend_scatter -- Section 2, Eq. 1 and the repair step.
 *
 * For each layer l in [layer_begin, layer_end):
 *   1. scatter: k_cache[l][h][sel_idx[m]] <- k_fresh[l][h][sel_idx[m] - s_1]
 *      and the same for V; every other row is unchanged.
 *   2. attend: for slot m (token t = sel_idx[m]) and query head h
 *      (KV head kv = h / (H_q/H_kv)), with q = q_fresh[l][h][t - s_1],
 *        out[l][h][m] = softmax_j(q . K[l][kv][j] / sqrt(D)) V[l][kv][j],
 *      j = 0 .. t (causal in cache order, self included), over the
 *      post-scatter cache.  Softmax and accumulation run in float32.
 *      lse[l][h][m] = log(sum_j exp(q . K[l][kv][j] / sqrt(D))).
 * Layers are independent, so one call over many layers equals one call per
 * layer; per-layer calls mirror the model's layer-by-layer recompute.
 *
 *   g              geometry (HOST)
 *   k_cache,v_cache DEVICE [L][H_kv][T][D], rows sel_idx overwritten in place
 *   layer_begin, layer_end  0 <= begin <= end <= L
 *   sel_idx        DEVICE int32 [n_sel], strictly ascending, in [s_1, T)
 *                  (as written by score_deviation_topk).  Not checked unless
 *                  the environment variable CS_DEBUG_VALIDATE is "1": then a
 *                  violation returns CS_ERR_INVALID_ARGUMENT before anything
 *                  else is enqueued, at the cost of a synchronisation of the
 *                  stream (a debugging aid; such calls must not overlap on one
 *                  GPU).  Unchecked, an index outside [s_1, T) is skipped and
 *                  an unsorted list gives wrong outputs, never an access
 *                  outside the caller's buffers.
 *   n_sel          0 <= n_sel <= n
 *   q_fresh        DEVICE [L][H_q][n][D] fresh queries (post-rotary, global)
 *   k_fresh,v_fresh DEVICE [L][H_kv][n][D] fresh keys / values
 *   out            DEVICE [L][H_q][n_sel][D] output, slot order of sel_idx
 *   lse            DEVICE float32 [L][H_q][n_sel] output, or NULL
 *   workspace      DEVICE scratch, >= selective_attend_scatter_workspace()
 *                  for the same n_sel and n_layers_per_call >= layer_end -
 *                  layer_begin (the size grows with the layer count); no
 *                  initial contents needed.  The call leaves its work plan at
 *                  the start of the workspace; a later call that finds there
 *                  a plan made from the same inputs (the row tiles' last
 *                  selected tokens, the row-tile and KV-head counts, the
 *                  partial-slot budget), whose checksum holds, keeps it
 *                  instead of planning again, so the layer calls of one
 *                  composition plan once.  Any other contents are
 *                  overwritten: the caller may use the workspace for anything
 *                  between calls.
 * Errors: CS_ERR_INVALID_ARGUMENT, CS_ERR_WORKSPACE_TOO_SMALL, CS_ERR_HIP. */
cs_status selective_attend_scatter_workspace(const cs_geometry* g, int64_t n_sel,
                                             int32_t n_layers_per_call,
                                             size_t* bytes);
cs_status selective_attend_scatter(const cs_geometry* g, void* k_cache,
                                   void* v_cache, int32_t layer_begin,
                                   int32_t layer_end, const int32_t* sel_idx,
                                   int64_t n_sel, const void* q_fresh,
                                   const void* k_fresh, const void* v_fresh,
                                   void* out, float* lse, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * selective_attend_scatter_noalloc -- selective_attend_scatter for callers
 * that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): the same scatter and
 * attention with no workspace argument.  It calls no hipMalloc, hipFree or
 * other allocating routine (kernel tracing is off for its launches).
 *
 * Its plan and partial results live in a 64 MiB array of device memory that
 * the library holds on every GPU it runs on until the process ends; its
 * device address is looked up once per GPU, on the first call with that GPU
 * current.  Every call on a GPU shares that GPU's array: calls that overlap
 * on one GPU (two streams, two threads) race and give wrong results.  Nothing
 * needs clearing between calls; the plan left in the array is kept by a later
 * call with the same inputs, as in a workspace.
 *
 * When the call's plan and partials would exceed the array, the key pieces
 * of long row tiles are made longer (fewer partials), so the output then
 * differs from selective_attend_scatter's by rounding only (same tolerance);
 * within the limit it is bit-identical.  A call whose plan alone exceeds the
 * array returns CS_ERR_UNSUPPORTED before anything is enqueued (this needs
 * several million selected rows).
 *
 * Arguments, layouts and the other errors are those of
 * selective_attend_scatter (contiguous cache only).                        */
cs_status selective_attend_scatter_noalloc(const cs_geometry* g, void* k_cache,
                                           void* v_cache, int32_t layer_begin,
                                           int32_t layer_end, const int32_t* sel_idx,
                                           int64_t n_sel, const void* q_fresh,
                                           const void* k_fresh, const void* v_fresh,
                                           void* out, float* lse, void* stream);

/* ---------------------------------------------------------------------------
 * Paged cache (Section 2: every chunk is prefilled and stored on its own, and
 * the stored caches are concatenated after re-basing, the step listed after
 * Eq. 6).  The *_paged calls
 * take the cache as the chunks' own buffers instead of one composed buffer,
 * so chunks loaded from storage are used where they landed:
 *   k_chunks, v_chunks   HOST arrays of geometry.n_chunks DEVICE pointers;
 *                        chunk c's keys (values) are [L][H_kv][len_c][D],
 *                        len_c = chunk_start[c+1] - chunk_start[c], dense,
 *                        row-major.  The arrays are read before the call
 *                        returns; the buffers are used in place.
 * Every other argument, the workspace sizes (the contiguous *_workspace
 * queries apply), the outputs and the errors are those of the contiguous call
 * of the same name, and the results are bit-identical to that call on the
 * concatenation of the chunks.
 * Limits: n_chunks <= 128 when dtype is CS_BF16 and head_dim is 128, <= 64
 * otherwise (else CS_ERR_UNSUPPORTED).  The attention calls on the bf16 /
 * head_dim 128 path read whole 64-key tiles from one chunk, so they need every
 * chunk_start to be a multiple of 64 (else CS_ERR_UNSUPPORTED).  A NULL array
 * or NULL chunk pointer is CS_ERR_INVALID_ARGUMENT.                          */
cs_status compose_rebase_k_paged(const cs_geometry* g, void* const* k_chunks,
                                 const int32_t* chunk_offsets,
                                 const int32_t* local_coords,
                                 int32_t* global_coords, void* stream);
cs_status compose_rebase_k_tokens_paged(const cs_geometry* g, void* const* k_chunks,
                                        const int32_t* token_offsets, void* stream);

/* compose_load_rebase_k_paged -- the chunks' load from host memory with the
 * re-basing of Eq. 3 done during the load (Section 2: chunks come back from
 * storage and are re-based before they are concatenated), so that the
 * rotation hides under the transfer of the values.
 *
 * Every chunk's keys are copied from the host to k_chunks[c] on copy_stream,
 * then every chunk's values to v_chunks[c]; once the keys have landed, stream
 * re-bases them exactly as compose_rebase_k_paged would (chunks with a zero
 * offset are copied only) while the values are still in transfer.  The
 * copies start after the work
 * enqueued on stream before the call, and when stream reaches the end of the
 * call's work every copy is complete: the call is one step of stream, and
 * later work on stream sees the whole composed cache.
 *   k_host, v_host  HOST arrays of n_chunks HOST pointers, chunk c's keys
 *                   (values) as [L][H_kv][len_c][D]; page-locked memory
 *                   (hipHostMalloc) lets the copies overlap the re-basing,
 *                   pageable memory works but serialises them.  Read before
 *                   the call's work completes on stream: keep them unchanged
 *                   until then.
 *   copy_stream     the stream of the copies; NULL or equal to stream: one
 *                   stream does everything in order.
 *   k_chunks, v_chunks, chunk_offsets, stream: as for compose_rebase_k_paged
 *                   (the destination buffers' prior contents are overwritten).
 * The results are bit-identical to copying the chunks and then calling
 * compose_rebase_k_paged.  Errors: those of compose_rebase_k_paged, plus
 * CS_ERR_INVALID_ARGUMENT for a NULL host array or chunk pointer. */
cs_status compose_load_rebase_k_paged(const cs_geometry* g, void* const* k_chunks,
                                      void* const* v_chunks, const void* const* k_host,
                                      const void* const* v_host,
                                      const int32_t* chunk_offsets,
                                      void* copy_stream, void* stream);
cs_status score_deviation_topk_paged(const cs_geometry* g, void* const* k_chunks,
                                     int32_t score_layer, const void* k_fresh,
                                     double rho, float* scores, int32_t* sel_idx,
                                     int64_t* n_sel, void* workspace,
                                     size_t workspace_bytes, void* stream);
cs_status selective_attend_scatter_paged(const cs_geometry* g, void* const* k_chunks,
                                         void* const* v_chunks, int32_t layer_begin,
                                         int32_t layer_end, const int32_t* sel_idx,
                                         int64_t n_sel, const void* q_fresh,
                                         const void* k_fresh, const void* v_fresh,
                                         void* out, float* lse, void* workspace,
                                         size_t workspace_bytes, void* stream);
cs_status selective_attend_scatter_rope_paged(const cs_geometry* g, void* const* k_chunks,
                                              void* const* v_chunks, int32_t layer_begin,
                                              int32_t layer_end, const int32_t* sel_idx,
                                              int64_t n_sel, const void* q_pre,
                                              const void* k_pre, const void* v_fresh,
                                              const int32_t* coords, void* out, float* lse,
                                              void* workspace, size_t workspace_bytes,
                                              void* stream);

/* ---------------------------------------------------------------------------
 * Answering over composed caches: batches of requests over a pool of pages.
 *
 * A page is a chunk buffer of the *_paged calls, [L][H_kv][P][D] with P tokens,
 * and a pool holds n_pages of them one behind the other, for keys and for
 * values.  The calls below take the geometry of ONE page (n_tokens = P; its
 * chunks, one from 0 to P for instance, are checked as everywhere and not
 * used), and a page can be handed to the *_paged calls as a chunk (k_chunks[c] =
 * k_pages + page x L x H_kv x P x D elements), so a memory is composed where it
 * lies.
 *
 * Token j of request b lies at offset j % P of page block_table[b][j / P].  A
 * request has cached_len[b] tokens behind it and new_len[b] new ones (rows) in
 * the step: the next token, a tree of drafted tokens, or a question's tokens.
 * The rows of all requests follow each other: request b owns rows
 * [row_start[b], row_start[b + 1]), and its i-th row is its token
 * cached_len[b] + i.  Which rows a row sees is a bit mask, so a step is
 *     batch_plan_pages       pages, slots, coordinates and masks (once a step)
 *     qk_norm_rope_append    per layer: norm, rotation, keys and values to pages
 *     tree_attend_paged      per layer: attention of the rows
 *     tree_commit_paged      the rows of an accepted path become cached tokens
 *
 * Requests may share pages that none of them writes: those that are full of
 * cached tokens.  A request writes the page that its last cached token does not
 * fill, and the ones behind it.
 *
 * All the arrays of cs_batch are DEVICE memory, dense, and are read when the
 * stream gets there, so a captured graph can be replayed with new lengths.
 * Their contents cannot be checked by the host.  Whatever they hold, no call
 * reads or writes outside the buffers it was given: a table entry or slot
 * outside the pool is left out (its keys are not seen, its rows not written).
 * max_rows only chooses between kernels: no results but for rounding depend on
 * it.  Calls may overlap where one does not write what another uses, and what a
 * call writes must not overlap what it reads but where that is allowed below.
 * A batch has at most 4,096 requests, and rows x (H_q + 2 H_kv) below 2^31
 * (CS_ERR_UNSUPPORTED beyond); the pool's two buffers are aligned to 16 bytes. */
typedef struct {
  void* k_pages;               /* DEVICE [n_pages][L][H_kv][P][D] */
  void* v_pages;               /* the same */
  int64_t n_pages;             /* n_pages x P < 2^31 */
} cs_page_pool;

typedef struct {
  int32_t n_requests;          /* B >= 0 */
  int32_t n_rows;              /* rows the row arrays have room for, >= row_start[B] */
  int32_t max_blocks;          /* entries of a block table's row */
  int32_t mask_words;          /* 64-bit words of a mask's row */
  int32_t max_rows;            /* the most rows one request is expected to have; 0: n_rows */
  const int32_t* cached_len;   /* [B] */
  int32_t* row_start;          /* [B + 1] */
  int32_t* block_table;        /* [B][max_blocks] */
  int32_t* slot;               /* [n_rows] page x P + offset of every row; -1: none */
  int32_t* coords;             /* [n_rows][3] (t, h, w) of every row */
  uint64_t* tree_mask;         /* [n_rows][mask_words]: bit w of row i: row i sees row w of its
                                  request; NULL: a row sees itself and the rows before it */
} cs_batch;

/* Rows of heads: element d of head h of row r is data[r x row_stride +
 * h x head_stride + d] (strides in elements, >= 0), so the slices of a
 * projection's rows are used where they are.                               */
typedef struct {
  void* data;                  /* DEVICE, geometry.dtype */
  int64_t row_stride, head_stride;
} cs_rows;

typedef struct {
  const int32_t* new_len;      /* DEVICE [B] rows of every request, >= 0 */
  const int32_t* n_blocks;     /* DEVICE [B] pages every request holds */
  int32_t* n_blocks_out;       /* DEVICE [B] the same after the step; not n_blocks */
  const int32_t* free_pages;   /* DEVICE [n_free] free pages, taken in order */
  int32_t n_free;
  const int32_t* free_head;    /* DEVICE [1] entries of free_pages already taken */
  int32_t* free_head_out;      /* DEVICE [1] the same after the step; not free_head */
  const int32_t* parent;       /* DEVICE [n_rows] parent of every row in its request's tree, a row
                                  before it, or -1: the cached tokens; NULL: the row before it */
  const int32_t* coord_base;   /* DEVICE [B] coordinate of a request's row 0, or NULL: cached_len */
  int32_t* status;             /* DEVICE [1] CS_PLAN_* flags are added here; the caller clears it */
} cs_page_plan;

enum {
  CS_PLAN_BAD_LENGTH = 1,      /* a length, page count or free_head is negative, the pages held do not
                                  hold the cached tokens, or a token index would reach 2^31 */
  CS_PLAN_TABLE_FULL = 2,      /* a request needs more than max_blocks pages */
  CS_PLAN_POOL_FULL = 4,       /* the free pages do not suffice */
  CS_PLAN_TOO_MANY_ROWS = 8,   /* more than n_rows rows */
  CS_PLAN_MASK_TOO_SMALL = 16, /* a request has more than 64 x mask_words rows */
  CS_PLAN_BAD_PARENT = 32,     /* a parent is neither -1 nor a row before its child: taken for -1 */
  CS_PLAN_BAD_PAGE = 64        /* a page taken from the free list, or a held one that a row of the step
                                  goes to, is outside the pool: used as it is, and left out by the other
                                  calls (pages of cached tokens alone are not looked at) */
};

/* ---------------------------------------------------------------------------
 * batch_plan_pages -- block tables, slots, coordinates and tree masks of a
 * step, from the requests' lengths.
 *
 * Request b needs ceil((cached_len[b] + new_len[b]) / P) pages; what it lacks is
 * taken from the free list, request by request in order, and put behind the
 * pages it holds.  Written: batch->row_start, the new entries of
 * batch->block_table (the others are left as they are), batch->slot,
 * batch->coords (all three axes coord_base[b] + the row's depth, its number of
 * ancestors), batch->tree_mask when it is not NULL (the row itself and its
 * ancestors), n_blocks_out, free_head_out and, when something is wrong, status.
 * Rows behind the last request's get slot -1; their coordinates and masks are
 * left as they are.  A step that cannot be planned (the flags up to
 * CS_PLAN_MASK_TOO_SMALL) takes nothing: row_start is zero throughout, so that
 * the step's other calls find no rows, every slot is -1, and n_blocks_out and
 * free_head_out repeat what was there.
 *
 *   page      geometry of a page (only n_tokens matters beside its checks)
 *   n_pages   pages of the pool
 *   batch     every pointer but tree_mask is required (where B, n_rows are not 0)
 * Errors: CS_ERR_INVALID_ARGUMENT for a bad geometry, size or NULL pointer, or
 * for plan->parent without batch->tree_mask.                               */
cs_status batch_plan_pages(const cs_geometry* page, int64_t n_pages, const cs_batch* batch,
                           const cs_page_plan* plan, void* stream);

/* ---------------------------------------------------------------------------
 * qk_norm_rope_append -- RMS norm of every query and key head, the rotation of
 * Eq. 2 at the row's coordinates, and the rows' keys and values put into their
 * pages, in one pass over the rows.
 *
 *   y = x / sqrt(mean_d x_d^2 + eps) * weight      (norm, per head; the squares are float32)
 *   (y_i, y_{i+D/2}) turned by coords[axis(i)] * theta_i   (as everywhere here)
 * Queries go to q_out, keys and (unchanged) values to slot[r] of the pool in
 * `layer`.  Everything between is float32 (the angles float64), rounded once.
 * Rows whose slot is outside the pool write no key and no value; a row's query
 * is written whatever its slot is, for the rows below row_start[B] alone.
 * Two rows with one slot leave a mixture of both there.
 *
 *   q, k, v            [n_rows][H_q | H_kv | H_kv][D]
 *   q_weight, k_weight DEVICE [D], geometry.dtype, or NULL: that side is
 *                      rotated without a norm
 *   eps                finite, >= 0
 *   q_out              [n_rows][H_q][D]; may be q itself (data and strides)
 * Uses batch->row_start, slot and coords.
 * Errors: CS_ERR_INVALID_ARGUMENT, CS_ERR_UNSUPPORTED (grid), CS_ERR_HIP.    */
cs_status qk_norm_rope_append(const cs_geometry* page, const cs_page_pool* pool, int32_t layer,
                              const cs_batch* batch, const cs_rows* q, const cs_rows* k, const cs_rows* v,
                              const void* q_weight, const void* k_weight, float eps,
                              const cs_rows* q_out, void* stream);

/* ---------------------------------------------------------------------------
 * tree_attend_paged -- attention (Eq. 1) of the step's rows over their
 * requests' pages, the step's own keys and values (already appended) included.
 *
 *   out[r][h] = softmax_j(q[r][h] . K[j] / sqrt(D)) V[j]
 * over the keys j that row i of request b sees: every j < cached_len[b], and
 * j = cached_len[b] + w for the rows w < new_len[b] that its mask names (w <= i
 * without a mask).  lse[r][h] = log(sum_j exp(q . K[j] / sqrt(D))).  Softmax and
 * accumulation run in float32; in bf16 the probabilities are rounded to bf16 for
 * the product with the values (the sum in the quotient and lse is of the
 * unrounded ones), and the parts of a row that several workgroups work on may be
 * kept in fp16 with an exponent for each row.  Sums of products with values are
 * divided at the end: |V| x keys up to 2^122 is safe.  A row that sees no key gets 0 and -inf.
 * Keys and values that a row does not see do not matter, infinities and NaN
 * included.  Of what it sees, a score of NaN or +inf makes the row NaN, lse too, and
 * so do scores of -inf where there are no others; beside others they are
 * keys of weight 0.  An element of a value that is infinite or NaN leaves that
 * element of out infinite or NaN.  Rows of out and lse at row_start[B] and behind it are left as
 * they are.  Results do not depend on timing.
 *
 *   q, out     [n_rows][H_q][D]; out may be q itself (data and strides)
 *   lse        DEVICE float32 [n_rows][H_q], or NULL
 *   workspace  DEVICE, >= tree_attend_paged_workspace() bytes, the same for every
 *              batch with rows of a geometry (none without); no initial
 *              contents needed; calls that overlap need one each
 * Uses batch->cached_len, row_start, block_table and tree_mask.
 * Errors: CS_ERR_INVALID_ARGUMENT, CS_ERR_WORKSPACE_TOO_SMALL,
 * CS_ERR_UNSUPPORTED (grid; max_blocks x P above 2^31 - 65,536), CS_ERR_HIP. */
cs_status tree_attend_paged_workspace(const cs_geometry* page, const cs_batch* batch, size_t* bytes);
cs_status tree_attend_paged(const cs_geometry* page, const cs_page_pool* pool, int32_t layer,
                            const cs_batch* batch, const cs_rows* q, const cs_rows* out, float* lse,
                            void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * tree_commit_paged -- the rows of an accepted path become cached tokens.
 *
 * For every request b and i < n_accepted[b], row accepted[b][i] of the request
 * (its token cached_len[b] + accepted[b][i]) moves to token cached_len[b] + i,
 * keys and values, in the layers [layer_begin, layer_end), and cached_len_out[b]
 * = cached_len[b] + n_accepted[b].  The keys' rotation stays, so accepted[b] is to
 * be a path: a row whose parent is the cached tokens, then a child of each row
 * before it (of a question, the first rows).  Then entry i has the coordinate of
 * depth i, which is the next one.  That it is a path is not checked: other rows
 * move as they are, with keys turned by the coordinates they were appended
 * with.  What is checked is that rows ascend: the list ends before the first entry
 * that does not or is no row of the request (then cached_len_out counts the
 * entries before it).  Every other token is left as it is.  Requests that share
 * a page they write race.
 *
 *   accepted        DEVICE int32 [B][max_accept]
 *   n_accepted      DEVICE int32 [B]
 *   cached_len_out  DEVICE int32 [B], not batch->cached_len; or NULL
 * Uses batch->cached_len, row_start and block_table.
 * Errors: CS_ERR_INVALID_ARGUMENT, CS_ERR_UNSUPPORTED (grid), CS_ERR_HIP.    */
cs_status tree_commit_paged(const cs_geometry* page, const cs_page_pool* pool, int32_t layer_begin,
                            int32_t layer_end, const cs_batch* batch, const int32_t* accepted,
                            int32_t max_accept, const int32_t* n_accepted, int32_t* cached_len_out,
                            void* stream);

/* Thread-local text describing the last non-OK status on this thread. */
const char* cs_last_error(void);

/* ---------------------------------------------------------------------------
 * Kernel tracing (measurement aid, off by default).
 * While enabled, every kernel the library launches carries a pair of
 * hipEvents that its own dispatch stamps at the kernel's start and end
 * (hipExtLaunchKernel: no extra packets on the stream, so tracing leaves the
 * timeline as it is).  cs_trace_collect() synchronises those events and
 * accumulates, per kernel name, the number of launches and their total
 * duration.  The trace state is shared by all threads and guarded by a
 * lock; a kernel's events reach the collector once its launch is enqueued,
 * so a collect running beside launches on other threads never waits on a
 * half-enqueued pair.  A collect that fails keeps the launches it had not
 * reached.
 *
 * cs_trace_only(names) narrows tracing to the kernels named in a
 * comma-separated list (NULL or "": every kernel); the list is copied.  The
 * events cost the GPU a few microseconds per traced launch, so a caller that
 * needs one kernel's durations can leave the others untraced. */
cs_status cs_trace_enable(int32_t on);
cs_status cs_trace_only(const char* names);
cs_status cs_trace_collect(void);
int32_t cs_trace_count(void);
cs_status cs_trace_get(int32_t i, const char** name, int64_t* launches,
                       double* total_ms);
void cs_trace_reset(void);

#ifdef __cplusplus
}
#endif

#endif /* CHRONOSTITCH_H */
