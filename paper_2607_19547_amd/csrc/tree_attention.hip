// Attention of a batch's rows over their requests' pages (Eq. 1): a single
// token, a tree of drafted tokens or a question's tokens per request.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "tree_attention.h"

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
  if (a.lse && tid == 0) a.lse[(int64_t)r * a.Hq + h] = !any ? -INFINITY : l == 0.f ? __builtin_nanf("") : m + logf(l);  // (0: only scores of -inf)
}

// ============================================================== matrix-instruction path
// Head dims that fill whole 64-byte pieces of a row (bf16: multiples of 32,
// float32: of 16, see has_instance), pages of a multiple of 16 tokens.
//
// A unit is one request, one KV head and a row tile of 16 NR query vectors
// (its rows x the G query heads that share the KV head).  A wavefront takes a
// tile of kTile keys: with the keys as the rows of the matrix instruction,
//   S^T = K Q^T       each lane holds 4 or 8 scores of ONE query vector
//   O^T += V^T P^T    with those scores' probabilities as the operand as they are
// since the order of the keys inside a product is free: lane group g = lane / 16
// holds keys 4 g .. 4 g + 3 of each 16, and loads those rows of V.  K and V go
// from memory straight into the operands' registers (a row's pieces of 16
// bytes belong to one lane); only V's 16-bit elements have to be paired by key,
// four byte permutes per product.  No LDS and no barrier in the loop, so a
// wavefront's loads run ahead of its arithmetic: while a tile is worked on, the
// next one's keys are in flight from the end of its scores on, and its values
// from the end of its products on.
//
// Bound by memory for few rows (every key and value is read once per row tile):
// 64 requests of 8,000 tokens, one row, 16 / 2 heads of 128 in bf16, 91 us with the
// merge, 5.8 TB/s.  A short launch is bound by its chain of loads and by fetching
// its instructions (8,211 tokens: 9.0 us, of them 5 without any key tile).  Float32
// with many rows is bound by the matrix instructions (20,000 tokens, 800 query
// vectors a KV head: 155 us, 106 TFLOP/s).
// The work, in key tiles over all units, is cut into equal runs, one for each
// workgroup, whatever the requests' lengths: a run ends inside a unit or spans
// several (a unit is a row tile, or two of a long chain: see Units).  A row tile
// that one workgroup has whole is finished there; of the others each piece leaves
// a partial (O, max, sum), and tree_combine merges them in key order, so results do
// not depend on timing.  Every workgroup finds its run from the lengths alone (one
// load and a prefix sum).
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
// The running maximum may grow by 2^5 before the accumulators are rescaled:
// probabilities stay far inside the range of both types.
constexpr float kRescaleLog2 = 5.f;

// Keys and values are fetched with the non-temporal hint (ONCE) where one row
// tile reads them all and they would not stay in the 256 MB cache anyway: 32
// requests of up to 16,384 tokens 50.8 -> 45.2 us, 64 of 8,000 103 -> 91 (5.8
// TB/s); 8,000 tokens in all 13.6 -> 14.2, so short batches go without.
constexpr double kOnceBytes = 24e6;
template <int BYTES>
struct Words {
  uint32_t w[BYTES / 4];
};
template <int BYTES, bool ONCE>
__device__ __forceinline__ Words<BYTES> load_words(__amdgpu_buffer_rsrc_t r, int off) {
  Words<BYTES> o;
  if constexpr (BYTES == 16) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, ONCE ? kNonTemporal : 0);
    for (int i = 0; i < 4; ++i) o.w[i] = v[i];
  } else if constexpr (BYTES == 12) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b96(r, off, 0, ONCE ? kNonTemporal : 0);
    for (int i = 0; i < 3; ++i) o.w[i] = v[i];
  } else if constexpr (BYTES == 8) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, ONCE ? kNonTemporal : 0);
    for (int i = 0; i < 2; ++i) o.w[i] = v[i];
  } else {
    o.w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, ONCE ? kNonTemporal : 0);
  }
  return o;
}

// Over the four lanes that hold one query vector: l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float group_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float group_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The place of a run's next key tile, `off` of request b with `left` to go, past
// requests' ends and the empty ends of pairs; n is 0 behind the last.  (A loop of
// its own: two ways back to the loop over the pieces cost 34 registers.)
template <bool PAIRS>
__device__ __forceinline__ Place next_place(const SplitArgs& a, int* b, int64_t* off, int64_t* left, Request* q) {
  Place x;
  x.n = 0;
#pragma unroll 1
  while (*b < a.t.B && *left > 0) {
    *q = load_request_scalar(a.t, *b);
    const Units units = unit_sizes<PAIRS>(a, *q);
    if (*off >= request_tiles(a, units)) {
      *off = 0;
      ++*b;
      continue;
    }
    x = place_at<PAIRS>(a, *q, units, *off);
    if (x.n) break;
    *off += x.t0;
    *left -= x.t0;
  }
  return x;
}

template <typename E, int D, int NR, bool ONCE>
__global__ __launch_bounds__(kThreads, 2) void tree_attend(const SplitArgs) {
  constexpr bool kBf16 = sizeof(E) == 2;
  constexpr int SUB = kBf16 ? 2 : 1;             // 16-key pieces of a tile
  constexpr int KT = 16 * SUB;
  constexpr int kRowB = D * (int)sizeof(E);
  constexpr int KS = kRowB / 64;                 // 64-byte pieces of a row
  constexpr int NB = kRowB > 256 ? kRowB / 256 : 1;  // blocks of a row that 16 lanes load
  constexpr int VB = kRowB / 16 / NB;            // bytes of a V row a lane loads per block
  constexpr int VW = VB / (int)sizeof(E);
  constexpr int NO = NB * VW;                    // output tiles: 16 elements x 16 query vectors
  constexpr int RT = 16 * NR;
  constexpr int NS = 4 * SUB;                    // scores of a lane per 16 query vectors
  constexpr int kPad = D + 4;
  static_assert(KS * 64 == kRowB && NO * 16 == D && VB % 4 == 0, "head dim");

  __shared__ float s_o[kWaves * 16 * kPad];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const int ln = lane & 15, lg = lane >> 4;
  // The arguments are read where they are used: a launch is short, and what it
  // spends on moving arguments in and out of scalar registers, and on fetching
  // the instructions that do, is part of its latency.
  typedef const __attribute__((address_space(4))) SplitArgs* ArgPtr;
  const ArgPtr argp = (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
  auto args = [&]() -> SplitArgs {
    ArgPtr p = argp;
    asm volatile("" : "+s"(p));
    return *(const SplitArgs*)p;
  };
  Run run;
  if (!find_run<(NR > 1), (NR > 1)>(args(), blockIdx.x, &run)) return;
  int64_t left = run.end - run.begin, off = run.off;
  int b = run.b;
  bool first_seg = true;

  while (left > 0) {
    const SplitArgs a = args();
    const TreeArgs& t = a.t;
    Request q;
    const Place place = next_place<(NR > 1)>(a, &b, &off, &left, &q);
    if (!place.n) break;
    const int h = place.h, rt = place.rt, t0 = place.t0, ntile = place.n;
    const int seg = (int)min(left, (int64_t)(ntile - t0));
    const int vectors = q.n * t.G;
    // rows see no key behind their own without a mask, so later tiles are left out
    const int i_last = a.group.div(min(rt * RT + RT, vectors) - 1);
    const int key_end = t.mask ? q.len : min(q.len, q.cached + i_last + 1);
    const int t_end = min(t0 + seg, (key_end + KT - 1) / KT);
    const int t_full = min(t.mask ? q.cached : q.cached + a.group.div(rt * RT) + 1, q.len) / KT;  // tiles before it: every row sees every key

    Words<16> qf[NR][KS];
    int row[NR];  // the lane's row in the request, per 16 query vectors
#pragma unroll
    for (int x = 0; x < NR; ++x) {
      const int qv = min(rt * RT + 16 * x + ln, vectors - 1), i = a.group.div(qv);
      row[x] = i;
      const char* qp = (const char*)t.q + ((int64_t)(q.r0 + i) * t.q_row + (h * t.G + qv - i * t.G) * t.q_head) * (int)sizeof(E);
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[x][k] = *(const Words<16>*)(qp + 64 * k + 16 * lg);
    }

    // Where the 16-key pieces of a tile lie: 16 rows of a page (pages are
    // multiples of 16 tokens), as many of them as the request has; none behind
    // the request's or the run's end.  The page numbers come through the scalar
    // cache, a tile ahead of the loads that need them, so that nothing waits
    // for the values in flight.
    const scalar_ptr pages = (scalar_ptr)(uint64_t)(t.table + (int64_t)b * t.max_blocks);
    const FastDiv page_div = t.page;
    const int64_t plane = ((int64_t)t.layer * t.Hkv + h) * page_div.d * kRowB, page_bytes = t.pool.page_bytes;
    const char *k_plane = t.pool.k + plane, *v_plane = t.pool.v + plane;
    const int n_pages = t.pool.n_pages;
    Words<16> kf[SUB][KS];
    Words<VB> vf[SUB * 4][NB];
    int64_t at[SUB];
    int bytes[SUB], page[SUB];
    auto fetch_pages = [&](int tile) {
#pragma unroll
      for (int s = 0; s < SUB; ++s) page[s] = pages[page_div.div(min(min(tile, t_end - 1) * KT + 16 * s, q.len - 1))];
    };
    auto places = [&](int tile) {
#pragma unroll
      for (int s = 0; s < SUB; ++s) {
        const int key = tile * KT + 16 * s;
        at[s] = page[s] * page_bytes + (int64_t)(key - page_div.div(key) * page_div.d) * kRowB;
        // (no bytes: no address is used)
        bytes[s] = tile < t_end && key < q.len && (unsigned)page[s] < (unsigned)n_pages ? min(q.len - key, 16) * kRowB : 0;
      }
    };
    auto load_k = [&]() {
#pragma unroll
      for (int s = 0; s < SUB; ++s) {
        const auto r = rows_rsrc(k_plane + at[s], bytes[s]);
#pragma unroll
        for (int k = 0; k < KS; ++k) kf[s][k] = load_words<16, ONCE>(r, ln * kRowB + 64 * k + 16 * lg);
      }
    };
    auto load_v = [&]() {
#pragma unroll
      for (int s = 0; s < SUB; ++s) {
        const auto r = rows_rsrc(v_plane + at[s], bytes[s]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int n = 0; n < NB; ++n) vf[4 * s + i][n] = load_words<VB, ONCE>(r, (4 * lg + i) * kRowB + n * 16 * VB + VB * ln);
      }
    };

    const float sc = t.scale * kLog2e;
    f32x4 o[NR][NO];
    float m[NR], l[NR];
    bool seen[NR];  // some key was visible
#pragma unroll
    for (int x = 0; x < NR; ++x) {
      m[x] = -INFINITY;
      l[x] = 0.f;
      seen[x] = false;
#pragma unroll
      for (int e = 0; e < NO; ++e) o[x][e] = f32x4{};
    }

    // value(j, n, w): word w of key j's block n; weight(x, j): of query vector and key
    auto pv = [&](auto value, auto weight, auto add) {
      if constexpr (kBf16) {
        bf16x8 pb[NR];
#pragma unroll
        for (int x = 0; x < NR; ++x)
#pragma unroll
          for (int j = 0; j < 8; ++j) pb[x][j] = (__bf16)weight(x, j);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < VW; ++e) {
            u32x4 va;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              va[j] = __builtin_amdgcn_perm(value(2 * j + 1, n, e / 2), value(2 * j, n, e / 2), e & 1 ? 0x07060302 : 0x05040100);
#pragma unroll
            for (int x = 0; x < NR; ++x)
              add(x, n * VW + e, [&](f32x4 c) {
                return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, va), pb[x], c, 0, 0, 0);
              });
          }
      } else {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < VW; ++e)
#pragma unroll
            for (int x = 0; x < NR; ++x)
              add(x, n * VW + e, [&](f32x4 c) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(value(j, n, e)), weight(x, j), c, 0, 0, 0);
                return c;
              });
      }
    };

    int tile = t0 + wave;
    if (tile < t_end && q.len > 0) {
      fetch_pages(tile);
      places(tile);
      load_k();
      load_v();
      fetch_pages(tile + kWaves);
    }
    // One body for every tile: the masked tiles' extra work is behind a branch,
    // so that their first one finds its instructions fetched (with bodies of
    // their own it cost 3 us).
#pragma unroll 1
    for (; tile < t_end; tile += kWaves) {
      const int key0 = tile * KT;
      f32x4 s[NR][SUB];
#pragma unroll
      for (int x = 0; x < NR; ++x)
#pragma unroll
        for (int y = 0; y < SUB; ++y) {
          s[x][y] = f32x4{};
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            if constexpr (kBf16) {
              s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[y][k]),
                                                                __builtin_bit_cast(bf16x8, qf[x][k]), s[x][y], 0, 0, 0);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                s[x][y] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[y][k].w[e]),
                                                               __uint_as_float(qf[x][k].w[e]), s[x][y], 0, 0, 0);
            }
          }
        }
      bool have[SUB];  // the 16 keys lie in a page of the pool
#pragma unroll
      for (int y = 0; y < SUB; ++y) have[y] = bytes[y] != 0;
      places(tile + kWaves);
      load_k();
      fetch_pages(tile + 2 * kWaves);

      float p[NR][NS];
#pragma unroll
      for (int x = 0; x < NR; ++x)
#pragma unroll
        for (int y = 0; y < SUB; ++y)
#pragma unroll
          for (int i = 0; i < 4; ++i) p[x][4 * y + i] = s[x][y][i];
      bool masked = tile >= t_full;
#pragma unroll
      for (int y = 0; y < SUB; ++y) masked = masked || !have[y];
      uint32_t vis[NR];  // bit 16 y + i: key 16 y + 4 lg + i
      if (masked) {
        const SplitArgs A = args();
        uint32_t there = 0;  // keys of the request that lie in the pool
#pragma unroll
        for (int y = 0; y < SUB; ++y)
          if (have[y]) there |= ((1u << min(max(q.len - key0 - 16 * y, 0), 16)) - 1) << (16 * y);
        const int w0 = key0 - q.cached, w = max(w0, 0);  // new row of the tile's first key
#pragma unroll
        for (int x = 0; x < NR; ++x) {
          uint64_t bits = 0;  // visible rows from w on
          if (A.t.mask) {
            const unsigned long long* mk = A.t.mask + (int64_t)(q.r0 + row[x]) * A.t.words;
            const int j = w >> 6, sft = w & 63;
            if (w0 > -KT && j < A.t.words) bits = mk[j] >> sft;
            if (w0 > -KT && sft && j + 1 < A.t.words) bits |= mk[j + 1] << (64 - sft);
          } else {
            const int n = row[x] - w + 1;
            bits = n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0ull;
          }
          if (w0 < 0) bits = -w0 >= 64 ? ~0ull : bits << -w0 | ((1ull << -w0) - 1);
          vis[x] = (uint32_t)bits & there;
          seen[x] = seen[x] || vis[x];
          vis[x] >>= 4 * lg;
#pragma unroll
          for (int j = 0; j < NS; ++j)
            if (!(vis[x] >> (16 * (j >> 2) + (j & 3)) & 1)) p[x][j] = -INFINITY;
        }
      } else {
#pragma unroll
        for (int x = 0; x < NR; ++x) seen[x] = true;
      }

#pragma unroll
      for (int x = 0; x < NR; ++x) {
        float mx = p[x][0];
#pragma unroll
        for (int j = 1; j < NS; ++j) mx = fmaxf(mx, p[x][j]);
        mx = group_max(mx) * sc;
        const bool grow = mx > m[x] + kRescaleLog2;
        if (__ballot(grow)) {
          const float m_new = grow ? mx : m[x];
          const float alpha = grow ? __builtin_amdgcn_exp2f(m[x] - m_new) : 1.f;
          l[x] *= alpha;
#pragma unroll
          for (int e = 0; e < NO; ++e) o[x][e] *= alpha;
          m[x] = m_new;
        }
        const float ref = m[x] == -INFINITY ? 0.f : m[x];
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          p[x][j] = __builtin_amdgcn_exp2f(fmaf(p[x][j], sc, -ref));
          l[x] += p[x][j];
        }
      }

      // Values that are not finite must not reach rows that do not see them
      // (0 x inf): rare, and only among the step's own rows.  0 x value is NaN
      // where there is one.
      if (masked) {
        float odd = 0.f;
#pragma unroll
        for (int j = 0; j < SUB * 4; ++j)
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int w = 0; w < VB / 4; ++w) {
              const uint32_t v = vf[j][n].w[w];
              if constexpr (kBf16)
                odd = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, v), bf16x2{(__bf16)0.f, (__bf16)0.f}, odd, false);
              else
                odd = fmaf(__uint_as_float(v), 0.f, odd);
            }
        if (__ballot(odd != odd)) {
          // How many values of +inf (or NaN), and of -inf (or NaN), each output
          // element gets from keys that its row sees; those give it the infinity,
          // both of them NaN.  The values themselves become zero.
#pragma unroll 1
          for (int sign = 0; sign < 2; ++sign) {
            auto flag16 = [&](uint32_t v) -> uint32_t {  // 1.0 in bf16 where the element counts
              const bool nan = (v & 0x7f80u) == 0x7f80u && (v & 0x7fu);
              return nan || (v & 0xffffu) == (sign ? 0xff80u : 0x7f80u) ? 0x3f80u : 0u;
            };
            auto flag = [&](uint32_t v) -> uint32_t {
              if constexpr (kBf16) return flag16(v) | flag16(v >> 16) << 16;
              const bool nan = (v & 0x7f800000u) == 0x7f800000u && (v & 0x7fffffu);
              return nan || v == (sign ? 0xff800000u : 0x7f800000u) ? 0x3f800000u : 0u;
            };
            pv([&](int j, int n, int w) { return flag(vf[j][n].w[w]); },
               [&](int x, int j) { return vis[x] >> (16 * (j >> 2) + (j & 3)) & 1 ? 1.f : 0.f; },
               [&](int x, int e, auto mul) {
                 const f32x4 c = mul(f32x4{});
#pragma unroll
                 for (int i = 0; i < 4; ++i)
                   if (c[i] > 0.f) o[x][e][i] += sign ? -INFINITY : INFINITY;
               });
          }
#pragma unroll
          for (int j = 0; j < SUB * 4; ++j)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
              for (int w = 0; w < VB / 4; ++w) {
                uint32_t& v = vf[j][n].w[w];
                if (kBf16) {
                  if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
                  if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
                } else if ((v & 0x7f800000u) == 0x7f800000u) {
                  v = 0;
                }
              }
        }
      }
      pv([&](int j, int n, int w) { return vf[j][n].w[w]; }, [&](int x, int j) { return p[x][j]; },
         [&](int x, int e, auto mul) { o[x][e] = mul(o[x][e]); });
      load_v();
    }

    // The wavefronts' results, 16 query vectors at a time, merged through LDS.
    const int64_t slot = 2 * (int64_t)run.w + (t0 == 0);  // (of a run's pieces, its first begins inside a row tile, its last ends there)
#pragma unroll
    for (int x = 0; x < NR; ++x) {
      float lt = group_sum(l[x]);
      if (seen[x] && m[x] == -INFINITY) {
        m[x] = kOnlyMinusInf;
        lt += 1.f;
      }
      if (x > 0 || !first_seg) __syncthreads();  // the previous 16 have been read
      if (lg == 0) {
        s_m[wave][ln] = m[x];
        s_l[wave][ln] = lt;
      }
      float* to = s_o + (wave * 16 + ln) * kPad + VW * 4 * lg;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < VW; ++e) to[n * 16 * VW + VW * i + e] = o[x][n * VW + e][i];
      __syncthreads();
      const SplitArgs A = args();
      const int r = tid >> 4, c = tid & 15;  // 16 threads a query vector, D / 16 elements each
      const int qv = rt * RT + 16 * x + r;
      if (qv < q.n * A.t.G) {
        constexpr int C = D / 16;
        float2 ml[kWaves];
        float v[kWaves][C];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          ml[w] = make_float2(s_m[w][r], s_l[w][r]);
#pragma unroll
          for (int e = 0; e < C; ++e) v[w][e] = s_o[(w * 16 + r) * kPad + c * C + e];
        }
        Merge<C> mg;
        mg.add(ml, v);
        if (seg == ntile) {
          const int i = A.group.div(qv), head = h * A.t.G + qv - i * A.t.G;
          const float by = mg.scale();
          E* op = (E*)A.t.out + (int64_t)(q.r0 + i) * A.t.o_row + head * A.t.o_head + c * C;
          if constexpr (kBf16) {
#pragma unroll
            for (int e = 0; e < C; e += 2) *(uint32_t*)(op + e) = pack_bf16x2(mg.acc[e] * by, mg.acc[e + 1] * by);
          } else {
#pragma unroll
            for (int e = 0; e < C; ++e) op[e] = mg.acc[e] * by;
          }
          if (A.t.lse && c == 0) A.t.lse[(int64_t)(q.r0 + i) * A.t.Hq + head] = mg.lse();
        } else {
          const int64_t pr = slot * RT + 16 * x + r;
          float* pp = A.part + pr * D + c * C;
#pragma unroll
          for (int e = 0; e < C; ++e) pp[e] = mg.acc[e];
          if (c == 0) *(float2*)(A.part_ml + pr * 2) = make_float2(mg.m, mg.sum);
        }
      }
    }
    first_seg = false;
    left -= seg;
    off += seg;
  }
}

// Merges the pieces of a unit that several workgroups worked on, in key order.
// Workgroup w has the border between runs w and w + 1.  The borders inside a
// unit, and blockIdx.y, share its query vectors.  32 lanes hold a vector's
// elements.  A unit of many pieces (few requests, long caches) has all eight
// groups of 32 lanes take pieces of one vector in turn; with few pieces a
// group takes a vector for itself.  The launch is a chain of loads from other
// XCDs' results, about 1 us each: lengths, then a round of pieces at a time,
// outputs and statistics together.
constexpr int kGroups = kThreads / 32;
constexpr int kManyPieces = 16;
constexpr int kRound = 8;  // pieces of a round
template <typename E, int D, bool PAIRS>
__global__ __launch_bounds__(kThreads) void tree_combine(const SplitArgs a) {
  constexpr int C = (D + 31) / 32;  // elements a lane holds
  __shared__ float s_o[kGroups][32 * C], s_m[kGroups], s_l[kGroups];
  const TreeArgs& t = a.t;
  const int w1 = blockIdx.x + 1;
  Run run;
  if (!find_run<PAIRS>(a, w1, &run)) return;
  const Request q = load_request_scalar(t, run.b);
  const Place at = place_at<PAIRS>(a, q, unit_sizes<PAIRS>(a, q), run.off);
  if (at.t0 == 0 || at.n == 0) return;  // the border lies between row tiles
  const int h = at.h, rt = at.rt;
  const int64_t len = run_length(a, run.total), unit0 = run.begin - at.t0, unit1 = unit0 + at.n;
  const int w0 = quotient(unit0, len), w_last = quotient(unit1 - 1, len);  // the runs of its first and last tile
  const int pieces = w_last - w0 + 1, borders = pieces - 1;
  const int vectors = min(1 << a.row_bits, q.n * t.G - (rt << a.row_bits));
  const int grp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool many = pieces > kManyPieces;
  const int step = many ? kGroups : 1, x0 = many ? grp : 0;
  // (many: every group has the same vectors, so the barriers below match)
  const int lot = w1 - 1 - w0 + borders * (many ? blockIdx.y : grp + kGroups * blockIdx.y);
  for (int r = lot; r < vectors; r += borders * gridDim.y * (many ? 1 : kGroups)) {
    Merge<C> mg;
    for (int c = x0; c < pieces; c += kRound * step) {
      float2 ml[kRound];
      float v[kRound][C];
#pragma unroll
      for (int y = 0; y < kRound; ++y) {
        const int x = min(c + y * step, pieces - 1);
        const int64_t at = ((2 * (int64_t)(w0 + x) + (x == 0)) << a.row_bits) + r;
        ml[y] = *(const float2*)(a.part_ml + at * 2);
        const float* pp = a.part + at * D + lane * C;
#pragma unroll
        for (int e = 0; e < C; ++e) v[y][e] = D % 32 == 0 || lane * C + e < D ? pp[e] : 0.f;
      }
#pragma unroll
      for (int y = 0; y < kRound; ++y)
        if (c + y * step >= pieces) ml[y] = make_float2(-INFINITY, 0.f);
      mg.add(ml, v);
    }
    if (many) {
      __syncthreads();  // the previous vector has been read
      if (lane == 0) {
        s_m[grp] = mg.m;
        s_l[grp] = mg.sum;
      }
#pragma unroll
      for (int e = 0; e < C; ++e) s_o[grp][lane * C + e] = mg.acc[e];
      __syncthreads();
      if (grp) continue;
      float2 ml[kGroups];
      float v[kGroups][C];
#pragma unroll
      for (int x = 0; x < kGroups; ++x) {
        ml[x] = make_float2(s_m[x], s_l[x]);
#pragma unroll
        for (int e = 0; e < C; ++e) v[x][e] = s_o[x][lane * C + e];
      }
      mg = Merge<C>();
      mg.add(ml, v);
    }
    const int qv = (rt << a.row_bits) + r, i = a.group.div(qv), head = h * t.G + qv - i * t.G;
    const float inv = mg.scale();
    E* op = (E*)t.out + (q.r0 + i) * t.o_row + head * t.o_head + lane * C;
#pragma unroll
    for (int e = 0; e < C; ++e)
      if (D % 32 == 0 || lane * C + e < D) put_elem(op + e, mg.acc[e] * inv);
    if (t.lse && lane == 0) t.lse[(int64_t)(q.r0 + i) * t.Hq + head] = mg.lse();
  }
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
  t.q = q.data;
  t.out = out.data;
  t.lse = lse;
  t.q_row = q.row_stride;
  t.q_head = q.head_stride;
  t.o_row = out.row_stride;
  t.o_head = out.head_stride;
  t.cached = b.cached_len;
  t.row_start = b.row_start;
  t.table = b.block_table;
  t.mask = (const unsigned long long*)b.tree_mask;
  t.pool = pool_view(g, pool);
  t.page = fast_div((int)g.T);
  t.B = b.n_requests;
  t.n_rows = b.n_rows;
  t.max_blocks = b.max_blocks;
  t.words = b.mask_words;
  t.layer = layer;
  t.Hq = g.Hq;
  t.Hkv = g.Hkv;
  t.G = g.G;
  t.D = g.D;
  t.scale = 1.f / sqrtf((float)g.D);
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
