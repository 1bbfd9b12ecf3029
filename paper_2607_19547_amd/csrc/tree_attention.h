// Shared by the sources of the batch attention: its arguments and how its work is cut.
#pragma once

#include <math.h>

#include <algorithm>

#include "packed.h"

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

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Request load_request(const TreeArgs& a, int b) {
  return request_of(a.row_start[b], a.row_start[b + 1], a.cached[b], a.n_rows, (int64_t)a.max_blocks * a.page.d);
}
// Arrays that no kernel of the call writes, at places that the whole wavefront
// shares: through the scalar cache.
typedef const __attribute__((address_space(4))) int32_t* scalar_ptr;
__device__ __forceinline__ Request load_request_scalar(const TreeArgs& a, int b) {
  const scalar_ptr rs = (scalar_ptr)(uint64_t)a.row_start, c = (scalar_ptr)(uint64_t)a.cached;
  return request_of(rs[b], rs[b + 1], c[b], a.n_rows, (int64_t)a.max_blocks * a.page.d);
}

// Whether row i of a request sees its new row w (w >= 0).
__device__ __forceinline__ bool sees(const TreeArgs& a, const Request& q, int i, int w) {
  if (!a.mask) return w <= i;
  if (w >> 6 >= a.words) return false;
  return (a.mask[(int64_t)(q.r0 + i) * a.words + (w >> 6)] >> (w & 63)) & 1;
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct SplitArgs {
  static constexpr bool kMemory = false;
  TreeArgs t;
  float* part;      // [2 workgroups][row tile][D] unnormalised partial outputs
  float* part_ml;   // [2 workgroups][row tile][2] their maximum (log2 units) and sum
  int min_tiles;    // key tiles of a run at least, where the units are that long
  FastDiv units;    // division by the units that there are about: the rows shared out evenly
  int row_bits;     // a row tile has 2^row_bits query vectors
  int tile_bits;    // a key tile has 2^tile_bits keys
  int run_bits;     // 2^run_bits runs at most
  int by_xcd;       // runs in a row on one XCD
  FastDiv group;    // division by G
};

// Memories whose first pages are packed, and of which rows see a span
// (tree_attend_packed).
struct MemoryArgs : SplitArgs {
  static constexpr bool kMemory = true;
  PackedView packed;
  const int32_t* blocks;  // packed pages of every request, or null
  int sinks, window;      // window 0: every key is seen
  int paged_bits;         // a key tile of ordinary pages counts as 2^paged_bits packed ones in the cutting of the work
  int unit_tiles;         // and a unit's start and end as that many
};
// Keys of a request that lie in packed pages: whole pages of cached tokens.
// (SCALAR: of a request that the whole wavefront shares)
template <bool SCALAR = true>
__device__ __forceinline__ int packed_keys(const MemoryArgs& a, const Request& q, int b) {
  if (!a.blocks) return 0;
  int n;
  if constexpr (SCALAR) n = ((scalar_ptr)(uint64_t)a.blocks)[b];
  else n = a.blocks[b];
  return min(min(max(n, 0), a.t.page.div(q.cached)), a.t.max_blocks) * a.t.page.d;
}
// Whether a key of the table lies in a page of its pool.
__device__ __forceinline__ bool in_pool(const MemoryArgs& a, int b, int key, int packed) {
  const int32_t pg = a.t.table[(int64_t)b * a.t.max_blocks + a.t.page.div(key)];
  return (unsigned)pg < (unsigned)(key < packed ? a.packed.n_pages : a.t.pool.n_pages);
}
constexpr int kFewTileBits = 5, kWideTileBits = 6;  // key tiles of 32 (a block of values) and of 64 keys
// What a row tile (rows [i0, i1]) leaves out between the sinks and its rows'
// windows, in whole key tiles of 2^BITS: tile t of its work is key tile t, or t + skip
// from `sinks` on.  Keys below `low`, and from `high` on, are hidden from no row of it
// (but for rows among the step's own keys, which are masked in any case).
struct Span {
  int sinks, skip, low, high;
  __device__ __forceinline__ int tile(int t) const { return t >= sinks ? t + skip : t; }
  // of the tiles that the work has, those before key tile `key_tile`
  __device__ __forceinline__ int before(int key_tile) const { return key_tile <= sinks ? key_tile : max(key_tile - skip, sinks); }
};
template <int BITS>
__device__ __forceinline__ Span span_of(const MemoryArgs& a, const Request& q, int i0, int i1) {
  Span s = {0, 0, 0x7fffffff, 0};
  if (!a.window) return s;
  // the first row's window begins here, and the last one's (a row of a mask sees 0 to n rows)
  const int64_t first = (int64_t)q.cached + (a.t.mask ? 0 : i0 + 1) - a.window;
  const int64_t last = (int64_t)q.cached + (a.t.mask ? q.n : i1 + 1) - a.window;
  s.sinks = (int)(((int64_t)min(a.sinks, q.len) + (1 << BITS) - 1) >> BITS);
  s.skip = max((int)(min(max(first, (int64_t)0), (int64_t)q.len) >> BITS) - s.sinks, 0);
  s.low = min(a.sinks, q.cached);
  s.high = (int)min(max(last, (int64_t)0), (int64_t)0x7fffffff);
  return s;
}
// The keys [lo, hi) that the window hides from row i of a request.
struct Hidden {
  int lo, hi;
  // bit w: key k0 + w, of `n` <= 64 keys
  __device__ __forceinline__ uint64_t bits(int k0, int n) const {
    const int a = min(max((int64_t)lo - k0, (int64_t)0), (int64_t)n), b = min(max((int64_t)hi - k0, (int64_t)0), (int64_t)n);
    if (a >= b) return 0;
    const uint64_t below = b == 64 ? ~0ull : (1ull << b) - 1;
    return below & ~((1ull << a) - 1);  // (a < b <= 64)
  }
};
__device__ __forceinline__ Hidden hidden_keys(const MemoryArgs& a, const Request& q, int i) {
  if (!a.window) return {0x7fffffff, 0};
  int64_t lo = a.sinks, hi = (int64_t)q.cached + i + 1 - a.window;
  if (a.t.mask) {
    // the row's visible rows, in order: word by word
    const unsigned long long* mk = a.t.mask + (int64_t)(q.r0 + i) * a.t.words;
    const int words = min(a.t.words, (q.n + 63) >> 6);
    auto word = [&](int w) -> uint64_t {
      const int n = q.n - 64 * w;
      return mk[w] & (n >= 64 ? ~0ull : (1ull << n) - 1);
    };
    int seen = 0;
#pragma unroll 1
    for (int w = 0; w < words; ++w) seen += __popcll(word(w));
    auto nth = [&](int64_t n) -> int64_t {  // place of the n-th (from 0) of them; behind all keys if there are not so many
      if (n >= seen) return 0x7fffffff;
#pragma unroll 1
      for (int w = 0; w < words; ++w) {
        uint64_t x = word(w);
        const int c = __popcll(x);
        if (n < c) {
#pragma unroll 1
          for (; n > 0; --n) x &= x - 1;
          return 64 * w + __builtin_ctzll(x);
        }
        n -= c;
      }
      return 0x7fffffff;
    };
    if (lo > q.cached) lo = q.cached + nth(lo - q.cached);
    hi = seen <= a.window ? (int64_t)q.cached + seen - a.window : q.cached + nth(seen - a.window);
  }
  return {(int)min(lo, (int64_t)0x7fffffff), (int)min(max(hi, (int64_t)0), (int64_t)0x7fffffff)};
}

constexpr int kNonTemporal = 2;  // the buffer loads' cache policy bit

__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
  return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) |
                   (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}
// A request's units for one KV head: `units` of them, `ntile` key tiles long each.
// Mostly a unit is one of the nrt row tiles.  Where the rows are a chain, later
// row tiles see more keys.  Row tiles p and nrt - 1 - p together see about as many
// for every p, so that there such a pair is a unit, as long as any pair can be
// (the few tiles that a pair has less stay empty), if that is less in all and
// there is enough to do to be worth the merges (kPairTiles).
// Tiles for each run, if all requests are alike, from which on chains' row tiles are
// paired.  Measured (us without / with pairs; bf16 x 128, 16 / 2 heads, no cache): 1,000
// rows (4 tiles) 29 / 39, 2,000 (16) 50 / 55, 4,000 (62) 130 / 108, 8,000 (246) 402 / 292.
// Not with row tiles of 16, which many rows have only where there is little to do: the
// code alone cost a single row of 8,000 tokens 0.4 us of 13.8.
constexpr int kPairTiles = 20;
struct Units {
  int nrt, units, ntile;
};
__device__ __forceinline__ int key_tiles(const SplitArgs& a, uint32_t keys) {
  return max((int)((keys + (1 << a.tile_bits) - 1) >> a.tile_bits), 1);
}
template <bool PAIRS, bool SCALAR = true, class A>
__device__ __forceinline__ Units unit_sizes(const A& a, const Request& q, int b) {
  Units s;
  s.units = s.nrt = (int)(((int64_t)q.n * a.t.G + (1 << a.row_bits) - 1) >> a.row_bits);
  s.ntile = key_tiles(a, q.len);
  bool whole = true;  // row tiles see everything before them (and are to be paired)
  if constexpr (A::kMemory) {
    int packed = packed_keys<SCALAR>(a, q, b) >> a.tile_bits;
    if (a.window) {
      // the sinks, and as many keys as the windows of a row tile's rows cover (as many more as it has rows)
      const int rows = a.t.mask ? q.n : min(q.n, (int)a.group.div((1 << a.row_bits) - 1) + 2);
      const int64_t keys = (int64_t)a.window + rows, tiles = (int64_t)min(a.sinks, q.len) + (1 << a.tile_bits) - 1 >> a.tile_bits;
      s.ntile = (int)min((int64_t)s.ntile, tiles + (keys + (2 << a.tile_bits) >> a.tile_bits));
      whole = false;
      // (later row tiles leave out more: the last has the fewest packed tiles)
      const int i0 = s.nrt ? a.group.div((s.nrt - 1) << a.row_bits) : 0;
      packed = a.tile_bits == kWideTileBits ? span_of<kWideTileBits>(a, q, i0, i0).before(packed) : span_of<kFewTileBits>(a, q, i0, i0).before(packed);
    }
    packed = min(packed, s.ntile);
    if (a.paged_bits) whole = false;  // (a pair's tiles count as one each)
    s.ntile = (int)min(packed + ((int64_t)(s.ntile - packed) << a.paged_bits), (int64_t)1 << 29);
  }
  if (PAIRS && whole && !a.t.mask && s.nrt > 1) {
    // the keys of both: the last rows of p and nrt - 1 - p are, added up, at most n + 2 row tiles' rows
    const int64_t keys = 2 * (int64_t)q.cached + 2 + q.n + a.group.div(2 << a.row_bits);
    const int pair = (int)min((keys + (2 << a.tile_bits) - 2) >> a.tile_bits, 2 * (int64_t)s.ntile), pairs = (s.nrt + 1) >> 1;
    const int64_t tiles = (int64_t)s.ntile * s.nrt;
    if ((int64_t)pair * pairs < tiles && (double)tiles * a.t.Hkv * a.t.B >= (double)(kPairTiles << a.run_bits)) {
      s.units = pairs;
      s.ntile = pair;
    }
  }
  if constexpr (A::kMemory) s.ntile += a.unit_tiles;
  return s;
}
__device__ __forceinline__ int64_t request_tiles(const SplitArgs& a, const Units& s) {
  return (int64_t)a.t.Hkv * s.units * s.ntile;
}
// x / d for 0 <= x < 2^53, d > 0 and a quotient below 2^31.
__device__ __forceinline__ int quotient(int64_t x, int64_t d) {
  const int u = (int)((double)x / (double)d);  // at most one too large, by rounding up
  return u * d > x ? u - 1 : u;
}
// Where the key tile at `off` of a request lies: the KV head, the row tile, the
// key tile, and the row tile's key tiles; in the empty end of a pair n is 0 and t0
// the tiles that are left of it.
struct Place {
  int h, rt, t0, n;
};
template <bool PAIRS, class A>
__device__ __forceinline__ Place place_at(const A& a, const Request& q, const Units& s, int64_t off) {
  const int u = uniform(quotient(off, s.ntile));
  Place x;
  x.t0 = uniform((int)(off - (int64_t)u * s.ntile));
  x.h = s.units == 1 ? u : uniform(u / s.units);
  x.rt = u - x.h * s.units;
  x.n = s.ntile;
  if constexpr (A::kMemory) {
    x.n -= a.unit_tiles;
    if (x.t0 >= x.n && !(PAIRS && s.units != s.nrt)) {
      x.n = 0;
      x.t0 = s.ntile - x.t0;
    }
  }
  if (PAIRS && s.units != s.nrt) {
    const int vectors = q.n * a.t.G;
    auto tiles = [&](int rt) {
      return key_tiles(a, min((uint32_t)q.len, (uint32_t)q.cached + a.group.div(min((uint32_t)(rt + 1) << a.row_bits, (uint32_t)vectors) - 1) + 1));
    };
    x.n = tiles(x.rt);
    if (x.t0 >= x.n) {
      const int other = s.nrt - 1 - x.rt, t0 = x.t0 - x.n;
      x.n = other > x.rt ? tiles(other) : 0;
      if (t0 < x.n) {
        x.rt = other;
        x.t0 = t0;
      } else {
        x.n = 0;
        x.t0 = s.ntile - x.t0;
      }
    }
  }
  return x;
}
// Key tiles of a run: the same for all, so that run w is [w x len, (w + 1) x len).
// A run of min_tiles pays for what its unit costs beside the tiles; where units
// are shorter than that, one costs as much by itself, and a run has one of them.
__device__ __forceinline__ int64_t run_length(const SplitArgs& a, int64_t total) {
  int at_least = a.min_tiles;
  if (total < (int64_t)a.min_tiles * a.units.d) at_least = a.units.div((int)total + a.units.d - 1);
  return max((int64_t)at_least, (total + (1 << a.run_bits) - 1) >> a.run_bits);
}

struct Run {
  int64_t begin, end, total, off;  // key tiles [begin, end) of `total`; begin is tile `off` of request b
  int b, w;
};
// The run of workgroup x.  Workgroups go to the eight XCDs in turn; by_xcd has runs
// in a row go to one, where the row tiles of a KV head find its keys in that XCD's L2
// cache.  Measured (us in turn / by XCD): 2 questions of 389 rows over 32,768 tokens, bf16
// x 64 259 / 206, x 128 222 / 218; 4 of 500 rows, x 128 58 / 52; but 8 of 400 rows, x 64,
// whose keys every L2 holds, 49 / 54, and trees of 61 rows over 65,501 tokens 59 / 60.
__device__ __forceinline__ int run_of(int x, int64_t total, int64_t len) {
  const int runs = quotient(total + len - 1, len), per = (runs + 7) >> 3;
  return (x >> 3) < per ? (x & 7) * per + (x >> 3) : runs;
}
// Run w; false where there is none.  Every wavefront finds it for itself: a
// lane adds up a few consecutive requests, a prefix sum over the lanes gives
// the lane whose requests hold the run's first tile, and that lane walks them.
// Nothing waits for another wavefront.
// (BLOCK: w is a workgroup's number)
template <bool PAIRS, bool BLOCK = false, class A>
__device__ __forceinline__ bool find_run(const A& a, int w, Run* run) {
  if (a.t.B == 1) {
    run->total = request_tiles(a, unit_sizes<PAIRS>(a, load_request_scalar(a.t, 0), 0));
    const int64_t len = run_length(a, run->total);
    if (BLOCK && a.by_xcd) w = run_of(w, run->total, len);
    run->w = w;
    run->begin = run->off = w * len;
    run->end = min(run->begin + len, run->total);
    run->b = 0;
    return run->begin < run->total;
  }
  const int lane = threadIdx.x & 63, per = (a.t.B + 63) >> 6;
  auto tiles = [&](int b) { return request_tiles(a, unit_sizes<PAIRS, false>(a, load_request(a.t, b), b)); };
  const int b0 = min(lane * per, a.t.B), b1 = min(b0 + per, a.t.B);
  int64_t sum = 0;
#pragma unroll 4
  for (int b = b0; b < b1; ++b) sum += tiles(b);
  // (in 32 bits where the lanes' sums allow it: six steps of one instruction)
  const int64_t upto = __ballot(sum >> 24) ? wave_scan64(sum) : (int64_t)wave_scan((unsigned)sum);
  const int64_t total = lane_value(upto, 63);
  const int64_t len = run_length(a, total);
  if (BLOCK && a.by_xcd) w = run_of(w, total, len);
  run->w = w;
  const int64_t begin = w * len;
  if (begin >= total) return false;
  const int at = __builtin_ctzll(__ballot(upto > begin));  // the first lane that reaches past it
  int64_t off = begin - lane_value(upto - sum, at);
  int b = at * per;
  if (per > 1)  // (the whole wavefront walks, off the scalar cache)
    for (; b < a.t.B - 1; ++b) {
      const int64_t x = request_tiles(a, unit_sizes<PAIRS>(a, load_request_scalar(a.t, b), b));
      if (off < x) break;
      off -= x;
    }
  run->begin = begin;
  run->end = min(begin + len, total);
  run->total = total;
  run->off = off;
  run->b = b;
  return true;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const char* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00020000);
}

// Pieces of one query vector's softmax, merged a round at a time: maxima (log2
// units) and sums, and C elements of the outputs.  A piece that saw no key has a
// maximum of -inf and a sum of 0.  One whose seen scores were all -inf (weight 0
// beside any other piece) has kOnlyMinusInf, below every finite score, and a sum
// above 0.  Maxima do not show NaN; a score of NaN is in the sum.  No weight is
// less than the smallest float (which adds at most 2^-21 for any finite output),
// so a sum or an output that is not finite stays so, wherever the work is cut.
constexpr float kOnlyMinusInf = -3.40282347e38f, kSmallest = 1.40129846e-45f;  // 2^-149
__device__ __forceinline__ float final_sum(float m, float sum) { return m == kOnlyMinusInf ? __builtin_nanf("") : sum; }
template <int C>
struct Merge {
  float m = -INFINITY, sum = 0.f, acc[C] = {};
  template <int U>
  __device__ __forceinline__ void add(const float2 (&ml)[U], const float (&v)[U][C]) {
    float mn = m;
#pragma unroll
    for (int y = 0; y < U; ++y) mn = fmaxf(mn, ml[y].x);
    // (two infinities: NaN, and the larger of it and kSmallest is that)
    const float back = fmaxf(__builtin_amdgcn_exp2f(m - mn), kSmallest);
    sum *= back;
#pragma unroll
    for (int e = 0; e < C; ++e) acc[e] *= back;
#pragma unroll
    for (int y = 0; y < U; ++y) {
      const float w = fmaxf(__builtin_amdgcn_exp2f(ml[y].x - mn), kSmallest);
      sum = fmaf(w, ml[y].y, sum);
#pragma unroll
      for (int e = 0; e < C; ++e) acc[e] = fmaf(w, v[y][e], acc[e]);
    }
    m = mn;
  }
  __device__ __forceinline__ float scale() const { return sum == 0.f ? 0.f : 1.f / final_sum(m, sum); }
  __device__ __forceinline__ float lse() const { return (m + __log2f(final_sum(m, sum))) * kLn2; }
};

// Units of a batch whose requests have all as many rows.
inline int even_units(const SplitArgs& a) {
  const int64_t vectors = (int64_t)a.t.n_rows * a.t.G, per_tile = (int64_t)a.t.B << a.row_bits;
  const int64_t units = std::max<int64_t>(1, (vectors + per_tile - 1) / per_tile) * a.t.B * a.t.Hkv;
  return (int)std::min<int64_t>(units, 1 << 26);  // (times min_tiles in 32 bits: more has runs enough)
}
// Workgroups that a launch needs at most: the runs there can be, from the rows
// and the block tables' room.  A batch with room for one run needs no merge.
template <class A>
inline int most_runs(const A& a) {
  double tiles = std::max<double>(1, ((double)a.t.max_blocks * a.t.page.d + (1 << a.tile_bits) - 1) / (1 << a.tile_bits));
  if constexpr (A::kMemory) tiles = tiles * (1 << a.paged_bits) + a.unit_tiles;
  const double units = ((double)a.t.n_rows * a.t.G / (1 << a.row_bits) + a.t.B) * a.t.Hkv;
  return (int)std::min<double>(1 << a.run_bits, std::max<double>(a.units.d, ceil(tiles * units / a.min_tiles)));
}

inline TreeArgs tree_args(const Geo& g, const cs_page_pool& pool, int layer, const cs_batch& b, const cs_rows& q,
                          const cs_rows& out, float* lse) {
  TreeArgs t;
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
  return t;
}

// The instance for many rows (bf16, head_dim 128): see tree_attention_wide.hip.
constexpr int kWideRowBits = 8, kWideRunBits = 8;
size_t tree_wide_workspace();
// once: keys and values with the non-temporal hint.  One row tile a request: 32 requests
// of 8,000 tokens, 8 rows 72 -> 64 us; two and more read them again (tree-sized steps
// of 65,000 tokens 59 -> 62).
constexpr double kWideOnceBytes = 64e6;
void launch_tree_wide(SplitArgs a, void* ws, bool once, hipStream_t s);
void launch_packed_wide(MemoryArgs a, void* ws, hipStream_t s);

}  // namespace cs
