// Shared by the sources of the batch attention: its arguments and how its work is cut.
#pragma once

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
template <bool PAIRS>
__device__ __forceinline__ Units unit_sizes(const SplitArgs& a, const Request& q) {
  Units s;
  s.units = s.nrt = (int)(((int64_t)q.n * a.t.G + (1 << a.row_bits) - 1) >> a.row_bits);
  s.ntile = key_tiles(a, q.len);
  if (PAIRS && !a.t.mask && s.nrt > 1) {
    // the keys of both: the last rows of p and nrt - 1 - p are, added up, at most n + 2 row tiles' rows
    const int64_t keys = 2 * (int64_t)q.cached + 2 + q.n + a.group.div(2 << a.row_bits);
    const int pair = (int)min((keys + (2 << a.tile_bits) - 2) >> a.tile_bits, 2 * (int64_t)s.ntile), pairs = (s.nrt + 1) >> 1;
    const int64_t tiles = (int64_t)s.ntile * s.nrt;
    if ((int64_t)pair * pairs < tiles && (double)tiles * a.t.Hkv * a.t.B >= (double)(kPairTiles << a.run_bits)) {
      s.units = pairs;
      s.ntile = pair;
    }
  }
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
template <bool PAIRS>
__device__ __forceinline__ Place place_at(const SplitArgs& a, const Request& q, const Units& s, int64_t off) {
  const int u = uniform(quotient(off, s.ntile));
  Place x;
  x.t0 = uniform((int)(off - (int64_t)u * s.ntile));
  x.h = s.units == 1 ? u : uniform(u / s.units);
  x.rt = u - x.h * s.units;
  x.n = s.ntile;
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
template <bool PAIRS, bool BLOCK = false>
__device__ __forceinline__ bool find_run(const SplitArgs& a, int w, Run* run) {
  if (a.t.B == 1) {
    run->total = request_tiles(a, unit_sizes<PAIRS>(a, load_request_scalar(a.t, 0)));
    const int64_t len = run_length(a, run->total);
    if (BLOCK && a.by_xcd) w = run_of(w, run->total, len);
    run->w = w;
    run->begin = run->off = w * len;
    run->end = min(run->begin + len, run->total);
    run->b = 0;
    return run->begin < run->total;
  }
  const int lane = threadIdx.x & 63, per = (a.t.B + 63) >> 6;
  auto tiles = [&](int b) { return request_tiles(a, unit_sizes<PAIRS>(a, load_request(a.t, b))); };
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
      const int64_t x = request_tiles(a, unit_sizes<PAIRS>(a, load_request_scalar(a.t, b)));
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
inline int most_runs(const SplitArgs& a) {
  const double tiles = std::max<double>(1, ((double)a.t.max_blocks * a.t.page.d + (1 << a.tile_bits) - 1) / (1 << a.tile_bits));
  const double units = ((double)a.t.n_rows * a.t.G / (1 << a.row_bits) + a.t.B) * a.t.Hkv;
  return (int)std::min<double>(1 << a.run_bits, std::max<double>(a.units.d, ceil(tiles * units / a.min_tiles)));
}

// The instance for many rows (bf16, head_dim 128): see tree_attention_wide.hip.
constexpr int kWideRowBits = 8, kWideTileBits = 6, kWideRunBits = 8;
size_t tree_wide_workspace();
// once: keys and values with the non-temporal hint.  One row tile a request: 32 requests
// of 8,000 tokens, 8 rows 72 -> 64 us; two and more read them again (tree-sized steps
// of 65,000 tokens 59 -> 62).
constexpr double kWideOnceBytes = 64e6;
void launch_tree_wide(SplitArgs a, void* ws, bool once, hipStream_t s);

}  // namespace cs
