// Attention of a batch's rows with the matrix instructions, row tiles of 16 to 64
// query vectors: the kernel and the merge of its pieces.
#pragma once

#include <math.h>

#include <type_traits>

#include "tree_attention.h"

namespace cs {

__device__ __forceinline__ void put_elem(float* p, float x) { *p = x; }
__device__ __forceinline__ void put_elem(uint16_t* p, float x) { *p = f32_to_bf16(x); }

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
constexpr int kMemoryTile = 1 << kFewTileBits;  // (packed pages)
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
template <bool PAIRS, class A>
__device__ __forceinline__ Place next_place(const A& a, int* b, int64_t* off, int64_t* left, Request* q) {
  Place x;
  x.n = 0;
#pragma unroll 1
  while (*b < a.t.B && *left > 0) {
    *q = load_request_scalar(a.t, *b);
    const Units units = unit_sizes<PAIRS>(a, *q, *b);
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

// PT: packed tiles of a wavefront's step, all of them in flight while the step before
// is worked on.  One does where there is little to do; much is bound by what is in
// flight, which with a tile of 4 KB for each wavefront is too little for 5 TB/s.
template <typename E, int D, int NR, bool ONCE, class Args = SplitArgs, int PT = 1>
__global__ __launch_bounds__(kThreads, 2) void tree_attend(const Args) {
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
  constexpr bool kMemory = Args::kMemory;
  static_assert(!(kMemory && ONCE), "packed tiles are loaded without the hint");
  constexpr int kSub = kMemory ? kMemoryTile / KT : 1;  // tiles here of a key tile of the work
  // Where a lane's 16 bytes k of a row lie.  With packed keys they are the elements
  // of its words of codes, which are next to each other (but for D = 96, see there).
  constexpr bool kRowRuns = kMemory && D % 32 == 0 && D != 96;
  static_assert(KS * 64 == kRowB && NO * 16 == D && VB % 4 == 0, "head dim");

  __shared__ float s_o[kWaves * 16 * kPad];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63;
  const int ln = lane & 15, lg = lane >> 4;
  // The arguments are read where they are used: a launch is short, and what it
  // spends on moving arguments in and out of scalar registers, and on fetching
  // the instructions that do, is part of its latency.
  typedef const __attribute__((address_space(4))) Args* ArgPtr;
  const ArgPtr argp = (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
  auto args = [&]() -> Args {
    ArgPtr p = argp;
    asm volatile("" : "+s"(p));
    return *(const Args*)p;
  };
  auto piece = [&](auto row, int k) {  // (a row's address or offset)
    if constexpr (kRowRuns) return row + (kRowB >> 2) * lg + 16 * k;
    else return row + 64 * k + 16 * lg;
  };
  Run run;
  if (!find_run<(NR > 1), (NR > 1)>(args(), blockIdx.x, &run)) return;
  int64_t left = run.end - run.begin, off = run.off;
  int b = run.b;
  bool first_seg = true;

  while (left > 0) {
    const Args a = args();
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
    Span span;
    int t_begin = t0, t_end = min(t0 + seg, (key_end + KT - 1) / KT), first_tile = t0, packed_end = 0;  // (tiles of KT keys; packed ones, of 32)
    if constexpr (kMemory) {
      span = span_of<kFewTileBits>(a, q, a.group.div(rt * RT), i_last);
      const int last = (key_end + kMemoryTile - 1) / kMemoryTile - span.skip;
      const int packed = span.before(packed_keys(a, q, b) >> kFewTileBits);
      auto tile_at = [&](int t) {  // of a place in the cut work
        return min(t <= packed ? t : packed + ((t - packed + (1 << a.paged_bits) - 1) >> a.paged_bits), last);
      };
      const int begin = tile_at(t0), end = tile_at(t0 + seg);
      first_tile = begin;
      packed_end = min(end, packed);
      t_begin = max(begin, packed_end) * kSub;
      t_end = end * kSub;
    }
    auto key_of = [&](int tile) {  // the first key of a tile
      if constexpr (kMemory) return (span.tile(tile / kSub) * kSub + tile % kSub) * KT;
      else return tile * KT;
    };
    const int t_full = min(t.mask ? q.cached : q.cached + a.group.div(rt * RT) + 1, q.len) / KT;  // tiles before it: every row sees every key

    Words<16> qf[NR][KS];
    int row[NR];  // the lane's row in the request, per 16 query vectors
#pragma unroll
    for (int x = 0; x < NR; ++x) {
      const int qv = min(rt * RT + 16 * x + ln, vectors - 1), i = a.group.div(qv);
      row[x] = i;
      const char* qp = (const char*)t.q + ((int64_t)(q.r0 + i) * t.q_row + (h * t.G + qv - i * t.G) * t.q_head) * (int)sizeof(E);
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[x][k] = *(const Words<16>*)piece(qp, k);
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
      for (int s = 0; s < SUB; ++s) page[s] = pages[page_div.div(min(key_of(min(tile, t_end - 1)) + 16 * s, q.len - 1))];
    };
    auto places = [&](int tile) {
#pragma unroll
      for (int s = 0; s < SUB; ++s) {
        const int key = key_of(tile) + 16 * s;
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
        for (int k = 0; k < KS; ++k) kf[s][k] = load_words<16, ONCE>(r, piece(ln * kRowB, k));
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

    // Packed tiles, 32 keys each: a word of codes of a key is a lane's part of one
    // 16 x 16 x 32 product, converted to bf16 where it lies.  Row r of the two
    // S^T tiles is key 2 r and key 2 r + 1, so that a lane's scores are those of keys
    // 8 lg .. 8 lg + 7, the eight tokens of its words of values.  In float32 queries
    // and probabilities are three bf16 terms each, which hold all 24 bits from 2^-110 on
    // (bf16 ends at 2^-133).  A query's first term is cut, not rounded: magnitudes
    // above 3.39e38 would round to infinity.
    if constexpr (kMemory && D % 32 == 0) {
      constexpr int KW = D / 32, NT = kBf16 ? 1 : 3;
      constexpr int KSW = KW == 8 ? 2 : KW == 3 ? 3 : 1;  // halfwords of key scales that a lane needs
      struct Tile {
        uint32_t k[2][KW], ks[KSW], v[NB][VW], vs[NB][(VW + 3) / 4];
        bool have;
      };
      constexpr int NP = 8 * PT;  // scores of a lane per query vector
      bf16x8 qt[NR][KW][NT];
#pragma unroll
      for (int x = 0; x < NR; ++x)
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          if constexpr (kBf16) {
            qt[x][w][0] = __builtin_bit_cast(bf16x8, qf[x][w]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float rest = __uint_as_float(qf[x][2 * w + (e >> 2)].w[e & 3]);
#pragma unroll
              for (int y = 0; y < NT; ++y) {
                qt[x][w][y][e] = (__bf16)(y ? rest : __uint_as_float(__float_as_uint(rest) & 0xffff0000u));
                rest -= (float)qt[x][w][y][e];
              }
            }
          }
        }
      const PackedView pk = a.packed;
      const int64_t plane4 = ((int64_t)t.layer * t.Hkv + h) * pk.plane_bytes();
      const int k_off = 2 * ln * (D / 2) + (kRowRuns ? 4 * KW * lg : 4 * lg);
      const int v_off = pk.v_codes() + (lg * D + VW * ln) * 4, vs_off = pk.v_scales() + VW * ln;
      const int ks_off = pk.k_scales() + 2 * ln + (kRowRuns ? kBlock * (KW * lg / 4) : 0);
      int page4[PT];
      auto fetch_page4 = [&](int tile) {
#pragma unroll
        for (int u = 0; u < PT; ++u) page4[u] = pages[page_div.div(span.tile(min(tile + kWaves * u, packed_end - 1)) * kMemoryTile)];
      };
      __amdgpu_buffer_rsrc_t codes[PT], scales[PT];
      Tile T[PT];
      auto place4 = [&](int tile) {
#pragma unroll
        for (int u = 0; u < PT; ++u) {
          const int at = tile + kWaves * u, key = span.tile(at) * kMemoryTile;
          const int x = (key - page_div.div(key) * page_div.d) >> kFewTileBits, c = x * (kMemoryTile * D / 2), s = x * D;
          T[u].have = at < packed_end && (unsigned)page4[u] < (unsigned)pk.n_pages;
          const char* p = pk.base + page4[u] * pk.page_bytes + plane4;  // (no bytes: no address is used)
          codes[u] = rows_rsrc(p + c, T[u].have ? pk.plane_bytes() - c : 0);
          scales[u] = rows_rsrc(p + s, T[u].have ? pk.plane_bytes() - s : 0);
        }
      };
      auto load_k4 = [&](Tile& T, __amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t scales) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int at = k_off + y * (D / 2);
          if constexpr (kRowRuns) {
#pragma unroll
            for (int w = 0; w < KW; w += 4) {
              const auto x = load_words<(KW < 4 ? 4 * KW : 16), false>(codes, at + 4 * w);
#pragma unroll
              for (int i = 0; i < (KW < 4 ? KW : 4); ++i) T.k[y][w + i] = x.w[i];
            }
          } else {
#pragma unroll
            for (int w = 0; w < KW; ++w) T.k[y][w] = load_words<4, false>(codes, at + 16 * w).w[0];
          }
        }
#pragma unroll
        for (int w = 0; w < KSW; ++w) T.ks[w] = __builtin_amdgcn_raw_buffer_load_b16(scales, ks_off + kBlock * w, 0, 0);
      };
      auto load_v4 = [&](Tile& T, __amdgpu_buffer_rsrc_t codes, __amdgpu_buffer_rsrc_t scales) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const int at = v_off + n * 64 * VW, as = vs_off + n * 16 * VW;
#pragma unroll
          for (int w = 0; w < VW; w += 4) {
            constexpr int last = VW % 4 ? VW % 4 : 4;
            if (w + 4 <= VW) {
              const auto x = load_words<16, false>(codes, at + 4 * w);
#pragma unroll
              for (int i = 0; i < 4; ++i) T.v[n][w + i < VW ? w + i : 0] = x.w[i];
            } else {
              const auto x = load_words<4 * last, false>(codes, at + 4 * w);
#pragma unroll
              for (int i = 0; i < last; ++i) T.v[n][w + i] = x.w[i];
            }
          }
          if constexpr (VW % 4 == 0) {
            const auto x = load_words<VW, false>(scales, as);
#pragma unroll
            for (int w = 0; w < VW / 4; ++w) T.vs[n][w] = x.w[w];
          } else {
#pragma unroll
            for (int w = 0; w < VW / 2; ++w) {
              const uint32_t x = __builtin_amdgcn_raw_buffer_load_b16(scales, as + 2 * w, 0, 0);
              if (w & 1) T.vs[n][w / 2] |= x << 16;
              else T.vs[n][w / 2] = x;
            }
          }
        }
      };
      auto v_scale = [&](const Tile& T, int n, int e) -> float {
        const uint32_t w = T.vs[n][e / 4];
        return __uint_as_float((e & 3) == 3 ? w >> 1 : w << (23 - 8 * (e & 3)));
      };
      // A tile's scores of query vector x become probabilities: the running maximum,
      // the accumulators rescaled when it grew, the sum.
      auto weigh = [&](int x, float (&p)[NP]) {
        float mx = p[0];
#pragma unroll
        for (int j = 1; j < NP; ++j) mx = fmaxf(mx, p[j]);
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
        for (int j = 0; j < NP; ++j) {
          p[j] = __builtin_amdgcn_exp2f(fmaf(p[j], sc, -ref));
          l[x] += p[j];
        }
      };
      int tile = first_tile + wave;
      if (tile < packed_end) {
        fetch_page4(tile);
        place4(tile);
#pragma unroll
        for (int u = 0; u < PT; ++u) load_k4(T[u], codes[u], scales[u]);
#pragma unroll
        for (int u = 0; u < PT; ++u) load_v4(T[u], codes[u], scales[u]);
        fetch_page4(tile + PT * kWaves);
      }
#pragma unroll 1
      for (; tile < packed_end; tile += PT * kWaves) {
        auto key_at = [&](int u) { return span.tile(tile + kWaves * u) * kMemoryTile; };
        bool have[PT], masked = false;
        f32x4 s[NR][PT][2];
#pragma unroll
        for (int u = 0; u < PT; ++u) {
          have[u] = T[u].have;
          masked = masked || !have[u] || (key_at(u) + kMemoryTile > span.low && key_at(u) < span.high);
#pragma unroll
          for (int x = 0; x < NR; ++x) s[x][u][0] = s[x][u][1] = f32x4{};
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int w = 0; w < KW; ++w) {
              const uint32_t ks = T[u].ks[KW == 8 ? w / 4 : KW == 3 ? w : 0];
              const bf16x8 kw = decode8(T[u].k[y][w], y ? scale_of<1>(ks) : scale_of<0>(ks));
#pragma unroll
              for (int x = 0; x < NR; ++x)
#pragma unroll
                for (int z = NT - 1; z >= 0; --z)
                  s[x][u][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kw, qt[x][w][z], s[x][u][y], 0, 0, 0);
            }
        }
        place4(tile + PT * kWaves);
#pragma unroll
        for (int u = 0; u < PT; ++u) load_k4(T[u], codes[u], scales[u]);
        fetch_page4(tile + 2 * PT * kWaves);
        float p[NR][NP];
#pragma unroll
        for (int x = 0; x < NR; ++x)
#pragma unroll
          for (int j = 0; j < NP; ++j) p[x][j] = s[x][j >> 3][j & 1][j >> 1 & 3];
        uint32_t vis[NR][PT];  // bit j: key 8 lg + j
        if (masked) {
          const Args A = args();
#pragma unroll
          for (int x = 0; x < NR; ++x)
#pragma unroll
            for (int u = 0; u < PT; ++u) {
              vis[x][u] = have[u] ? ~(uint32_t)hidden_keys(A, q, row[x]).bits(key_at(u), kMemoryTile) : 0u;
              seen[x] = seen[x] || vis[x][u];
              vis[x][u] >>= 8 * lg;
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (!(vis[x][u] >> j & 1)) p[x][8 * u + j] = -INFINITY;
            }
        } else {
#pragma unroll
          for (int x = 0; x < NR; ++x) seen[x] = true;
        }
#pragma unroll
        for (int x = 0; x < NR; ++x) weigh(x, p[x]);
#pragma unroll
        for (int u = 0; u < PT; ++u) {
          // A block of values that is NaN must not reach rows that see none of its keys.
          if (masked) {
            uint32_t nan = 0;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
              for (int w = 0; w < (VW + 3) / 4; ++w) nan |= ((T[u].vs[n][w] & 0x7f7f7f7fu) + 0x01010101u) & T[u].vs[n][w] & 0x80808080u;
            if (__ballot(nan != 0)) {
#pragma unroll
              for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int e = 0; e < VW; ++e) {
                  const uint32_t byte = T[u].vs[n][e / 4] >> (8 * (e & 3)) & 255;
                  const __bf16 odd = byte == kNanScale ? (__bf16)1.f : (__bf16)0.f;
                  bf16x8 va, pb;
#pragma unroll
                  for (int j = 0; j < 8; ++j) va[j] = odd;
                  if (byte == kNanScale) T[u].vs[n][e / 4] &= ~(255u << (8 * (e & 3)));
#pragma unroll
                  for (int x = 0; x < NR; ++x) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) pb[j] = vis[x][u] >> j & 1 ? (__bf16)1.f : (__bf16)0.f;
                    const f32x4 c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb, f32x4{}, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                      if (c[i] > 0.f) o[x][n * VW + e][i] = __builtin_nanf("");
                  }
                }
            }
          }
          bf16x8 pb[NR][NT];
#pragma unroll
          for (int x = 0; x < NR; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              float rest = p[x][8 * u + j];
#pragma unroll
              for (int z = 0; z < NT; ++z) {
                pb[x][z][j] = (__bf16)rest;
                if (z + 1 < NT) rest -= (float)pb[x][z][j];
              }
            }
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < VW; ++e) {
              const bf16x8 va = decode8(T[u].v[n][e], v_scale(T[u], n, e));
#pragma unroll
              for (int x = 0; x < NR; ++x)
#pragma unroll
                for (int z = NT - 1; z >= 0; --z)
                  o[x][n * VW + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[x][z], o[x][n * VW + e], 0, 0, 0);
            }
          load_v4(T[u], codes[u], scales[u]);
        }
      }
    }
    int tile = t_begin + wave;
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
      const int key0 = key_of(tile);
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
      bool masked = kMemory ? key0 >= t_full * KT || (key0 + KT > span.low && key0 < span.high) : tile >= t_full;
#pragma unroll
      for (int y = 0; y < SUB; ++y) masked = masked || !have[y];
      uint32_t vis[NR];  // bit 16 y + i: key 16 y + 4 lg + i
      if (masked) {
        const Args A = args();
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
          if constexpr (kMemory) vis[x] &= ~(uint32_t)hidden_keys(A, q, row[x]).bits(key0, KT);
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
      const Args A = args();
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
template <typename E, int D, bool PAIRS, class Args = SplitArgs>
__global__ __launch_bounds__(kThreads) void tree_combine(const Args a) {
  constexpr int C = (D + 31) / 32;  // elements a lane holds
  __shared__ float s_o[kGroups][32 * C], s_m[kGroups], s_l[kGroups];
  const TreeArgs& t = a.t;
  const int w1 = blockIdx.x + 1;
  Run run;
  if (!find_run<PAIRS>(a, w1, &run)) return;
  const Request q = load_request_scalar(t, run.b);
  const Place at = place_at<PAIRS>(a, q, unit_sizes<PAIRS>(a, q, run.b), run.off);
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

}  // namespace cs
