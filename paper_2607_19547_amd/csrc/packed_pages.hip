// Pages into 4 bits and back (keys turned on the way, Eq. 3).
//
// A plane's elements are taken 16,384 at a time by a workgroup, whatever the page
// and head sizes are: planes of small pages share one, large ones are split.
// Both ways a thread has whole 32-bit words of codes: eight elements of a key's
// row, or eight tokens of some channels of the values, whose block of 32 tokens
// lies in the four lanes of a quad.
//
// Bound by memory: 128 pages of 64 tokens, 36 layers of 2 heads of 128 in bf16 are packed
// in 74 us (302 MB read, 80 written, 5.2 TB/s); 256 come back and are turned in 171 us (161
// and 604 MB, 4.5 TB/s).  A page alone takes 6.4 us and 4.8 (turned 7.4: float64 sines), the
// chain of its entry, its elements and the stores.  With the places found per item, and
// loads a few at a time, packing took 107 us.
#include <algorithm>
#include <type_traits>

#include "packed.h"

namespace cs {

constexpr int kPageThreads = 256;
constexpr int kShare = 16384;       // elements of a workgroup, of keys and of values
constexpr int kLeastPlane = 1024;   // 32 x 32
constexpr int kMostPlanes = kShare / kLeastPlane + 1;  // that a workgroup has a part of

struct PagesArgs {
  const int32_t *src, *dst;
  PoolView pool;
  PackedView packed;
  int planes;               // entries x layers x KV heads
  FastDiv plane_units;      // a plane in units of kLeastPlane elements
  FastDiv per_entry, heads, head_words, pieces;  // planes of an entry; KV heads; D / 8; 16-byte pieces of a row
  FastDiv plane_words, plane_values;             // a plane's words of codes; its value items
  int Hkv, lb;
};
struct TurnArgs : PagesArgs {
  const int32_t* offsets;
  int sec0, sec01;
  double theta[256];
};

// The planes that a workgroup's elements lie in: `plane` the first, `within` its
// elements before the workgroup's own.
struct Share {
  int plane, within, n;  // (n of them)
};
__device__ __forceinline__ Share share_of(const PagesArgs& a) {
  Share s;
  const int unit = (int)blockIdx.x * (kShare / kLeastPlane);  // (below 2^31: see the launch)
  s.plane = a.plane_units.div(unit);
  s.within = (unit - s.plane * a.plane_units.d) * kLeastPlane;
  const int left = a.planes - s.plane, reach = a.plane_units.div(s.within / kLeastPlane + kShare / kLeastPlane - 1) + 1;
  s.n = min(left, reach);
  return s;
}
// Where they are in the pool (keys and values alike) and in the packed pool, and
// their entries; at -1 those that are left out.
struct Places {
  int64_t pool[kMostPlanes], packed[kMostPlanes];
  int entry[kMostPlanes];
};
template <bool PACK>
__device__ __forceinline__ void find_places(const PagesArgs& a, const Share& s, Places* at) {
  const int x = threadIdx.x;
  if (x < s.n) {
    const int plane = s.plane + x, e = a.per_entry.div(plane), lh = plane - e * a.per_entry.d;
    const int p = (PACK ? a.src : a.dst)[e], p4 = (PACK ? a.dst : a.src)[e];
    const int l = a.heads.div(lh), h = lh - l * a.heads.d;
    const int64_t nth = (int64_t)(a.lb + l) * a.Hkv + h;
    const bool ok = (unsigned)p < (unsigned)a.pool.n_pages && (unsigned)p4 < (unsigned)a.packed.n_pages;
    at->pool[x] = ok ? p * a.pool.page_bytes + nth * a.pool.P * a.pool.row_bytes : -1;
    at->packed[x] = p4 * a.packed.page_bytes + nth * a.packed.plane_bytes();
    at->entry[x] = e;
  }
}

// A 16-byte piece of a row: 8 or 4 elements.
template <typename E>
struct Piece {
  static constexpr int N = 16 / sizeof(E);
};
// Item x of a workgroup, in items of 1 / PER of an element: its plane among the
// workgroup's (below s.n, or the item is none) and its place there.
template <int PER>
__device__ __forceinline__ int item_at(const Share& s, const FastDiv& per_plane, int x, int* at) {
  const int off = s.within / PER + x, pl = per_plane.div(off);
  *at = off - pl * per_plane.d;
  return pl;
}

// One block's scale byte from the bits of its largest magnitude (float32; an
// infinity or NaN has the largest of all): the least e from -125 to 125 with amax <=
// 7 x 2^e, or 125 (codes saturate).
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  const int e = (int)((amax + 0x1fffffu) >> 23) - 2;  // (1.75 = 7 / 4 has the mantissa 0x600000)
  return amax >= 0x7f800000u ? kNanScale : (uint32_t)min(max(e, kLeastScale), kMostScale);
}
// Over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));  // quad_perm 1, 0, 3, 2
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));  // 2, 3, 0, 1
}
// Codes of two elements into byte B of w.
template <int B>
__device__ __forceinline__ uint32_t encode2(uint32_t w, uint32_t pair, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, pair), scale, B);
}
template <int B>
__device__ __forceinline__ uint32_t encode2(uint32_t w, float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, a, b, scale, B);
}

template <typename E, bool ONCE>
__global__ __launch_bounds__(kPageThreads) void pack_pages_kernel(const PagesArgs a) {
  constexpr bool kBf16 = sizeof(E) == 2;
  constexpr int W = Piece<E>::N;  // channels of a value item
  constexpr int KI = kShare / 8 / kPageThreads, VI = kShare / (8 * W) / kPageThreads;  // items of a thread
  constexpr int KL = kBf16 ? 1 : 2;                                                    // loads of a key item
  __shared__ Places place;
  const int tid = threadIdx.x, D = a.packed.D;
  const Share sh = share_of(a);
  find_places<true>(a, sh, &place);
  __syncthreads();
  auto load = [&](const char* from) -> u32x4 {
    if constexpr (ONCE) return __builtin_nontemporal_load((const u32x4*)from);
    else return *(const u32x4*)from;
  };
  // all loads first: values, eight tokens of W channels per item (a quad's lanes
  // have a block's tokens), and keys, a word of codes
  u32x4 vw[VI][8], kw[KI][KL];
  int v_at[VI], v_pl[VI], k_at[KI], k_pl[KI];
#pragma unroll
  for (int y = 0; y < VI; ++y) {
    v_pl[y] = item_at<8 * W>(sh, a.plane_values, tid + kPageThreads * y, &v_at[y]);
    const int64_t at = v_pl[y] < sh.n ? place.pool[v_pl[y]] : -1;
    if (at < 0) {
      v_pl[y] = -1;
      continue;
    }
    const int tg = v_at[y] & 3, blk = a.pieces.div(v_at[y] >> 2), c = (v_at[y] >> 2) - blk * a.pieces.d;
    const char* from = a.pool.v + at + ((int64_t)(blk * kBlock + 8 * tg) * D + W * c) * sizeof(E);
#pragma unroll
    for (int j = 0; j < 8; ++j) vw[y][j] = load(from + (int64_t)j * D * sizeof(E));
  }
#pragma unroll
  for (int y = 0; y < KI; ++y) {
    k_pl[y] = item_at<8>(sh, a.plane_words, tid + kPageThreads * y, &k_at[y]);
    const int64_t at = k_pl[y] < sh.n ? place.pool[k_pl[y]] : -1;
    if (at < 0) {
      k_pl[y] = -1;
      continue;
    }
#pragma unroll
    for (int j = 0; j < KL; ++j) kw[y][j] = load(a.pool.k + at + (int64_t)k_at[y] * 8 * sizeof(E) + 16 * j);
  }
#pragma unroll
  for (int y = 0; y < VI; ++y) {
    if (v_pl[y] < 0) continue;
    char* to = a.packed.base + place.packed[v_pl[y]];
    const int tg = v_at[y] & 3, blk = a.pieces.div(v_at[y] >> 2), c = (v_at[y] >> 2) - blk * a.pieces.d;
    uint32_t codes[W], es[W];
#pragma unroll
    for (int d = 0; d < W; ++d) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t w = vw[y][j][kBf16 ? d / 2 : d];
        m = max(m, kBf16 ? (d & 1 ? w : w << 16) & 0x7fff0000u : w & 0x7fffffffu);
      }
      es[d] = scale_byte(quad_max(m));
      const float scale = __uint_as_float(es[d] << 23);
      uint32_t code = 0;
      if constexpr (kBf16) {
        auto two = [&](int j) { return __builtin_amdgcn_perm(vw[y][j + 1][d / 2], vw[y][j][d / 2], d & 1 ? 0x07060302 : 0x05040100); };
        code = encode2<0>(code, two(0), scale);
        code = encode2<1>(code, two(2), scale);
        code = encode2<2>(code, two(4), scale);
        code = encode2<3>(code, two(6), scale);
      } else {
        auto el = [&](int j) { return __uint_as_float(vw[y][j][d]); };
        code = encode2<0>(code, el(0), el(1), scale);
        code = encode2<1>(code, el(2), el(3), scale);
        code = encode2<2>(code, el(4), el(5), scale);
        code = encode2<3>(code, el(6), el(7), scale);
      }
      codes[d] = es[d] == kNanScale ? 0u : code;
    }
    u32x4* word = (u32x4*)(to + a.packed.v_codes() + ((int64_t)(blk * 4 + tg) * D + W * c) * 4);
#pragma unroll
    for (int g = 0; g < W / 4; ++g) word[g] = u32x4{codes[4 * g], codes[4 * g + 1], codes[4 * g + 2], codes[4 * g + 3]};
    if (tg == 0) {
      uint32_t* sc = (uint32_t*)(to + a.packed.v_scales() + blk * D + W * c);
#pragma unroll
      for (int g = 0; g < W / 4; ++g) sc[g] = es[4 * g] | es[4 * g + 1] << 8 | es[4 * g + 2] << 16 | es[4 * g + 3] << 24;
    }
  }
#pragma unroll
  for (int y = 0; y < KI; ++y) {
    if (k_pl[y] < 0) continue;
    char* to = a.packed.base + place.packed[k_pl[y]];
    const int row = a.head_words.div(k_at[y]), c = k_at[y] - row * a.head_words.d;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kBf16) m = max(m, max(kw[y][0][i] << 16 & 0x7fff0000u, kw[y][0][i] & 0x7fff0000u));
      else m = max(m, max(kw[y][0][i] & 0x7fffffffu, kw[y][KL - 1][i] & 0x7fffffffu));
    }
    const uint32_t e = scale_byte(quad_max(m));
    const float scale = __uint_as_float(e << 23);
    uint32_t code = 0;
    if constexpr (kBf16) {
      code = encode2<0>(code, kw[y][0][0], scale);
      code = encode2<1>(code, kw[y][0][1], scale);
      code = encode2<2>(code, kw[y][0][2], scale);
      code = encode2<3>(code, kw[y][0][3], scale);
    } else {
      auto el = [&](int i) { return __uint_as_float(kw[y][i >> 2][i & 3]); };
      code = encode2<0>(code, el(0), el(1), scale);
      code = encode2<1>(code, el(2), el(3), scale);
      code = encode2<2>(code, el(4), el(5), scale);
      code = encode2<3>(code, el(6), el(7), scale);
    }
    *(uint32_t*)(to + 4 * (int64_t)k_at[y]) = e == kNanScale ? 0u : code;
    if ((c & 3) == 0) to[a.packed.k_scales() + (row >> 5) * D + (c >> 2) * kBlock + (row & 31)] = (char)e;
  }
}

// Rotation: a thread has the same eight elements of both halves of a key.  The
// cos/sin tables of the workgroup's entries are made in LDS while its codes are
// on their way.
template <typename E, bool TURN, bool ONCE>
__global__ __launch_bounds__(kPageThreads) void unpack_pages_kernel(const std::conditional_t<TURN, TurnArgs, PagesArgs> a) {
  constexpr bool kBf16 = sizeof(E) == 2;
  constexpr int W = Piece<E>::N;
  constexpr int KI = kShare / 16 / kPageThreads, VI = kShare / (8 * W) / kPageThreads;  // items of a thread
  extern __shared__ float2 tab[];
  __shared__ Places place;
  const int tid = threadIdx.x, D = a.packed.D, half = D >> 1;
  const Share sh = share_of(a);
  find_places<false>(a, sh, &place);
  __syncthreads();
  // all loads first: keys, two words of codes per item, of elements 8 c and
  // D / 2 + 8 c, and values, eight tokens of W channels
  uint32_t wa[KI], wb[KI], ea[KI], eb[KI], ve[VI][W / 4];
  u32x4 vw[VI][W / 4];
  int v_at[VI], v_pl[VI], k_at[KI], k_pl[KI];
#pragma unroll
  for (int y = 0; y < KI; ++y) {
    const int off = 2 * (sh.within / 16 + tid + kPageThreads * y);
    k_pl[y] = a.plane_words.div(off);
    k_at[y] = (off - k_pl[y] * a.plane_words.d) >> 1;
    if (k_pl[y] >= sh.n || place.pool[k_pl[y]] < 0) {
      k_pl[y] = -1;
      continue;
    }
    const char* from = a.packed.base + place.packed[k_pl[y]];
    const int row = a.head_words.div(2 * k_at[y]), c = k_at[y] - row * (a.head_words.d >> 1);
    wa[y] = *(const uint32_t*)(from + (int64_t)row * half + 4 * c);
    wb[y] = *(const uint32_t*)(from + (int64_t)row * half + (half >> 1) + 4 * c);
    const unsigned char* sc = (const unsigned char*)from + a.packed.k_scales() + (row >> 5) * D + (row & 31);
    ea[y] = sc[(c >> 2) * kBlock];
    eb[y] = sc[((half + 8 * c) >> 5) * kBlock];
  }
#pragma unroll
  for (int y = 0; y < VI; ++y) {
    v_pl[y] = item_at<8 * W>(sh, a.plane_values, tid + kPageThreads * y, &v_at[y]);
    if (v_pl[y] >= sh.n || place.pool[v_pl[y]] < 0) {
      v_pl[y] = -1;
      continue;
    }
    const char* from = a.packed.base + place.packed[v_pl[y]];
    const int tg = a.pieces.div(v_at[y]), c = v_at[y] - tg * a.pieces.d;  // eight tokens, piece of the row
#pragma unroll
    for (int g = 0; g < W / 4; ++g) {
      vw[y][g] = *(const u32x4*)(from + a.packed.v_codes() + ((int64_t)tg * D + W * c + 4 * g) * 4);
      ve[y][g] = *(const uint32_t*)(from + a.packed.v_scales() + (tg >> 2) * D + W * c + 4 * g);
    }
  }
  const int entry0 = sh.n > 0 ? place.entry[0] : 0;
  if constexpr (TURN) {
    const int n = sh.n > 0 ? place.entry[sh.n - 1] - entry0 + 1 : 0;
    for (int x = tid; x < n * half; x += kPageThreads) {
      const int e = x / half, i = x - e * half;
      tab[x] = cos_sin_of((double)a.offsets[3 * (int64_t)(entry0 + e) + axis_of(i, a.sec0, a.sec01)] * a.theta[i]);
    }
    __syncthreads();
  }
  auto store = [&](char* to, u32x4 v) {
    if constexpr (ONCE) __builtin_nontemporal_store(v, (u32x4*)to);
    else *(u32x4*)to = v;
  };
#pragma unroll
  for (int y = 0; y < VI; ++y) {
    if (v_pl[y] < 0) continue;
    const int tg = a.pieces.div(v_at[y]), c = v_at[y] - tg * a.pieces.d;
    char* to = a.pool.v + place.pool[v_pl[y]] + ((int64_t)(8 * tg) * D + W * c) * sizeof(E);
    u32x4 row[8];
#pragma unroll
    for (int g = 0; g < W / 4; ++g) {
      const u32x4 w = vw[y][g];
      const uint32_t s = ve[y][g];
      const bf16x8 d0 = decode8(w[0], scale_of<0>(s)), d1 = decode8(w[1], scale_of<1>(s));
      const bf16x8 d2 = decode8(w[2], scale_of<2>(s)), d3 = decode8(w[3], scale_of<3>(s));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (kBf16) {
          row[j][2 * g] = __builtin_bit_cast(uint32_t, bf16x2{d0[j], d1[j]});
          row[j][2 * g + 1] = __builtin_bit_cast(uint32_t, bf16x2{d2[j], d3[j]});
        } else {
          row[j] = __builtin_bit_cast(u32x4, f32x4{(float)d0[j], (float)d1[j], (float)d2[j], (float)d3[j]});
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) store(to + (int64_t)j * D * sizeof(E), row[j]);
  }
#pragma unroll
  for (int y = 0; y < KI; ++y) {
    if (k_pl[y] < 0) continue;
    const int row = a.head_words.div(2 * k_at[y]), c = k_at[y] - row * (a.head_words.d >> 1);
    const bf16x8 ya = decode8(wa[y], scale_of<0>(ea[y])), yb = decode8(wb[y], scale_of<0>(eb[y]));
    char* to = a.pool.k + place.pool[k_pl[y]] + ((int64_t)row * D + 8 * c) * sizeof(E);
    float fa[8], fb[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      fa[i] = (float)ya[i];
      fb[i] = (float)yb[i];
    }
    if constexpr (TURN) {
      const int e = place.entry[k_pl[y]];
      const int32_t* o = a.offsets + 3 * (int64_t)e;
      if (o[0] | o[1] | o[2]) {
        const float2* t = tab + (e - entry0) * half + 8 * c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 cs = t[i];
          const float p = fmaf(fa[i], cs.x, -(fb[i] * cs.y)), q = fmaf(fa[i], cs.y, fb[i] * cs.x);
          fa[i] = p;
          fb[i] = q;
        }
      }
    }
    char* to_b = to + half * sizeof(E);
    if constexpr (kBf16) {
      u32x4 ra, rb;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ra[i] = pack_bf16x2(fa[2 * i], fa[2 * i + 1]);
        rb[i] = pack_bf16x2(fb[2 * i], fb[2 * i + 1]);
      }
      store(to, ra);
      store(to_b, rb);
    } else {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        store(to + 16 * g, __builtin_bit_cast(u32x4, f32x4{fa[4 * g], fa[4 * g + 1], fa[4 * g + 2], fa[4 * g + 3]}));
        store(to_b + 16 * g, __builtin_bit_cast(u32x4, f32x4{fb[4 * g], fb[4 * g + 1], fb[4 * g + 2], fb[4 * g + 3]}));
      }
    }
  }
}

// ------------------------------------------------------------------ launch
PackedView packed_view(const Geo& g, const cs_packed_pool& p) {
  PackedView v;
  v.base = (char*)p.pages;
  v.n_pages = (int)p.n_pages;
  v.P = (int)g.T;
  v.D = g.D;
  v.page_bytes = (int64_t)g.L * g.Hkv * v.plane_bytes();
  return v;
}

static cs_status pages_args(const Geo& g, const cs_page_pool& pool, const cs_packed_pool& packed, const PagesJob& job,
                            const char* what, PagesArgs* a, unsigned* blocks) {
  const int64_t per_entry = (int64_t)(job.le - job.lb) * g.Hkv, plane = g.T * g.D;
  const int64_t most = (int64_t(1) << 31) - 1;  // entries, planes and units of them are counted in 32 bits
  if (per_entry > most / job.n || per_entry * job.n > most / (plane / kLeastPlane) - kShare / kLeastPlane)
    return fail(CS_ERR_UNSUPPORTED, std::string(what) + ": pages x layers x KV heads x a plane / 1,024 must be below 2^31");
  const int64_t planes = per_entry * job.n, n = (planes * (plane / kLeastPlane) + kShare / kLeastPlane - 1) / (kShare / kLeastPlane);
  const cs_status st = check_grid(n, 1, 1, kPageThreads, what);
  if (st) return st;
  *blocks = (unsigned)n;
  a->src = job.src;
  a->dst = job.dst;
  a->pool = pool_view(g, pool);
  a->packed = packed_view(g, packed);
  a->planes = (int)planes;
  a->plane_units = fast_div((int)(plane / kLeastPlane));
  a->per_entry = fast_div((int)per_entry);
  a->heads = fast_div(g.Hkv);
  a->head_words = fast_div(g.D / 8);
  a->pieces = fast_div(g.D * g.esize / 16);
  a->plane_words = fast_div((int)(plane / 8));
  a->plane_values = fast_div((int)(plane / 8 / (16 / g.esize)));
  a->Hkv = g.Hkv;
  a->lb = job.lb;
  return CS_OK;
}

// Pool pages with the non-temporal hint where they would not stay in the 256 MB
// cache anyway: 128 pages of 36 layers packed and brought back (604 MB of them) 172 ->
// 132 us, 256 brought back and turned 176 -> 172.
constexpr int64_t kOnceBytes = 128000000;
static bool once(const PagesArgs& a, const Geo& g) { return 2 * (int64_t)a.planes * g.T * g.D * g.esize >= kOnceBytes; }

template <typename E, bool ONCE>
static void run_pack(const PagesArgs& a, unsigned blocks, hipStream_t s) {
  TraceScope tr("pack_pages", s);
  CS_LAUNCH(tr, (pack_pages_kernel<E, ONCE>), dim3(blocks), dim3(kPageThreads), 0, s, a);
}
cs_status launch_pack(const Geo& g, const cs_page_pool& pool, const cs_packed_pool& packed, const PagesJob& job,
                      hipStream_t s, bool check_only) {
  PagesArgs a;
  unsigned blocks;
  const cs_status st = pages_args(g, pool, packed, job, "pack", &a, &blocks);
  if (st || check_only) return st;
  if (g.dtype == CS_BF16) once(a, g) ? run_pack<uint16_t, true>(a, blocks, s) : run_pack<uint16_t, false>(a, blocks, s);
  else once(a, g) ? run_pack<float, true>(a, blocks, s) : run_pack<float, false>(a, blocks, s);
  return check_launch("pack launch");
}

template <typename E, bool ONCE>
static void run_unpack(const TurnArgs& a, unsigned blocks, hipStream_t s) {
  TraceScope tr("unpack_pages", s);
  // (entries of a workgroup's planes, first and last in part)
  const int64_t planes = std::min<int64_t>(kMostPlanes, kShare / ((int64_t)a.packed.P * a.packed.D) + 2);
  const int64_t entries = (planes + a.per_entry.d - 1) / a.per_entry.d + 1;
  const size_t lds = (size_t)entries * (a.packed.D / 2) * sizeof(float2);
  if (a.offsets) CS_LAUNCH(tr, (unpack_pages_kernel<E, true, ONCE>), dim3(blocks), dim3(kPageThreads), lds, s, a);
  else CS_LAUNCH(tr, (unpack_pages_kernel<E, false, ONCE>), dim3(blocks), dim3(kPageThreads), 0, s, (const PagesArgs&)a);
}
cs_status launch_unpack(const Geo& g, const cs_packed_pool& packed, const cs_page_pool& pool, const PagesJob& job,
                        const double* theta, hipStream_t s, bool check_only) {
  TurnArgs a;
  unsigned blocks;
  const cs_status st = pages_args(g, pool, packed, job, "unpack", &a, &blocks);
  if (st || check_only) return st;
  a.offsets = job.offsets;
  a.sec0 = g.sec[0];
  a.sec01 = g.sec[0] + g.sec[1];
  for (int i = 0; i < g.P; ++i) a.theta[i] = theta[i];
  if (g.dtype == CS_BF16) once(a, g) ? run_unpack<uint16_t, true>(a, blocks, s) : run_unpack<uint16_t, false>(a, blocks, s);
  else once(a, g) ? run_unpack<float, true>(a, blocks, s) : run_unpack<float, false>(a, blocks, s);
  return check_launch("unpack launch");
}

}  // namespace cs
