// Pages into 4 bits and back (keys turned on the way, Eq. 3).
//
// A plane's elements are taken 16,384 at a time by a workgroup, whatever the page
// and head sizes are: planes of small pages share one, large ones are split.
// Both ways a thread has whole 32-bit words of codes: eight elements of a key's
// row, or eight tokens of some channels of the values, whose block of 32 tokens
// lies in the four lanes of a quad.
#include "packed.h"

namespace cs {

constexpr int kPageThreads = 256;
constexpr int kShare = 16384;  // elements of a workgroup, of keys and of values

struct PagesArgs {
  const int32_t *src, *dst, *offsets;
  PoolView pool;
  PackedView packed;
  int64_t planes;           // entries x layers x KV heads
  FastDiv per_entry, heads, head_words, quads;  // planes of an entry; KV heads; D / 8; 16-byte pieces of a row
  FastDiv plane_words, plane_values;            // a plane's words of codes; its value items
  int Hkv, lb;
  int sec0, sec01;
  double theta[256];
};

// A 16-byte piece of a row: 8 or 4 elements.
template <typename E>
struct Piece {
  static constexpr int N = 16 / sizeof(E);
  u32x4 w;
};

// One block's scale byte from the bits of its largest magnitude (float32; an
// infinity or NaN has the largest of all): the least e with amax <= 7 x 2^e.
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

// Where a workgroup's elements lie: offset `off` of them from its first plane's
// start.
struct PlaneAt {
  int64_t plane;
  int at;  // item of the plane
};

// The pages of plane `plane` of the job, false where an entry is left out.
template <bool PACK>
__device__ __forceinline__ bool plane_bases(const PagesArgs& a, int plane, char** k, char** v, char** packed, int* entry) {
  const int e = a.per_entry.div(plane), x = plane - e * a.per_entry.d;
  const int l = a.heads.div(x), h = x - l * a.heads.d;
  const int s = a.src[e], d = a.dst[e], bf = PACK ? s : d, fp = PACK ? d : s;
  *entry = e;
  if ((unsigned)bf >= (unsigned)a.pool.n_pages || (unsigned)fp >= (unsigned)a.packed.n_pages) return false;
  const int64_t lh = (int64_t)(a.lb + l) * a.Hkv + h;
  const int64_t at = bf * a.pool.page_bytes + lh * a.pool.P * a.pool.row_bytes;
  *k = a.pool.k + at;
  *v = a.pool.v + at;
  *packed = a.packed.base + fp * a.packed.page_bytes + lh * a.packed.plane_bytes();
  return true;
}

template <typename E>
__global__ __launch_bounds__(kPageThreads) void pack_pages_kernel(const PagesArgs a) {
  constexpr bool kBf16 = sizeof(E) == 2;
  constexpr int W = Piece<E>::N;  // channels of a value item
  const int tid = threadIdx.x, D = a.packed.D;
  const int64_t first = (int64_t)blockIdx.x * kShare, pd = (int64_t)a.packed.P * D;
  const int64_t plane0 = first / pd;
  const int within = (int)(first - plane0 * pd);
  char *k, *v, *to;
  int entry;
  // keys: a word of codes per item
#pragma unroll 4
  for (int x = tid; x < kShare / 8; x += kPageThreads) {
    const int off = within / 8 + x, pl = a.plane_words.div(off), at = off - pl * a.plane_words.d;
    if (plane0 + pl >= a.planes || !plane_bases<true>(a, (int)(plane0 + pl), &k, &v, &to, &entry)) continue;
    const int row = a.head_words.div(at), c = at - row * a.head_words.d;
    u32x4 w[kBf16 ? 1 : 2];
    w[0] = *(const u32x4*)(k + (int64_t)at * 8 * sizeof(E));
    if constexpr (!kBf16) w[1] = *(const u32x4*)(k + (int64_t)at * 8 * sizeof(E) + 16);
    uint32_t m = 0;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      if constexpr (kBf16) m = max(m, max(w[0][y] << 16 & 0x7fff0000u, w[0][y] & 0x7fff0000u));
      else m = max(m, max(w[0][y] & 0x7fffffffu, w[1][y] & 0x7fffffffu));
    }
    const uint32_t e = scale_byte(quad_max(m));
    const float scale = __uint_as_float(e << 23);
    uint32_t code = 0;
    if constexpr (kBf16) {
      code = encode2<0>(code, w[0][0], scale);
      code = encode2<1>(code, w[0][1], scale);
      code = encode2<2>(code, w[0][2], scale);
      code = encode2<3>(code, w[0][3], scale);
    } else {
      code = encode2<0>(code, __uint_as_float(w[0][0]), __uint_as_float(w[0][1]), scale);
      code = encode2<1>(code, __uint_as_float(w[0][2]), __uint_as_float(w[0][3]), scale);
      code = encode2<2>(code, __uint_as_float(w[1][0]), __uint_as_float(w[1][1]), scale);
      code = encode2<3>(code, __uint_as_float(w[1][2]), __uint_as_float(w[1][3]), scale);
    }
    *(uint32_t*)(to + 4 * at) = e == kNanScale ? 0u : code;
    if ((c & 3) == 0) to[a.packed.k_scales() + (row >> 5) * D + (c >> 2) * kBlock + (row & 31)] = (char)e;
  }
  // values: eight tokens of W channels per item, the quad's lanes have a block's tokens
#pragma unroll 1
  for (int x = tid; x < kShare / (8 * W); x += kPageThreads) {
    const int off = within / (8 * W) + x, pl = a.plane_values.div(off), at = off - pl * a.plane_values.d;
    if (plane0 + pl >= a.planes || !plane_bases<true>(a, (int)(plane0 + pl), &k, &v, &to, &entry)) continue;
    const int tg = at & 3, blk = a.quads.div(at >> 2), c = (at >> 2) - blk * a.quads.d;  // token group of its block, piece of the row
    const char* from = v + ((int64_t)(blk * kBlock + 8 * tg) * D + W * c) * sizeof(E);
    u32x4 w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = *(const u32x4*)(from + (int64_t)j * D * sizeof(E));
    uint32_t codes[W], es[W];
#pragma unroll
    for (int d = 0; d < W; ++d) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, kBf16 ? (d & 1 ? w[j][d / 2] & 0x7fff0000u : w[j][d / 2] << 16 & 0x7fff0000u) : w[j][d] & 0x7fffffffu);
      es[d] = scale_byte(quad_max(m));
      const float scale = __uint_as_float(es[d] << 23);
      uint32_t code = 0;
      if constexpr (kBf16) {
        auto two = [&](int j) { return __builtin_amdgcn_perm(w[j + 1][d / 2], w[j][d / 2], d & 1 ? 0x07060302 : 0x05040100); };
        code = encode2<0>(code, two(0), scale);
        code = encode2<1>(code, two(2), scale);
        code = encode2<2>(code, two(4), scale);
        code = encode2<3>(code, two(6), scale);
      } else {
        code = encode2<0>(code, __uint_as_float(w[0][d]), __uint_as_float(w[1][d]), scale);
        code = encode2<1>(code, __uint_as_float(w[2][d]), __uint_as_float(w[3][d]), scale);
        code = encode2<2>(code, __uint_as_float(w[4][d]), __uint_as_float(w[5][d]), scale);
        code = encode2<3>(code, __uint_as_float(w[6][d]), __uint_as_float(w[7][d]), scale);
      }
      codes[d] = es[d] == kNanScale ? 0u : code;
    }
    u32x4* word = (u32x4*)(to + a.packed.v_codes() + ((int64_t)(blk * 4 + tg) * D + W * c) * 4);
#pragma unroll
    for (int y = 0; y < W / 4; ++y) word[y] = u32x4{codes[4 * y], codes[4 * y + 1], codes[4 * y + 2], codes[4 * y + 3]};
    if (tg == 0) {
      uint32_t* sc = (uint32_t*)(to + a.packed.v_scales() + blk * D + W * c);
#pragma unroll
      for (int y = 0; y < W / 4; ++y) sc[y] = es[4 * y] | es[4 * y + 1] << 8 | es[4 * y + 2] << 16 | es[4 * y + 3] << 24;
    }
  }
}

// Rotation: a thread has the same eight elements of both halves of a key.  The
// cos/sin tables of the workgroup's entries (its elements are of 1 + kShare /
// 1,024 planes at most, so of no more entries) are made in LDS first.
template <typename E, bool TURN>
__global__ __launch_bounds__(kPageThreads) void unpack_pages_kernel(const PagesArgs a) {
  constexpr bool kBf16 = sizeof(E) == 2;
  constexpr int W = Piece<E>::N;
  extern __shared__ float2 tab[];
  const int tid = threadIdx.x, D = a.packed.D, half = D >> 1;
  const int64_t first = (int64_t)blockIdx.x * kShare, pd = (int64_t)a.packed.P * D;
  const int64_t plane0 = first / pd;
  const int within = (int)(first - plane0 * pd);
  char *k, *v, *from;
  int entry;
  const int entry0 = a.per_entry.div((int)plane0);
  if constexpr (TURN) {
    const int64_t last = min(plane0 + (within + kShare - 1) / pd, a.planes - 1);
    const int n = a.per_entry.div((int)last) - entry0 + 1;
    for (int x = tid; x < n * half; x += kPageThreads) {
      const int e = x / half, i = x - e * half;
      tab[x] = cos_sin_of((double)a.offsets[3 * (int64_t)(entry0 + e) + axis_of(i, a.sec0, a.sec01)] * a.theta[i]);
    }
    __syncthreads();
  }
  // keys: two words of codes per item, of elements 8 c and D / 2 + 8 c
#pragma unroll 4
  for (int x = tid; x < kShare / 16; x += kPageThreads) {
    const int off = within / 16 + x, pl = a.plane_words.div(2 * off), at = off - pl * (a.plane_words.d >> 1);
    if (plane0 + pl >= a.planes || !plane_bases<false>(a, (int)(plane0 + pl), &k, &v, &from, &entry)) continue;
    const int row = a.head_words.div(2 * at), c = at - row * (a.head_words.d >> 1);
    const uint32_t wa = *(const uint32_t*)(from + (int64_t)row * half + 4 * c);
    const uint32_t wb = *(const uint32_t*)(from + (int64_t)row * half + (half >> 1) + 4 * c);
    const unsigned char* sc = (const unsigned char*)from + a.packed.k_scales() + (row >> 5) * D + (row & 31);
    const float sa = scale_of<0>(sc[(c >> 2) * kBlock]), sb = scale_of<0>(sc[((half + 8 * c) >> 5) * kBlock]);
    bf16x8 ya = decode8(wa, sa), yb = decode8(wb, sb);
    char* to = k + ((int64_t)row * D + 8 * c) * sizeof(E);
    float fa[8], fb[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      fa[i] = (float)ya[i];
      fb[i] = (float)yb[i];
    }
    if constexpr (TURN) {
      const int32_t* o = a.offsets + 3 * (int64_t)entry;
      if (o[0] | o[1] | o[2]) {
        const float2* t = tab + (entry - entry0) * half + 8 * c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 cs = t[i];
          const float p = fmaf(fa[i], cs.x, -(fb[i] * cs.y)), q = fmaf(fa[i], cs.y, fb[i] * cs.x);
          fa[i] = p;
          fb[i] = q;
        }
      }
    }
    if constexpr (kBf16) {
      u32x4 ra, rb;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ra[i] = pack_bf16x2(fa[2 * i], fa[2 * i + 1]);
        rb[i] = pack_bf16x2(fb[2 * i], fb[2 * i + 1]);
      }
      *(u32x4*)to = ra;
      *(u32x4*)(to + half * sizeof(E)) = rb;
    } else {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        ((f32x4*)to)[y] = f32x4{fa[4 * y], fa[4 * y + 1], fa[4 * y + 2], fa[4 * y + 3]};
        ((f32x4*)(to + half * sizeof(E)))[y] = f32x4{fb[4 * y], fb[4 * y + 1], fb[4 * y + 2], fb[4 * y + 3]};
      }
    }
  }
  // values: eight tokens of W channels per item
#pragma unroll 1
  for (int x = tid; x < kShare / (8 * W); x += kPageThreads) {
    const int off = within / (8 * W) + x, pl = a.plane_values.div(off), at = off - pl * a.plane_values.d;
    if (plane0 + pl >= a.planes || !plane_bases<false>(a, (int)(plane0 + pl), &k, &v, &from, &entry)) continue;
    const int tg = a.quads.div(at), c = at - tg * a.quads.d;  // eight tokens, piece of the row
    const u32x4* word = (const u32x4*)(from + a.packed.v_codes() + ((int64_t)tg * D + W * c) * 4);
    const uint32_t* sc = (const uint32_t*)(from + a.packed.v_scales() + (tg >> 2) * D + W * c);
    char* to = v + ((int64_t)(8 * tg) * D + W * c) * sizeof(E);
    u32x4 y[8];
#pragma unroll
    for (int g = 0; g < W / 4; ++g) {
      const u32x4 w = word[g];
      const uint32_t s = sc[g];
      const bf16x8 d0 = decode8(w[0], scale_of<0>(s)), d1 = decode8(w[1], scale_of<1>(s));
      const bf16x8 d2 = decode8(w[2], scale_of<2>(s)), d3 = decode8(w[3], scale_of<3>(s));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (kBf16) {
          y[j][2 * g] = __builtin_bit_cast(uint32_t, bf16x2{d0[j], d1[j]});
          y[j][2 * g + 1] = __builtin_bit_cast(uint32_t, bf16x2{d2[j], d3[j]});
        } else {
          y[j] = __builtin_bit_cast(u32x4, f32x4{(float)d0[j], (float)d1[j], (float)d2[j], (float)d3[j]});
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) *(u32x4*)(to + (int64_t)j * D * sizeof(E)) = y[j];
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
                            const double* theta, const char* what, PagesArgs* a, unsigned* blocks) {
  const int64_t per_entry = (int64_t)(job.le - job.lb) * g.Hkv, planes = per_entry * job.n;
  if (per_entry >= (int64_t(1) << 31) || planes >= (int64_t(1) << 31))
    return fail(CS_ERR_UNSUPPORTED, std::string(what) + ": pages x layers x KV heads must be below 2^31");
  const int64_t elements = planes * g.T * g.D;  // (planes below 2^31, a plane below 2^30)
  const int64_t n = (elements + kShare - 1) / kShare;
  const cs_status st = check_grid(n, 1, 1, kPageThreads, what);
  if (st) return st;
  *blocks = (unsigned)n;
  a->src = job.src;
  a->dst = job.dst;
  a->offsets = job.offsets;
  a->pool = pool_view(g, pool);
  a->packed = packed_view(g, packed);
  a->planes = planes;
  a->per_entry = fast_div((int)per_entry);
  a->heads = fast_div(g.Hkv);
  a->head_words = fast_div(g.D / 8);
  a->quads = fast_div(g.D * g.esize / 16);
  a->plane_words = fast_div((int)(g.T * g.D / 8));
  a->plane_values = fast_div((int)(g.T * g.D / 8 / (16 / g.esize)));
  a->Hkv = g.Hkv;
  a->lb = job.lb;
  a->sec0 = g.sec[0];
  a->sec01 = g.sec[0] + g.sec[1];
  for (int i = 0; i < g.P; ++i) a->theta[i] = theta ? theta[i] : 0.;
  return CS_OK;
}

cs_status launch_pack(const Geo& g, const cs_page_pool& pool, const cs_packed_pool& packed, const PagesJob& job,
                      hipStream_t s, bool check_only) {
  PagesArgs a;
  unsigned blocks;
  const cs_status st = pages_args(g, pool, packed, job, nullptr, "pack", &a, &blocks);
  if (st || check_only) return st;
  TraceScope tr("pack_pages", s);
  if (g.dtype == CS_BF16) CS_LAUNCH(tr, pack_pages_kernel<uint16_t>, dim3(blocks), dim3(kPageThreads), 0, s, a);
  else CS_LAUNCH(tr, pack_pages_kernel<float>, dim3(blocks), dim3(kPageThreads), 0, s, a);
  return check_launch("pack launch");
}

template <typename E>
static void run_unpack(const PagesArgs& a, unsigned blocks, int half, hipStream_t s) {
  TraceScope tr("unpack_pages", s);
  // (entries of a workgroup's planes, first and last in part: see the kernel)
  const int64_t planes = kShare / ((int64_t)a.packed.P * a.packed.D) + 2, entries = (planes + a.per_entry.d - 1) / a.per_entry.d + 1;
  const size_t lds = (size_t)entries * half * sizeof(float2);
  if (a.offsets) CS_LAUNCH(tr, (unpack_pages_kernel<E, true>), dim3(blocks), dim3(kPageThreads), lds, s, a);
  else CS_LAUNCH(tr, (unpack_pages_kernel<E, false>), dim3(blocks), dim3(kPageThreads), 0, s, a);
}
cs_status launch_unpack(const Geo& g, const cs_packed_pool& packed, const cs_page_pool& pool, const PagesJob& job,
                        const double* theta, hipStream_t s, bool check_only) {
  PagesArgs a;
  unsigned blocks;
  const cs_status st = pages_args(g, pool, packed, job, theta, "unpack", &a, &blocks);
  if (st || check_only) return st;
  if (g.dtype == CS_BF16) run_unpack<uint16_t>(a, blocks, g.P, s);
  else run_unpack<float>(a, blocks, g.P, s);
  return check_launch("unpack launch");
}

}  // namespace cs
