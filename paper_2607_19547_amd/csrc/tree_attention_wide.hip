// Attention of a batch's rows over their requests' pages for requests of many
// rows: trees of drafted tokens and questions (bf16, head_dim 128).
//
// With many query vectors the products bound the work, not the reading of the
// keys, so a K/V tile is staged in LDS once for 256 query vectors of a KV head:
// eight wavefronts of 32, two per SIMD.  Per 64-key tile a wavefront computes
//   S^T = K Q^T       (v_mfma_f32_32x32x16_bf16, K from LDS, Q in registers)
//   O^T += V^T P^T    (V^T by transposing reads of LDS, P^T from the scores' registers)
// with the softmax on the 32 scores of one query that a lane holds, in one
// block with the next tile's S^T, so that exponentials and products overlap.
// Tiles come by buffer-to-LDS loads into a ring of four, three ahead: one
// wavefront brings 8 keys, whose page it looks up through the scalar cache
// (pages are multiples of 16 tokens); rows behind the request's end, and rows
// of no page of the pool, read as zeros.
//
// Bound by the matrix instructions and the exponentials between them, at the
// clock that their power leaves: two questions of 389 rows over 32,768 tokens, 16 /
// 2 heads, 210 us, 1.0 PFLOP/s (1.07 with the rows that fill the last row tile; a
// product of two 8,192 x 8,192 matrices runs at 1.11); about 2 us a tile.  Starting a
// launch and leaving its pieces takes as long as 8 tiles.
//
// The work is cut as in the kernel for few rows (equal runs of key tiles, one
// run for each of 256 workgroups, one workgroup per CU).  A piece of a unit
// leaves its outputs, in the accumulators' own layout, divided by 2^e, so that a
// query vector's largest lies in [2^14, 2^15), and rounded to fp16: 11 bits
// of every element down to 2^-28 of that largest, an eighth of the output's
// own rounding, for half the bytes of float32 (a launch of 256 pieces leaves 17
// MB and the merge reads them: see tree_combine_wide).
#include <math.h>

#include <type_traits>

#include "tree_attention.h"

namespace cs {

constexpr int kKT = 64;                  // keys per tile
constexpr int kWideWaves = 8;
constexpr int kWideThreads = 64 * kWideWaves;
constexpr int kRow = 256;                // bytes of a K/V row
constexpr int kHiLds = 65536;            // LDS bytes below the K ring (the V ring)
constexpr float kRescaleLog2 = 5.f;      // growth of the running maximum before the accumulators are rescaled
constexpr int kWideRuns = 1 << kWideRunBits;
constexpr int kPartHalfs = 256 * 128;    // a partial's outputs
constexpr int kPartExp = 15;             // their largest is below 2^15
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) void lds_void;

// Lanes l and l ^ 32 hold the same query.
__device__ __forceinline__ float pair_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <bool ONCE>
__global__ __launch_bounds__(kWideThreads) void tree_attend_wide(const SplitArgs a0) {
  // LDS rows are 256 bytes, a key each, their 16-byte chunks permuted so that
  // the operand reads are free of bank conflicts (K: chunk c of row r at c ^
  // (r & 15); V: at c ^ 4 (r & 3)).  The V ring takes the low 64 KB, where the
  // DS instructions' 16-bit offsets reach; variables are laid out by name.
  __shared__ __attribute__((aligned(1024))) char lo_v0[kKT * kRow], lo_v1[kKT * kRow], lo_v2[kKT * kRow], lo_v3[kKT * kRow];
  __shared__ __attribute__((aligned(1024))) char up_k0[kKT * kRow], up_k1[kKT * kRow], up_k2[kKT * kRow], up_k3[kKT * kRow];
  auto kbuf = [&](auto B) -> char* {
    if constexpr (decltype(B)::value == 0) return up_k0;
    else if constexpr (decltype(B)::value == 1) return up_k1;
    else if constexpr (decltype(B)::value == 2) return up_k2;
    else return up_k3;
  };
  auto vbuf = [&](auto B) -> char* {
    if constexpr (decltype(B)::value == 0) return lo_v0;
    else if constexpr (decltype(B)::value == 1) return lo_v1;
    else if constexpr (decltype(B)::value == 2) return lo_v2;
    else return lo_v3;
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;

  // The arguments are read again where they are used, so that the tile loop
  // keeps none of them in registers.
  typedef const __attribute__((address_space(4))) SplitArgs* ArgPtr;
  const ArgPtr argp = (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
  auto args = [&]() -> SplitArgs {
    ArgPtr p = argp;
    asm volatile("" : "+s"(p));
    return *(const SplitArgs*)p;
  };
  const int tid = threadIdx.x, wave = uniform(tid >> 6), lane = tid & 63, ql = lane & 31, hi = lane >> 5;

  Run run;
  if (!find_run<true, true>(a0, blockIdx.x, &run)) return;
  int64_t left = run.end - run.begin, off = run.off;
  int b = run.b;

  int koff[8];  // K operand: row ql, chunk 2s + hi (row 32 + ql has the same swizzle)
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    koff[s] = ql * kRow + 16 * ((2 * s + hi) ^ (ql & 15));
    // opaque to constant folding, so that each read keeps this register as its
    // base and puts (slot - kHiLds) in the instruction's offset field
    asm("v_add_u32 %0, 0x10000, %1" : "=v"(koff[s]) : "v"(koff[s]));
  }
  const int vl = lane & 15, dh = (lane >> 4) & 1;
  int voff[4];  // V transposing reads: rows 4hi + vl/4 (+16ks, +8), dims 32d + 16dh + 4(vl%4)
#pragma unroll
  for (int d = 0; d < 4; ++d)
    voff[d] = (4 * hi + (vl >> 2)) * kRow + 16 * ((4 * d + 2 * dh + ((vl & 3) >> 1)) ^ ((vl >> 2) << 2)) + 8 * (vl & 1);
  int soff_k[2], soff_v[2];  // this lane's chunk within the wavefront's 8 keys, per load
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r = 4 * j + (lane >> 4), tr = 8 * wave + r, p = lane & 15;
    soff_k[j] = r * kRow + 16 * (p ^ (tr & 15));
    soff_v[j] = r * kRow + 16 * (p ^ ((tr & 3) << 2));
  }
  const float sc = a0.t.scale * kLog2e;

  while (left > 0) {
    Request q;
    int h, rt, t0, ntile;
    {
      const SplitArgs A = args();
      if (b >= A.t.B) break;  // (lengths that changed meanwhile)
      q = load_request_scalar(A.t, b);
      const Units units = unit_sizes<true>(A, q);
      if (off >= request_tiles(A, units)) {  // behind this request's units
        off = 0;
        ++b;
        continue;
      }
      const Place place = place_at<true>(A, q, units, off);
      h = place.h;
      rt = place.rt;
      t0 = place.t0;
      ntile = place.n;
      if (!ntile) {  // the empty end of a pair
        off += t0;
        left -= t0;
        continue;
      }
    }
    const int seg = (int)min(left, (int64_t)(ntile - t0));
    // all_see: keys that every row sees; g_row: the lane's row; w_seen: keys behind it are seen by no row of the wavefront
    int n_kt, key_begin, all_see, g_row, w_seen, bad;
    bf16x8 qb[8];
    {
      const SplitArgs A = args();
      const int vectors = q.n * A.t.G;
      // rows see no key behind their own without a mask, so later tiles are left out
      const int i_last = A.group.div(min((rt + 1) * 256, vectors) - 1);
      const int key_end = A.t.mask ? q.len : min(q.len, q.cached + i_last + 1);
      all_see = min(A.t.mask ? q.cached : q.cached + A.group.div(rt * 256) + 1, q.len);
      key_begin = t0 * kKT;
      n_kt = max(min(t0 + seg, (key_end + kKT - 1) / kKT) - t0, 0);
      const int v0 = rt * 256 + 32 * wave;
      const int qv = min(v0 + ql, vectors - 1);
      g_row = A.group.div(qv);
      w_seen = v0 >= vectors ? -1 : A.t.mask ? q.len : q.cached + uniform(A.group.div(min(v0 + 31, vectors - 1)));
    }

    // this wavefront's 8 keys of tile i: their page, and the loads into a ring
    // slot (what they need of the arguments stays in scalar registers: read
    // again in every step it would hold the step up)
    int page_next = 0;
    FastDiv page;
    scalar_ptr table;
    const char *k_plane, *v_plane;
    int64_t page_bytes;
    int n_pages;
    {
      const SplitArgs A = args();
      page = A.t.page;
      table = (scalar_ptr)(uint64_t)(A.t.table + (int64_t)b * A.t.max_blocks);
      const int64_t plane = ((int64_t)A.t.layer * A.t.Hkv + h) * page.d * kRow;
      k_plane = A.t.pool.k + plane;
      v_plane = A.t.pool.v + plane;
      page_bytes = A.t.pool.page_bytes;
      n_pages = A.t.pool.n_pages;
    }
    const int last_key = q.len - 1, key_wave = key_begin + 8 * wave;
    auto find_page = [&](int i) {
      if (last_key >= 0) page_next = table[page.div(min(key_wave + i * kKT, last_key))];
    };
    auto fetch = [&](int i, char* Kd, char* Vd) {
      const int key = key_wave + i * kKT;
      const bool ok = i < n_kt && key <= last_key && (unsigned)page_next < (unsigned)n_pages;
      const int64_t at = page_next * page_bytes + (int64_t)(key - page.div(key) * page.d) * kRow;
      const int bytes = ok ? min(last_key + 1 - key, 8) * kRow : 0;  // (no bytes: no address is used)
      const auto rk = rows_rsrc(k_plane + at, bytes), rv = rows_rsrc(v_plane + at, bytes);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r0 = 8 * wave + 4 * j;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void*)(Kd + r0 * kRow), 16, soff_k[j], 0, 0, ONCE ? kNonTemporal : 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void*)(Vd + r0 * kRow), 16, soff_v[j], 0, 0, ONCE ? kNonTemporal : 0);
      }
      find_page(i + 1);
    };
    find_page(0);
    fetch(0, up_k0, lo_v0);
    fetch(1, up_k1, lo_v1);
    {
      const SplitArgs A = args();
      const int qv = min(rt * 256 + 32 * wave + ql, q.n * A.t.G - 1);
      const uint16_t* qp = (const uint16_t*)A.t.q + (int64_t)(q.r0 + g_row) * A.t.q_row +
                           (h * A.t.G + qv - g_row * A.t.G) * A.t.q_head + 8 * hi;
#pragma unroll
      for (int s = 0; s < 8; ++s) qb[s] = *(const bf16x8*)(qp + 16 * s);
      // pages of this piece that are none of the pool
      bad = 0;
      if (n_kt > 0) {
        const int p0 = A.t.page.div(key_begin), p1 = A.t.page.div(min(key_begin + n_kt * kKT, q.len) - 1);
        const int32_t* tb = A.t.table + (int64_t)b * A.t.max_blocks;
        for (int x = p0 + tid; x <= p1; x += kWideThreads) bad |= tb[x] < 0 || tb[x] >= A.t.pool.n_pages;
      }
    }
    fetch(2, up_k2, lo_v2);
    bad = __syncthreads_or(bad);

    f32x16 o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] = f32x16{};
    float m_use = -INFINITY, l_run = 0.f;
    bool seen = false;

    auto qk = [&](const char* K, f32x16& s0, f32x16& s1) {
      s0 = f32x16{};
      s1 = f32x16{};
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const bf16x8 k0 = *(const bf16x8*)(K - kHiLds + koff[s]);
        const bf16x8 k1 = *(const bf16x8*)(K - kHiLds + 32 * kRow + koff[s]);
        s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, qb[s], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, qb[s], s1, 0, 0, 0);
      }
    };
    // V operand of 16 keys ks and 32 dims d
    auto v_operand = [&](const char* V, int ks, int d) {
      const char* vp = V + ks * 16 * kRow + voff[d];
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(vp));
      const bf16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(vp + 8 * kRow));
      return __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    // Tiles with the step's own rows, the request's end or keys in no page of
    // the pool: the keys that the lane's row does not see get -inf.
    // Accumulator register r of block y holds key kt + 32 y + 8 (r / 4) + 4 hi + r % 4.
    auto visible = [&](int kt) -> uint64_t {  // bit 32 y + 8 (r / 4) + r % 4 belongs to register r of block y
      const SplitArgs A = args();
      uint64_t vis;
      {
        const int w0 = kt - q.cached, w = max(w0, 0);
        uint64_t bits = 0;
        if (A.t.mask) {
          const unsigned long long* mk = A.t.mask + (int64_t)(q.r0 + g_row) * A.t.words;
          const int j = w >> 6, sft = w & 63;
          if (w0 > -kKT && j < A.t.words) bits = mk[j] >> sft;
          if (w0 > -kKT && sft && j + 1 < A.t.words) bits |= mk[j + 1] << (64 - sft);
        } else {
          const int n = g_row - w + 1;
          bits = n >= 64 ? ~0ull : n > 0 ? (1ull << n) - 1 : 0ull;
        }
        vis = w0 <= -64 ? ~0ull : w0 < 0 ? bits << -w0 | ((1ull << -w0) - 1) : bits;
        const int n = q.len - kt;
        vis &= n >= 64 ? ~0ull : (1ull << n) - 1;
        if (bad) {
          const scalar_ptr tb = (scalar_ptr)(uint64_t)(A.t.table + (int64_t)b * A.t.max_blocks);
          for (int y = 0; y < 4; ++y) {
            const int pg = tb[A.t.page.div(min(kt + 16 * y, q.len - 1))];
            if (pg < 0 || pg >= A.t.pool.n_pages) vis &= ~(0xffffull << (16 * y));
          }
        }
      }
      seen = seen || vis != 0;
      return vis >> (4 * hi);
    };
    auto mask = [&](int kt, f32x16& s0, f32x16& s1) {
      const uint64_t mine = visible(kt);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int bit = 8 * (r >> 2) + (r & 3);
        if (!((uint32_t)mine >> bit & 1)) s0[r] = -INFINITY;
        if (!((uint32_t)(mine >> 32) >> bit & 1)) s1[r] = -INFINITY;
      }
    };
    // Values that are not finite must not reach rows that do not see them
    // (0 x inf).  Where the tile has one (every wavefront finds the same), the
    // products count, for each output element, the values of +inf (or NaN) and
    // of -inf (or NaN) that its row sees; those give it the infinity, both of
    // them NaN.  Then the values become zero in LDS.  (After the accumulators
    // are rescaled for the tile: their first factor is 0.)
    auto not_finite = [&](char* V, int kt) {
      uint32_t odd = 0;
      int x = lane;
      asm volatile("" : "+v"(x));  // (worked out here, not kept through the tiles)
      for (; x < kKT * kRow / 16; x += 64) {
        const u32x4 v = *(const u32x4*)(V + 16 * x);
#pragma unroll
        for (int y = 0; y < 4; ++y) odd |= (v[y] & 0x7f807f80u) + 0x00800080u;
      }
      if (__ballot(odd & 0x80008000u)) {
        const uint64_t mine = visible(kt);
#pragma unroll 1
        for (int sign = 0; sign < 2; ++sign) {
          auto flag = [&](uint32_t v) -> uint32_t {  // 1.0 in bf16 where the element counts
            const bool nan = (v & 0x7f80u) == 0x7f80u && (v & 0x7fu);
            return nan || (v & 0xffffu) == (sign ? 0xff80u : 0x7f80u) ? 0x3f80u : 0u;
          };
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            f32x16 c = f32x16{};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
              u32x4 va = __builtin_bit_cast(u32x4, v_operand(V, ks, d)), pb;
#pragma unroll
              for (int y = 0; y < 4; ++y) va[y] = flag(va[y]) | flag(va[y] >> 16) << 16;
              // the operand's elements x are registers 8 (ks & 1) + x of block ks / 2
              const uint32_t bits = (uint32_t)(mine >> (32 * (ks >> 1) + 16 * (ks & 1)));
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const int b0 = 8 * (y >> 1) + 2 * (y & 1);
                pb[y] = (bits >> b0 & 1 ? 0x3f80u : 0u) | (bits >> (b0 + 1) & 1 ? 0x3f800000u : 0u);
              }
              c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, va), __builtin_bit_cast(bf16x8, pb), c, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (c[r] > 0.f) o[d][r] += sign ? -INFINITY : INFINITY;
          }
        }
        __syncthreads();  // every wavefront has read the tile
        for (int x = tid; x < kKT * kRow / 4; x += kWideThreads) {
          uint32_t v = *(const uint32_t*)(V + 4 * x);
          if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
          if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
          *(uint32_t*)(V + 4 * x) = v;
        }
        __syncthreads();
      }
    };

    // Running maximum of the tile; rescales the accumulators when it grew by more than 2^5.
    auto tile_max = [&](f32x16& s0, f32x16& s1) {
      float t8[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) t8[r] = fmaxf(fmaxf(s0[r], s0[r + 8]), s1[r]);
      float t4[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) t4[r] = fmaxf(fmaxf(t8[2 * r], t8[2 * r + 1]), s1[r + 8]);
      const float t2a = fmaxf(fmaxf(t4[0], t4[1]), s1[12]), t2b = fmaxf(fmaxf(t4[2], t4[3]), s1[13]);
      const float mx = fmaxf(fmaxf(fmaxf(t2a, t2b), s1[14]), s1[15]);
      const float mt = pair_max(mx) * sc;
      const bool need = mt > m_use + kRescaleLog2;
      if (__ballot(need)) {
        const float m_new = need ? mt : m_use;
        const float alpha = need ? __builtin_amdgcn_exp2f(m_use - m_new) : 1.f;
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= alpha;
        m_use = m_new;
      }
    };
    auto qk_head = [&](const char* K, f32x16& n0, f32x16& n1) {
      n0 = f32x16{};
      n1 = f32x16{};
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const bf16x8 k0 = *(const bf16x8*)(K - kHiLds + koff[s]);
        const bf16x8 k1 = *(const bf16x8*)(K - kHiLds + 32 * kRow + koff[s]);
        n0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, qb[s], n0, 0, 0, 0);
        n1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, qb[s], n1, 0, 0, 0);
      }
    };
    // Probabilities of the current tile, O^T += V^T P^T, and k-steps 2..7 of
    // the next tile's S^T in one straight-line block.
    auto exp_pv_qk = [&](const char* V, const char* K, f32x16& s0, f32x16& s1, f32x16& n0, f32x16& n1) {
      __builtin_amdgcn_iglp_opt(3);
      const float nm = m_use == -INFINITY ? 0.f : -m_use;
      bf16x8 pb[4];
      float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const f32x16& sv = ks < 2 ? s0 : s1;
        const int base = 8 * (ks & 1);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sv[base + x], sc, nm));
          ls[ks] += p;  // (the sum of the unrounded probabilities)
          pb[ks][x] = (__bf16)p;
        }
        if (ks < 3) {
#pragma unroll
          for (int s = 2 * ks + 2; s < 2 * ks + 4; ++s) {
            const bf16x8 k0 = *(const bf16x8*)(K - kHiLds + koff[s]);
            const bf16x8 k1 = *(const bf16x8*)(K - kHiLds + 32 * kRow + koff[s]);
            n0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, qb[s], n0, 0, 0, 0);
            n1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, qb[s], n1, 0, 0, 0);
          }
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(V, ks, d), pb[ks], o[d], 0, 0, 0);
      }
      l_run += (ls[0] + ls[1]) + (ls[2] + ls[3]);
    };

    // Tile i is in ring slot C, tile i + 1 in N; tile i + 3 goes to S (read last
    // in step i - 1).  Each wavefront waits for its part of tile i + 2 (all but
    // its four newest loads) before the barrier.
    auto step = [&](auto C, auto N, auto S, int i, f32x16& c0, f32x16& c1, f32x16& n0, f32x16& n1) {
      fetch(i + 3, kbuf(S), vbuf(S));
      if (w_seen >= 0) {
        qk_head(kbuf(N), n0, n1);
        tile_max(c0, c1);
        exp_pv_qk(vbuf(C), kbuf(N), c0, c1, n0, n1);
      }
      asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
      __builtin_amdgcn_s_barrier();
    };
    // First the tiles that every row sees whole, their ring slots known to the
    // compiler, a tile's scores computed a step ahead; then, in a plain loop, the
    // few with the step's own rows.
    const int n_clear = bad ? 0 : min(max(all_see / kKT - t0, 0), n_kt);
    f32x16 sa0, sa1, sb0, sb1;
    asm volatile("s_waitcnt vmcnt(4)" ::: "memory");  // tiles 0 and 1 and the queries have landed
    __builtin_amdgcn_s_barrier();
    if (n_clear > 0) qk(up_k0, sa0, sa1);
    for (int i = 0; i < n_clear; i += 4) {
      step(I0{}, I1{}, I3{}, i, sa0, sa1, sb0, sb1);
      if (i + 1 >= n_clear) break;
      step(I1{}, I2{}, I0{}, i + 1, sb0, sb1, sa0, sa1);
      if (i + 2 >= n_clear) break;
      step(I2{}, I3{}, I1{}, i + 2, sa0, sa1, sb0, sb1);
      if (i + 3 >= n_clear) break;
      step(I3{}, I0{}, I2{}, i + 3, sb0, sb1, sa0, sa1);
    }
    seen = n_clear > 0;
    auto k_at = [&](int x) -> char* { return x & 2 ? (x & 1 ? up_k3 : up_k2) : (x & 1 ? up_k1 : up_k0); };
    auto v_at = [&](int x) -> char* { return x & 2 ? (x & 1 ? lo_v3 : lo_v2) : (x & 1 ? lo_v1 : lo_v0); };
#pragma unroll 1
    for (int i = n_clear; i < n_kt; ++i) {
      const int kt = key_begin + i * kKT;
      fetch(i + 3, k_at(i + 3), v_at(i + 3));
      char* V = v_at(i);
      if (kt <= w_seen) {
        qk(k_at(i), sa0, sa1);
        mask(kt, sa0, sa1);
        tile_max(sa0, sa1);
      }
      not_finite(V, kt);  // (has barriers: every wavefront)
      if (kt <= w_seen) {
        const float nm = m_use == -INFINITY ? 0.f : -m_use;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          bf16x8 pb;
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const float p = __builtin_amdgcn_exp2f(fmaf((ks < 2 ? sa0 : sa1)[8 * (ks & 1) + x], sc, nm));
            l_run += p;
            pb[x] = (__bf16)p;
          }
#pragma unroll
          for (int d = 0; d < 4; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(V, ks, d), pb, o[d], 0, 0, 0);
        }
      }
      asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
      __builtin_amdgcn_s_barrier();
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    // Results: accumulator register r of block d holds dim 32d + 8(r/4) + 4hi + r%4.
    const SplitArgs A = args();
    const int vectors = q.n * A.t.G, qv = rt * 256 + 32 * wave + ql;
    float lt = pair_sum(l_run);
    if (seen && m_use == -INFINITY) {
      m_use = kOnlyMinusInf;
      lt += 1.f;
    }
    if (seg == ntile) {
      // Through LDS, so that the stores write whole lines (stores of the lanes' own
      // 8 bytes, a row each: 61 questions of 388 rows 157 us, so 146).
      // A wavefront has 8 KB of the ring to itself, chunk c of a row at c ^ (row & 15).
      __builtin_amdgcn_s_barrier();  // the last loads of every wavefront have landed
      asm volatile("" ::: "memory");
      lt = final_sum(m_use, lt);
      const float inv = lt == 0.f ? 0.f : 1.f / lt;
      char* rows = v_at(wave >> 1) + (wave & 1) * 32 * kRow;
      int at = lane;
      asm volatile("" : "+v"(at));  // (places worked out here, not kept through the tiles)
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          u32x2 w;
          w[0] = pack_bf16x2(o[d][4 * r] * inv, o[d][4 * r + 1] * inv);
          w[1] = pack_bf16x2(o[d][4 * r + 2] * inv, o[d][4 * r + 3] * inv);
          *(u32x2*)(rows + (at & 31) * kRow + 16 * ((4 * d + r) ^ (at & 15)) + 8 * (at >> 5)) = w;
        }
      if (A.t.lse && hi == 0 && qv < vectors)
        A.t.lse[(int64_t)(q.r0 + g_row) * A.t.Hq + h * A.t.G + qv - g_row * A.t.G] = (m_use + __log2f(lt)) * kLn2;
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int r = 4 * y + (at >> 4), v = rt * 256 + 32 * wave + r, i = A.group.div(v);
        const u32x4 w = *(const u32x4*)(rows + r * kRow + 16 * ((at & 15) ^ (r & 15)));
        if (v < vectors)
          *(u32x4*)((uint16_t*)A.t.out + (int64_t)(q.r0 + i) * A.t.o_row + (h * A.t.G + v - i * A.t.G) * A.t.o_head + 8 * (at & 15)) = w;
      }
    } else {
      const int64_t slot = 2 * (int64_t)run.w + (t0 == 0);
      float amax = 0.f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) amax = fmaxf(amax, fabsf(o[d][r]) < INFINITY ? fabsf(o[d][r]) : 0.f);
      const int e = __builtin_amdgcn_frexp_expf(pair_max(amax)) - kPartExp;  // (of zero: 0)
      if (hi == 0) *(float4*)(A.part_ml + (slot * 256 + 32 * wave + ql) * 4) = make_float4(m_use, lt, (float)e, 0.f);
      _Float16* pp = (_Float16*)A.part + slot * kPartHalfs + wave * (8 * 512) + lane * 8;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          f16x8 w;
#pragma unroll
          for (int x = 0; x < 8; ++x) w[x] = (_Float16)__builtin_ldexpf(o[d][8 * r + x], -e);
          *(f16x8*)(pp + (2 * d + r) * 512) = w;
        }
    }
    left -= seg;
    off += seg;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // the ring is free (the stores need not have landed)
    asm volatile("" ::: "memory");
  }
}

// Merges the pieces of a unit, in key order.  A strip is what one store of a
// wavefront left, 1 KB in a row: 8 elements of 32 query vectors' halves.  The
// unit's 64 strips are shared by the workgroups of the borders inside it,
// blockIdx.y among them.  With few pieces a wavefront takes a strip through all
// of them; with many, four wavefronts take the pieces of a strip in turn.
constexpr int kStripThreads = 256;
constexpr int kStripShare = 4;
constexpr int kRound = 8;
__global__ __launch_bounds__(kStripThreads) void tree_combine_wide(const SplitArgs a) {
  __shared__ float s_acc[4][8][64], s_m[4][64], s_l[4][64];
  const TreeArgs& t = a.t;
  const int w1 = blockIdx.x + 1;
  Run run;
  if (!find_run<true>(a, w1, &run)) return;
  const Request q = load_request_scalar(t, run.b);
  const Place at = place_at<true>(a, q, unit_sizes<true>(a, q), run.off);
  if (at.t0 == 0 || at.n == 0) return;  // the border lies between row tiles
  const int h = at.h, rt = at.rt;
  const int64_t len = run_length(a, run.total), unit0 = run.begin - at.t0;
  const int w0 = quotient(unit0, len), w_last = quotient(unit0 + at.n - 1, len);
  const int pieces = w_last - w0 + 1, borders = pieces - 1;
  const int vectors = min(256, q.n * t.G - rt * 256);
  const int lane = threadIdx.x & 63, ql = lane & 31, hi = lane >> 5, grp = uniform(threadIdx.x >> 6);
  const bool many = pieces > kRound;
  const int step = many ? 4 : 1, strips = (vectors + 31) / 32 * 8;
  const int lot = (w1 - 1 - w0) * kStripShare + blockIdx.y;
  for (int strip = many ? lot : lot * 4 + grp; strip < strips; strip += borders * kStripShare * (many ? 1 : 4)) {
    const int wave = strip >> 3, c = strip & 7, r = 32 * wave + ql;
    Merge<8> mg;
    for (int x0 = many ? grp : 0; x0 < pieces; x0 += kRound * step) {
      float4 st[kRound];
      f16x8 v16[kRound];
#pragma unroll
      for (int y = 0; y < kRound; ++y) {
        const int x = min(x0 + y * step, pieces - 1);
        const int64_t slot = 2 * (int64_t)(w0 + x) + (x == 0);
        st[y] = *(const float4*)(a.part_ml + (slot * 256 + r) * 4);
        v16[y] = *(const f16x8*)((const _Float16*)a.part + slot * kPartHalfs + strip * 512 + lane * 8);
      }
      float2 ml[kRound];
      float v[kRound][8];
#pragma unroll
      for (int y = 0; y < kRound; ++y) {
        ml[y] = x0 + y * step < pieces ? make_float2(st[y].x, st[y].y) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[y][e] = __builtin_ldexpf((float)v16[y][e], (int)st[y].z);
      }
      mg.add(ml, v);
    }
    if (many) {
      __syncthreads();  // the previous strip has been read
      s_m[grp][lane] = mg.m;
      s_l[grp][lane] = mg.sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) s_acc[grp][e][lane] = mg.acc[e];
      __syncthreads();
      if (grp) continue;
      float2 ml[4];
      float v[4][8];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        ml[x] = make_float2(s_m[x][lane], s_l[x][lane]);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[x][e] = s_acc[x][e][lane];
      }
      mg = Merge<8>();
      mg.add(ml, v);
    }
    if (r >= vectors) continue;
    const int qv = rt * 256 + r, i = a.group.div(qv), head = h * t.G + qv - i * t.G;
    const float inv = mg.scale();
    uint16_t* op = (uint16_t*)t.out + (int64_t)(q.r0 + i) * t.o_row + head * t.o_head + 16 * c + 4 * hi;
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // elements 4x .. 4x + 3 are dims 16c + 8x + 4hi ..
      u32x2 w;
      w[0] = pack_bf16x2(mg.acc[4 * x] * inv, mg.acc[4 * x + 1] * inv);
      w[1] = pack_bf16x2(mg.acc[4 * x + 2] * inv, mg.acc[4 * x + 3] * inv);
      *(u32x2*)(op + 8 * x) = w;
    }
    if (t.lse && c == 0 && hi == 0) t.lse[(int64_t)(q.r0 + i) * t.Hq + head] = mg.lse();
  }
}

size_t tree_wide_workspace() { return 2 * (size_t)kWideRuns * (kPartHalfs * sizeof(_Float16) + 4 * 256 * sizeof(float)) + 512; }

void launch_tree_wide(SplitArgs a, void* ws, bool once, hipStream_t s) {
  a.row_bits = kWideRowBits;
  a.tile_bits = kWideTileBits;
  a.run_bits = kWideRunBits;
  a.min_tiles = 4;
  a.units = fast_div(even_units(a));
  a.by_xcd = !a.t.mask;
  a.part = (float*)(((uintptr_t)ws + 255) & ~(uintptr_t)255);
  a.part_ml = a.part + 2 * (size_t)kWideRuns * kPartHalfs / 2;
  const int runs = most_runs(a);
  {
    TraceScope tr("tree_attend_wide", s);
    if (once) CS_LAUNCH(tr, tree_attend_wide<true>, dim3((runs + 7) / 8 * 8), dim3(kWideThreads), 0, s, a);
    else CS_LAUNCH(tr, tree_attend_wide<false>, dim3((runs + 7) / 8 * 8), dim3(kWideThreads), 0, s, a);
  }
  if (runs == 1) return;
  TraceScope tr("tree_combine_wide", s);
  CS_LAUNCH(tr, tree_combine_wide, dim3(runs - 1, kStripShare), dim3(kStripThreads), 0, s, a);
}

}  // namespace cs
