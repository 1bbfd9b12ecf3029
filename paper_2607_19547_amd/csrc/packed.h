// Pages held in 4 bits: their layout, and the conversions.
//
// An element is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6, negatives) times a power of two
// 2^(byte - 127) that a block of 32 shares.  Keys are products' rows over D, so
// their blocks lie along a token's row; values are summed over tokens, so
// theirs lie along 32 tokens of a channel: in both a block is one operand's
// piece of a matrix instruction's sum, and a lane needs one scale for all that
// it converts.  gfx950's conversions take the code's byte and the scale's
// exponent at once (v_cvt_scalef32_*: round to nearest even, saturating; a scale
// byte of 255 gives NaN), and every value is exact in bf16.
#pragma once

#include "batch.h"

namespace cs {

constexpr int kBlock = 32;          // elements that share a scale
constexpr int kNanScale = 255;      // a block with an infinity or a NaN
constexpr int kLeastScale = 2, kMostScale = 252;  // 2^-125 .. 2^125: every value is a normal bf16 number

// A plane (layer, KV head) of a packed page: key codes [P][D/2], key scales
// [P/32][D/32][32], value codes [P/8][D][4] (byte w: tokens 2 w and 2 w + 1 of
// eight, the even one in the low half, as the even element of keys), value scales [P/32][D].
struct PackedView {
  char* base;
  int64_t page_bytes;
  int n_pages, P, D;
  __host__ __device__ __forceinline__ int codes() const { return P * D / 2; }
  __host__ __device__ __forceinline__ int scales() const { return P * D / kBlock; }
  __host__ __device__ __forceinline__ int k_scales() const { return codes(); }
  __host__ __device__ __forceinline__ int v_codes() const { return codes() + scales(); }
  __host__ __device__ __forceinline__ int v_scales() const { return 2 * codes() + scales(); }
  __host__ __device__ __forceinline__ int plane_bytes() const { return 2 * (codes() + scales()); }
};
PackedView packed_view(const Geo& g, const cs_packed_pool& p);

// The scale's exponent where the conversions read it (they take nothing else of
// the float): byte I of w.
template <int I>
__device__ __forceinline__ float scale_of(uint32_t w) {
  return __uint_as_float(I == 3 ? w >> 1 : w << (23 - 8 * I));
}
// Eight codes as bf16, one scale.
__device__ __forceinline__ bf16x8 decode8(uint32_t w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// One code (the slow kernel's).
__device__ __forceinline__ float decode1(uint32_t code, uint32_t scale_byte) {
  const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code & 15, scale_of<0>(scale_byte), 0);
  return v[0];
}

// ------------------------------------------------------------------ launches
// With check_only set a launcher validates its launch sizes and enqueues nothing.
struct PagesJob {
  const int32_t *src, *dst;  // DEVICE [n]
  const int32_t* offsets;    // DEVICE [n][3], or null
  int n, lb, le;
};
cs_status launch_pack(const Geo& g, const cs_page_pool& pool, const cs_packed_pool& packed, const PagesJob& job,
                      hipStream_t s, bool check_only);
cs_status launch_unpack(const Geo& g, const cs_packed_pool& packed, const cs_page_pool& pool, const PagesJob& job,
                        const double* theta, hipStream_t s, bool check_only);

}  // namespace cs
