// Rows and weights in 8 bits: e4m3 values with a float32 scale for each group of
// 128 columns (rows) or block of 128 x 128 (weights).
//
//   s = max(max |v| / 448, 2^-126),  q = e4m3(v / s), nearest, ties to even.
//
// 448 is the largest e4m3 value.  The smallest scale is the smallest normal
// number, so that a group of zeros divides like any other.
#pragma once

#include "device_common.h"

namespace dattri {
namespace dev {

constexpr int kGroup8 = 128;

// max(m, |v|); a NaN is left to its own element.
__device__ inline float max_mag(float m, float v) { return fmaxf(m, fabsf(v)); }

__device__ inline float scale8(float top) { return fmaxf(top / 448.f, 0x1p-126f); }

// v / s as a float32 division rounds it, from r = 1 / s rounded: the remainder
// of v r is exact in one fma (four operations; a division takes ten).  Its last
// bit is worth ulp(v r) ulp(s), which for scales under 2^-92 lies below float32's
// smallest value at quotients that e4m3 still tells apart (2^-10 and up): small
// scales and their values are first multiplied by a power of two, which changes
// no quotient.  An infinite scale leaves 0 or NaN as the division does.
struct Quotient8 {
  float up, s, r;
  __device__ explicit Quotient8(float scale) : up(scale < 0x1p-64f ? 0x1p64f : 1.f), s(scale * up), r(1.f / s) {}
  __device__ float of(float v) const {
    v *= up;
    const float q = v * r, e = fmaf(fmaf(-q, s, v), r, q);
    return s < __builtin_inff() ? e : q;
  }
};

// e4m3 of a and b (RNE) in the low (HI false) or high half of `old`.
template <bool HI>
__device__ inline int pack8(float a, float b, int old) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, HI);
}

__device__ inline float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

}  // namespace dev
}  // namespace dattri
