// What becomes of four neighbouring elements (m, n .. n + 3) of a linear
// layer's product: bias, activation, residual, the kept pre-activation; the
// slope of the activation below; or the float32 weight gradient.  Everything is
// float32 until the one rounding to the output's type.
#pragma once

#include "activation.h"
#include "device_common.h"
#include "model_ops.h"

namespace dattri {
namespace dev {

template <int ELT>
__device__ inline float load_elt(const void* p, int64_t i) {
  return ELT == 2 ? bf16_bits_to_f32(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}
template <int ELT>
__device__ inline void store_elt(void* p, int64_t i, float v) {
  if (ELT == 2)
    ((uint16_t*)p)[i] = (uint16_t)pack_bf16(v, 0.f);
  else
    ((float*)p)[i] = v;
}

// Four elements from index i; `vec`: one aligned load or store, else the first `cnt` one by one.
template <int ELT>
__device__ inline f32x4 load4_elt(const void* p, int64_t i, bool vec, int cnt) {
  if (vec) {
    if constexpr (ELT == 2) {
      const i32x2 w = *(const i32x2*)((const uint16_t*)p + i);
      const uint32_t a = (uint32_t)w.x, b = (uint32_t)w.y;
      return f32x4{__builtin_bit_cast(float, a << 16), __builtin_bit_cast(float, a & 0xFFFF0000u),
                   __builtin_bit_cast(float, b << 16), __builtin_bit_cast(float, b & 0xFFFF0000u)};
    } else {
      return *(const f32x4*)((const float*)p + i);
    }
  }
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < cnt) v[e] = load_elt<ELT>(p, i + e);
  return v;
}
template <int ELT>
__device__ inline void store4_elt(void* p, int64_t i, f32x4 v, bool vec, int cnt) {
  if (vec) {
    if constexpr (ELT == 2)
      *(i32x2*)((uint16_t*)p + i) = i32x2{(int)pack_bf16(v.x, v.y), (int)pack_bf16(v.z, v.w)};
    else
      *(f32x4*)((float*)p + i) = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < cnt) store_elt<ELT>(p, i + e, v[e]);
}

// m < M and n < N; a.vec: every row of the epilogue's buffers starts on four elements.
template <int OP, int ELT>
__device__ inline void epilogue4(const GemmArgs& a, int m, int n, f32x4 v) {
  const int cnt = a.N - n;
  const bool vec = a.vec && cnt >= 4;
  if constexpr (OP == DATTRI_LINEAR_FORWARD) {
    if (a.bias) v += load4_elt<ELT>(a.bias, n, vec, cnt);
    if (a.Z) store4_elt<ELT>(a.Z, m * a.ldz + n, v, vec, cnt);
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (a.R) r = load4_elt<ELT>(a.R, m * a.ldr + n, vec, cnt);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = act_value<ELT>(v[e], a.act);
    if (a.R) v += r;
    store4_elt<ELT>(a.out, m * a.ldo + n, v, vec, cnt);
  } else if constexpr (OP == DATTRI_LINEAR_INPUT_GRAD) {
    const bool slope = a.out2 && a.act != DATTRI_ACT_NONE;
    f32x4 z = {0.f, 0.f, 0.f, 0.f};
    if (slope) z = load4_elt<ELT>(a.Z, m * a.ldz + n, vec, cnt);
    if (a.R) v += load4_elt<ELT>(a.R, m * a.ldr + n, vec, cnt);
    if (a.out) store4_elt<ELT>(a.out, m * a.ldo + n, v, vec, cnt);
    if (!a.out2) return;
    if (slope) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float s = act_slope<ELT>(z[e], a.act);
        v[e] = a.act == DATTRI_ACT_RELU && s == 0.f ? 0.f : v[e] * s;  // a closed relu passes nothing, not 0 * inf
      }
    }
    store4_elt<ELT>(a.out2, m * a.ldo2 + n, v, vec, cnt);
  } else {
    if (a.accumulate) v += load4_elt<4>(a.out, m * a.ldo + n, vec, cnt);
    store4_elt<4>(a.out, m * a.ldo + n, v, vec, cnt);
  }
}

}  // namespace dev
}  // namespace dattri
