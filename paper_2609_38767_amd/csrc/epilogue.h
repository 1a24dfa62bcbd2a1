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

// v = act(v) and v *= act'(z) for U times four values, one choice of activation for all.
template <int ELT, int U>
__device__ inline void act_values(f32x4 (&v)[U], int act) {
  with_act(act, [&](auto kind) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[u][e] = act_value<ELT>(v[u][e], decltype(kind)::value);
  });
}
template <int ELT, int U>
__device__ inline void slope_values(f32x4 (&v)[U], const f32x4 (&z)[U], int act) {
  with_act(act, [&](auto kind) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float s = act_slope<ELT>(z[u][e], decltype(kind)::value);
        // a closed relu passes nothing, not 0 * inf
        v[u][e] = decltype(kind)::value == DATTRI_ACT_RELU && s == 0.f ? 0.f : v[u][e] * s;
      }
  });
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
    f32x4 y[1] = {v};
    act_values<ELT, 1>(y, a.act);
    v = y[0];
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
      f32x4 p[1] = {v};
      const f32x4 at[1] = {z};
      slope_values<ELT, 1>(p, at, a.act);
      v = p[0];
    }
    store4_elt<ELT>(a.out2, m * a.ldo2 + n, v, vec, cnt);
  } else {
    if (a.accumulate) v += load4_elt<4>(a.out, m * a.ldo + n, vec, cnt);
    store4_elt<4>(a.out, m * a.ldo + n, v, vec, cnt);
  }
}

// Four elements of a buffer from byte offset `off` (range checked): neighbours
// (APART 1), or APART elements from each other, of which the first `cnt` exist.
template <int ELT, int APART>
__device__ inline f32x4 buffer_load4(rsrc_t r, uint32_t off, int cnt) {
  if constexpr (APART > 1) {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t o = e < cnt ? off + e * APART * ELT : kOOB;
      v[e] = ELT == 2 ? bf16_bits_to_f32(load2(r, o)) : __builtin_bit_cast(float, load4(r, o));
    }
    return v;
  } else if constexpr (ELT == 2) {
    const i32x2 w = load8(r, off);
    const uint32_t a = (uint32_t)w.x, b = (uint32_t)w.y;
    return f32x4{__builtin_bit_cast(float, a << 16), __builtin_bit_cast(float, a & 0xFFFF0000u),
                 __builtin_bit_cast(float, b << 16), __builtin_bit_cast(float, b & 0xFFFF0000u)};
  } else {
    return __builtin_bit_cast(f32x4, load16(r, off));
  }
}
template <int ELT, int APART>
__device__ inline void buffer_store4(rsrc_t r, uint32_t off, f32x4 v, int cnt) {
  if constexpr (APART > 1) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t o = e < cnt ? off + e * APART * ELT : kOOB;
      if constexpr (ELT == 2)
        __builtin_amdgcn_raw_buffer_store_b16((short)pack_bf16(v[e], 0.f), r, o, 0, 0);
      else
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(int, (float)v[e]), r, o, 0, 0);
    }
  } else if constexpr (ELT == 2) {
    __builtin_amdgcn_raw_buffer_store_b64(i32x2{(int)pack_bf16(v.x, v.y), (int)pack_bf16(v.z, v.w)}, r, off, 0, 0);
  } else {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(i32x4, v), r, off, 0, 0);
  }
}

// A buffer of the epilogue seen from a tile: rows m0 .. (rows of them exist),
// columns n0 .. n0 + width - 1.  Rows past the last are out of its range.
template <int ELT>
struct TileRows {
  rsrc_t r;
  uint32_t ld;
  __device__ TileRows(const void* p, int64_t ld_elts, int m0, int n0, int rows, int width) {
    ld = (uint32_t)(ld_elts * ELT);
    r = make_rsrc((const uint8_t*)p + ((int64_t)m0 * ld_elts + n0) * ELT,
                  p ? (uint32_t)(rows - 1) * ld + (uint32_t)width * ELT : 0u);
  }
};

// epilogue4 for U rows at once: v[u] are the elements of rows at[u] and columns
// col, col + APART, ... of the tile at (m0, n0); APART 1: all buffers' rows on
// four elements and four columns left.  Rows past the tile's may be passed: what
// they store is dropped by the range checks.
template <int OP, int ELT, int U, int APART>
struct TileEpilogue {
  static constexpr int OELT = OP == DATTRI_LINEAR_WEIGHT_GRAD ? 4 : ELT;
  const GemmArgs& a;
  TileRows<OELT> out;
  TileRows<ELT> out2, z, r;
  f32x4 bias;
  uint32_t n;
  int cnt;  // columns that exist
  __device__ TileEpilogue(const GemmArgs& a_, int m0, int n0, int rows, int width, int col)
      : a(a_), out(a_.out, a_.ldo, m0, n0, rows, width), out2(a_.out2, a_.ldo2, m0, n0, rows, width),
        z(a_.Z, a_.ldz, m0, n0, rows, width), r(a_.R, a_.ldr, m0, n0, rows, width), bias{0.f, 0.f, 0.f, 0.f},
        n((uint32_t)col), cnt(APART > 1 ? min(4, (width - col + APART - 1) / APART) : 4) {
    if (OP == DATTRI_LINEAR_FORWARD && a.bias) {
      if constexpr (APART == 1) {
        bias = load4_elt<ELT>(a.bias, n0 + col, true, 4);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < cnt) bias[e] = load_elt<ELT>(a.bias, n0 + col + e * APART);
      }
    }
  }
  __device__ void run(const int (&at)[U], f32x4 (&v)[U]) const {
    f32x4 x[U], y[U];
    if (OP != DATTRI_LINEAR_WEIGHT_GRAD && a.R) {
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = buffer_load4<ELT, APART>(r.r, at[u] * r.ld + n * ELT, cnt);
    }
    if constexpr (OP == DATTRI_LINEAR_FORWARD) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] += bias;
      if (a.Z) {
#pragma unroll
        for (int u = 0; u < U; ++u) buffer_store4<ELT, APART>(z.r, at[u] * z.ld + n * ELT, v[u], cnt);
      }
      act_values<ELT, U>(v, a.act);
      if (a.R) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] += x[u];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) buffer_store4<ELT, APART>(out.r, at[u] * out.ld + n * ELT, v[u], cnt);
    } else if constexpr (OP == DATTRI_LINEAR_INPUT_GRAD) {
      const bool slope = a.out2 && a.act != DATTRI_ACT_NONE;
      if (slope) {
#pragma unroll
        for (int u = 0; u < U; ++u) y[u] = buffer_load4<ELT, APART>(z.r, at[u] * z.ld + n * ELT, cnt);
      }
      if (a.R) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] += x[u];
      }
      if (a.out) {
#pragma unroll
        for (int u = 0; u < U; ++u) buffer_store4<ELT, APART>(out.r, at[u] * out.ld + n * ELT, v[u], cnt);
      }
      if (slope) slope_values<ELT, U>(v, y, a.act);
      if (a.out2) {
#pragma unroll
        for (int u = 0; u < U; ++u) buffer_store4<ELT, APART>(out2.r, at[u] * out2.ld + n * ELT, v[u], cnt);
      }
    } else {
      if (a.accumulate) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] += buffer_load4<4, APART>(out.r, at[u] * out.ld + n * 4, cnt);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) buffer_store4<4, APART>(out.r, at[u] * out.ld + n * 4, v[u], cnt);
    }
  }
};

}  // namespace dev
}  // namespace dattri
