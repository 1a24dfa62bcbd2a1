// Activations of the linear layers' epilogue and their slopes, in float32.
//
// gelu(z) = z Phi(z) with Phi(z) = (1 + erf(z / sqrt 2)) / 2;
// its tanh form equals z s(2u), s the logistic function,
// u = sqrt(2/pi) (z + 0.044715 z^3), since (1 + tanh u) / 2 = s(2u);
// silu(z) = z s(z).  ELT 2 (bf16 results) takes the hardware's exp2 and
// reciprocal, off by a few 2^-23 (exp2 below 2^-126 is zero), and for Phi(-z) =
// exp(-z^2 / 2) t P(t), t = 1 / (1 + q z), z >= 0, the P of degree 6 (and q) whose
// largest relative error over 0 <= z <= 13.5 is least: 6.2e-7, in float32 with
// its exp 8.1e-6 = 2^-16.9 at most and nowhere 7 2^-24 of 1, so the tail keeps
// what bf16 can hold (a P of least absolute error was off by 0.4% at -6 and 3%
// at -12).  8192 x 14336
// outputs: erfcf took 207 us beside the product.  ELT 4 takes the library
// functions and a division.
// s is formed from exp(-|x|), which cannot overflow; a factor that has reached
// zero ends its product, so infinite z and finite z whose cube overflows give
// the limits (0 or z, slopes 0 or 1) and not 0 * inf.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "dattri.h"

namespace dattri {
namespace dev {

constexpr float kSqrt2OverPi = 0.7978845608028654f, kGeluCubic = 0.044715f, kSqrtHalf = 0.7071067811865476f,
                kInvSqrt2Pi = 0.3989422804014327f;

template <int ELT>
__device__ inline float exp_of(float x) {
  if constexpr (ELT == 2) return __builtin_amdgcn_exp2f(x * 1.4426950408889634f);
  return expf(x);
}
// 1 / (1 + exp(-x))
template <int ELT>
__device__ inline float logistic(float x) {
  const float e = exp_of<ELT>(-fabsf(x));
  const float r = ELT == 2 ? __builtin_amdgcn_rcpf(1.f + e) : 1.f / (1.f + e);
  return x < 0.f ? e * r : r;
}

// Phi(z), and in *e exp(-z^2 / 2)
template <int ELT>
__device__ inline float normal_cdf(float z, float* e) {
  *e = exp_of<ELT>(-0.5f * z * z);
  if constexpr (ELT == 4) return 0.5f * erfcf(-z * kSqrtHalf);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.265f, fabsf(z), 1.f));
  float p = fmaf(t, -0.067787044f, 0.19527316f);
  p = fmaf(t, p, -0.06636296f);
  p = fmaf(t, p, 0.14249335f);
  p = fmaf(t, p, 0.08294658f);
  p = fmaf(t, p, 0.107836775f);
  p = fmaf(t, p, 0.10559983f);
  const float tail = t * p * *e;  // Phi(-|z|)
  return z < 0.f ? tail : 1.f - tail;
}

// z * w with w = 0 winning over an infinite z
__device__ inline float decayed(float z, float w) { return w == 0.f ? 0.f : z * w; }

template <int ELT>
__device__ inline float act_value(float z, int act) {
  switch (act) {
    case DATTRI_ACT_RELU:
      return z < 0.f ? 0.f : z;  // NaN stays
    case DATTRI_ACT_GELU: {
      float e;
      return decayed(z, normal_cdf<ELT>(z, &e));
    }
    case DATTRI_ACT_GELU_TANH:
      return decayed(z, logistic<ELT>(2.f * kSqrt2OverPi * (z + kGeluCubic * z * z * z)));
    case DATTRI_ACT_SILU:
      return decayed(z, logistic<ELT>(z));
    default:
      return z;
  }
}

template <int ELT>
__device__ inline float act_slope(float z, int act) {
  switch (act) {
    case DATTRI_ACT_RELU:
      return z <= 0.f ? 0.f : 1.f;
    case DATTRI_ACT_GELU: {
      float e;
      const float p = normal_cdf<ELT>(z, &e);
      return p + decayed(z, kInvSqrt2Pi * e);
    }
    case DATTRI_ACT_GELU_TANH: {  // s(2u) + z 2u' s(2u) (1 - s(2u))
      const float x = 2.f * kSqrt2OverPi * (z + kGeluCubic * z * z * z), s = logistic<ELT>(x), t = logistic<ELT>(-x);
      return s + decayed(z * (2.f * kSqrt2OverPi * (1.f + 3.f * kGeluCubic * z * z)), s * t);
    }
    case DATTRI_ACT_SILU: {
      const float s = logistic<ELT>(z), t = logistic<ELT>(-z);
      return s + decayed(z, s * t);
    }
    default:
      return 1.f;
  }
}

// f(activation as a constant)
template <class F>
__device__ inline void with_act(int act, F f) {
  switch (act) {
    case DATTRI_ACT_RELU:
      return f(std::integral_constant<int, DATTRI_ACT_RELU>{});
    case DATTRI_ACT_GELU:
      return f(std::integral_constant<int, DATTRI_ACT_GELU>{});
    case DATTRI_ACT_GELU_TANH:
      return f(std::integral_constant<int, DATTRI_ACT_GELU_TANH>{});
    case DATTRI_ACT_SILU:
      return f(std::integral_constant<int, DATTRI_ACT_SILU>{});
    default:
      return;
  }
}

}  // namespace dev
}  // namespace dattri
