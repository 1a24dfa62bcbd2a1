// Linear layers with a fused epilogue and their backward products.
#include <algorithm>

#include "activation.h"
#include "api_common.h"
#include "device_common.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;

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

// What becomes of the product's element (m, n).
template <int OP, int ELT>
__device__ inline void epilogue_one(const GemmArgs& a, int m, int n, float v) {
  if constexpr (OP == DATTRI_LINEAR_FORWARD) {
    if (a.bias) v += load_elt<ELT>(a.bias, n);
    if (a.Z) store_elt<ELT>(a.Z, m * a.ldz + n, v);
    v = act_value<ELT>(v, a.act);
    if (a.R) v += load_elt<ELT>(a.R, m * a.ldr + n);
    store_elt<ELT>(a.out, m * a.ldo + n, v);
  } else if constexpr (OP == DATTRI_LINEAR_INPUT_GRAD) {
    if (a.R) v += load_elt<ELT>(a.R, m * a.ldr + n);
    const float slope = a.out2 && a.act != DATTRI_ACT_NONE ? act_slope<ELT>(load_elt<ELT>(a.Z, m * a.ldz + n), a.act)
                                                            : 1.f;
    if (a.out) store_elt<ELT>(a.out, m * a.ldo + n, v);
    if (a.out2) store_elt<ELT>(a.out2, m * a.ldo2 + n, a.act == DATTRI_ACT_RELU ? (slope == 0.f ? 0.f : v) : v * slope);
  } else {
    float* o = (float*)a.out + m * a.ldo + n;
    *o = a.accumulate ? *o + v : v;
  }
}

// 64 x 64 tile, 256 threads of 4 x 4 outputs, float32 products, K in steps of 16
// staged in LDS as float32.
template <int OP, int ELT>
__global__ __launch_bounds__(256) void gemm_simple_kernel(GemmArgs a, int tiles_n) {
  constexpr bool kAc = OP != DATTRI_LINEAR_WEIGHT_GRAD, kBc = OP == DATTRI_LINEAR_FORWARD;
  __shared__ float sa[16][65], sb[16][65];
  const int m0 = (int)(blockIdx.x / tiles_n) * 64, n0 = (int)(blockIdx.x % tiles_n) * 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  auto fill = [&](const void* P, int64_t ld, bool kc, int r0, int rows, int k0, float (&s)[16][65]) {
    for (int i = threadIdx.x; i < 1024; i += 256) {
      const int r = kc ? i >> 4 : i & 63, k = kc ? i & 15 : i >> 6;
      float v = 0.f;
      if (r0 + r < rows && k0 + k < a.K)
        v = load_elt<ELT>(P, kc ? (int64_t)(r0 + r) * ld + k0 + k : (int64_t)(k0 + k) * ld + r0 + r);
      s[k][r] = v;
    }
  };
  for (int k0 = 0; k0 < a.K; k0 += 16) {
    fill(a.A, a.lda, kAc, m0, a.M, k0, sa);
    fill(a.B, a.ldb, kBc, n0, a.N, k0, sb);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      float x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = sa[k][4 * ty + i];
        y[i] = sb[k][tx + 16 * i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + 4 * ty + i, n = n0 + tx + 16 * j;
      if (m < a.M && n < a.N) epilogue_one<OP, ELT>(a, m, n, acc[i][j]);
    }
}

// One thread per column, rows in order.
template <int ELT>
__global__ __launch_bounds__(256) void column_sums_kernel(const void* __restrict__ G, int64_t ld, int64_t rows,
                                                          int cols, float* __restrict__ out, int accumulate) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  float s = 0.f;
  for (int64_t r = 0; r < rows; ++r) s += load_elt<ELT>(G, r * ld + c);
  out[c] = accumulate ? out[c] + s : s;
}

size_t linear_workspace_need(dattri_linear_op op, int64_t rows, int64_t d_in, int64_t d_out, int elt, bool aligned) {
  return 0;
}

hipError_t launch_column_sums(int elt, const void* G, int64_t ld_g, int64_t rows, int64_t cols, float* out,
                              bool accumulate, uint8_t* ws, hipStream_t s) {
  auto k = elt == 2 ? column_sums_kernel<2> : column_sums_kernel<4>;
  hipLaunchKernelGGL(k, dim3((unsigned)((cols + 255) / 256)), dim3(256), 0, s, G, ld_g, rows, (int)cols, out,
                     (int)accumulate);
  return hipGetLastError();
}

hipError_t launch_gemm(dattri_linear_op op, int elt, const GemmArgs& a, uint8_t* ws, hipStream_t s) {
  const int64_t tm = (a.M + 63) / 64, tn = (a.N + 63) / 64;
  if (tm * tn > INT32_MAX) return hipErrorInvalidValue;
  auto go = [&](auto k) {
    hipLaunchKernelGGL(k, dim3((unsigned)(tm * tn)), dim3(256), 0, s, a, (int)tn);
    return hipGetLastError();
  };
  if (op == DATTRI_LINEAR_FORWARD) return elt == 2 ? go(gemm_simple_kernel<0, 2>) : go(gemm_simple_kernel<0, 4>);
  if (op == DATTRI_LINEAR_INPUT_GRAD) return elt == 2 ? go(gemm_simple_kernel<1, 2>) : go(gemm_simple_kernel<1, 4>);
  return elt == 2 ? go(gemm_simple_kernel<2, 2>) : go(gemm_simple_kernel<2, 4>);
}

}  // namespace dattri
