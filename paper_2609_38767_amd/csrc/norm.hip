// Root-mean-square norm of rows with the residual's addition, its gradient, and
// rows and weights in 8 bits.
//
//   h = x + r,  u = 1 / sqrt(mean_j h_j^2 + eps),  y_j = h_j u w_j
//   a_j = g_j w_j:  dh_j = u (a_j - h_j u^2 mean_j(a_j h_j)) + p_j,  dw_j = sum_rows g_j h_j u
//
// A workgroup per row that reads it twice: for its sums, in float64, and for its
// outputs.  A wave takes 128 neighbouring columns at a time, 64 apart per lane, so
// that the largest magnitude of a group of 8-bit values is one reduction.
#include "api_common.h"
#include "device_common.h"
#include "eight.h"
#include "epilogue.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;

namespace {

// Sums over the workgroup of four waves, in a fixed order; all threads get them.
__device__ inline double block_sum(double v) {
  __shared__ double red[4];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// q and s of a wave's group: lane holds columns lane and lane + 64 of it.
__device__ inline void store_group8(uint8_t* q, float* s, int lane, int left, float v0, float v1) {
  const float sc = scale8(wave_max(max_mag(max_mag(0.f, v0), v1))), r = 1.f / sc;
  const int w = pack8<false>(over_scale(v0, sc, r), over_scale(v1, sc, r), 0);
  if (lane < left) q[lane] = (uint8_t)w;
  if (lane + 64 < left) q[lane + 64] = (uint8_t)(w >> 8);
  if (lane == 0) *s = sc;
}

}  // namespace

template <int ELT>
__global__ __launch_bounds__(256) void rms_norm_long_kernel(NormArgs a) {
  const int64_t row = row_block();
  if (row >= a.rows) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto value = [&](int j) {
    float h = load_elt<ELT>(a.X, row * a.ldx + j);
    if (a.R) h += load_elt<ELT>(a.R, row * a.ldr + j);
    return h;
  };
  double s = 0.;
  for (int j = threadIdx.x; j < a.d; j += 256) {
    const double h = value(j);
    s = fma(h, h, s);
  }
  const float u = 1.f / sqrtf((float)(block_sum(s) / a.d) + a.eps);
  for (int c = wave * kGroup8; c < a.d; c += 4 * kGroup8) {
    float y[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = c + lane + 64 * e;
      if (j >= a.d) continue;
      const float h = value(j);
      y[e] = h * u * load_elt<ELT>(a.W, j);
      if (a.H) store_elt<ELT>(a.H, row * a.ldh + j, h);
      if (a.Y) store_elt<ELT>(a.Y, row * a.ldy + j, y[e]);
    }
    if (a.Q) store_group8(a.Q + row * a.ldq + c, a.S + row * a.lds + c / kGroup8, lane, a.d - c, y[0], y[1]);
  }
}

template <int ELT>
__global__ __launch_bounds__(256) void norm_grad_long_kernel(NormGradArgs a) {
  const int64_t row = row_block();
  if (row >= a.rows) return;
  double s = 0., t = 0.;
  for (int j = threadIdx.x; j < a.d; j += 256) {
    const double h = load_elt<ELT>(a.H, row * a.ldh + j), g = load_elt<ELT>(a.G, row * a.ldg + j);
    s = fma(h, h, s);
    t = fma(g * load_elt<ELT>(a.W, j), h, t);
  }
  s = block_sum(s);
  t = block_sum(t);
  const float u = 1.f / sqrtf((float)(s / a.d) + a.eps), c = u * u * (float)(t / a.d);
  if (a.U && threadIdx.x == 0) a.U[row] = u;
  for (int j = threadIdx.x; j < a.d; j += 256) {
    const float h = load_elt<ELT>(a.H, row * a.ldh + j);
    float v = u * fmaf(-h, c, load_elt<ELT>(a.G, row * a.ldg + j) * load_elt<ELT>(a.W, j));
    if (a.P) v += load_elt<ELT>(a.P, row * a.ldp + j);
    store_elt<ELT>(a.D, row * a.ldd + j, v);
  }
}

// Column sums of g h u over rows [y per, (y + 1) per): a wave owns 64 columns and
// every fourth row.
template <int ELT>
__global__ __launch_bounds__(256) void norm_weight_kernel(NormGradArgs a, int64_t per, float* __restrict__ out,
                                                          int accumulate) {
  __shared__ float red[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  const int64_t r0 = blockIdx.y * per, r1 = min(a.rows, r0 + per);
  float s = 0.f;
  if (c < a.d)
#pragma unroll 4
    for (int64_t r = r0 + wave; r < r1; r += 4)
      s = fmaf(load_elt<ELT>(a.G, r * a.ldg + c), load_elt<ELT>(a.H, r * a.ldh + c) * a.U[r], s);
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < a.d) {
    s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
    float* o = out + (int64_t)blockIdx.y * a.d + c;
    *o = accumulate ? *o + s : s;
  }
}

// A wave per 64 columns and four interleaved runs of the parts.
__global__ __launch_bounds__(256) void norm_join_kernel(const float* __restrict__ part, int n_parts, int cols,
                                                        float* __restrict__ out, int accumulate) {
  __shared__ float red[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < cols)
#pragma unroll 4
    for (int y = wave; y < n_parts; y += 4) s += part[(int64_t)y * cols + c];
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) {
    s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
    out[c] = accumulate ? out[c] + s : s;
  }
}

// A wave per group of a row.
template <int ELT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void* __restrict__ X, int64_t ldx, int64_t rows,
                                                            int d, uint8_t* __restrict__ Q, int64_t ldq,
                                                            float* __restrict__ S, int64_t lds) {
  const int lane = threadIdx.x & 63;
  const int64_t groups = (d + kGroup8 - 1) / kGroup8, i = row_block() * 4 + (threadIdx.x >> 6);
  if (i >= rows * groups) return;
  const int64_t row = i / groups;
  const int g = (int)(i - row * groups), c = g * kGroup8;
  float v[2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    v[e] = c + lane + 64 * e < d ? load_elt<ELT>(X, row * ldx + c + lane + 64 * e) : 0.f;
  store_group8(Q + row * ldq + c, S + row * lds + g, lane, d - c, v[0], v[1]);
}

// A workgroup per block of 128 x 128, read twice (64 KB at most).
template <int ELT>
__global__ __launch_bounds__(256) void quantize_weight_kernel(const void* __restrict__ W, int64_t ldw, int rows,
                                                              int d, uint8_t* __restrict__ Q, int64_t ldq,
                                                              float* __restrict__ S, int64_t lds) {
  __shared__ float red[4];
  const int64_t blocks = (d + kGroup8 - 1) / kGroup8, i = row_block(), bo = i / blocks;
  if (bo >= (rows + kGroup8 - 1) / kGroup8) return;
  const int bi = (int)(i - bo * blocks), r0 = (int)bo * kGroup8, c = bi * kGroup8 + (threadIdx.x & 127);
  const int n = min(kGroup8, rows - r0);
  float top = 0.f;
  if (c < d)
#pragma unroll 8
    for (int r = threadIdx.x >> 7; r < n; r += 2) top = max_mag(top, load_elt<ELT>(W, (r0 + r) * ldw + c));
  top = wave_max(top);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  const float s = scale8(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]))), inv = 1.f / s;
  if (threadIdx.x == 0) S[bo * lds + bi] = s;
  if (c < d)
#pragma unroll 8
    for (int r = threadIdx.x >> 7; r < n; r += 2)
      Q[(r0 + r) * ldq + c] = (uint8_t)pack8<false>(over_scale(load_elt<ELT>(W, (r0 + r) * ldw + c), s, inv), 0.f, 0);
}

hipError_t launch_rms_norm(int elt, const NormArgs& a, hipStream_t s) {
  dim3 grid;
  const hipError_t e = row_grid(a.rows, &grid);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(elt == 2 ? rms_norm_long_kernel<2> : rms_norm_long_kernel<4>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

namespace {

// Rows per part of the weight gradient, and parts: eight workgroups per CU of 64 rows or more.
void weight_shape(int64_t rows, int64_t d, int64_t* per, int64_t* parts) {
  const int64_t p = std::max<int64_t>(1, std::min<int64_t>(2048 / ((d + 63) / 64), rows / 64));
  *per = std::max<int64_t>(1, (rows + p - 1) / p);
  *parts = std::max<int64_t>(1, (rows + *per - 1) / *per);
}

}  // namespace

NormGradLayout norm_grad_layout(int64_t rows, int64_t d, bool weight) {
  NormGradLayout l = {};
  if (!weight) return l;
  int64_t per, parts;
  weight_shape(rows, d, &per, &parts);
  l.off_part = align_up((size_t)rows * 4);
  l.total = l.off_part + align_up(parts > 1 ? (size_t)parts * d * 4 : 0);
  return l;
}

hipError_t launch_norm_grad(int elt, NormGradArgs a, float* dw, bool accumulate, uint8_t* ws, hipStream_t s) {
  hipError_t e;
  a.U = dw ? (float*)ws : nullptr;
  if (a.rows > 0) {
    dim3 grid;
    if ((e = row_grid(a.rows, &grid)) != hipSuccess) return e;
    hipLaunchKernelGGL(elt == 2 ? norm_grad_long_kernel<2> : norm_grad_long_kernel<4>, grid, dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (!dw) return hipSuccess;
  int64_t per, parts;
  weight_shape(a.rows, a.d, &per, &parts);
  float* part = (float*)(ws + norm_grad_layout(a.rows, a.d, true).off_part);
  const unsigned strips = (unsigned)((a.d + 63) / 64);
  hipLaunchKernelGGL(elt == 2 ? norm_weight_kernel<2> : norm_weight_kernel<4>, dim3(strips, (unsigned)parts), dim3(256),
                     0, s, a, per, parts > 1 ? part : dw, parts > 1 ? 0 : (int)accumulate);
  if ((e = hipGetLastError()) != hipSuccess || parts == 1) return e;
  hipLaunchKernelGGL(norm_join_kernel, dim3(strips), dim3(256), 0, s, part, (int)parts, (int)a.d, dw, (int)accumulate);
  return hipGetLastError();
}

hipError_t launch_quantize_rows(int elt, const void* X, int64_t ldx, int64_t rows, int64_t d, uint8_t* Q, int64_t ldq,
                                float* S, int64_t lds, hipStream_t s) {
  dim3 grid;
  const hipError_t e = row_grid((rows * ((d + kGroup8 - 1) / kGroup8) + 3) / 4, &grid);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(elt == 2 ? quantize_rows_kernel<2> : quantize_rows_kernel<4>, grid, dim3(256), 0, s, X, ldx, rows,
                     (int)d, Q, ldq, S, lds);
  return hipGetLastError();
}

hipError_t launch_quantize_weight(int elt, const void* W, int64_t ldw, int64_t rows, int64_t d, uint8_t* Q, int64_t ldq,
                                  float* S, int64_t lds, hipStream_t s) {
  dim3 grid;
  const hipError_t e = row_grid(((rows + kGroup8 - 1) / kGroup8) * ((d + kGroup8 - 1) / kGroup8), &grid);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(elt == 2 ? quantize_weight_kernel<2> : quantize_weight_kernel<4>, grid, dim3(256), 0, s, W, ldw,
                     (int)rows, (int)d, Q, ldq, S, lds);
  return hipGetLastError();
}

}  // namespace dattri
