// Product of 8-bit rows and 8-bit weights with a scale for every 128 of k:
//   Z[m][n] = sum_b sx[m][b] sw[n / 128][b] sum_{k in b} X[m][k] W[n][k] + bias[n],  Y = act(Z) + R.
//
// Few rows: a wave owns 16 weight rows and 16 MB rows of X.  Both come straight
// from memory into registers: lane l holds row l % 16 and 16-byte chunks l / 16
// and 4 + l / 16 of a block of 128 k (the same for both operands, so that every
// product meets its own), the matrix cores sum the block from zero, and one fma
// adds it times its two scales.  Four neighbouring n of one m per lane go to the
// epilogue.
//
// What sums a block depends on the results' type.  The 8-bit matrix instructions
// add the products of eight neighbouring k (the sum of eights is float32's) with
// 13 bits below the largest of them: bits under 2^-13 of the power of two in
// it are dropped (measured: 2^16 + 2^2 gives 2^16, 2^16 + 2^3 keeps all, within
// eight; nothing is lost from one eight to the next; the same for the 32- and
// the 128-deep instruction, with scales or without).  That is far below bf16's
// own 2^-8, so bf16 results take one v_mfma_f32_16x16x128_f8f6f4.  Float32
// results would show it (3e-5 of a sum of 16 products): there the values go to
// bf16, which holds them exactly, and to bf16's instructions, whose products and
// sums keep all of float32, at half the rate.
#include "api_common.h"
#include "device_common.h"
#include "eight.h"
#include "epilogue.h"
#include "internal.h"
#include "linear_tile.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Eight e4m3 values as bf16, exactly.
__device__ inline bf16x8 widen8(int lo, int hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, 1.f, false),
               b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)lo, 1.f, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, 1.f, false),
               d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)hi, 1.f, true);
  return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// Sum over 128 k of a 16 x 16 block, from zero: chunks w0, x0 and w1, x1 of every lane.
template <int ELT>
__device__ inline f32x4 block_dot(i32x4 w0, i32x4 w1, i32x4 x0, i32x4 x1) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if constexpr (ELT == 2) {
    const i32x8 w = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w}, x = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, s, 0, 0, 0, 0, 0, 0);
  }
  s = mfma_bf16_16(widen8(w0.x, w0.y), widen8(x0.x, x0.y), s);
  s = mfma_bf16_16(widen8(w0.z, w0.w), widen8(x0.z, x0.w), s);
  s = mfma_bf16_16(widen8(w1.x, w1.y), widen8(x1.x, x1.y), s);
  return mfma_bf16_16(widen8(w1.z, w1.w), widen8(x1.z, x1.w), s);
}

}  // namespace

template <int ELT>
__global__ __launch_bounds__(256) void linear8_few_kernel(GemmArgs a, Scales8 sc) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15,
            c = lane >> 4;
  const int n0 = (blockIdx.x * 4 + wave) * 16, m0 = (int)(blockIdx.z * gridDim.y + blockIdx.y) * 16;
  if (n0 >= a.N || m0 >= a.M) return;
  // rows past the last repeat it; their sums are not stored
  const uint8_t* w = (const uint8_t*)a.B + (int64_t)min(n0 + r16, a.N - 1) * a.ldb;
  const int m = min(m0 + r16, a.M - 1);
  const uint8_t* x = (const uint8_t*)a.A + m * a.lda;
  const float *sx = sc.x + m * sc.ldx, *sw = sc.w + (n0 / kGroup8) * sc.ldw;
  auto piece = [&](const uint8_t* p, int k) {
    const i32x4 z = {0, 0, 0, 0};
    return k < a.K ? *(const i32x4*)(p + k) : z;
  };
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int b = 0, k = 16 * c; b * kGroup8 < a.K; ++b, k += kGroup8) {
    const f32x4 d = block_dot<ELT>(piece(w, k), piece(w, k + 64), piece(x, k), piece(x, k + 64));
    const float s = sx[b] * sw[b];
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = fmaf(d[e], s, sum[e]);
  }
  const int n = n0 + 4 * c;
  if (m0 + r16 < a.M && n < a.N) epilogue4<DATTRI_LINEAR_FORWARD, ELT>(a, m0 + r16, n, sum);
}

namespace {

struct Layout8 {
  bool pack_x, pack_w;
  size_t off_x, off_w, total;
};
Layout8 layout8(int64_t rows, int64_t d_in, int64_t d_out, bool aligned) {
  Layout8 l = {};
  l.pack_x = l.pack_w = !aligned || d_in % 16;
  const int64_t w = (d_in + 15) / 16 * 16;
  l.off_w = align_up(l.pack_x ? (size_t)rows * w : 0);
  l.total = l.off_w + align_up(l.pack_w ? (size_t)d_out * w : 0);
  return l;
}

}  // namespace

size_t linear8_workspace_need(int64_t rows, int64_t d_in, int64_t d_out, bool aligned) {
  return layout8(rows, d_in, d_out, aligned).total;
}

hipError_t launch_linear8(int elt, bool aligned, GemmArgs a, const Scales8& sc, uint8_t* ws, hipStream_t s) {
  const Layout8 l = layout8(a.M, a.K, a.N, aligned);
  auto on4 = [&](const void* p, int64_t ld) { return !p || ((uintptr_t)p % (4 * elt) == 0 && ld % 4 == 0); };
  a.vec = on4(a.bias, 0) && on4(a.R, a.ldr) && on4(a.Z, a.ldz) && on4(a.out, a.ldo);
  if (l.pack_x) {
    const tile::Repack rx = tile::repack_of(&a.A, &a.lda, a.K, a.M, 1, ws + l.off_x),
                       rw = tile::repack_of(&a.B, &a.ldb, a.K, a.N, 1, ws + l.off_w);
    dim3 grid;
    hipError_t e = row_grid((rx.rows + rw.rows + 3) / 4, &grid);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(tile::repack_kernel<1>, grid, dim3(256), 0, s, rx, rw);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    a.K = (int)a.lda;
  }
  const unsigned mb = (unsigned)(((int64_t)a.M + 15) / 16), my = std::min(mb, 65535u);
  hipLaunchKernelGGL(elt == 2 ? linear8_few_kernel<2> : linear8_few_kernel<4>,
                     dim3((unsigned)((a.N + 63) / 64), my, (mb + my - 1) / my), dim3(256), 0, s, a, sc);
  return hipGetLastError();
}

}  // namespace dattri
