// Linear layers with a fused epilogue and their backward products:
//   C[m][n] = sum_k A(m, k) B(n, k), then epilogue4.
//
// Tiles: linear_tile.h.
//
// What bounds it: 8192 x 4096 -> 14336 bf16, medians of five: forward 774 us
// (1240 TFLOP/s; the vendor library 654), input gradient 735 (1310; 726), weight
// gradient 764 (1260; 971).  The matrix cores are 70, 73 and 67% busy, at a
// clock that the load holds at 1.7 GHz.  The weight gradient's 896 tiles are 3.5 rounds
// of 256 CUs.  Float32, 4096 cubed: 145-151 TFLOP/s (the library 147-150).
#include <algorithm>
#include <cmath>

#include "api_common.h"
#include "device_common.h"
#include "epilogue.h"
#include "internal.h"
#include "linear_shape.h"
#include "linear_tile.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;
using namespace tile;

// WM x WN waves; BM x BN blocks of 32 x 32 each.  Grid (tiles, splits of k,
// more tiles): split y runs stages [y * sps, min((y + 1) * sps, all)); with
// several splits (OP kPartial) part holds them as [split][M][ld_part].
template <int OP, bool AC, bool BC, int ELT, int KW, int WM, int WN, int BM, int BN>
__global__ __launch_bounds__(256, BM * BN >= 16 ? 1 : 2) void gemm_kernel(GemmArgs a, int nm, int nn, int sps,
                                                                          float* __restrict__ part, int64_t ld_part) {
  constexpr int BK = KW / ELT;
  typedef TileBuffers<AC, BC, ELT, KW, WM, WN, BM, BN> Buffers;
  DATTRI_TILE_BUFFERS(Buffers);
  const int64_t tile = (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
  if (tile >= (int64_t)nm * nn) return;
  int mt, nt;
  tile_of((int)tile, nm, nn, &mt, &nt);
  const int all = (int)(((int64_t)a.K + BK - 1) / BK), s0 = blockIdx.y * sps, ns = min(sps, all - s0);
  const int k_end = (int)min((int64_t)a.K, (int64_t)(s0 + ns) * BK);
  tile_product<OP, AC, BC, ELT, KW, WM, WN, BM, BN>(a, mt * WM * BM * 32, nt * WN * BN * 32, s0, ns, k_end,
                                                    part + (int64_t)blockIdx.y * a.M * ld_part, ld_part, x0, x1, x2, x3);
}

// Column sums over rows [y * per, (y + 1) * per): a wave owns 64 C columns, C
// neighbours per lane, and every fourth row of the range; the waves' sums are
// added in wave order.  8192 x 14336 bf16 (235 MB): one column per lane took 80
// us, two bytes per lane and load.
template <int ELT, int C>
__global__ __launch_bounds__(256) void column_sums_kernel(const void* __restrict__ G, int64_t ld, int64_t rows,
                                                          int cols, int64_t per, float* __restrict__ out,
                                                          int accumulate) {
  constexpr int kAhead = 8;
  __shared__ float red[4][64 * C];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (blockIdx.x * 64 + lane) * C;
  const int64_t r0 = blockIdx.y * per, r1 = min(rows, r0 + per);
  f32x4 s[2] = {};
  auto get = [&](int64_t r) {
    if constexpr (C == 4) return load4_elt<ELT>(G, r * ld + c, true, 4);
    return f32x4{load_elt<ELT>(G, r * ld + c), 0.f, 0.f, 0.f};
  };
  if (c < cols) {
    int64_t r = r0 + wave;
    for (; r + 4 * (kAhead - 1) < r1; r += 4 * kAhead) {
      f32x4 v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = get(r + 4 * u);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) s[u & 1] += v[u];
    }
    for (; r < r1; r += 4) s[0] += get(r);
  }
  s[0] += s[1];
#pragma unroll
  for (int e = 0; e < C; ++e) red[wave][e * 64 + lane] = s[0][e];
  __syncthreads();
  if (wave == 0 && c < cols) {
#pragma unroll
    for (int e = 0; e < C; ++e) {
      const int i = e * 64 + lane;
      const float v = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
      float* o = out + (int64_t)blockIdx.y * cols + c + e;
      *o = accumulate ? *o + v : v;
    }
  }
}

// A wave per 64 columns and four interleaved runs of the parts.
__global__ __launch_bounds__(256) void column_join_kernel(const float* __restrict__ part, int n_parts, int cols,
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

namespace {

// Column sums: rows per part, parts.  Parts of at least 64 rows until there are
// eight workgroups per CU.
void column_shape(int64_t rows, int64_t cols, int64_t* per, int64_t* parts) {
  const int64_t strips = (cols + 255) / 256;
  const int64_t p = std::max<int64_t>(1, std::min<int64_t>(2048 / strips, rows / 64));
  *per = std::max<int64_t>(1, (rows + p - 1) / p);
  *parts = std::max<int64_t>(1, (rows + *per - 1) / *per);
}

struct LinearLayout {
  int64_t M, N, K;
  bool ac, bc;          // operands k contiguous
  int64_t a_rows, a_w, b_rows, b_w;  // as stored
  bool pack_a, pack_b;
  size_t off_a, off_b, off_part, off_cols, total;
  GemmShape g;
};
LinearLayout linear_layout(dattri_linear_op op, int64_t rows, int64_t d_in, int64_t d_out, int elt, bool aligned) {
  LinearLayout L = {};
  L.ac = op != DATTRI_LINEAR_WEIGHT_GRAD;
  L.bc = op == DATTRI_LINEAR_FORWARD;
  L.M = op == DATTRI_LINEAR_WEIGHT_GRAD ? d_out : rows;
  L.N = op == DATTRI_LINEAR_FORWARD ? d_out : d_in;
  L.K = op == DATTRI_LINEAR_FORWARD ? d_in : op == DATTRI_LINEAR_INPUT_GRAD ? d_out : rows;
  L.a_rows = L.ac ? L.M : L.K;
  L.a_w = L.ac ? L.K : L.M;
  L.b_rows = L.bc ? L.N : L.K;
  L.b_w = L.bc ? L.K : L.N;
  L.pack_a = !aligned || (L.a_w * elt) % 16;
  L.pack_b = !aligned || (L.b_w * elt) % 16;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align_up(off + bytes);
    return at;
  };
  auto packed = [&](int64_t r, int64_t w) { return (size_t)r * (size_t)((w * elt + 15) / 16 * 16); };
  L.off_a = take(L.pack_a ? packed(L.a_rows, L.a_w) : 0);
  L.off_b = take(L.pack_b ? packed(L.b_rows, L.b_w) : 0);
  L.g = gemm_shape(std::max<int64_t>(L.M, 1), L.N, L.K, elt, L.ac, L.bc);
  L.off_part = take(L.g.splits > 1 ? (size_t)L.g.splits * L.M * ((L.N + 3) / 4 * 4) * 4 : 0);
  L.off_cols = off;
  if (op == DATTRI_LINEAR_WEIGHT_GRAD) {
    int64_t per, parts;
    column_shape(rows, d_out, &per, &parts);
    take(parts > 1 ? (size_t)parts * d_out * 4 : 0);
  }
  L.total = off;
  return L;
}

unsigned flat_grid(int64_t n) { return (unsigned)std::min<int64_t>((n + 255) / 256, 16384); }

template <int OP, bool AC, bool BC, int ELT, int KW, int WM, int WN, int BM, int BN>
hipError_t launch_tiles(const GemmArgs& a, const GemmShape& g, float* part, int64_t ldp, hipStream_t s) {
  dim3 grid(1, g.splits);
  const hipError_t e = row_grid(g.nm * g.nn, &grid, 256, true);
  if (e != hipSuccess) return e;
  if (g.splits > 1)
    hipLaunchKernelGGL((gemm_kernel<kPartial, AC, BC, ELT, KW, WM, WN, BM, BN>), grid, dim3(256), 0, s, a, (int)g.nm,
                       (int)g.nn, g.sps, part, ldp);
  else
    hipLaunchKernelGGL((gemm_kernel<OP, AC, BC, ELT, KW, WM, WN, BM, BN>), grid, dim3(256), 0, s, a, (int)g.nm, (int)g.nn,
                       g.sps, part, ldp);
  return hipGetLastError();
}

template <int OP, int ELT>
hipError_t launch_product(const GemmArgs& a, const GemmShape& g, float* part, hipStream_t s) {
  constexpr bool AC = OP != DATTRI_LINEAR_WEIGHT_GRAD, BC = OP == DATTRI_LINEAR_FORWARD;
  if (g.nm * g.nn > INT32_MAX) return hipErrorInvalidValue;
  const int64_t ldp = (a.N + 3) / 4 * 4;
  hipError_t e = hipErrorInvalidValue;
  if (g.v == kBig)
    e = launch_tiles<OP, AC, BC, ELT, stage_bytes(AC, BC, ELT, 256), 2, 2, 4, 4>(a, g, part, ldp, s);
  else if (g.v == kMid)
    e = launch_tiles<OP, AC, BC, ELT, stage_bytes(AC, BC, ELT, 128), 2, 2, 2, 2>(a, g, part, ldp, s);
  else if constexpr (AC) {
    if (g.v == kSlim)
      e = launch_tiles<OP, AC, BC, ELT, 64, 2, 2, 1, 2>(a, g, part, ldp, s);
    else
      e = launch_tiles<OP, AC, BC, ELT, 64, 1, 4, 1, 1>(a, g, part, ldp, s);
  }
  if (e != hipSuccess || g.splits == 1) return e;
  hipLaunchKernelGGL((gemm_join_kernel<OP, ELT>), dim3(flat_grid((int64_t)a.M * (ldp / 4))), dim3(256), 0, s, a, part,
                     ldp, g.splits);
  return hipGetLastError();
}

hipError_t launch_column_sums(int elt, const void* G, int64_t ld_g, int64_t rows, int64_t cols, float* out,
                              bool accumulate, float* part, hipStream_t s) {
  int64_t per, parts;
  column_shape(rows, cols, &per, &parts);
  const bool four = (uintptr_t)G % (4 * elt) == 0 && ld_g % 4 == 0 && cols % 4 == 0;
  auto k = elt == 2 ? (four ? column_sums_kernel<2, 4> : column_sums_kernel<2, 1>)
                    : (four ? column_sums_kernel<4, 4> : column_sums_kernel<4, 1>);
  const int64_t wide = four ? 256 : 64;
  hipLaunchKernelGGL(k, dim3((unsigned)((cols + wide - 1) / wide), (unsigned)parts), dim3(256), 0, s, G, ld_g, rows, (int)cols,
                     per, parts > 1 ? part : out, parts > 1 ? 0 : (int)accumulate);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  hipLaunchKernelGGL(column_join_kernel, dim3((unsigned)((cols + 63) / 64)), dim3(256), 0, s, part, (int)parts,
                     (int)cols, out, (int)accumulate);
  return hipGetLastError();
}

}  // namespace

size_t linear_workspace_need(dattri_linear_op op, int64_t rows, int64_t d_in, int64_t d_out, int elt, bool aligned) {
  if (linear_few(op, rows, d_out)) return 0;
  return linear_layout(op, rows, d_in, d_out, elt, aligned).total;
}

hipError_t launch_linear(dattri_linear_op op, int elt, bool aligned, GemmArgs a, float* dbias, uint8_t* ws,
                         hipStream_t s) {
  const bool wgrad = op == DATTRI_LINEAR_WEIGHT_GRAD;
  const int64_t rows = wgrad ? a.K : a.M, d_out = op == DATTRI_LINEAR_FORWARD ? a.N : wgrad ? a.M : a.K,
                d_in = op == DATTRI_LINEAR_FORWARD ? a.K : a.N;
  const int oelt = wgrad ? 4 : elt;
  auto on4 = [](const void* p, int64_t ld, int e) { return !p || ((uintptr_t)p % (4 * e) == 0 && ld % 4 == 0); };
  a.vec = on4(a.bias, 0, elt) && on4(a.R, a.ldr, elt) && on4(a.Z, a.ldz, elt) && on4(a.out, a.ldo, oelt) &&
          on4(a.out2, a.ldo2, elt);
  if (linear_few(op, rows, d_out)) return launch_linear_few(elt, a, aligned && (d_in * elt) % 16 == 0, s);
  const LinearLayout L = linear_layout(op, rows, d_in, d_out, elt, aligned);
  hipError_t e;
  if (dbias) {
    e = launch_column_sums(elt, a.A, a.lda, rows, d_out, dbias, a.accumulate, (float*)(ws + L.off_cols), s);
    if (e != hipSuccess || !a.out) return e;
  }
  if (L.pack_a || L.pack_b) {
    Repack ra = {}, rb = {};
    if (L.pack_a) ra = repack_of(&a.A, &a.lda, L.a_w, L.a_rows, elt, ws + L.off_a);
    if (L.pack_b) rb = repack_of(&a.B, &a.ldb, L.b_w, L.b_rows, elt, ws + L.off_b);
    const int64_t n = ra.rows + rb.rows;
    if (n > 0) {
      dim3 grid;
      e = row_grid((n + 3) / 4, &grid);
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(elt == 2 ? repack_kernel<2> : repack_kernel<4>, grid, dim3(256), 0, s, ra, rb);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  float* part = (float*)(ws + L.off_part);
  if (op == DATTRI_LINEAR_FORWARD)
    return elt == 2 ? launch_product<DATTRI_LINEAR_FORWARD, 2>(a, L.g, part, s)
                    : launch_product<DATTRI_LINEAR_FORWARD, 4>(a, L.g, part, s);
  if (op == DATTRI_LINEAR_INPUT_GRAD)
    return elt == 2 ? launch_product<DATTRI_LINEAR_INPUT_GRAD, 2>(a, L.g, part, s)
                    : launch_product<DATTRI_LINEAR_INPUT_GRAD, 4>(a, L.g, part, s);
  return elt == 2 ? launch_product<DATTRI_LINEAR_WEIGHT_GRAD, 2>(a, L.g, part, s)
                  : launch_product<DATTRI_LINEAR_WEIGHT_GRAD, 4>(a, L.g, part, s);
}

}  // namespace dattri
