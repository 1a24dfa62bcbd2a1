// Forward product of a few rows against a wide layer (a single token while
// serving): Y[m][n] = act(sum_k X[m][k] W[n][k] + bias[n]) + R, m < M <= 4.
//
// The weights are read once and are all there is to read, so a wave takes four
// of their rows and M sums each: 16 bytes of every row and of every X row per
// lane and step (X stays in the caches), products in float32, one sum over the
// wave at the end, and lane m finishes row m's four outputs.  No partial
// sums go to memory and no second launch follows.  Rows not on 16 bytes
// are read element by element, 64 neighbours at a time.
//
// What bounds it: HBM.  4096 -> 14336 bf16 (117 MB of weights, not cached): one
// row 22.3 us (5.3 TB/s), four rows 26.6; five rows, by the tile kernel, 31.2.
#include "device_common.h"
#include "epilogue.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;

namespace {

constexpr int kRowsPerWave = 4;

template <int ELT>
__device__ inline float dot_piece(i32x4 x, i32x4 w, float s) {
  if constexpr (ELT == 2) {
    const uint32_t a[4] = {(uint32_t)x.x, (uint32_t)x.y, (uint32_t)x.z, (uint32_t)x.w};
    const uint32_t b[4] = {(uint32_t)w.x, (uint32_t)w.y, (uint32_t)w.z, (uint32_t)w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s = fmaf(__builtin_bit_cast(float, a[e] << 16), __builtin_bit_cast(float, b[e] << 16), s);
      s = fmaf(__builtin_bit_cast(float, a[e] & 0xFFFF0000u), __builtin_bit_cast(float, b[e] & 0xFFFF0000u), s);
    }
  } else {
    const f32x4 a = __builtin_bit_cast(f32x4, x), b = __builtin_bit_cast(f32x4, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) s = fmaf(a[e], b[e], s);
  }
  return s;
}

template <int ELT, int M, bool ALIGNED>
__global__ __launch_bounds__(256) void linear_few_kernel(GemmArgs a) {
  constexpr int EPL = ALIGNED ? 16 / ELT : 1, kStep = 64 * EPL, kAhead = M == 1 ? 4 : 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = (blockIdx.x * 4 + wave) * kRowsPerWave;
  if (n0 >= a.N) return;
  const uint8_t* w[kRowsPerWave];
#pragma unroll
  for (int r = 0; r < kRowsPerWave; ++r)  // rows past the last repeat it; their sums are not stored
    w[r] = (const uint8_t*)a.B + (int64_t)min(n0 + r, a.N - 1) * a.ldb * ELT;
  const uint8_t* x = (const uint8_t*)a.A;
  float s[M][kRowsPerWave] = {};
  int k = lane * EPL;
  // kAhead pieces of every row in flight; the last ones one by one
  auto pieces = [&](auto count) {
    constexpr int U = decltype(count)::value;
    if constexpr (ALIGNED) {
      i32x4 wv[U][kRowsPerWave], xv[U][M];
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int r = 0; r < kRowsPerWave; ++r) wv[u][r] = *(const i32x4*)(w[r] + (int64_t)(k + u * kStep) * ELT);
#pragma unroll
        for (int m = 0; m < M; ++m) xv[u][m] = *(const i32x4*)(x + (m * a.lda + k + u * kStep) * ELT);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
          for (int r = 0; r < kRowsPerWave; ++r) s[m][r] = dot_piece<ELT>(xv[u][m], wv[u][r], s[m][r]);
    } else {
      float wv[U][kRowsPerWave], xv[U][M];
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int r = 0; r < kRowsPerWave; ++r) wv[u][r] = load_elt<ELT>(w[r], k + u * kStep);
#pragma unroll
        for (int m = 0; m < M; ++m) xv[u][m] = load_elt<ELT>(x, m * a.lda + k + u * kStep);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
          for (int r = 0; r < kRowsPerWave; ++r) s[m][r] = fmaf(xv[u][m], wv[u][r], s[m][r]);
    }
  };
  for (; k + (kAhead - 1) * kStep < a.K; k += kAhead * kStep) pieces(std::integral_constant<int, kAhead>{});
  for (; k < a.K; k += kStep) pieces(std::integral_constant<int, 1>{});
  f32x4 mine = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) {
      float v = s[m][r];
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
      if (lane == m) mine[r] = v;
    }
  if (lane < M) epilogue4<DATTRI_LINEAR_FORWARD, ELT>(a, lane, n0, mine);
}

template <int ELT, int M>
void launch(const GemmArgs& a, bool aligned, hipStream_t s) {
  const dim3 grid((unsigned)((a.N + 4 * kRowsPerWave - 1) / (4 * kRowsPerWave)));
  if (aligned)
    hipLaunchKernelGGL((linear_few_kernel<ELT, M, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((linear_few_kernel<ELT, M, false>), grid, dim3(256), 0, s, a);
}

}  // namespace

// A wave for four weight rows: from 2048 rows on there are two waves per CU,
// below that the tile kernels' splits of k read faster.
bool linear_few(dattri_linear_op op, int64_t rows, int64_t d_out) {
  return op == DATTRI_LINEAR_FORWARD && rows <= 4 && d_out >= 2048;
}

hipError_t launch_linear_few(int elt, const GemmArgs& a, bool aligned, hipStream_t s) {
  if (elt == 2)
    a.M == 1 ? launch<2, 1>(a, aligned, s) : a.M == 2 ? launch<2, 2>(a, aligned, s)
    : a.M == 3 ? launch<2, 3>(a, aligned, s) : launch<2, 4>(a, aligned, s);
  else
    a.M == 1 ? launch<4, 1>(a, aligned, s) : a.M == 2 ? launch<4, 2>(a, aligned, s)
    : a.M == 3 ? launch<4, 3>(a, aligned, s) : launch<4, 4>(a, aligned, s);
  return hipGetLastError();
}

}  // namespace dattri
