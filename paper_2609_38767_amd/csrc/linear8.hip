// Product of 8-bit rows and 8-bit weights with a scale for every 128 of k:
//   Z[m][n] = sum_b sx[m][b] sw[n / 128][b] sum_{k in b} X[m][k] W[n][k] + bias[n],  Y = act(Z) + R.
//
// Few rows: a wave owns 16 weight rows and up to 16 rows of X.  Both come straight
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
// the 128-deep instruction, with scales or without).  For results as large as their
// terms that is far below bf16's own 2^-8, so bf16 results take one
// v_mfma_f32_16x16x128_f8f6f4; where terms cancel it is not: the loss, up to 7
// 2^-13 of the largest product of each eight, goes by the terms and the rounding
// by the result, and who needs more takes float32 results.  Those would show it
// anywhere (3e-5 of a sum of 16 products): there the values go to bf16, which
// holds them exactly, and to bf16's instructions, whose products and sums keep
// all of float32, at half the rate.
//
// What bounds it.  16384 x 14336 -> 4096, bf16 results: 835 us (2.30 PFLOP/s; the
// vendor library's 8-bit product with one scale for each whole operand 597).  By
// the counters both hold the clock at 1.5 to 1.6 GHz, where the matrix cores are
// busy 62% of the time here and 88% there: the scales' fma and the addresses take
// five times the vector instructions, 46% of the issue cycles, and the waves wait
// for 31% of theirs; LDS conflicts are none, HBM traffic is the same.  At 16384 x
// 4096 -> 4096 (259 us) copies for timing without its loads took 221, without the
// scales' fma 240, without barriers and waits 251: no one of them alone ends it.
// Float32 results 1713 us (1.12 PFLOP/s).  Weights out of the caches, 4096 ->
// 14336: one row 14.4 us (4.1 TB/s), 16 rows, by tiles, 16.7, 64 rows 20.3.
#include <algorithm>
#include <type_traits>

#include "api_common.h"
#include "device_common.h"
#include "eight.h"
#include "epilogue.h"
#include "internal.h"
#include "linear8_shape.h"
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

// A 32-row block of a stage: two halves of 64 k, lane l: row l % 32, and of each
// half chunks l / 32 and 2 + l / 32.
struct Block8 {
  i32x8 k[2];
};
// Half h of block i; at: this lane's four chunks of X's first block of the wave, by: from there to the operand's.
__device__ DATTRI_INLINE inline i32x8 read_half(const uint8_t* buf, const uint32_t (&at)[4], int by, int i, int h) {
  const i32x4 c = *(const i32x4*)(buf + (at[2 * h] + by) + i * (32 * 128)),
              d = *(const i32x4*)(buf + (at[2 * h + 1] + by) + i * (32 * 128));
  return i32x8{c.x, c.y, c.z, c.w, d.x, d.y, d.z, d.w};
}
// Keeps what is made of v inside the loop: the sums leave few registers for
// addresses that could be formed again.
__device__ DATTRI_INLINE inline void renew(uint32_t& v) { asm volatile("" : "+v"(v)); }
// c + the products of 64 k of a 32 x 32 block.
template <int ELT>
__device__ DATTRI_INLINE inline f32x16 half_sum(const i32x8& w, const i32x8& x, f32x16 c) {
  if constexpr (ELT == 2) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, 0, 0, 0, 0);
  } else {
#pragma unroll
    for (int q = 0; q < 8; q += 2)
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w[q], w[q + 1]), widen8(x[q], x[q + 1]), c, 0, 0, 0);
    return c;
  }
}

}  // namespace

// Eight waves of a workgroup share 16 weight rows and all rows of X, 16 at most:
// wave w takes the groups of k w, w + 8, ...; the waves' sums are added in their
// order.  (One row of 4096 -> 14336, calls of several inputs in turn: 13.4 us,
// with four waves 14.4, with sixteen 18.4; 4096 -> 4096, whose workgroups are one
// per CU, weights in the caches, 5.0, with sixteen 5.5.)
template <int ELT>
__global__ __launch_bounds__(512) void linear8_few_kernel(GemmArgs a, Scales8 sc) {
  constexpr int W = 8, kAhead = 4;  // groups in flight per wave
  __shared__ f32x4 red[W][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15,
            c = lane >> 4;
  const int n0 = blockIdx.x * 16, groups = (int)(((int64_t)a.K + kGroup8 - 1) / kGroup8);
  // rows past the last repeat it; their sums are not stored
  const int64_t row = min(m, a.M - 1);
  const uint8_t *w = (const uint8_t*)a.B + (int64_t)min(n0 + m, a.N - 1) * a.ldb + 16 * c,
                *x = (const uint8_t*)a.A + row * a.lda + 16 * c;
  const float *sw = sc.w + (n0 / kGroup8) * sc.ldw, *sx = sc.x + row * sc.ldx;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  auto take = [&](int b0, auto count) DATTRI_INLINE {
    constexpr int U = decltype(count)::value;
    i32x4 wv[U][2], xv[U][2];
    float f[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int b = b0 + u * W;
      const int64_t k = (int64_t)b * kGroup8;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        wv[u][h] = xv[u][h] = i32x4{0, 0, 0, 0};
        if (k + 64 * h + 16 * c < a.K) {
          wv[u][h] = *(const i32x4*)(w + k + 64 * h);
          xv[u][h] = *(const i32x4*)(x + k + 64 * h);
        }
      }
      f[u] = sx[b] * sw[b];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const f32x4 d = block_dot<ELT>(wv[u][0], wv[u][1], xv[u][0], xv[u][1]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(d[e], f[u], sum[e]);
    }
  };
  int b = wave;
  for (; b + (kAhead - 1) * W < groups; b += kAhead * W) take(b, std::integral_constant<int, kAhead>{});
  for (; b < groups; b += W) take(b, std::integral_constant<int, 1>{});
  red[wave][lane] = sum;
  __syncthreads();
  const int n = n0 + 4 * c;
  if (wave > 0 || m >= a.M || n >= a.N) return;
#pragma unroll
  for (int q = 1; q < W; ++q) sum += red[q][lane];
  epilogue4<DATTRI_LINEAR_FORWARD, ELT>(a, m, n, sum);
}

// Tiles: WM x WN waves with BM x BN blocks of 32 x 32 each, stages of 128 bytes of
// k (one group of scales) in a ring of BUF buffers, rows and scales by direct
// loads.  At the last block column of a stage everything of it is in registers:
// its buffer takes the loads of the stage a ring further on, which have BUF - 1
// stages to arrive, and the next stage's first fragments are read between its
// products.  A block's products start from zero; while the next block's run, the
// fma of its 16 sums with the two scales' product joins them to the accumulators.
// Four buffers where a stage is short (128 x 128: 0.25 us of products against
// loads of 1 us or more): 1531 x 1001 -> 2305 took 19.8 us with two.
template <int OP, int ELT, int WM, int WN, int BM, int BN, int BUF>
__global__ __launch_bounds__(WM* WN * 64) void linear8_kernel(GemmArgs a, Scales8 sc, int nm, int nn, int sps,
                                                              float* __restrict__ part, int64_t ld_part) {
  constexpr int TM = WM * BM * 32, TN = WN * BN * 32, kWaves = WM * WN;
  static_assert(TM / 64 < kWaves && BN * 32 <= 128 && 128 % (BN * 32) == 0 && BM * BN % 2 == 0, "tile shape");
  typedef tile::Side<1, true, TM, 128, kWaves> SA;
  typedef tile::Side<1, true, TN, 128, kWaves> SB;
  constexpr int kRowBytes = SA::kBytes + SB::kBytes, kStage = kRowBytes + TM * 4 + 256;
  constexpr int kSlab = 32 * TN * 4;
  constexpr int kBuf = std::max(kStage, BUF == 4 ? kSlab : WM * kSlab), kLoads = SA::kLoads + SB::kLoads + 1;
  __shared__ __align__(1024) uint8_t x0[kBuf], x1[kBuf], x2[BUF == 4 ? kBuf : 16], x3[BUF == 4 ? kBuf : 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN, l32 = lane & 31;
  const int64_t tile = (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
  if (tile >= (int64_t)nm * nn) return;
  int mt, nt;
  tile::tile_of((int)tile, nm, nn, &mt, &nt);
  const int m0 = mt * TM, n0 = nt * TN;
  const int all = (int)(((int64_t)a.K + 127) / 128), s0 = blockIdx.y * sps, ns = min(sps, all - s0);
  const int k_end = (int)min((int64_t)a.K, (int64_t)(s0 + ns) * 128);
  SA sa;
  SB sb;
  sa.init(a.A, a.lda, m0, a.M, k_end, wave, lane);
  sb.init(a.B, a.ldb, n0, a.N, k_end, wave, lane);

  // Scales of a stage: the first TM / 64 waves load those of 64 rows each, the
  // others those of the tile's blocks of 128 columns.  Rows past the last repeat it.
  const bool of_x = wave < TM / 64;
  const float* const sbase = of_x ? sc.x + (int64_t)m0 * sc.ldx : sc.w + (int64_t)(n0 / kGroup8) * sc.ldw;
  const int srows = of_x ? min(TM, a.M - m0) : (min(TN, a.N - n0) + kGroup8 - 1) / kGroup8;
  const uint32_t sld = (uint32_t)((of_x ? sc.ldx : sc.ldw) * 4);
  const uint32_t soff = (uint32_t)min(of_x ? wave * 64 + lane : lane, srows - 1) * sld;
  const int sat = kRowBytes + (of_x ? wave * 256 : TM * 4);
  // loads From .. To - 1 of stage st: the scales, X's, W's
  auto issue = [&](int st, uint8_t* x, auto From, auto To) DATTRI_INLINE {
    constexpr int from = decltype(From)::value, to = decltype(To)::value;
    const rsrc_t ra = sa.range(s0 + st), rb = sb.range(s0 + st);
    if constexpr (from == 0 && to > 0) {
      const rsrc_t rs = make_rsrc(sbase + s0 + st, st < ns ? (uint32_t)(srows - 1) * sld + 4 : 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, DATTRI_LDS_PTR(x + sat), 4, soff, 0, 0, 0);
    }
    tile::unrolled<kLoads - 1>([&](auto J) DATTRI_INLINE {
      constexpr int j = decltype(J)::value;
      if constexpr (j + 1 >= from && j + 1 < to) {
        if constexpr (j < SA::kLoads)
          sa.load(ra, s0 + st, x, wave, j);
        else
          sb.load(rb, s0 + st, x + SA::kBytes, wave, j - SA::kLoads);
      }
    });
  };
  typedef std::integral_constant<int, 0> zero_t;
  typedef std::integral_constant<int, 1> one_t;
  typedef std::integral_constant<int, kLoads> all_t;

  f32x16 acc[BN][BM], sum[2];
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    sum[0][v] = sum[1][v] = 0.f;
#pragma unroll
    for (int i = 0; i < BN; ++i)
#pragma unroll
      for (int j = 0; j < BM; ++j) acc[i][j][v] = 0.f;
  }
  // X's fragments: the next block column's beside this one's, or (256 x 256, whose sums take the registers) in its place
  constexpr int kSlots = TM == 256 ? 1 : 2;
  Block8 fa[kSlots], fb[BN];
  // scales: of the blocks whose sums wait, of this block column, of the next one, the stage's and the next stage's weight's
  float before = 0.f, now = 0.f, then = 0.f, of_w = 0.f;
  uint32_t at[4], at_s = (wm * BM * 32 + l32) * 4;
#pragma unroll
  for (int q = 0; q < 4; ++q) at[q] = (wm * BM * 32 + l32) * 128 + (((2 * q + (lane >> 5)) ^ SA::swz(l32)) << 4);
  const int to_b = SA::kBytes + (wn * BN - wm * BM) * 32 * 128;  // rows of both operands are swizzled alike
  auto read_a = [&](const uint8_t* x, int j, int h) DATTRI_INLINE { return read_half(x, at, 0, j, h); };
  auto read_b = [&](const uint8_t* x, int i, int h) DATTRI_INLINE { return read_half(x, at, to_b, i, h); };
  auto read_s = [&](const uint8_t* x, int j) DATTRI_INLINE {
    return *(const float*)(x + kRowBytes + at_s + j * 128);
  };
  auto read_w = [&](const uint8_t* x) DATTRI_INLINE {
    return *(const float*)(x + kRowBytes + TM * 4 + (wn * BN * 32 / kGroup8) * 4);
  };
  // Stage st (in cx; P: its parity); the stage after it is in nx by its last block column.
  auto stage = [&](auto P, int st, uint8_t* cx, const uint8_t* nx) DATTRI_INLINE {
#pragma unroll
    for (int q = 0; q < 4; ++q) renew(at[q]);
    renew(at_s);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      renew(sa.off[q]);
      renew(sb.off[q]);
    }
    // Half a block's products at a time, and while they run half of the sums of the block before (in front of the
    // first: zeros), the reads of what comes next and the loads.  For bf16 results the order is fixed (left to itself
    // the compiler puts sums right behind the products that they wait for: 1024 x 4096 -> 4096 27.6 us, 25.3 so); the
    // float32 ones, with their conversions, are better left to it (42 and 45).
    constexpr bool kOrdered = ELT == 2;
    tile::unrolled<BM * BN * 2>([&](auto Q) DATTRI_INLINE {
      constexpr int q = decltype(Q)::value, h = q & 1, b = q >> 1, j = b / BN, i = b % BN;
      constexpr int pj = b ? (b - 1) / BN : BM - 1, pi = b ? (b - 1) % BN : BN - 1;
      constexpr int slot = (j + decltype(P)::value * BM) % kSlots;
      constexpr bool last = j + 1 == BM;
      if constexpr (last && i == 0 && h == 0) {
        wait_vmcnt_dma<(BUF - 2) * kLoads>();  // the next stage has landed
        tile::stage_barrier();
      }
      if constexpr (h == 0)
        sum[b & 1] = half_sum<ELT>(fb[i].k[0], fa[slot].k[0], f32x16{});
      else
        sum[b & 1] = half_sum<ELT>(fb[i].k[1], fa[slot].k[1], sum[b & 1]);
      if constexpr (kOrdered) __builtin_amdgcn_sched_barrier(0);
      if constexpr (i == (kSlots == 1 ? BN - 1 : 0)) {  // one slot: the fragment has met its last block
        if constexpr (last)
          fa[(slot + 1) % kSlots].k[h] = read_a(nx, 0, h);
        else
          fa[(slot + 1) % kSlots].k[h] = read_a(cx, j + 1, h);
      }
      if constexpr (last) {
        constexpr int part = i * 2 + h, parts = BN * 2;
        issue(st + BUF, cx, std::integral_constant<int, kLoads * part / parts>{},
              std::integral_constant<int, kLoads*(part + 1) / parts>{});
        fb[i].k[h] = read_b(nx, i, h);
      }
      if constexpr (i == 0 && h == 0) {
        if constexpr (last) {
          now = then * of_w;
          then = read_s(nx, 0);
          of_w = read_w(nx);
        } else {
          now = then * of_w;
          then = read_s(cx, j + 1);
        }
      }
#pragma unroll
      for (int v = 8 * h; v < 8 * h + 8; ++v) acc[pi][pj][v] = fmaf(sum[1 - (b & 1)][v], before, acc[pi][pj][v]);
      if constexpr (h == 1) before = now;
      if constexpr (kOrdered) __builtin_amdgcn_sched_barrier(0);
    });
  };
  if (ns > 0) {
    issue(0, x0, zero_t{}, all_t{});
    issue(1, x1, zero_t{}, all_t{});
    if constexpr (BUF == 4) {
      issue(2, x2, zero_t{}, all_t{});
      issue(3, x3, zero_t{}, all_t{});
    }
    wait_vmcnt_dma<(BUF - 1) * kLoads>();
    tile::plain_barrier();
    then = read_s(x0, 0);
    of_w = read_w(x0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      fa[0].k[h] = read_a(x0, 0, h);
#pragma unroll
      for (int i = 0; i < BN; ++i) fb[i].k[h] = read_b(x0, i, h);
    }
    for (int st = 0; st < ns; st += BUF) {  // a last round that is not full ends in stages of zeros
      stage(zero_t{}, st, x0, x1);
      if constexpr (BUF == 4) {
        stage(one_t{}, st + 1, x1, x2);
        stage(zero_t{}, st + 2, x2, x3);
        stage(one_t{}, st + 3, x3, x0);
      } else {
        stage(one_t{}, st + 1, x1, x0);
      }
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[BN - 1][BM - 1][v] = fmaf(sum[1][v], before, acc[BN - 1][BM - 1][v]);
    tile::wait_all();
  }
  tile::finish_tile<OP, ELT, WM, WN, BM, BN>(a, acc, m0, n0, part + (int64_t)blockIdx.y * a.M * ld_part, ld_part,
                                             [&](int j, int wm) {
                                               uint8_t* const y = j & 1 ? x1 : x0;
                                               return BUF == 4 && wm ? (j & 1 ? x3 : x2) : y + wm * kSlab;
                                             });
}

namespace {

struct Layout8 {
  bool pack;
  size_t off_x, off_w, off_part, total;
  Shape8 g;
};
Layout8 layout8(int64_t rows, int64_t d_in, int64_t d_out, int elt, bool aligned) {
  Layout8 l = {};
  l.pack = !aligned || d_in % 16;
  const int64_t w = (d_in + 15) / 16 * 16;
  l.off_w = align_up(l.pack ? (size_t)rows * w : 0);
  l.off_part = l.off_w + align_up(l.pack ? (size_t)d_out * w : 0);
  l.g = shape8(std::max<int64_t>(rows, 1), d_out, d_in, elt);
  l.total = l.off_part + align_up(l.g.splits > 1 ? (size_t)l.g.splits * rows * ((d_out + 3) / 4 * 4) * 4 : 0);
  return l;
}

template <int ELT, int WM, int WN, int BM, int BN, int BUF>
hipError_t launch_tiles(const GemmArgs& a, const Scales8& sc, const Shape8& g, float* part, int64_t ldp, hipStream_t s) {
  constexpr int kThreads = WM * WN * 64;
  if (g.nm * g.nn > INT32_MAX) return hipErrorInvalidValue;
  dim3 grid(1, g.splits);
  hipError_t e = row_grid(g.nm * g.nn, &grid, kThreads, true);
  if (e != hipSuccess) return e;
  if (g.splits == 1) {
    hipLaunchKernelGGL((linear8_kernel<DATTRI_LINEAR_FORWARD, ELT, WM, WN, BM, BN, BUF>), grid, dim3(kThreads), 0, s, a, sc,
                       (int)g.nm, (int)g.nn, g.sps, part, ldp);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((linear8_kernel<tile::kPartial, ELT, WM, WN, BM, BN, BUF>), grid, dim3(kThreads), 0, s, a, sc,
                     (int)g.nm, (int)g.nn, g.sps, part, ldp);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int64_t quads = (int64_t)a.M * (ldp / 4);
  hipLaunchKernelGGL((tile::gemm_join_kernel<DATTRI_LINEAR_FORWARD, ELT>),
                     dim3((unsigned)std::min<int64_t>((quads + 255) / 256, 16384)), dim3(256), 0, s, a, part, ldp,
                     g.splits);
  return hipGetLastError();
}

template <int ELT>
hipError_t launch_few(const GemmArgs& a, const Scales8& sc, hipStream_t s) {
  hipLaunchKernelGGL(linear8_few_kernel<ELT>, dim3((unsigned)(((int64_t)a.N + 15) / 16)), dim3(512), 0, s, a, sc);
  return hipGetLastError();
}

template <int ELT>
hipError_t launch_product(const GemmArgs& a, const Scales8& sc, const Shape8& g, float* part, hipStream_t s) {
  const int64_t ldp = (a.N + 3) / 4 * 4;
  // 128 x 128: eight waves and four buffers for bf16 results (1536 x 4096 -> 2304: 26.8 us, with four waves and two
  // buffers 29.2); float32 results, whose stages are twice as long, the other way (16384 x 4096 -> 4096: 519 and 600)
  if (g.v == kMid)
    return ELT == 2 ? launch_tiles<2, 2, 4, 2, 1, 4>(a, sc, g, part, ldp, s)
                    : launch_tiles<4, 2, 2, 2, 2, 2>(a, sc, g, part, ldp, s);
  if (g.v == kSlim) return launch_tiles<ELT, 2, 2, 1, 2, 4>(a, sc, g, part, ldp, s);
  if constexpr (ELT == 2)
    if (g.v == kBig) return launch_tiles<ELT, 2, 4, 4, 2, 2>(a, sc, g, part, ldp, s);
  return launch_few<ELT>(a, sc, s);
}

}  // namespace

size_t linear8_workspace_need(int64_t rows, int64_t d_in, int64_t d_out, int elt, bool aligned) {
  return layout8(rows, d_in, d_out, elt, aligned).total;
}

hipError_t launch_linear8(int elt, bool aligned, GemmArgs a, const Scales8& sc, uint8_t* ws, hipStream_t s) {
  const Layout8 l = layout8(a.M, a.K, a.N, elt, aligned);
  auto on4 = [&](const void* p, int64_t ld) { return !p || ((uintptr_t)p % (4 * elt) == 0 && ld % 4 == 0); };
  a.vec = on4(a.bias, 0) && on4(a.R, a.ldr) && on4(a.Z, a.ldz) && on4(a.out, a.ldo);
  if (l.pack) {
    // the layout has room for both as soon as one is off 16 bytes
    tile::Repack rx = {}, rw = {};
    const int64_t d_in = a.K;
    if (!tile::on_chunks(a.A, a.lda, d_in, 1)) rx = tile::repack_of(&a.A, &a.lda, d_in, a.M, 1, ws + l.off_x);
    if (!tile::on_chunks(a.B, a.ldb, d_in, 1)) rw = tile::repack_of(&a.B, &a.ldb, d_in, a.N, 1, ws + l.off_w);
    dim3 grid;
    hipError_t e = row_grid((rx.rows + rw.rows + 3) / 4, &grid);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(tile::repack_kernel<1>, grid, dim3(256), 0, s, rx, rw);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    a.K = (int)((d_in + 15) / 16 * 16);
  }
  float* part = (float*)(ws + l.off_part);
  return elt == 2 ? launch_product<2>(a, sc, l.g, part, s) : launch_product<4>(a, sc, l.g, part, s);
}

}  // namespace dattri
