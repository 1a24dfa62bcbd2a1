// Linear layers of experts and their backward products: rows sorted by expert,
// any number of rows for each, the boundaries on the GPU.
//   forward      Z[t] = X[t] W_e^T + b_e     input gradient   D[t] = G[t] W_e + R[t]
//   weight gradient   dW_e = sum_t G[t]^T X[t]     t in [offsets[e], offsets[e + 1])
//
// The tiles are those of the linear layers (linear_tile.h).  Nothing of the
// boundaries is known on the host, so a product over rows is launched with as
// many tiles as any boundaries can need; every wave adds up the segments' tiles
// and finds its own.  Rows in front of the first boundary and behind the last
// one are segments too, whose products have no k: they come out as those of an
// expert with zero weights and bias.  Boundaries are clamped to the rows and to
// each other, so wrong ones give wrong rows, never an access out of range.
//
// What bounds it: the matrix cores, as the linear layers' products, and the last
// round of tiles, whose prologue and epilogue overlap nothing.  bf16, over several
// sets of row counts: eight experts of 4096 -> 14336, 16384 rows: forward 1570 to
// 1615 us (1.2 PFLOP/s; with experts of equal size 1535, one dense layer 1490),
// input gradient 1710 to 1750 alone, 1820 to 1880 with a residual and a slope
// (equal 1555 alone), weight gradient 1690 (equal 1665); 64 experts of 4096 -> 1024,
// 32768 rows, with bias, silu and the kept pre-activation: 365 to 417, for 2.2 to
// 2.3 rounds of tiles take 2.5 or 3 (equal experts, two rounds, 299).  Few rows:
// memory.  16 rows that meet 14 experts of 4096 -> 14336 298 us, 5.5 TB/s of those
// experts' weights.
#include <algorithm>

#include "api_common.h"
#include "device_common.h"
#include "epilogue.h"
#include "expert_shape.h"
#include "internal.h"
#include "linear_shape.h"
#include "linear_tile.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;
using namespace tile;

namespace {

__device__ inline int boundary(const ExpertArgs& x, int i) {
  const int64_t v = x.offset_bytes == 8 ? ((const int64_t*)x.offsets)[i] : ((const int32_t*)x.offsets)[i];
  return (int)min(max(v, (int64_t)0), (int64_t)x.rows);
}

// Segment s of experts + 2: the rows in front, the experts' and the rows behind.
struct Segment {
  int begin, end;
};
__device__ inline Segment segment(const ExpertArgs& x, int s) {
  const int begin = s == 0 ? 0 : boundary(x, s - 1);
  return Segment{begin, max(begin, s > x.experts ? x.rows : boundary(x, s))};
}

// Tile row `at` of all segments' tile rows.
struct Place {
  int segment, m0, end;
};
// Sums stop at the largest number of tile rows that ordered boundaries give, so
// others may not overflow them, and what is found below it is a tile row of its
// segment.
template <int TM>
struct Segments {
  const ExpertArgs& x;
  int lane;
  Segment first;  // of the first 64 segments, this lane's
  __device__ Segment load(int s) const { return s < x.experts + 2 ? segment(x, s) : Segment{0, 0}; }
  __device__ Segments(const ExpertArgs& x_, int lane_) : x(x_), lane(lane_) { first = load(lane); }
  template <Rows R>
  __device__ static int tiles(const Segment& g) {
    return tile_rows(R, g.end - g.begin, TM);
  }
  template <Rows R>
  __device__ int most() const {
    const int full = x.rows / TM, some = min(x.experts + 2, x.rows);
    return R == kRest ? some : full + some;
  }
  template <Rows R>
  __device__ int total() const {
    int n = tiles<R>(first);
    for (int s = 64; s < x.experts + 2; s += 64) n = min(n + tiles<R>(load(s + lane)), most<R>());
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n = min(n + __shfl_xor(n, o), most<R>());
    return __builtin_amdgcn_readfirstlane(n);
  }
  template <Rows R>
  __device__ Place find(int at) const {  // at < total
    int before = 0;
    for (int s = 0;; s += 64) {
      const Segment g = s ? load(s + lane) : first;
      int upto = min(before + tiles<R>(g), most<R>());  // of the segments up to this lane's
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(upto - before, o);
        if (lane >= o) upto = min(upto + v, most<R>());
      }
      const uint64_t here = __ballot(upto > at);
      if (here) {
        const int l = __builtin_ctzll(here), in_front = l ? __builtin_amdgcn_readlane(upto, l - 1) : before,
                  begin = __builtin_amdgcn_readlane(g.begin, l), end = __builtin_amdgcn_readlane(g.end, l);
        return Place{s + l, R == kRest ? begin + (end - begin) / TM * TM : begin + (at - in_front) * TM, end};
      }
      before = __builtin_amdgcn_readlane(upto, 63);
      if (s + 64 >= x.experts + 2) return Place{0, 0, 0};
    }
  }
};

}  // namespace

// Products over rows: grid as many tiles as there can be (tiles, splits of k, more
// tiles); split y runs stages [y * sps, (y + 1) * sps), with several splits (OP
// kPartial) part holds them as [split][rows][ld_part].
// Of 256 x 256 tiles a segment's last is half empty on average: where it would be
// half empty or more, a tile of 128 x 256 takes its place, behind the others, in
// half the time.  (Tiles of 128 x 128 for all last rows: 64 experts of 4096 ->
// 1024, 32768 rows, 455 us, whole tiles 371; alone on a CU they are slow.)
template <int OP, bool BC, int ELT, int KW, int WM, int WN, int BM, int BN>
__global__ __launch_bounds__(256, BM * BN >= 16 ? 1 : 2) void expert_rows_kernel(GemmArgs a, ExpertArgs x, int nn,
                                                                                 int sps, float* __restrict__ part,
                                                                                 int64_t ld_part) {
  constexpr int TM = WM * BM * 32, TN = WN * BN * 32, BK = KW / ELT;
  constexpr bool kHalves = TM == 256;
  typedef TileBuffers<true, BC, ELT, KW, WM, WN, BM, BN> Buffers;
  DATTRI_TILE_BUFFERS(Buffers);
  const Segments<TM> all(x, threadIdx.x & 63);
  const int64_t tile = (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
  auto run = [&](const Place& p, auto product) DATTRI_INLINE {
    const int e = p.segment - 1;
    a.M = p.end;
    if (e < 0 || e >= x.experts) {
      a.K = 0;
      a.bias = nullptr;
    } else {
      a.B = (const uint8_t*)a.B + (int64_t)e * x.stride * ELT;
      if (a.bias) a.bias = (const uint8_t*)a.bias + (int64_t)e * a.N * ELT;
    }
    const int all = (int)(((int64_t)a.K + BK - 1) / BK), s0 = blockIdx.y * sps, ns = min(sps, all - s0);
    product(s0, ns, (int)min((int64_t)a.K, (int64_t)(s0 + ns) * BK));
  };
  part += (int64_t)blockIdx.y * x.rows * ld_part;
  const int n = all.template total<kHalves ? kFull : kAll>();
  int mt, nt;
  if (tile < (int64_t)n * nn) {
    tile_of((int)tile, n, nn, &mt, &nt);
    const Place p = all.template find<kHalves ? kFull : kAll>(mt);
    run(p, [&](int s0, int ns, int k_end) DATTRI_INLINE {
      tile_product<OP, true, BC, ELT, KW, WM, WN, BM, BN>(a, p.m0, nt * TN, s0, ns, k_end, part, ld_part, x0, x1, x2, x3);
    });
    return;
  }
  if constexpr (kHalves) {
    const int64_t half = tile - (int64_t)n * nn;
    const int rest = all.template total<kRest>();
    if (half >= (int64_t)rest * nn) return;
    tile_of((int)half, rest, nn, &mt, &nt);
    const Place p = all.template find<kRest>(mt);
    run(p, [&](int s0, int ns, int k_end) DATTRI_INLINE {
      tile_product<OP, true, BC, ELT, KW, 2, 2, 2, 4>(a, p.m0, nt * TN, s0, ns, k_end, part, ld_part, x0, x1, x2, x3);
    });
  }
}

// Weight gradients: experts times nm times nn tiles, grid as above; the splits of k
// cut each expert's rows, part holds [split][experts * M][ld_part].
template <int OP, int ELT, int KW, int WM, int WN, int BM, int BN>
__global__ __launch_bounds__(256, BM * BN >= 16 ? 1 : 2) void expert_weight_kernel(GemmArgs a, ExpertArgs x, int nm,
                                                                                   int nn, float* __restrict__ part,
                                                                                   int64_t ld_part) {
  constexpr int BK = KW / ELT, kRound = buffers_of(KW);
  typedef TileBuffers<false, false, ELT, KW, WM, WN, BM, BN> Buffers;
  DATTRI_TILE_BUFFERS(Buffers);
  const int64_t tile = (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
  if (tile >= (int64_t)x.experts * nm * nn) return;
  const int e = (int)(tile / (nm * nn));
  int mt, nt;
  tile_of((int)(tile - (int64_t)e * nm * nn), nm, nn, &mt, &nt);
  const Segment g = segment(x, e + 1);
  if (OP != kPartial && a.accumulate && g.begin == g.end) return;
  a.K = g.end - g.begin;
  a.A = (const uint8_t*)a.A + (int64_t)g.begin * a.lda * ELT;
  a.B = (const uint8_t*)a.B + (int64_t)g.begin * a.ldb * ELT;
  a.out = (float*)a.out + (int64_t)e * x.stride;
  part += ((int64_t)blockIdx.y * x.experts + e) * a.M * ld_part;
  const int all = (int)(((int64_t)a.K + BK - 1) / BK), splits = gridDim.y,
            sps = splits > 1 ? ((all + splits - 1) / splits + kRound - 1) / kRound * kRound : all;
  const int s0 = (int)min((int64_t)blockIdx.y * sps, (int64_t)all), ns = min(sps, all - s0);
  tile_product<OP, false, false, ELT, KW, WM, WN, BM, BN>(a, mt * WM * BM * 32, nt * WN * BN * 32, s0, ns,
                                                          (int)min((int64_t)a.K, (int64_t)(s0 + ns) * BK), part, ld_part,
                                                          x0, x1, x2, x3);
}

// Rows (a) and weights (b, `per` rows of each expert) repacked in one launch, of
// the weights only those of experts that have rows: the others are not read.
template <int ELT>
__global__ __launch_bounds__(256) void expert_repack_kernel(Repack a, Repack b, ExpertArgs x, int per) {
  const int64_t at = repack_at();
  if (at >= a.rows + b.rows) return;
  if (at >= a.rows) {
    const Segment g = segment(x, (int)((uint32_t)(at - a.rows) / (uint32_t)per) + 1);
    if (g.begin == g.end) return;
  }
  repack_row<ELT>(at < a.rows ? a : b, at < a.rows ? at : at - a.rows);
}

// Sums of a split product over rows in split order, and the epilogue with the
// bias of the row's expert: the last one whose rows begin at or before it.
template <int OP, int ELT>
__global__ __launch_bounds__(256) void expert_join_kernel(GemmArgs a, ExpertArgs x, const float* __restrict__ part,
                                                          int64_t ld_part, int splits) {
  const int nv = (a.N + 3) / 4;
  const int64_t total = (int64_t)a.M * nv, step = (int64_t)a.M * ld_part;
  const uint8_t* const bias = (const uint8_t*)a.bias;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int m = (int)(i / nv), n = (int)(i - (int64_t)m * nv) * 4;
    const float* p = part + m * ld_part + n;
    f32x4 s = *(const f32x4*)p;
#pragma unroll 4
    for (int y = 1; y < splits; ++y) s += *(const f32x4*)(p + y * step);
    if (bias) {
      int lo = -1, hi = x.experts;  // boundary(lo) <= m < boundary(hi + 1), experts + 1 boundaries
      while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (boundary(x, mid) <= m) lo = mid;
        else hi = mid - 1;
      }
      a.bias = lo < 0 || lo >= x.experts ? nullptr : bias + (int64_t)lo * a.N * ELT;
    }
    epilogue4<OP, ELT>(a, m, n, s);
  }
}

// Column sums of an expert's rows: grid (64 C columns, parts, experts); part y of
// parts takes its share of the expert's rows, a wave every fourth of them, C
// neighbouring columns per lane.  Sums of one part go to out, else part holds
// [parts][experts][cols].  16384 x 14336 bf16 of eight experts took 125 us with
// one column per lane.
template <int ELT, int C>
__global__ __launch_bounds__(256) void expert_columns_kernel(const void* __restrict__ G, int64_t ld, ExpertArgs x,
                                                             int cols, float* __restrict__ part,
                                                             float* __restrict__ out, int accumulate) {
  constexpr int kAhead = 8;
  __shared__ float red[4][64 * C];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (blockIdx.x * 64 + lane) * C, e = blockIdx.z;
  const Segment g = segment(x, e + 1);
  const int64_t per = ((int64_t)g.end - g.begin + gridDim.y - 1) / gridDim.y, r0 = g.begin + blockIdx.y * per,
                r1 = min((int64_t)g.end, r0 + per);
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
  for (int k = 0; k < C; ++k) red[wave][k * 64 + lane] = s[0][k];
  __syncthreads();
  if (wave == 0 && c < cols) {
    const int64_t at = (int64_t)e * cols + c;
#pragma unroll
    for (int k = 0; k < C; ++k) {
      const int i = k * 64 + lane;
      const float v = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
      if (gridDim.y > 1)
        part[(int64_t)blockIdx.y * x.experts * cols + at + k] = v;
      else
        out[at + k] = accumulate ? out[at + k] + v : v;
    }
  }
}

__global__ __launch_bounds__(256) void expert_columns_join_kernel(const float* __restrict__ part, int parts, int64_t n,
                                                                  float* __restrict__ out, int accumulate) {
  const int64_t i = row_block() * 256 + threadIdx.x;
  if (i >= n) return;
  float s = 0.f;
#pragma unroll 4
  for (int y = 0; y < parts; ++y) s += part[y * n + i];
  out[i] = accumulate ? out[i] + s : s;
}

namespace {

int64_t column_parts(int64_t rows, int64_t experts, int64_t cols) {
  return std::max<int64_t>(1, std::min<int64_t>(4096 / ((cols + 255) / 256 * experts), rows / experts / 64));
}

struct ExpertLayout {
  int64_t a_rows, a_w, b_rows, b_w;  // as stored
  bool pack_a, pack_b;
  size_t off_a, off_b, off_part, off_cols, total;
  ExpertShape g;
};
ExpertLayout expert_layout(dattri_linear_op op, int64_t rows, int64_t experts, int64_t d_in, int64_t d_out, int elt,
                           bool aligned) {
  ExpertLayout L = {};
  const bool wgrad = op == DATTRI_LINEAR_WEIGHT_GRAD;
  L.a_rows = rows;
  L.a_w = op == DATTRI_LINEAR_FORWARD ? d_in : d_out;
  L.b_rows = wgrad ? rows : experts * d_out;
  L.b_w = d_in;
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
  const int64_t m = wgrad ? d_out : rows, n = op == DATTRI_LINEAR_FORWARD ? d_out : d_in,
                k = op == DATTRI_LINEAR_FORWARD ? d_in : wgrad ? rows : d_out;
  L.g = expert_shape(wgrad, rows, experts, m, n, k, elt, op == DATTRI_LINEAR_FORWARD);
  L.off_part = take(L.g.splits > 1 ? (size_t)L.g.splits * (wgrad ? experts * m : m) * ((n + 3) / 4 * 4) * 4 : 0);
  L.off_cols = off;
  if (wgrad) {
    const int64_t parts = column_parts(rows, experts, d_out);
    take(parts > 1 ? (size_t)parts * experts * d_out * 4 : 0);
  }
  L.total = off;
  return L;
}

// OP kPartial: partial sums of splits to part, else the whole product.
template <int OP, int REAL, int ELT, int KW, int WM, int WN, int BM, int BN>
hipError_t launch_grid(const GemmArgs& a, const ExpertArgs& x, int splits, float* part, int64_t ldp, hipStream_t s) {
  constexpr int TM = WM * BM * 32, TN = WN * BN * 32;
  const int64_t nn = ((int64_t)a.N + TN - 1) / TN;
  dim3 grid(1, (unsigned)splits);
  if constexpr (REAL == DATTRI_LINEAR_WEIGHT_GRAD) {
    const int64_t nm = ((int64_t)a.M + TM - 1) / TM;
    if (nm * nn > INT32_MAX) return hipErrorInvalidValue;
    const hipError_t e = row_grid(x.experts * nm * nn, &grid, 256, true);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((expert_weight_kernel<OP, ELT, KW, WM, WN, BM, BN>), grid, dim3(256), 0, s, a, x, (int)nm,
                       (int)nn, part, ldp);
  } else {
    // every segment with rows has at most one tile row more than its rows fill
    const int64_t n = (x.rows / TM + std::min<int64_t>(x.experts + 2, x.rows)) * nn;
    if (n > INT32_MAX) return hipErrorInvalidValue;
    const hipError_t e = row_grid(n, &grid, 256, true);
    if (e != hipSuccess) return e;
    const int64_t stages = ((int64_t)a.K * ELT + KW - 1) / KW, round = buffers_of(KW),
                  sps = splits > 1 ? ((stages + splits - 1) / splits + round - 1) / round * round : stages;
    hipLaunchKernelGGL((expert_rows_kernel<OP, REAL == DATTRI_LINEAR_FORWARD, ELT, KW, WM, WN, BM, BN>), grid,
                       dim3(256), 0, s, a, x, (int)nn, (int)sps, part, ldp);
  }
  return hipGetLastError();
}

template <int OP, int ELT, int KW, int WM, int WN, int BM, int BN>
hipError_t launch_tiles(const GemmArgs& a, const ExpertArgs& x, int splits, float* part, hipStream_t s) {
  const int64_t ldp = ((int64_t)a.N + 3) / 4 * 4;
  if constexpr (expert_splits(BM * BN == 16 ? kBig : BM * BN == 4 ? kMid : BM * BN == 2 ? kSlim : kFew, ELT)) {
    if (splits > 1) {
      const hipError_t e = launch_grid<kPartial, OP, ELT, KW, WM, WN, BM, BN>(a, x, splits, part, ldp, s);
      if (e != hipSuccess) return e;
      GemmArgs j = a;  // all rows of the buffers
      if (OP == DATTRI_LINEAR_WEIGHT_GRAD) j.M = (int)(x.experts * (int64_t)a.M);
      const dim3 grid((unsigned)std::min<int64_t>(((int64_t)j.M * (ldp / 4) + 255) / 256, 16384));
      if constexpr (OP == DATTRI_LINEAR_WEIGHT_GRAD)
        hipLaunchKernelGGL((gemm_join_kernel<OP, ELT>), grid, dim3(256), 0, s, j, part, ldp, splits);
      else
        hipLaunchKernelGGL((expert_join_kernel<OP, ELT>), grid, dim3(256), 0, s, j, x, part, ldp, splits);
      return hipGetLastError();
    }
  }
  return launch_grid<OP, OP, ELT, KW, WM, WN, BM, BN>(a, x, 1, nullptr, 0, s);
}

template <int OP, int ELT>
hipError_t launch_product(const GemmArgs& a, const ExpertArgs& x, const ExpertShape& g, float* part, hipStream_t s) {
  constexpr bool AC = OP != DATTRI_LINEAR_WEIGHT_GRAD, BC = OP == DATTRI_LINEAR_FORWARD;
  if constexpr (AC || ELT == 2)
    if (g.v == kBig) return launch_tiles<OP, ELT, stage_bytes(AC, BC, ELT, 256), 2, 2, 4, 4>(a, x, 1, part, s);
  if (g.v == kMid) return launch_tiles<OP, ELT, stage_bytes(AC, BC, ELT, 128), 2, 2, 2, 2>(a, x, g.splits, part, s);
  if constexpr (AC || ELT == 4)
    if (g.v == kSlim) return launch_tiles<OP, ELT, 64, 2, 2, 1, 2>(a, x, g.splits, part, s);
  if constexpr (AC) return launch_tiles<OP, ELT, 64, 1, 4, 1, 1>(a, x, g.splits, part, s);
  return hipErrorInvalidValue;
}

}  // namespace

size_t expert_workspace_need(dattri_linear_op op, int64_t rows, int64_t experts, int64_t d_in, int64_t d_out, int elt,
                             bool aligned) {
  return expert_layout(op, rows, experts, d_in, d_out, elt, aligned).total;
}

hipError_t launch_expert(dattri_linear_op op, int elt, bool aligned, GemmArgs a, ExpertArgs x, float* dbias,
                         uint8_t* ws, hipStream_t s) {
  const bool wgrad = op == DATTRI_LINEAR_WEIGHT_GRAD;
  const int64_t d_out = op == DATTRI_LINEAR_FORWARD ? a.N : wgrad ? a.M : a.K,
                d_in = op == DATTRI_LINEAR_FORWARD ? a.K : a.N;
  const int oelt = wgrad ? 4 : elt;
  auto on4 = [](const void* p, int64_t ld, int e) { return !p || ((uintptr_t)p % (4 * e) == 0 && ld % 4 == 0); };
  a.vec = on4(a.bias, a.N, elt) && on4(a.R, a.ldr, elt) && on4(a.Z, a.ldz, elt) && on4(a.out, a.ldo, oelt) &&
          on4(a.out2, a.ldo2, elt) && (!wgrad || x.stride % 4 == 0);
  const ExpertLayout L = expert_layout(op, x.rows, x.experts, d_in, d_out, elt, aligned);
  hipError_t e;
  if (dbias) {
    const int64_t parts = column_parts(x.rows, x.experts, d_out), n = (int64_t)x.experts * d_out;
    float* part = (float*)(ws + L.off_cols);
    const bool four = on4(a.A, a.lda, elt) && d_out % 4 == 0;
    auto k = elt == 2 ? (four ? expert_columns_kernel<2, 4> : expert_columns_kernel<2, 1>)
                      : (four ? expert_columns_kernel<4, 4> : expert_columns_kernel<4, 1>);
    const int64_t wide = four ? 256 : 64;
    hipLaunchKernelGGL(k, dim3((unsigned)((d_out + wide - 1) / wide), (unsigned)parts, (unsigned)x.experts), dim3(256), 0,
                       s, a.A, a.lda, x, (int)d_out, part, dbias, (int)a.accumulate);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (parts > 1) {
      dim3 grid;
      if ((e = row_grid((n + 255) / 256, &grid)) != hipSuccess) return e;
      hipLaunchKernelGGL(expert_columns_join_kernel, grid, dim3(256), 0, s, part, (int)parts, n, dbias,
                         (int)a.accumulate);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (!a.out) return hipSuccess;
  }
  if (L.pack_a || L.pack_b) {
    Repack ra = {}, rb = {};
    // the layout has room for both as soon as one is off 16 bytes
    if (!on_chunks(a.A, a.lda, L.a_w, elt)) ra = repack_of(&a.A, &a.lda, L.a_w, L.a_rows, elt, ws + L.off_a);
    if (!on_chunks(a.B, a.ldb, L.b_w, elt)) {
      rb = repack_of(&a.B, &a.ldb, L.b_w, L.b_rows, elt, ws + L.off_b);
      if (!wgrad) x.stride = a.ldb * d_out;
    }
    const int64_t n = ra.rows + rb.rows;
    if (n > 0) {
      dim3 grid;
      if ((e = row_grid((n + 3) / 4, &grid)) != hipSuccess) return e;
      if (wgrad)
        hipLaunchKernelGGL(elt == 2 ? repack_kernel<2> : repack_kernel<4>, grid, dim3(256), 0, s, ra, rb);
      else
        hipLaunchKernelGGL(elt == 2 ? expert_repack_kernel<2> : expert_repack_kernel<4>, grid, dim3(256), 0, s, ra, rb, x,
                           (int)d_out);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  float* part = (float*)(ws + L.off_part);
  if (op == DATTRI_LINEAR_FORWARD)
    return elt == 2 ? launch_product<DATTRI_LINEAR_FORWARD, 2>(a, x, L.g, part, s)
                    : launch_product<DATTRI_LINEAR_FORWARD, 4>(a, x, L.g, part, s);
  if (op == DATTRI_LINEAR_INPUT_GRAD)
    return elt == 2 ? launch_product<DATTRI_LINEAR_INPUT_GRAD, 2>(a, x, L.g, part, s)
                    : launch_product<DATTRI_LINEAR_INPUT_GRAD, 4>(a, x, L.g, part, s);
  return elt == 2 ? launch_product<DATTRI_LINEAR_WEIGHT_GRAD, 2>(a, x, L.g, part, s)
                  : launch_product<DATTRI_LINEAR_WEIGHT_GRAD, 4>(a, x, L.g, part, s);
}

}  // namespace dattri
