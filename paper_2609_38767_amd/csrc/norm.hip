// Root-mean-square norm of rows with the residual's addition, its gradient, and
// rows and weights in 8 bits.
//
//   h = x + r,  u = 1 / sqrt(mean_j h_j^2 + eps),  y_j = h_j u w_j
//   a_j = g_j w_j:  dh_j = u (a_j - h_j u^2 mean_j(a_j h_j)) + p_j,  dw_j = sum_rows g_j h_j u
//
// Rows that fit the registers of up to 1024 threads are read once: T threads hold
// a row, C pieces of 16 bytes each (or of two elements where rows are not on 16
// bytes), from the sums to the outputs.  Longer rows are read twice, by a
// workgroup each.  A group of 8-bit values is 128 neighbouring columns of one
// wave's piece, so its largest magnitude is one reduction over 16, 32 or 64 lanes.
//
// What bounds it: memory.  16384 rows of 4096 bf16: sum, norm and 8 bits 72 us
// (471 MB, 6.5 TB/s), gradients 89 + 5 (537 MB, 6.0); 65536 rows of 128 12.1 us
// (67 MB); 8192 rows of 4099, most of them off 16 bytes, 54 us (5.0 TB/s), the
// gradients 67.  One row of 4096 2.1 us: the launch.  Rows that no registers hold
// are read twice: 4096 of 40000 float32 834 us, 3.9 TB/s of what it then moves.
// Times of variants below are of kernels alone, measured in turn: between runs the
// gradient's kernel moves from 83 to 89 us, so each is to be read beside its pair.
#include <algorithm>
#include <type_traits>

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
  const float sc = scale8(wave_max(max_mag(max_mag(0.f, v0), v1)));
  const Quotient8 by(sc);
  const int w = pack8<false>(by.of(v0), by.of(v1), 0);
  if (lane < left) q[lane] = (uint8_t)w;
  if (lane + 64 < left) q[lane + 64] = (uint8_t)(w >> 8);
  if (lane == 0) *s = sc;
}

// Sum or maximum over 16 lanes by data-parallel moves: the quad's neighbours, the
// other quad of eight, the other eight.
template <class F>
__device__ inline float over16(float v, F f) {
  auto moved = [](float x, auto ctrl) {
    const int i = __builtin_bit_cast(int, x);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  v = f(v, moved(v, std::integral_constant<int, 0xB1>{}));   // quad_perm 1 0 3 2
  v = f(v, moved(v, std::integral_constant<int, 0x4E>{}));   // quad_perm 2 3 0 1
  v = f(v, moved(v, std::integral_constant<int, 0x141>{}));  // row_half_mirror
  return f(v, moved(v, std::integral_constant<int, 0x140>{}));  // row_mirror
}
// Sum over T lanes, 64 at most.
template <int T>
__device__ inline float lanes_sum(float v) {
  v = over16(v, [](float a, float b) { return a + b; });
  if constexpr (T > 16) v += __shfl_xor(v, 16);
  if constexpr (T > 32) v += __shfl_xor(v, 32);
  return v;
}

// A thread's pieces of a row of d elements held by T threads; T below 64: a wave
// holds 64 / T rows (VEC only).
template <int ELT, bool VEC, int T>
struct RowOf {
  static constexpr int N = VEC ? 16 / ELT : 2;  // elements of a piece
  // rows of a workgroup (one as soon as its waves have to meet), of a wave
  static constexpr int kRows = T <= 64 ? 256 / T : 1, kPerWave = T < 64 ? 64 / T : 1;
  static constexpr int kThreads = T <= 64 ? 256 : T;
  static_assert(T >= (VEC ? kGroup8 / N : 64), "a group of 8-bit values in one row's lanes");
  typedef std::conditional_t<VEC, i32x4, i32x2> Raw;
  int t, sub, d;  // place in the row, row of the wave
  __device__ explicit RowOf(int d_) : t(threadIdx.x % T), sub(T < 64 ? (threadIdx.x & 63) / T : 0), d(d_) {}
  // The wave's first row of the workgroup's rows from r0.
  __device__ static int64_t first(int64_t r0) {
    return r0 + (T <= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 64 / T : 0);
  }
  // Column of element e of piece c.  VEC: N neighbours per lane; else 64 apart, lanes neighbours.
  __device__ int col(int c, int e) const {
    return VEC ? (c * T + t) * N + e : (c * (T / 64) + (t >> 6)) * kGroup8 + (t & 63) + 64 * e;
  }
  // The wave's rows as a buffer that ends with the last one: what lies behind
  // reads as zero and is not written.  (Rows of their own end at d by themselves;
  // where several share a buffer the column is looked at.)
  struct Buffer {
    rsrc_t r;
    uint32_t row;
  };
  __device__ Buffer buffer(const void* p, int64_t row0, int64_t ld, int64_t rows, int elt = ELT) const {
    const uint32_t stride = (uint32_t)(ld * elt);
    const int n = kPerWave > 1 ? (int)min((int64_t)kPerWave, rows - row0) : 1;
    return Buffer{make_rsrc((const uint8_t*)p + row0 * ld * elt, (uint32_t)(n - 1) * stride + (uint32_t)d * elt),
                  kPerWave > 1 ? sub * stride : 0};
  }
  __device__ uint32_t at(const Buffer& b, int c, int e, int elt = ELT) const {
    const uint32_t o = b.row + (uint32_t)col(c, e) * elt;
    return kPerWave > 1 && col(c, e) >= d ? kOOB : o;
  }
  // ONCE: past the caches
  template <bool ONCE = false>
  __device__ Raw load(const Buffer& b, int c) const {
    constexpr int kAux = ONCE ? 2 : 0;  // non-temporal
    if constexpr (VEC)
      return __builtin_amdgcn_raw_buffer_load_b128(b.r, at(b, c, 0), 0, kAux);
    else
      return i32x2{(int)(ELT == 2 ? load2(b.r, at(b, c, 0)) : load4(b.r, at(b, c, 0))),
                   (int)(ELT == 2 ? load2(b.r, at(b, c, 1)) : load4(b.r, at(b, c, 1)))};
  }
  __device__ static void floats(Raw r, float (&v)[N]) {
    if constexpr (!VEC) {
#pragma unroll
      for (int e = 0; e < 2; ++e) v[e] = __builtin_bit_cast(float, ELT == 2 ? r[e] << 16 : r[e]);
    } else if constexpr (ELT == 2) {
      const uint32_t w[4] = {(uint32_t)r.x, (uint32_t)r.y, (uint32_t)r.z, (uint32_t)r.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __builtin_bit_cast(float, w[e] << 16);
        v[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xFFFF0000u);
      }
    } else {
      const f32x4 f = __builtin_bit_cast(f32x4, r);
      v[0] = f.x;
      v[1] = f.y;
      v[2] = f.z;
      v[3] = f.w;
    }
  }
  __device__ void store(const Buffer& b, int c, const float (&v)[N]) const {
    if constexpr (!VEC) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if constexpr (ELT == 2)
          __builtin_amdgcn_raw_buffer_store_b16((short)pack_bf16(v[e], 0.f), b.r, at(b, c, e), 0, 0);
        else
          __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(int, (float)v[e]), b.r, at(b, c, e), 0, 0);
    } else {
      i32x4 w;
      if constexpr (ELT == 2)
        w = i32x4{(int)pack_bf16(v[0], v[1]), (int)pack_bf16(v[2], v[3]), (int)pack_bf16(v[4], v[5]),
                  (int)pack_bf16(v[6], v[7])};
      else
        w = __builtin_bit_cast(i32x4, f32x4{v[0], v[1], v[2], v[3]});
      __builtin_amdgcn_raw_buffer_store_b128(w, b.r, at(b, c, 0), 0, 0);
    }
  }
  // The piece in 8 bits: values to q, the group's scale to the row's scales s (`here`: the row exists).
  __device__ void store8(const Buffer& q, float* s, bool here, int c, const float (&v)[N]) const {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) top = max_mag(top, v[e]);
    top = over16(top, [](float a, float b) { return fmaxf(a, b); });
    if constexpr (N < 8) top = fmaxf(top, __shfl_xor(top, 16));
    if constexpr (N < 4) top = fmaxf(top, __shfl_xor(top, 32));
    const float sc = scale8(top);
    const Quotient8 by(sc);
    if constexpr (!VEC) {
      const int w = pack8<false>(by.of(v[0]), by.of(v[1]), 0);
      __builtin_amdgcn_raw_buffer_store_b8((char)w, q.r, at(q, c, 0, 1), 0, 0);
      __builtin_amdgcn_raw_buffer_store_b8((char)(w >> 8), q.r, at(q, c, 1, 1), 0, 0);
    } else {
      int w[N / 4];
#pragma unroll
      for (int e = 0; e < N / 4; ++e)
        w[e] = pack8<true>(by.of(v[4 * e + 2]), by.of(v[4 * e + 3]),
                           pack8<false>(by.of(v[4 * e]), by.of(v[4 * e + 1]), 0));
      if constexpr (N == 8)
        __builtin_amdgcn_raw_buffer_store_b64(i32x2{w[0], w[1]}, q.r, at(q, c, 0, 1), 0, 0);
      else
        __builtin_amdgcn_raw_buffer_store_b32(w[0], q.r, at(q, c, 0, 1), 0, 0);
    }
    if (here && col(c, 0) % kGroup8 == 0 && col(c, 0) < d) s[col(c, 0) / kGroup8] = sc;
  }
};

// Sums of S values each over the T threads of a row, waves in order; every
// thread gets them.  `red` holds [2][T / 64][S], `turn` alternates from call to call.
template <int T, int S>
__device__ inline void row_sums(float (&v)[S], float* red, int turn) {
#pragma unroll
  for (int k = 0; k < S; ++k) v[k] = lanes_sum<T>(v[k]);
  if constexpr (T > 64) {
    constexpr int W = T / 64;
    float* at = red + (turn & 1) * W * S;
    const int t = threadIdx.x % T;
    if ((t & 63) == 0)
#pragma unroll
      for (int k = 0; k < S; ++k) at[(t >> 6) * S + k] = v[k];
    lds_barrier();
#pragma unroll
    for (int k = 0; k < S; ++k) {
      v[k] = at[k];
#pragma unroll
      for (int w = 1; w < W; ++w) v[k] += at[w * S + k];
    }
  }
}

}  // namespace

template <int ELT, bool VEC, bool ONCE, int T, int C>
__global__ __launch_bounds__(T <= 64 ? 256 : T) void rms_norm_kernel(NormArgs a) {
  typedef RowOf<ELT, VEC, T> Row;
  constexpr int N = Row::N;
  __shared__ float red[T > 64 ? T / 64 : 1];
  const Row p(a.d);
  const int64_t row0 = Row::first(row_block() * Row::kRows), row = row0 + p.sub;
  if (row0 >= a.rows) return;  // T up to 64: whole waves, which meet no barrier
  const bool here = row < a.rows;
  const auto x = p.buffer(a.X, row0, a.ldx, a.rows), r = p.buffer(a.R, row0, a.ldr, a.rows);
  const typename Row::Buffer w1 = {p.buffer(a.W, 0, 0, 1).r, 0};
  typename Row::Raw rx[C], rr[C], rw[C];
#pragma unroll
  for (int c = 0; c < C; ++c) rx[c] = p.template load<ONCE>(x, c);
  if (a.R)
#pragma unroll
    for (int c = 0; c < C; ++c) rr[c] = p.template load<ONCE>(r, c);
#pragma unroll
  for (int c = 0; c < C; ++c) rw[c] = p.load(w1, c);
  float h[C][N], s[1] = {0.f};
#pragma unroll
  for (int c = 0; c < C; ++c) {
    Row::floats(rx[c], h[c]);
    if (a.R) {
      float v[N];
      Row::floats(rr[c], v);
#pragma unroll
      for (int e = 0; e < N; ++e) h[c][e] += v[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) s[0] = fmaf(h[c][e], h[c][e], s[0]);
  }
  row_sums<T>(s, red, 0);
  const float u = 1.f / sqrtf(s[0] / a.d + a.eps);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (a.H) p.store(p.buffer(a.H, row0, a.ldh, a.rows), c, h[c]);
    float w[N];
    Row::floats(rw[c], w);
#pragma unroll
    for (int e = 0; e < N; ++e) h[c][e] = h[c][e] * u * w[e];
    if (a.Y) p.store(p.buffer(a.Y, row0, a.ldy, a.rows), c, h[c]);
    if (a.Q) p.store8(p.buffer(a.Q, row0, a.ldq, a.rows, 1), a.S + row * a.lds, here, c, h[c]);
  }
}

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

// The workgroups walk the rows; each keeps its columns' share of dW and leaves it
// as one row of part (null: dW is not wanted).
template <int ELT, bool VEC, bool ONCE, int T, int C>
__global__ __launch_bounds__(T <= 64 ? 256 : T) void norm_grad_kernel(NormGradArgs a, float* __restrict__ part) {
  typedef RowOf<ELT, VEC, T> Row;
  constexpr int N = Row::N, kRows = Row::kRows;
  constexpr bool kAhead = C <= 2;  // the next row is on its way while this one is worked on
  __shared__ float red[T > 64 ? 4 * T / 64 : 1];
  __shared__ float share[kRows > 1 ? kRows * T * N : 1];
  const Row p(a.d);
  typename Row::Raw rw[C];
  const typename Row::Buffer w1 = {p.buffer(a.W, 0, 0, 1).r, 0};
#pragma unroll
  for (int c = 0; c < C; ++c) rw[c] = p.load(w1, c);
  float dw[C][N] = {};
  struct Three {
    typename Row::Raw g[C], h[C], p[C];
  };
  auto fetch = [&](int64_t row0) {
    Three v = {};
    if (row0 < a.rows) {
      const auto g = p.buffer(a.G, row0, a.ldg, a.rows), h = p.buffer(a.H, row0, a.ldh, a.rows),
                 q = p.buffer(a.P, row0, a.ldp, a.rows);
#pragma unroll
      for (int c = 0; c < C; ++c) v.g[c] = p.template load<ONCE>(g, c);
#pragma unroll
      for (int c = 0; c < C; ++c) v.h[c] = p.template load<ONCE>(h, c);
      if (a.P)
#pragma unroll
        for (int c = 0; c < C; ++c) v.p[c] = p.template load<ONCE>(q, c);
    }
    return v;
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int turn = 0;
  Three next = fetch(Row::first((int64_t)blockIdx.x * kRows));
  // T > 64: all rows of a workgroup meet the barriers of row_sums, so it runs as long as its first has a row
  for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < a.rows; r0 += step, ++turn) {
    const int64_t row0 = Row::first(r0);
    if (!kAhead && turn) next = fetch(row0);
    Three now = next;
    auto &rg = now.g, &rh = now.h, &rp = now.p;
    if (kAhead) next = fetch(row0 + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float vg[N], vh[N], vw[N];
      Row::floats(rg[c], vg);
      Row::floats(rh[c], vh);
      Row::floats(rw[c], vw);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        s[0] = fmaf(vh[e], vh[e], s[0]);
        s[1] = fmaf(vg[e] * vw[e], vh[e], s[1]);
      }
    }
    row_sums<T>(s, red, turn);
    // places of the wave behind the last row hold zeros: no 0 / 0 of theirs goes to dW
    const float u = T < 64 && row0 + p.sub >= a.rows ? 0.f : 1.f / sqrtf(s[0] / a.d + a.eps), k = u * u * (s[1] / a.d);
    if (row0 >= a.rows) continue;  // rows of the wave that are not there are zeros, and are not written
    const auto out = p.buffer(a.D, row0, a.ldd, a.rows);
    // 1024 threads: the floats of before are formed again rather than kept, for bf16 takes half the registers (4096 rows
    // of 16384 with the joining of dW 118 us, kept 211; with 256 threads, 16384 rows of 4096, 99.6 and 93.0)
    if constexpr (T == 1024)
#pragma unroll
      for (int c = 0; c < C; ++c) asm volatile("" : "+v"(rg[c]), "+v"(rh[c]), "+v"(rw[c]));
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float vg[N], vh[N], vw[N], vp[N];
      Row::floats(rg[c], vg);
      Row::floats(rh[c], vh);
      Row::floats(rw[c], vw);
      Row::floats(rp[c], vp);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        dw[c][e] = fmaf(vg[e], vh[e] * u, dw[c][e]);
        vg[e] = u * fmaf(-vh[e], k, vg[e] * vw[e]);
        if (a.P) vg[e] += vp[e];
      }
      p.store(out, c, vg);
    }
  }
  if (!part) return;
  float* out = part + (int64_t)blockIdx.x * a.d;
  const int sub = T <= 64 ? threadIdx.x / T : 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if constexpr (kRows > 1) {  // the rows' shares in order
      __syncthreads();
#pragma unroll
      for (int e = 0; e < N; ++e) share[(sub * N + e) * T + p.t] = dw[c][e];
      __syncthreads();
      if (sub == 0)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          float v = share[e * T + p.t];
#pragma unroll
          for (int k = 1; k < kRows; ++k) v += share[(k * N + e) * T + p.t];
          dw[c][e] = v;
        }
    }
    if (sub == 0)
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (p.col(c, e) < a.d) out[p.col(c, e)] = dw[c][e];
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

// 32 columns per workgroup and 32 interleaved runs of the parts.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* __restrict__ part, int n_parts, int cols,
                                                         float* __restrict__ out, int accumulate) {
  __shared__ float red[32][33];
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols)
#pragma unroll 8
    for (int y = run; y < n_parts; y += 32) s += part[(int64_t)y * cols + c];
  red[run][lane] = s;
  __syncthreads();
  const int at = threadIdx.x >> 5, w = blockIdx.x * 32 + at;  // column `at`, summed by 32 lanes
  s = red[lane][at];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0 && w < cols) out[w] = accumulate ? out[w] + s : s;
}

// A wave takes kQuantize pieces of a row, n_waves waves a row.
constexpr int kQuantize = 4;
template <int ELT, bool VEC>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void* __restrict__ X, int64_t ldx, int64_t rows,
                                                            int d, int n_waves, uint8_t* __restrict__ Q, int64_t ldq,
                                                            float* __restrict__ S, int64_t lds) {
  typedef RowOf<ELT, VEC, 64> Row;
  const int64_t i = row_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = i / n_waves;
  if (row >= rows) return;
  const int c0 = (int)(i - row * n_waves) * kQuantize;
  const Row p(d);
  const auto x = p.buffer(X, row, ldx, rows), q = p.buffer(Q, row, ldq, rows, 1);
  typename Row::Raw r[kQuantize];
#pragma unroll
  for (int c = 0; c < kQuantize; ++c) r[c] = p.load(x, c0 + c);
#pragma unroll
  for (int c = 0; c < kQuantize; ++c) {
    float v[Row::N];
    Row::floats(r[c], v);
    p.store8(q, S + row * lds, true, c0 + c, v);
  }
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
  const float s = scale8(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
  const Quotient8 by(s);
  if (threadIdx.x == 0) S[bo * lds + bi] = s;
  if (c < d)
#pragma unroll 8
    for (int r = threadIdx.x >> 7; r < n; r += 2)
      Q[(r0 + r) * ldq + c] = (uint8_t)pack8<false>(by.of(load_elt<ELT>(W, (r0 + r) * ldw + c)), 0.f, 0);
}

namespace {

// Bytes read and written from which on rows are loaded past the caches, which
// cannot hold them for the next reader: 16384 rows of 4096 bf16, norm to 8 bits
// (471 MB) 71 us, through the caches 79; gradient (537 MB) 83 and 106.
constexpr int64_t kOnceBytes = (int64_t)256 << 20;

// Pieces of a row.
int64_t pieces_of(int elt, bool vec, int64_t d) { return vec ? d / (16 / elt) : (d + kGroup8 - 1) / kGroup8 * 64; }

// f(T, C) with the threads and pieces per thread that hold rows of n pieces;
// false if none do.  Several short rows in a wave: as few lanes each as hold a
// group of 8-bit values.  Four waves per row as soon as each has a piece for
// every lane: 16384 rows of 4096 bf16, norm to 8 bits 71 us, with one wave 74;
// gradient 83 and 116, whose sums of dW a wave has fewer of.
// Rows off 16 bytes, whose pieces are two elements: eight pieces per thread, for
// fewer sums across waves and more loads under way, where there are rows enough.
// us of the norm, with two pieces per thread in brackets: 40000 rows of 1001 bf16
// 33 (52), gradient 47 (102); 8192 of 3001 26 (48) and 39 (66); 8192 of 4099
// float32 53 (72), but its gradient 92 (85).  Few rows: 1024 of 769 float32 to 8
// bits 5.5 (4.3), gradient 8.0 (8.4); 300 of 1023 5.0 (3.4) and 7.1 (6.6).  Of 1025
// to 2048 columns a wave takes sixteen pieces for the gradient, whose workgroups
// (kGradGroups) of 128 threads would leave half the CUs' places empty: 20000 rows
// of 1501 bf16 43, with 128 threads 70.
constexpr int kGradMost = 16384;  // columns of the longest row of a gradient that they hold
template <int ELT, bool VEC, bool GRAD, class F>
bool with_shape(int64_t n, int64_t rows, F f) {
  constexpr int kMost = GRAD && VEC ? kGradMost * ELT / 16 : 8192;
#define SHAPE(T, C)                  \
  if constexpr ((T) * (C) <= kMost)  \
    if (n <= (T) * (C)) return f(std::integral_constant<int, T>{}, std::integral_constant<int, C>{}), true
  if constexpr (VEC) {
    SHAPE(8 * ELT, 1);
    SHAPE(8 * ELT, 2);
  }
  SHAPE(64, 1);
  SHAPE(64, 2);
  if (!VEC || n < 256) SHAPE(64, 4);
  if constexpr (!VEC)
    if (rows >= (GRAD ? 400 : 2048)) {
      SHAPE(64, 8);
      SHAPE(GRAD ? 64 : 128, GRAD ? 16 : 8);
      SHAPE(256, 8);
      if constexpr (!GRAD || ELT == 2) SHAPE(512, 8);
    }
  SHAPE(256, 2);
  SHAPE(512, 2);
  SHAPE(1024, 2);
  SHAPE(1024, 4);
  SHAPE(1024, 8);
#undef SHAPE
  return false;
}

bool on(const void* p, int64_t ld, int elt, int bytes) {
  return !p || ((uintptr_t)p % bytes == 0 && ld * elt % bytes == 0);
}

template <int ELT, bool VEC, bool ONCE>
hipError_t launch_norm_as(const NormArgs& a, hipStream_t s) {
  hipError_t e = hipSuccess;
  const int64_t n = pieces_of(ELT, VEC, a.d);
  const bool held = with_shape<ELT, VEC, false>(n, a.rows, [&](auto T, auto C) {
    typedef RowOf<ELT, VEC, decltype(T)::value> Row;
    dim3 grid;
    if ((e = row_grid((a.rows + Row::kRows - 1) / Row::kRows, &grid, Row::kThreads)) != hipSuccess) return;
    hipLaunchKernelGGL((rms_norm_kernel<ELT, VEC, ONCE, decltype(T)::value, decltype(C)::value>), grid,
                       dim3(Row::kThreads), 0, s, a);
    e = hipGetLastError();
  });
  if (held) return e;
  dim3 grid;
  if ((e = row_grid(a.rows, &grid)) != hipSuccess) return e;
  hipLaunchKernelGGL((rms_norm_long_kernel<ELT>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(int elt, const NormArgs& a, hipStream_t s) {
  const bool vec = a.d % (16 / elt) == 0 && on(a.X, a.ldx, elt, 16) && on(a.R, a.ldr, elt, 16) && on(a.W, 0, elt, 16) &&
                   on(a.Y, a.ldy, elt, 16) && on(a.H, a.ldh, elt, 16) && on(a.Q, a.ldq, 1, 16 / elt);
  const int64_t per = 1 + (a.R != nullptr) + (a.Y != nullptr) + (a.H != nullptr);
  const bool once = a.rows * a.d * (per * elt + (a.Q != nullptr)) > kOnceBytes;
  if (!vec) return elt == 2 ? launch_norm_as<2, false, false>(a, s) : launch_norm_as<4, false, false>(a, s);
  return elt == 2 ? (once ? launch_norm_as<2, true, true>(a, s) : launch_norm_as<2, true, false>(a, s))
                  : (once ? launch_norm_as<4, true, true>(a, s) : launch_norm_as<4, true, false>(a, s));
}

namespace {

// Workgroups of the gradient where registers hold the rows: two per CU (16384
// rows of 4096 bf16: 83 us, with one 87, three 89, four 97).  Whether they do
// does not go by the buffers' alignment here, so a layout fits any.
constexpr int kGradGroups = 512;
bool grad_held(int64_t d) { return d <= kGradMost; }

// Rows per part of a long row's weight gradient, and parts: eight workgroups per CU of 64 rows or more.
void weight_shape(int64_t rows, int64_t d, int64_t* per, int64_t* parts) {
  const int64_t p = std::max<int64_t>(1, std::min<int64_t>(2048 / ((d + 63) / 64), rows / 64));
  *per = std::max<int64_t>(1, (rows + p - 1) / p);
  *parts = std::max<int64_t>(1, (rows + *per - 1) / *per);
}

}  // namespace

NormGradLayout norm_grad_layout(int64_t rows, int64_t d, bool weight) {
  NormGradLayout l = {};
  if (!weight) return l;
  if (grad_held(d)) {
    l.total = align_up((size_t)std::min<int64_t>(kGradGroups, rows) * d * 4);
    return l;
  }
  int64_t per, parts;
  weight_shape(rows, d, &per, &parts);
  l.off_part = align_up((size_t)rows * 4);
  l.total = l.off_part + align_up(parts > 1 ? (size_t)parts * d * 4 : 0);
  return l;
}

namespace {

hipError_t join(const float* part, int64_t parts, int64_t d, float* dw, bool accumulate, hipStream_t s) {
  hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)((d + 31) / 32)), dim3(1024), 0, s, part, (int)parts, (int)d, dw,
                     (int)accumulate);
  return hipGetLastError();
}

template <int ELT, bool VEC, bool ONCE>
hipError_t launch_grad_as(const NormGradArgs& a, float* dw, bool accumulate, uint8_t* ws, hipStream_t s) {
  hipError_t e = hipSuccess;
  int64_t groups = 0;
  with_shape<ELT, VEC, true>(pieces_of(ELT, VEC, a.d), a.rows, [&](auto T, auto C) {
    typedef RowOf<ELT, VEC, decltype(T)::value> Row;
    groups = std::min<int64_t>(kGradGroups, (a.rows + Row::kRows - 1) / Row::kRows);
    if (groups == 0) return;
    hipLaunchKernelGGL((norm_grad_kernel<ELT, VEC, ONCE, decltype(T)::value, decltype(C)::value>),
                       dim3((unsigned)groups), dim3(Row::kThreads), 0, s, a, dw ? (float*)ws : nullptr);
    e = hipGetLastError();
  });
  if (e != hipSuccess || !dw) return e;
  return join((const float*)ws, groups, a.d, dw, accumulate, s);
}

}  // namespace

hipError_t launch_norm_grad(int elt, NormGradArgs a, float* dw, bool accumulate, uint8_t* ws, hipStream_t s) {
  if (grad_held(a.d)) {
    const bool vec = a.d % (16 / elt) == 0 && on(a.G, a.ldg, elt, 16) && on(a.H, a.ldh, elt, 16) &&
                     on(a.W, 0, elt, 16) && on(a.P, a.ldp, elt, 16) && on(a.D, a.ldd, elt, 16);
    const bool once = a.rows * a.d * elt * (3 + (a.P != nullptr)) > kOnceBytes;
    if (!vec)
      return elt == 2 ? launch_grad_as<2, false, false>(a, dw, accumulate, ws, s)
                      : launch_grad_as<4, false, false>(a, dw, accumulate, ws, s);
    if (elt == 2)
      return once ? launch_grad_as<2, true, true>(a, dw, accumulate, ws, s)
                  : launch_grad_as<2, true, false>(a, dw, accumulate, ws, s);
    return once ? launch_grad_as<4, true, true>(a, dw, accumulate, ws, s)
                : launch_grad_as<4, true, false>(a, dw, accumulate, ws, s);
  }
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
  hipLaunchKernelGGL(elt == 2 ? norm_weight_kernel<2> : norm_weight_kernel<4>,
                     dim3((unsigned)((a.d + 63) / 64), (unsigned)parts), dim3(256), 0, s, a, per,
                     parts > 1 ? part : dw, parts > 1 ? 0 : (int)accumulate);
  if ((e = hipGetLastError()) != hipSuccess || parts == 1) return e;
  return join(part, parts, a.d, dw, accumulate, s);
}

hipError_t launch_quantize_rows(int elt, const void* X, int64_t ldx, int64_t rows, int64_t d, uint8_t* Q, int64_t ldq,
                                float* S, int64_t lds, hipStream_t s) {
  const bool vec = d % (16 / elt) == 0 && on(X, ldx, elt, 16) && on(Q, ldq, 1, 16 / elt);
  const int n_waves = (int)((pieces_of(elt, vec, d) + 64 * kQuantize - 1) / (64 * kQuantize));
  dim3 grid;
  const hipError_t e = row_grid((rows * n_waves + 3) / 4, &grid);
  if (e != hipSuccess) return e;
  auto k = elt == 2 ? (vec ? quantize_rows_kernel<2, true> : quantize_rows_kernel<2, false>)
                    : (vec ? quantize_rows_kernel<4, true> : quantize_rows_kernel<4, false>);
  hipLaunchKernelGGL(k, grid, dim3(256), 0, s, X, ldx, rows, (int)d, n_waves, Q, ldq, S, lds);
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
