// Norm of many gradients together, and clipping.
//
//   norm = sqrt(sum g^2),  coef = min(1, max_norm / (norm + 1e-6)),  out = coef g
//
// The tensors of a launch come as a kernel argument (no table on the device to
// keep in step with buffers that move); their elements are cut into chunks of
// kClipChunk, dealt to the workgroups in turn.  Squares are summed in float64:
// float32 squares of large gradients overflow long before the gradients do,
// and the sum of 10^9 terms keeps its digits whatever the order.  Every
// workgroup writes one partial sum; one workgroup adds them up and writes norm
// and coefficient (4096 sums: every scaling workgroup adding them up for itself
// took 14 us where nothing was to be scaled).
//
// What bounds it: memory.  The norm has to be known before the first gradient
// is scaled, so what the caches do not hold is read twice.  872 M elements, bf16
// into float32: squares 252-262 us (6.7-6.9 TB/s), scaling 973 us (5.4 TB/s read
// and written).
#include "api_common.h"
#include "device_common.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;

// The chunk's tensor, its first element and how many elements it has.
struct Chunk {
  int tensor;
  int64_t begin;
  int count;
};
__device__ inline Chunk find_chunk(const ClipList& l, int c) {
  int lo = 0, hi = l.n - 1;  // the last tensor whose first chunk is <= c
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (l.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  const int64_t begin = (int64_t)(c - l.first[lo]) * kClipChunk;
  return Chunk{lo, begin, (int)min((int64_t)kClipChunk, (l.t[lo].size_flags >> 2) - begin)};
}

__device__ inline double sq(float x, double s) { return fma((double)x, (double)x, s); }

template <int ELT>
__device__ inline void unpack(i32x4 w, float (&v)[16 / ELT]) {
  if constexpr (ELT == 2) {
    const uint32_t u[4] = {(uint32_t)w.x, (uint32_t)w.y, (uint32_t)w.z, (uint32_t)w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __builtin_bit_cast(float, u[e] << 16);
      v[2 * e + 1] = __builtin_bit_cast(float, u[e] & 0xFFFF0000u);
    }
  } else {
    const f32x4 f = __builtin_bit_cast(f32x4, w);
    v[0] = f.x;
    v[1] = f.y;
    v[2] = f.z;
    v[3] = f.w;
  }
}
template <int ELT>
__device__ inline float load_one(const uint8_t* p, int i) {
  return ELT == 2 ? bf16_bits_to_f32(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}

constexpr int kBatch = 8;  // 16-byte loads in flight per thread

// STREAM: loads past the caches, for sets that no cache holds until the second
// pass.  bf16, norm alone: 288 MB 49 us, 50 through the caches; 480 MB 78 and 88;
// 1.74 GB 267 and 302.  Scaled into float32: 220 and 239, 359 and 381, 1275 and
// 1321 us.  Stores past the caches instead are slower (1.74 GB: 1927).  A
// template argument: under a run-time flag the compiler merges both loads into
// a plain one.
template <bool STREAM>
__device__ inline i32x4 load_piece(const uint8_t* p) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load((const i32x4*)p);
  else
    return *(const i32x4*)p;
}

template <int ELT, bool STREAM>
__device__ inline double chunk_squares(const uint8_t* p, int count) {
  constexpr int EPL = 16 / ELT, kStep = 256 * EPL * kBatch;
  double s[2] = {0., 0.};
  int done = 0;
  if ((uintptr_t)p % 16 == 0) {
    for (; done + kStep <= count; done += kStep) {
      i32x4 w[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        w[u] = load_piece<STREAM>(p + (int64_t)(done + (u * 256 + threadIdx.x) * EPL) * ELT);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        float v[EPL];
        unpack<ELT>(w[u], v);
#pragma unroll
        for (int e = 0; e < EPL; ++e) s[e & 1] = sq(v[e], s[e & 1]);
      }
    }
    const int end = count / EPL * EPL;
    for (int i = done + threadIdx.x * EPL; i < end; i += 256 * EPL) {
      float v[EPL];
      unpack<ELT>(*(const i32x4*)(p + (int64_t)i * ELT), v);
#pragma unroll
      for (int e = 0; e < EPL; ++e) s[e & 1] = sq(v[e], s[e & 1]);
    }
    done = end;
  }
#pragma unroll 4
  for (int i = done + threadIdx.x; i < count; i += 256) s[0] = sq(load_one<ELT>(p, i), s[0]);
  return s[0] + s[1];
}

// Sum over the workgroup's W waves in a fixed order; thread 0 gets it.
template <int W>
__device__ inline double block_sum(double s) {
  __shared__ double red[W];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = red[0];
#pragma unroll
  for (int w = 1; w < W; ++w) s += red[w];
  return s;
}

template <bool STREAM>
__global__ __launch_bounds__(256) void clip_squares_kernel(ClipList l, double* __restrict__ partials) {
  double s = 0.;
  const int chunks = l.first[l.n];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Chunk k = find_chunk(l, c);
    const ClipTensor& t = l.t[k.tensor];
    const int elt = t.size_flags & 1 ? 4 : 2;
    const uint8_t* p = (const uint8_t*)t.src + k.begin * elt;
    s += elt == 4 ? chunk_squares<4, STREAM>(p, k.count) : chunk_squares<2, STREAM>(p, k.count);
  }
  s = block_sum<4>(s);
  if (threadIdx.x == 0) partials[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void clip_norm_kernel(const double* __restrict__ partials, int n, float max_norm,
                                                         float* __restrict__ norm_coef) {
  double s = 0.;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 1024) s += partials[i];
  const double norm = sqrt(block_sum<16>(s));
  if (threadIdx.x != 0) return;
  const double c = (double)max_norm / (norm + 1e-6);
  norm_coef[0] = (float)norm;
  // a NaN norm stays in the coefficient; without a bound there is nothing to scale
  norm_coef[1] = max_norm == __builtin_inff() && norm == norm ? 1.f : c >= 1. ? 1.f : (float)c;
}

// One thread's 16 bytes of gradients, scaled, at element i of the output.
template <int ELT, int OELT>
__device__ inline void scale_piece(i32x4 w, float coef, uint8_t* q, int i) {
  constexpr int EPL = 16 / ELT;
  float v[EPL];
  unpack<ELT>(w, v);
#pragma unroll
  for (int e = 0; e < EPL; ++e) v[e] *= coef;
  auto put = [&](auto x, uint8_t* at) { *(decltype(x)*)at = x; };
  if constexpr (OELT == 4) {
#pragma unroll
    for (int e = 0; e < EPL; e += 4) put(f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]}, q + (int64_t)(i + e) * 4);
  } else if constexpr (EPL == 8) {
    put(i32x4{(int)pack_bf16(v[0], v[1]), (int)pack_bf16(v[2], v[3]), (int)pack_bf16(v[4], v[5]),
              (int)pack_bf16(v[6], v[7])}, q + (int64_t)i * 2);
  } else {
    put(i32x2{(int)pack_bf16(v[0], v[1]), (int)pack_bf16(v[2], v[3])}, q + (int64_t)i * 2);
  }
}

template <int ELT, int OELT, bool STREAM>
__device__ inline void scale_chunk(const uint8_t* p, uint8_t* q, int count, float coef) {
  constexpr int EPL = 16 / ELT, kStep = 256 * EPL * kBatch;
  int done = 0;
  if ((uintptr_t)p % 16 == 0 && (uintptr_t)q % 16 == 0) {
    for (; done + kStep <= count; done += kStep) {
      i32x4 w[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        w[u] = load_piece<STREAM>(p + (int64_t)(done + (u * 256 + threadIdx.x) * EPL) * ELT);
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        scale_piece<ELT, OELT>(w[u], coef, q, done + (u * 256 + threadIdx.x) * EPL);
    }
    const int end = count / EPL * EPL;
    for (int i = done + threadIdx.x * EPL; i < end; i += 256 * EPL)
      scale_piece<ELT, OELT>(*(const i32x4*)(p + (int64_t)i * ELT), coef, q, i);
    done = end;
  }
#pragma unroll 4
  for (int i = done + threadIdx.x; i < count; i += 256) {
    const float v = load_one<ELT>(p, i) * coef;
    if (OELT == 4)
      ((float*)q)[i] = v;
    else
      ((uint16_t*)q)[i] = (uint16_t)pack_bf16(v, 0.f);
  }
}

// One workgroup per chunk (872 M elements of bf16 to float32: 976 us, 1066 by
// 2048 workgroups of many chunks), from the last chunk to the first: the norm's
// pass has left the last ones in the caches.
template <bool STREAM>
__global__ __launch_bounds__(256) void clip_scale_kernel(ClipList l, const float* __restrict__ norm_coef) {
  const float coef = norm_coef[1];
  const Chunk k = find_chunk(l, (int)(gridDim.x - 1 - blockIdx.x));
  const ClipTensor& t = l.t[k.tensor];
  if (t.dst == t.src && coef == 1.f) return;  // multiplying by one changes nothing
  const bool f = t.size_flags & 1, of = t.size_flags & 2;
  const uint8_t* p = (const uint8_t*)t.src + k.begin * (f ? 4 : 2);
  uint8_t* q = (uint8_t*)t.dst + k.begin * (of ? 4 : 2);
  if (f && of) scale_chunk<4, 4, STREAM>(p, q, k.count, coef);
  else if (f) scale_chunk<4, 2, STREAM>(p, q, k.count, coef);
  else if (of) scale_chunk<2, 4, STREAM>(p, q, k.count, coef);
  else scale_chunk<2, 2, STREAM>(p, q, k.count, coef);
}

hipError_t launch_clip_squares(const ClipList& l, int groups, double* partials, bool stream, hipStream_t s) {
  if (stream)
    hipLaunchKernelGGL(clip_squares_kernel<true>, dim3(groups), dim3(256), 0, s, l, partials);
  else
    hipLaunchKernelGGL(clip_squares_kernel<false>, dim3(groups), dim3(256), 0, s, l, partials);
  return hipGetLastError();
}
hipError_t launch_clip_norm(const double* partials, int n_partials, float max_norm, float* norm_coef, hipStream_t s) {
  hipLaunchKernelGGL(clip_norm_kernel, dim3(1), dim3(1024), 0, s, partials, n_partials, max_norm, norm_coef);
  return hipGetLastError();
}
hipError_t launch_clip_scale(const ClipList& l, const float* norm_coef, bool stream, hipStream_t s) {
  if (stream)
    hipLaunchKernelGGL(clip_scale_kernel<true>, dim3(l.first[l.n]), dim3(256), 0, s, l, norm_coef);
  else
    hipLaunchKernelGGL(clip_scale_kernel<false>, dim3(l.first[l.n]), dim3(256), 0, s, l, norm_coef);
  return hipGetLastError();
}

}  // namespace dattri
