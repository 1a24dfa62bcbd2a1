// Embedding lookup and its table gradient.
//
// Lookup: out[i] = scale * table[tokens[i]].  One wave per (row, strip of 512
// columns), 16-byte loads and stores where rows are on 16 bytes.
//
// Gradient: grad_table[v] = scale * sum over positions i with tokens[i] = v of
// grad_out[i].  The positions are sorted by token with a stable radix sort
// (digits of at most 9 bits; counts per workgroup, one scan, ranks within a
// wave by ballots: no float and no ordering depends on timing), so the
// positions of a row form a run in ascending order.  A run is summed as the
// positions up to the next multiple of kRun, whole groups of kRun positions
// whose sums another kernel has formed (so a token that is most of the batch
// does not wait on one wave), and the positions left; the order is that of the
// positions in fixed groups, whatever the launch.
//
// What bounds it: the lookup and the sums read and write each row once; for a
// whole table the zeros of rows without tokens are most of the bytes.
#include <algorithm>

#include "api_common.h"
#include "device_common.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;

constexpr int kStrip = 512;       // columns per wave: 8 per lane
constexpr int kRun = 32;          // positions per group of a long run
constexpr int kMaxDigit = 9;      // bits per sorting pass
constexpr int kBins = 1 << kMaxDigit;
constexpr int kSortItems = 4096;  // least positions per sorting workgroup
constexpr int kSortBlocks = 2048; // most sorting workgroups

// The eight columns a lane owns of a strip: 8 in a row (16 bytes of bf16),
// twice 4 in a row (16 bytes of float32, or 8 of bf16 against 16 of a float32
// output), or one in every 64 (rows not on 16 bytes).
enum Cols { kCols8, kCols4, kCols1 };
template <Cols C>
__device__ inline int col_of(int base, int lane, int e) {
  if constexpr (C == kCols8) return base + 8 * lane + e;
  if constexpr (C == kCols4) return base + 256 * (e >> 2) + 4 * lane + (e & 3);
  return base + 64 * e + lane;
}

// float32 values of a lane's eight columns; columns >= d read as zero (d is a
// multiple of 8 for kCols8, of 4 for kCols4).
template <int ELT, Cols C>
__device__ inline void load_cols(const uint8_t* row, int base, int lane, int d, float (&v)[8]) {
  if constexpr (C == kCols8) {
    const int c = base + 8 * lane;
    i32x4 w = {0, 0, 0, 0};
    if (c < d) w = *(const i32x4*)(row + (int64_t)c * 2);
    const uint32_t u[4] = {(uint32_t)w.x, (uint32_t)w.y, (uint32_t)w.z, (uint32_t)w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __builtin_bit_cast(float, u[e] << 16);
      v[2 * e + 1] = __builtin_bit_cast(float, u[e] & 0xFFFF0000u);
    }
  } else if constexpr (C == kCols4) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = base + 256 * h + 4 * lane;
      if constexpr (ELT == 2) {
        i32x2 w = {0, 0};
        if (c < d) w = *(const i32x2*)(row + (int64_t)c * 2);
        const uint32_t a = (uint32_t)w.x, b = (uint32_t)w.y;
        v[4 * h] = __builtin_bit_cast(float, a << 16);
        v[4 * h + 1] = __builtin_bit_cast(float, a & 0xFFFF0000u);
        v[4 * h + 2] = __builtin_bit_cast(float, b << 16);
        v[4 * h + 3] = __builtin_bit_cast(float, b & 0xFFFF0000u);
      } else {
        f32x4 w = {0.f, 0.f, 0.f, 0.f};
        if (c < d) w = *(const f32x4*)(row + (int64_t)c * 4);
        v[4 * h] = w.x;
        v[4 * h + 1] = w.y;
        v[4 * h + 2] = w.z;
        v[4 * h + 3] = w.w;
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = base + 64 * e + lane;
      v[e] = 0.f;
      if (c < d)
        v[e] = ELT == 2 ? bf16_bits_to_f32(*(const uint16_t*)(row + (int64_t)c * 2))
                        : *(const float*)(row + (int64_t)c * 4);
    }
  }
}

template <int ELT, Cols C>
__device__ inline void store_cols(uint8_t* row, int base, int lane, int d, const float (&v)[8]) {
  if constexpr (C == kCols8) {
    const int c = base + 8 * lane;
    const i32x4 w = {(int)pack_bf16(v[0], v[1]), (int)pack_bf16(v[2], v[3]), (int)pack_bf16(v[4], v[5]),
                     (int)pack_bf16(v[6], v[7])};
    if (c < d) *(i32x4*)(row + (int64_t)c * 2) = w;
  } else if constexpr (C == kCols4) {
    static_assert(ELT == 4, "four columns in a row are written as float32");
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = base + 256 * h + 4 * lane;
      const f32x4 w = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
      if (c < d) *(f32x4*)(row + (int64_t)c * 4) = w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = base + 64 * e + lane;
      if (c < d) {
        if (ELT == 2)
          *(uint16_t*)(row + (int64_t)c * 2) = (uint16_t)pack_bf16(v[e], 0.f);
        else
          *(float*)(row + (int64_t)c * 4) = v[e];
      }
    }
  }
}

__device__ inline int64_t token_at(const void* tokens, int token_bytes, int64_t i) {
  return token_bytes == 8 ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
}

template <int ELT, Cols C>
__global__ __launch_bounds__(256) void embedding_kernel(const uint8_t* __restrict__ table, int64_t ld_table,
                                                        int64_t vocab, int d, const void* __restrict__ tokens,
                                                        int token_bytes, int64_t units, int strips, float scale,
                                                        uint8_t* __restrict__ out, int64_t ld_out) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t u = (int64_t)blockIdx.x * 4 + wave;
  if (u >= units) return;
  const int64_t i = u / strips;
  const int base = (int)(u - i * strips) * kStrip;
  const int64_t t = token_at(tokens, token_bytes, i);
  float v[8] = {};
  if (t >= 0 && t < vocab) {
    load_cols<ELT, C>(table + t * ld_table * ELT, base, lane, d, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= scale;
  }
  store_cols<ELT, C>(out + i * ld_out * ELT, base, lane, d, v);
}

hipError_t launch_embedding(int elt, const void* table, int64_t ld_table, int64_t vocab, int64_t d, const void* tokens,
                            int token_bytes, int64_t n, float scale, void* out, int64_t ld_out, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  const int strips = (int)((d + kStrip - 1) / kStrip);
  const int64_t units = n * strips, blocks = (units + 3) / 4;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  const bool al = (uintptr_t)table % 16 == 0 && (uintptr_t)out % 16 == 0 && (ld_table * elt) % 16 == 0 &&
                  (ld_out * elt) % 16 == 0 && (d * elt) % 16 == 0;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, (const uint8_t*)table, ld_table, vocab, (int)d,
                       tokens, token_bytes, units, strips, scale, (uint8_t*)out, ld_out);
    return hipGetLastError();
  };
  if (elt == 2) return al ? go(embedding_kernel<2, kCols8>) : go(embedding_kernel<2, kCols1>);
  return al ? go(embedding_kernel<4, kCols4>) : go(embedding_kernel<4, kCols1>);
}

// ---------------------------------------------------------------- sorting
// Keys are tokens, with vocab in the place of every token outside the table,
// so those sort to the end.
__device__ inline uint32_t key_at(const void* tokens, int token_bytes, int64_t vocab, int64_t i) {
  const int64_t t = token_at(tokens, token_bytes, i);
  return t >= 0 && t < vocab ? (uint32_t)t : (uint32_t)vocab;
}

struct SortPass {
  const void* tokens;  // first pass: keys from the tokens, positions in order
  int token_bytes;
  int64_t vocab;
  const uint32_t* key_in;
  const int* pos_in;
  uint32_t* key_out;
  int* pos_out;
  uint32_t* hist;  // [digit][workgroup]
  int n, items, blocks, shift, bits;
};
__device__ inline uint32_t pass_key(const SortPass& p, int i) {
  return p.tokens ? key_at(p.tokens, p.token_bytes, p.vocab, i) : p.key_in[i];
}

__global__ __launch_bounds__(256) void sort_count_kernel(SortPass p) {
  __shared__ uint32_t h[kBins];
  const int bins = 1 << p.bits;
  for (int b = threadIdx.x; b < bins; b += 256) h[b] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * p.items, i1 = min((int64_t)p.n, i0 + p.items);
  for (int64_t i = i0 + threadIdx.x; i < i1; i += 256)
    atomicAdd(&h[(pass_key(p, (int)i) >> p.shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += 256) p.hist[(int64_t)b * p.blocks + blockIdx.x] = h[b];
}

// Exclusive scan of the counts in place, digit-major: where each workgroup's
// first position of each digit goes.
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t* hist, int total) {
  __shared__ uint32_t sums[16];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int per = (total + 1023) / 1024, a = min(total, t * per), b = min(total, a + per);
  uint32_t s = 0;
  for (int i = a; i < b; ++i) s += hist[i];
  uint32_t x = s;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  uint32_t run = x - s;
  for (int w = 0; w < wave; ++w) run += sums[w];
  for (int i = a; i < b; ++i) {
    const uint32_t c = hist[i];
    hist[i] = run;
    run += c;
  }
}

// The wave's 64 digits (lanes not in `valid` take no part): how many lower
// lanes have this lane's digit, and how many lanes have it.
__device__ inline void digit_rank(uint32_t digit, int bits, uint64_t valid, int lane, int* rank, int* count) {
  uint64_t peers = valid;
  for (int b = 0; b < bits; ++b) {
    const bool one = (digit >> b) & 1u;
    const uint64_t m = __ballot(one);
    peers &= one ? m : ~m;
  }
  *rank = __popcll(peers & ((1ull << lane) - 1ull));
  *count = __popcll(peers);
}

__global__ __launch_bounds__(256) void sort_scatter_kernel(SortPass p) {
  __shared__ uint32_t off[4][kBins];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << p.bits;
  for (int b = threadIdx.x; b < 4 * kBins; b += 256) off[b / kBins][b % kBins] = 0;
  __syncthreads();
  const int per = p.items / 4;  // a multiple of 64
  const int64_t i0 = (int64_t)blockIdx.x * p.items + (int64_t)wave * per, i1 = min((int64_t)p.n, i0 + per);
  for (int64_t i = i0 + lane; i < i1; i += 64) atomicAdd(&off[wave][(pass_key(p, (int)i) >> p.shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += 256) {
    uint32_t run = p.hist[(int64_t)b * p.blocks + blockIdx.x];
    for (int w = 0; w < 4; ++w) {
      const uint32_t c = off[w][b];
      off[w][b] = run;
      run += c;
    }
  }
  __syncthreads();
  for (int64_t j = i0; j < i1; j += 64) {  // uniform per wave
    const int64_t i = j + lane;
    const bool ok = i < i1;
    const uint32_t key = ok ? pass_key(p, (int)i) : 0u;
    const int pos = !ok ? 0 : p.tokens ? (int)i : p.pos_in[i];
    const uint32_t digit = (key >> p.shift) & (bins - 1);
    int rank, count;
    digit_rank(digit, p.bits, __ballot(ok), lane, &rank, &count);
    const uint32_t to = off[wave][digit] + rank;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (ok && rank == 0) off[wave][digit] += count;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (ok) {
      p.key_out[to] = key;
      p.pos_out[to] = pos;
    }
  }
}

// ------------------------------------------------------------------- sums
template <int ELT, Cols C>
__device__ inline void add_positions(const uint8_t* g, int64_t ld, const int* pos, int a, int b, int base, int lane,
                                     int d, float (&acc)[8]) {
  constexpr int U = 4;  // rows in flight
  int i = a;
  for (; i + U <= b; i += U) {
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) load_cols<ELT, C>(g + (int64_t)pos[i + u] * ld * ELT, base, lane, d, v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += v[u][e];
  }
  for (; i < b; ++i) {
    float v[8];
    load_cols<ELT, C>(g + (int64_t)pos[i] * ld * ELT, base, lane, d, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += v[e];
  }
}

// Sums of the groups of kRun sorted positions that hold one token only.
template <int ELT, Cols C>
__global__ __launch_bounds__(256) void embgrad_groups_kernel(const uint8_t* __restrict__ g, int64_t ld, int d,
                                                             const uint32_t* __restrict__ key,
                                                             const int* __restrict__ pos, int n_groups, uint32_t vocab,
                                                             float* __restrict__ part, int64_t ld_part) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j = blockIdx.x * 4 + wave;
  if (j >= n_groups) return;
  const int a = j * kRun;
  const uint32_t v = key[a];
  if (v >= vocab || key[a + kRun - 1] != v) return;
  const int base = blockIdx.y * kStrip;
  float acc[8] = {};
  add_positions<ELT, C>(g, ld, pos, a, a + kRun, base, lane, d, acc);
  store_cols<4, C>((uint8_t*)(part + (int64_t)j * ld_part), base, lane, d, acc);
}

constexpr int kRowsPerBlock = 16;
// grid (table rows / 16, column groups): each wave owns four rows.
template <int ELT, Cols C>
__global__ __launch_bounds__(256) void embgrad_rows_kernel(const uint8_t* __restrict__ g, int64_t ld, int d,
                                                           const uint32_t* __restrict__ key,
                                                           const int* __restrict__ pos, int n,
                                                           const float* __restrict__ part, int64_t ld_part,
                                                           float scale, int64_t vocab, int strips_each,
                                                           float* __restrict__ out, int64_t ld_out, int accumulate) {
  __shared__ int start[kRowsPerBlock + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t v0 = (int64_t)blockIdx.x * kRowsPerBlock;
  if (threadIdx.x <= kRowsPerBlock) {  // first sorted position with a key >= v
    const uint32_t v = (uint32_t)min(v0 + threadIdx.x, vocab);
    int lo = 0, hi = n;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (key[mid] < v) lo = mid + 1;
      else hi = mid;
    }
    start[threadIdx.x] = lo;
  }
  __syncthreads();
  const int c0 = blockIdx.y * strips_each * kStrip, c1 = min(d, c0 + strips_each * kStrip);
  for (int r = wave; r < kRowsPerBlock; r += 4) {
    const int64_t v = v0 + r;
    if (v >= vocab) break;
    const int a = __builtin_amdgcn_readfirstlane(start[r]), b = __builtin_amdgcn_readfirstlane(start[r + 1]);
    if (accumulate && a == b) continue;
    const int ga = (a + kRun - 1) / kRun, gb = b / kRun;  // whole groups ga .. gb - 1
    for (int base = c0; base < c1; base += kStrip) {
      float acc[8] = {};
      if (ga < gb) {
        add_positions<ELT, C>(g, ld, pos, a, ga * kRun, base, lane, d, acc);
        for (int j = ga; j < gb; ++j) {
          float w[8];
          load_cols<4, C>((const uint8_t*)(part + (int64_t)j * ld_part), base, lane, d, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += w[e];
        }
        add_positions<ELT, C>(g, ld, pos, gb * kRun, b, base, lane, d, acc);
      } else {
        add_positions<ELT, C>(g, ld, pos, a, b, base, lane, d, acc);
      }
      uint8_t* row = (uint8_t*)(out + v * ld_out);
      float old[8] = {};
      if (accumulate) load_cols<4, C>(row, base, lane, d, old);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = fmaf(scale, acc[e], old[e]);
      store_cols<4, C>(row, base, lane, d, acc);
    }
  }
}

namespace {
int key_bits(int64_t vocab) {  // of the largest key, vocab
  int b = 1;
  while ((vocab >> b) != 0) ++b;
  return b;
}
// positions per sorting workgroup: a multiple of kSortItems, at most kSortBlocks workgroups
int64_t sort_items(int64_t n) {
  const int64_t units = (n + kSortItems - 1) / kSortItems;
  return (units + kSortBlocks - 1) / kSortBlocks * kSortItems;
}
int64_t part_ld(int64_t d) { return (d + 3) / 4 * 4; }
}  // namespace

EmbGradLayout embedding_grad_layout(int64_t n, int64_t vocab, int64_t d) {
  EmbGradLayout L;
  size_t off = 0;
  for (int i = 0; i < 2; ++i) {
    L.off_key[i] = off;
    off = align_up(off + (size_t)n * 4);
    L.off_pos[i] = off;
    off = align_up(off + (size_t)n * 4);
  }
  const int64_t items = std::max<int64_t>(sort_items(n), 1), blocks = (n + items - 1) / items;
  L.off_hist = off;
  off = align_up(off + (size_t)blocks * kBins * 4);
  L.off_part = off;
  off = align_up(off + (size_t)(n / kRun) * part_ld(d) * 4);
  L.total = std::max<size_t>(off, kAlign);
  return L;
}

hipError_t launch_embedding_grad(int elt, const void* grad_out, int64_t ld_grad, const void* tokens, int token_bytes,
                                 int64_t n, float scale, int64_t vocab, int64_t d, float* grad_table, int64_t ld_table,
                                 bool accumulate, uint8_t* ws, hipStream_t s) {
  if (vocab <= 0 || (n <= 0 && accumulate)) return hipSuccess;
  const EmbGradLayout L = embedding_grad_layout(n, vocab, d);
  uint32_t* key[2] = {(uint32_t*)(ws + L.off_key[0]), (uint32_t*)(ws + L.off_key[1])};
  int* pos[2] = {(int*)(ws + L.off_pos[0]), (int*)(ws + L.off_pos[1])};
  int cur = 0;
  if (n > 0) {
    const int bits = key_bits(vocab), passes = (bits + kMaxDigit - 1) / kMaxDigit, each = (bits + passes - 1) / passes;
    SortPass p = {};
    p.vocab = vocab;
    p.token_bytes = token_bytes;
    p.hist = (uint32_t*)(ws + L.off_hist);
    p.n = (int)n;
    p.items = (int)sort_items(n);
    p.blocks = (int)((n + p.items - 1) / p.items);
    for (int k = 0; k < passes; ++k) {
      p.tokens = k == 0 ? tokens : nullptr;
      p.key_in = key[cur];
      p.pos_in = pos[cur];
      p.key_out = key[1 - cur];
      p.pos_out = pos[1 - cur];
      p.shift = k * each;
      p.bits = std::min(each, bits - k * each);
      hipLaunchKernelGGL(sort_count_kernel, dim3(p.blocks), dim3(256), 0, s, p);
      hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), 0, s, p.hist, p.blocks << p.bits);
      hipLaunchKernelGGL(sort_scatter_kernel, dim3(p.blocks), dim3(256), 0, s, p);
      cur = 1 - cur;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int strips = (int)((d + kStrip - 1) / kStrip);
  const int64_t ldp = part_ld(d), n_groups = n / kRun;
  const bool al = (uintptr_t)grad_out % (4 * elt) == 0 && ld_grad % 4 == 0 && (uintptr_t)grad_table % 16 == 0 &&
                  ld_table % 4 == 0 && d % 4 == 0;
  float* part = (float*)(ws + L.off_part);
  const int64_t blocks = (vocab + kRowsPerBlock - 1) / kRowsPerBlock;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  auto go = [&](auto groups_kernel, auto rows_kernel) {
    if (n_groups > 0)
      hipLaunchKernelGGL(groups_kernel, dim3((unsigned)((n_groups + 3) / 4), strips), dim3(256), 0, s,
                         (const uint8_t*)grad_out, ld_grad, (int)d, key[cur], pos[cur], (int)n_groups, (uint32_t)vocab,
                         part, ldp);
    const int strips_each = 4, groups = (strips + strips_each - 1) / strips_each;
    hipLaunchKernelGGL(rows_kernel, dim3((unsigned)blocks, groups), dim3(256), 0, s, (const uint8_t*)grad_out, ld_grad,
                       (int)d, key[cur], pos[cur], (int)n, part, ldp, scale, vocab, strips_each, grad_table, ld_table,
                       (int)accumulate);
    return hipGetLastError();
  };
  if (elt == 2)
    return al ? go(embgrad_groups_kernel<2, kCols4>, embgrad_rows_kernel<2, kCols4>)
              : go(embgrad_groups_kernel<2, kCols1>, embgrad_rows_kernel<2, kCols1>);
  return al ? go(embgrad_groups_kernel<4, kCols4>, embgrad_rows_kernel<4, kCols4>)
            : go(embgrad_groups_kernel<4, kCols1>, embgrad_rows_kernel<4, kCols1>);
}

}  // namespace dattri
