// Embedding lookup and its table gradient.
//
// Lookup: out[i] = scale * table[tokens[i]].  One wave per (row, strip of 512
// columns), 16-byte loads and stores where rows are on 16 bytes.
//
// Gradient: grad_table[v] = scale * sum over positions i with tokens[i] = v of
// grad_out[i].  The positions are sorted by token with a stable radix sort
// (digits of at most 9 bits; ranks within a wave by ballots: no float and no
// order depends on timing), so the positions of a row form a run in ascending
// order.  A run is summed as the positions up to the next multiple of kRun,
// whole groups of kRun positions whose sums another kernel has formed (so a
// token that is most of the batch does not wait on one wave), and the positions
// left; the order is that of the positions in fixed groups, whatever the launch.
// A whole table is zeroed first, by workgroups that ride in the launch of the
// sort's first kernel: the sort is a few waves' latency, the zeros are bandwidth.
//
// What bounds it: the lookup and the sums read and write each row once; for a
// whole table the zeros of rows without tokens are most of the bytes.  16384
// tokens, 128000 x 4096 bf16: lookup 32 us by itself, 45 with its operands out of
// the caches; gradient: sort and 2.1 GB of zeros in one launch 338 us (6.2 TB/s),
// groups 18, rows 74.
#include <algorithm>

#include "api_common.h"
#include "device_common.h"
#include "model_ops.h"

namespace dattri {
using namespace dev;

constexpr int kStrip = 512;       // lookup: columns per wave, 8 per lane
constexpr int kRun = 32;          // positions per group of a long run
constexpr int kMaxDigit = 9;      // bits per sorting pass
constexpr int kBins = 1 << kMaxDigit;
constexpr int kSortItems = 4096;  // least positions per sorting workgroup
constexpr int kSortBlocks = 2048; // most sorting workgroups

// The E columns a lane owns of a strip of 64 E: 8 in a row (16 bytes of bf16),
// runs of 4 (16 bytes of float32, or 8 of bf16 against 16 of a float32 output),
// or one in every 64 (rows not on 16 bytes).
enum Cols { kCols8, kCols4, kCols1 };
// float32 values of a lane's columns; columns >= d read as zero (d is a
// multiple of 8 for kCols8, of 4 for kCols4).
template <int ELT, Cols C, int E>
__device__ inline void load_cols(const uint8_t* row, int base, int lane, int d, float (&v)[E]) {
  if constexpr (C == kCols8) {
    static_assert(E == 8, "one run of 8");
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
    for (int h = 0; h < E / 4; ++h) {
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
    for (int e = 0; e < E; ++e) {
      const int c = base + 64 * e + lane;
      v[e] = 0.f;
      if (c < d)
        v[e] = ELT == 2 ? bf16_bits_to_f32(*(const uint16_t*)(row + (int64_t)c * 2))
                        : *(const float*)(row + (int64_t)c * 4);
    }
  }
}

template <int ELT, Cols C, int E>
__device__ inline void store_cols(uint8_t* row, int base, int lane, int d, const float (&v)[E]) {
  if constexpr (C == kCols8) {
    const int c = base + 8 * lane;
    const i32x4 w = {(int)pack_bf16(v[0], v[1]), (int)pack_bf16(v[2], v[3]), (int)pack_bf16(v[4], v[5]),
                     (int)pack_bf16(v[6], v[7])};
    if (c < d) *(i32x4*)(row + (int64_t)c * 2) = w;
  } else if constexpr (C == kCols4) {
    static_assert(ELT == 4, "four columns in a row are written as float32");
#pragma unroll
    for (int h = 0; h < E / 4; ++h) {
      const int c = base + 256 * h + 4 * lane;
      const f32x4 w = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
      if (c < d) *(f32x4*)(row + (int64_t)c * 4) = w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
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
  const int64_t u = row_block() * 4 + wave;
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
  const int64_t units = n * strips;
  dim3 grid;
  const hipError_t e = row_grid((units + 3) / 4, &grid);
  if (e != hipSuccess) return e;
  const bool al = (uintptr_t)table % 16 == 0 && (uintptr_t)out % 16 == 0 && (ld_table * elt) % 16 == 0 &&
                  (ld_out * elt) % 16 == 0 && (d * elt) % 16 == 0;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (const uint8_t*)table, ld_table, vocab, (int)d,
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

// The table to be zeroed (out null: none).
struct Fill {
  float* out;
  int64_t ld, rows;
  int d;
};
// Share `b` of `nb` of it, by T threads, in pieces of 8 T stores (2 GiB in 331
// us by 1020 workgroups of 1024; store by store around the chip 403: memory
// takes neighbouring lines better together).
template <int T>
__device__ inline void fill_zero(const Fill& f, int64_t b, int64_t nb) {
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const int t = threadIdx.x;
  if (f.ld == f.d) {  // one block of memory
    const int64_t total = f.rows * f.d, head = min(total, (int64_t)(((16 - (uintptr_t)f.out % 16) % 16) / 4));
    const int64_t n4 = (total - head) / 4, tail = total - head - 4 * n4;
    f32x4* p = (f32x4*)(f.out + head);
    for (int64_t c = b; c * (8 * T) < n4; c += nb)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int64_t i = (c * 8 + u) * T + t;
        if (i < n4) p[i] = zero;
      }
    if (b == 0 && t < head) f.out[t] = 0.f;
    if (b == 0 && t < tail) f.out[head + 4 * n4 + t] = 0.f;
    return;
  }
  for (int64_t r = b * (T / 64) + t / 64; r < f.rows; r += nb * (T / 64))
    for (int c = t % 64; c < f.d; c += 64) f.out[r * f.ld + c] = 0.f;
}

// Zeros alone: no token points anywhere, so there is nothing to sort.
__global__ __launch_bounds__(1024) void zero_table_kernel(Fill f) { fill_zero<1024>(f, blockIdx.x, gridDim.x); }

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

__global__ __launch_bounds__(256) void sort_count_kernel(SortPass p, Fill f) {
  __shared__ uint32_t h[kBins];
  if ((int)blockIdx.x >= p.blocks) return fill_zero<256>(f, blockIdx.x - p.blocks, gridDim.x - p.blocks);
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

// The whole sort in one workgroup: up to kSmallSort positions, each packed with
// its key into 32 bits.  Wave w holds positions w * per .. + per - 1, 64 at a
// time; a pass counts and ranks them per wave, scans the counts digit by digit
// and moves the items through LDS.  509 positions take 10 us with their table's
// zeros (30 MB), the six launches of the passes above 29.
constexpr int kSmallSort = 16384, kPosBits = 14, kSmallRounds = kSmallSort / 1024;
__global__ __launch_bounds__(1024) void sort_small_kernel(const void* __restrict__ tokens, int token_bytes,
                                                          int64_t vocab, int n, int passes, int bits,
                                                          uint32_t* __restrict__ key_out, int* __restrict__ pos_out,
                                                          Fill f) {
  __shared__ uint32_t items[kSmallSort];
  __shared__ uint32_t off[16][kBins];
  __shared__ uint32_t sums[16];
  if (blockIdx.x > 0) return fill_zero<1024>(f, blockIdx.x - 1, gridDim.x - 1);
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, bins = 1 << bits;
  const int rounds = (n + 1023) / 1024, first = wave * rounds * 64 + lane;
  uint32_t v[kSmallRounds];
  int rank[kSmallRounds];
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r)
    if (r < rounds) {
      const int i = first + r * 64;
      v[r] = i < n ? key_at(tokens, token_bytes, vocab, i) << kPosBits | (uint32_t)i : 0u;
    }
  for (int p = 0; p < passes; ++p) {
    const int shift = kPosBits + p * bits;
    for (int b = t; b < 16 * kBins; b += 1024) off[b / kBins][b % kBins] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r)
      if (r < rounds) {
        const bool ok = first + r * 64 < n;
        const uint32_t digit = (v[r] >> shift) & (bins - 1);
        int below, count;
        digit_rank(digit, bits, __ballot(ok), lane, &below, &count);
        const uint32_t base = off[wave][digit];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (ok && below == 0) off[wave][digit] = base + count;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        rank[r] = (int)base + below;
      }
    __syncthreads();
    // exclusive scan of the counts, digit by digit and wave by wave: thread t has waves 8 (t % 2) .. + 7 of digit t / 2
    uint32_t c[8], s = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      c[w] = off[8 * (t & 1) + w][t >> 1];
      s += c[w];
    }
    uint32_t x = s;
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    uint32_t run = x - s;
    for (int w = 0; w < wave; ++w) run += sums[w];
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      off[8 * (t & 1) + w][t >> 1] = run;
      run += c[w];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r)
      if (r < rounds && first + r * 64 < n) items[off[wave][(v[r] >> shift) & (bins - 1)] + rank[r]] = v[r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r)
      if (r < rounds && first + r * 64 < n) v[r] = items[first + r * 64];
  }
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r)
    if (r < rounds && first + r * 64 < n) {
      key_out[first + r * 64] = v[r] >> kPosBits;
      pos_out[first + r * 64] = (int)(v[r] & ((1u << kPosBits) - 1u));
    }
}

// ------------------------------------------------------------------- sums
// acc += rows row(a) .. row(b - 1), in order, F of them loaded before they are added.
template <int ELT, Cols C, int F, int E, class Row>
__device__ inline void add_rows(Row row, int a, int b, int base, int lane, int d, float (&acc)[E]) {
  for (int i = a; i < b; i += F) {
    float v[F][E];
#pragma unroll
    for (int u = 0; u < F; ++u) {
      if (i + u < b) {  // uniform
        load_cols<ELT, C>(row(i + u), base, lane, d, v[u]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[u][e] = 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < F; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += v[u][e];
  }
}

// Sums of the groups of kRun sorted positions that hold one token only: all
// rows of a group in flight at once, 256 columns per wave.
template <int ELT, Cols C>
__global__ __launch_bounds__(256) void embgrad_groups_kernel(const uint8_t* __restrict__ g, int64_t ld, int d,
                                                             const uint32_t* __restrict__ key,
                                                             const int* __restrict__ pos, int n_groups, uint32_t vocab,
                                                             float* __restrict__ part, int64_t ld_part, int strips) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = row_block() * 4 + wave, group = unit / strips;
  if (group >= n_groups) return;
  const int j = (int)group, base = (int)(unit - group * strips) * 256, a = j * kRun;
  const int at = pos[a + (lane & (kRun - 1))];
  const uint32_t v = key[a];
  if (v >= vocab || key[a + kRun - 1] != v) return;
  float acc[4] = {};
  add_rows<ELT, C, kRun>([&](int i) { return g + (int64_t)__builtin_amdgcn_readlane(at, i) * ld * ELT; }, 0, kRun, base,
                         lane, d, acc);
  store_cols<4, C>((uint8_t*)(part + (int64_t)j * ld_part), base, lane, d, acc);
}

// One wave per (sorted position, strip of 64 E columns), a row's strips next to
// each other (strips of all rows one after the other took 117 us where this
// takes 84: memory takes a whole row better at once).  The waves at the start
// of a run sum it.
template <int ELT, Cols C, int E>
__global__ __launch_bounds__(256) void embgrad_rows_kernel(const uint8_t* __restrict__ g, int64_t ld, int d,
                                                           const uint32_t* __restrict__ key,
                                                           const int* __restrict__ pos, int n,
                                                           const float* __restrict__ part, int64_t ld_part,
                                                           float scale, uint32_t vocab, float* __restrict__ out,
                                                           int64_t ld_out, int accumulate, int strips) {
  constexpr int F = 64 / E;  // rows in flight
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = row_block() * 4 + wave, first = unit / strips;
  const int base = (int)(unit - first * strips) * (64 * E);
  if (first >= n) return;
  const int a = (int)first;
  // keys and positions of the next 64 places, asked for before the first key is known
  const int64_t mine = min(first + lane, (int64_t)n - 1);
  const uint32_t next = key[mine];
  const int at = pos[mine];
  const uint32_t before = a > 0 ? key[a - 1] : vocab;
  const uint32_t v = __builtin_amdgcn_readfirstlane(next);
  if (v >= vocab || before == v) return;
  const uint64_t other = __ballot(first + lane >= n || next != v);
  int b;
  if (other) {
    b = a + __builtin_ctzll(other);
  } else {  // a longer run: its end by bisection
    int lo = a + 64, hi = n;
    while (lo < hi) {
      const int mid = lo + ((hi - lo) >> 1);
      if (key[mid] == v) lo = mid + 1;
      else hi = mid;
    }
    b = lo;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  auto near = [&](int i) { return g + (int64_t)__builtin_amdgcn_readlane(at, i - a) * ld * ELT; };
  auto far = [&](int i) { return g + (int64_t)pos[i] * ld * ELT; };
  const int ga = a / kRun + (a % kRun != 0), gb = b / kRun;  // whole groups ga .. gb - 1
  float acc[E] = {};
  if (ga < gb) {
    add_rows<ELT, C, F>(near, a, ga * kRun, base, lane, d, acc);
    add_rows<4, C, F>([&](int j) { return (const uint8_t*)(part + (int64_t)j * ld_part); }, ga, gb, base, lane, d, acc);
    add_rows<ELT, C, F>(far, gb * kRun, b, base, lane, d, acc);
  } else {
    add_rows<ELT, C, F>(near, a, b, base, lane, d, acc);
  }
  uint8_t* to = (uint8_t*)(out + (int64_t)v * ld_out);
  float old[E] = {};
  if (accumulate) load_cols<4, C>(to, base, lane, d, old);
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = fmaf(scale, acc[e], old[e]);
  store_cols<4, C>(to, base, lane, d, acc);
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
  const Fill f = {accumulate ? nullptr : grad_table, ld_table, vocab, (int)d};
  // workgroups that zero the table: 64 KiB each at least, four rounds of the chip at most
  const int64_t share = (vocab * d * 4 + 65535) / 65536;
  auto fills = [&](int64_t most) { return accumulate ? 0u : (unsigned)std::min(share, most); };
  if (n <= 0) {
    hipLaunchKernelGGL(zero_table_kernel, dim3(fills(1024)), dim3(1024), 0, s, f);
    return hipGetLastError();
  }
  const int bits = key_bits(vocab);
  if (n <= kSmallSort && bits + kPosBits <= 32) {
    const int passes = (bits + kMaxDigit - 1) / kMaxDigit;
    hipLaunchKernelGGL(sort_small_kernel, dim3(1 + fills(1023)), dim3(1024), 0, s, tokens, token_bytes, vocab, (int)n,
                       passes, (bits + passes - 1) / passes, key[0], pos[0], f);
  } else {
    const int passes = (bits + kMaxDigit - 1) / kMaxDigit, each = (bits + passes - 1) / passes;
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
      hipLaunchKernelGGL(sort_count_kernel, dim3(p.blocks + (k == 0 ? fills(4096) : 0u)), dim3(256), 0, s, p, f);
      hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), 0, s, p.hist, p.blocks << p.bits);
      hipLaunchKernelGGL(sort_scatter_kernel, dim3(p.blocks), dim3(256), 0, s, p);
      cur = 1 - cur;
    }
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t ldp = part_ld(d), n_groups = n / kRun;
  const bool al = (uintptr_t)grad_out % (4 * elt) == 0 && ld_grad % 4 == 0 && (uintptr_t)grad_table % 16 == 0 &&
                  ld_table % 4 == 0 && d % 4 == 0;
  float* part = (float*)(ws + L.off_part);
  // 16 columns per lane while that leaves the chip 32 waves per CU (16384
  // positions x 4096 columns: 74 us, 8 columns 84, 4 93), else 4 (509 x 769: 6 us, 16 11)
  const bool wide = n * ((d + 1023) / 1024) >= 8192;
  auto go = [&](auto groups_kernel, auto wide_kernel, auto narrow_kernel) {
    const int row_cols = wide ? 16 : 4;
    const int64_t gs = (d + 255) / 256, rs = (d + 64 * row_cols - 1) / (64 * row_cols);
    dim3 gb, rb;
    hipError_t e = row_grid((n * rs + 3) / 4, &rb);
    if (e == hipSuccess && n_groups > 0) e = row_grid((n_groups * gs + 3) / 4, &gb);
    if (e != hipSuccess) return e;
    if (n_groups > 0)
      hipLaunchKernelGGL(groups_kernel, gb, dim3(256), 0, s, (const uint8_t*)grad_out, ld_grad, (int)d,
                         key[cur], pos[cur], (int)n_groups, (uint32_t)vocab, part, ldp, (int)gs);
    hipLaunchKernelGGL(wide ? wide_kernel : narrow_kernel, rb, dim3(256), 0, s, (const uint8_t*)grad_out, ld_grad,
                       (int)d, key[cur], pos[cur], (int)n, part, ldp, scale, (uint32_t)vocab, grad_table, ld_table,
                       (int)accumulate, (int)rs);
    return hipGetLastError();
  };
  if (elt == 2)
    return al ? go(embgrad_groups_kernel<2, kCols4>, embgrad_rows_kernel<2, kCols4, 16>,
                    embgrad_rows_kernel<2, kCols4, 4>)
              : go(embgrad_groups_kernel<2, kCols1>, embgrad_rows_kernel<2, kCols1, 16>,
                    embgrad_rows_kernel<2, kCols1, 4>);
  return al ? go(embgrad_groups_kernel<4, kCols4>, embgrad_rows_kernel<4, kCols4, 16>,
                    embgrad_rows_kernel<4, kCols4, 4>)
            : go(embgrad_groups_kernel<4, kCols1>, embgrad_rows_kernel<4, kCols1, 16>,
                    embgrad_rows_kernel<4, kCols1, 4>);
}

}  // namespace dattri
