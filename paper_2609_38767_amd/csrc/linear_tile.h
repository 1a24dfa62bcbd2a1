// The tile of a product of the linear layers, with its epilogue:
//   C[m][n] = sum_k A(m, k) B(n, k), then TileEpilogue.
//
// Four waves (one per SIMD) each own BN x BM blocks of 32 x 32
// outputs; the blocks' rows run along n and their columns along m, so a lane
// holds four neighbouring n of one m.  bf16 products are
// v_mfma_f32_32x32x16_bf16, float32 ones v_mfma_f32_32x32x2f32.  Operands come
// to LDS by direct loads (16 bytes per lane) in stages of KW bytes of k, in the
// order they have in memory:
//   k contiguous: [row][KW bytes], 16-byte chunks XORed by row; a fragment is
//     one 16-byte read per lane: 8 bf16, or 4 float32 that serve four MFMA
//     (slot j of half-wave h is k = 4h + j for both operands);
//   k strided: [k][row], read across with the transposing LDS read (bf16) or
//     by 4-byte reads of 32 neighbouring rows (float32); chunks XORed by k.
// Every read then meets each bank once.
//
// A ring of 256 / KW stage buffers, 32 bytes of k per K step.  Fragments are
// read one step ahead; the one barrier of a stage sits before its last step,
// where the stage is in registers: its buffer then takes the loads of the stage
// a ring further on, half of them in that step and half in the next, dealt out
// evenly (the wait counts: with four buffers the loads of two stages may still be
// under way).  Four buffers of 64 bytes give a load four to six steps to arrive.
// Where both operands of a 256 x 256 bf16 tile have k contiguous, 64 bytes are
// half a cache line and double the requests to L2 (8192 x 4096 -> 14336: 827 us);
// there two buffers of 128 bytes, two to four steps for a load, take 739.
//
// Rows past M or N and k past K read as zero, so no product meets what lies
// behind a row.
//
// The accumulators leave through LDS, 32 columns of blocks at a time as float32
// rows, so that the epilogue is one short loop over whole rows: its loads and
// stores of Z, R and the outputs are contiguous per wave.
#pragma once

#include <algorithm>
#include <type_traits>
#include <utility>

#include "device_common.h"
#include "epilogue.h"
#include "internal.h"
#include "linear_shape.h"
#include "model_ops.h"

namespace dattri {
namespace tile {
using namespace dev;

constexpr int kPartial = 3;  // epilogue of a split product: float32 partial tile

typedef short i16x4 __attribute__((ext_vector_type(4)));

__device__ inline void wait_all() {  // this wave's loads are in LDS, its LDS reads done
  __builtin_amdgcn_s_waitcnt(0x70);  // vmcnt 0, lgkmcnt 0, other counters untouched
}
__device__ inline void plain_barrier() { asm volatile("s_barrier" ::: "memory"); }
__device__ inline void stage_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Fragment halves that an LDS read written out below puts in place behind the
// compiler's back: only touched after landed() has waited for them.
struct Raw {
  i16x4 lo, hi;
};
// Transposing LDS read: lane 4r + c of every 16 addresses four bf16 of k row r,
// lane j receives the four k of column j.  Written out because the compiler,
// which cannot tell what bytes the builtin reads, waits for every direct load
// in flight (vmcnt 0) before it: 654 TFLOP/s where this reaches 1300.
template <int OFF>
__device__ inline i16x4 read_across(uint32_t lds) {
  i16x4 v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(lds), "i"(OFF));
  return v;
}
// All LDS reads of this wave are done; the fragments may be used.
__device__ inline void landed(Raw (&f)[4]) {
  asm volatile("s_waitcnt lgkmcnt(0)"
               : "+v"(f[0].lo), "+v"(f[0].hi), "+v"(f[1].lo), "+v"(f[1].hi), "+v"(f[2].lo), "+v"(f[2].hi),
                 "+v"(f[3].lo), "+v"(f[3].hi));
}
__device__ inline void landed(Raw (&f)[2]) {
  asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0].lo), "+v"(f[0].hi), "+v"(f[1].lo), "+v"(f[1].hi));
}
__device__ inline void landed(Raw (&f)[1]) {
  asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0].lo), "+v"(f[0].hi));
}
template <int N>
__device__ inline void landed(i32x4 (&)[N]) {}  // the compiler waits by itself
__device__ inline i32x4 operand(i32x4 f) { return f; }
__device__ inline i32x4 operand(const Raw& f) {
  const i32x2 x = __builtin_bit_cast(i32x2, f.lo), y = __builtin_bit_cast(i32x2, f.hi);
  return i32x4{x.x, x.y, y.x, y.y};
}

// The main loop's pieces keep accumulators and fragments in registers only if
// every one of them is inlined, whatever its size.
#define DATTRI_INLINE __attribute__((always_inline))

// f(0), ..., f(N - 1) with constants for arguments
template <class F, int... I>
__device__ DATTRI_INLINE inline void unrolled(F& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ DATTRI_INLINE inline void unrolled(F f) {
  unrolled(f, std::make_integer_sequence<int, N>{});
}

// One operand's share of a tile: R rows (of the operand's own index) of which
// `rows` exist, k contiguous (KC) or strided; KW bytes of k per stage, loaded by
// WAVES waves.
template <int ELT, bool KC, int R, int KW, int WAVES = 4>
struct Side {
  static constexpr int EPL = 16 / ELT, BK = KW / ELT;    // elements per chunk, k per stage
  static constexpr int kBytes = R * KW;                  // of a stage
  static constexpr int kPieces = kBytes / 1024;          // direct loads of 1 KiB
  static constexpr int kLoads = kPieces > WAVES ? kPieces / WAVES : 1;  // per wave; two pieces: each loaded by two waves
  static constexpr int CH = R * ELT / 16;                // chunks per k row (strided)

  // A direct load moves 64 chunks: kRows rows of a stage buffer (of the operand
  // or of k).  The chunks of row r are XORed by swz(r), which differs between
  // even and odd loads at most.
  static constexpr int kPer = KC ? KW / 16 : CH, kRows = 64 / kPer;  // chunks per row

  const uint8_t* base;  // the tile's first row (KC) or column (strided) at k = 0
  uint32_t ld;          // bytes
  int rows, K;
  uint32_t off[2];  // this lane's chunk of an even and an odd load, from the load's first row
  int kc[2];        // KC: its k within the stage

  __device__ static int swz(int r) {
    if constexpr (KC) return KW == 128 ? (r >> 1) & 7 : (r >> 2) & 3;
    return (ELT == 2 ? 2 * (r & 3) + 8 * (r & 1) : 8 * ((r >> 2) & 1)) & (CH - 1);
  }

  __device__ void init(const void* p, int64_t ld_elts, int row0, int n_rows, int K_, int wave, int lane) {
    ld = (uint32_t)(ld_elts * ELT);
    rows = min(R, n_rows - row0);
    K = K_;
    base = (const uint8_t*)p + (KC ? (int64_t)row0 * ld : (int64_t)row0 * ELT);
    const int r = lane / kPer, c = lane % kPer;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int x = c ^ swz((wave * kLoads + v) * kRows + r);
      off[v] = r * ld + (x << 4);
      kc[v] = x * EPL;
    }
  }

  // What stage st may read: from its first k to the last row's end (rows are
  // whole 16-byte chunks, repacked ones end in zeros); past the last k nothing.
  // Fits 32 bits: 256 rows stay below 4 GiB, st * BK is past K by a few stages at most.
  __device__ rsrc_t range(int st) const {
    const int left = (int)((uint32_t)K - (uint32_t)st * BK);
    if constexpr (KC) {
      const uint32_t bytes = (uint32_t)(rows - 1) * ld + ((uint32_t)left * ELT + 15) / 16 * 16;
      return make_rsrc(base + (int64_t)st * KW, left > 0 ? bytes : 0);
    } else {
      const uint32_t bytes = (uint32_t)(min(left, BK) - 1) * ld + ((uint32_t)rows * ELT + 15) / 16 * 16;
      return make_rsrc(base + (int64_t)st * BK * ld, left > 0 ? bytes : 0);
    }
  }
  // Direct load j of stage st (r: its range) into `buf`, this side's part of a
  // stage buffer.  Rows past the last (KC) and k past K read as zero; KC, where
  // the next row lies behind K: by an offset out of range.
  __device__ void load(rsrc_t r, int st, uint8_t* buf, int wave, int j) const {
    const int at = (wave * kLoads + j) % kPieces;
    uint32_t o = off[j & 1] + (uint32_t)(at * kRows) * ld;
    if (KC && kc[j & 1] >= (int)((uint32_t)K - (uint32_t)st * BK)) o = kOOB;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, DATTRI_LDS_PTR(buf + at * 1024), 16, o, 0, 0, 0);
  }

  typedef std::conditional_t<!KC && ELT == 2, Raw, i32x4> Frag;

  // Fragment of K step s of the 32-row block at row w0 + 32 i: lane l holds row
  // l % 32 and the step's k of half-wave l / 32.
  template <int S>
  __device__ static Frag read(const uint8_t* buf, int w0, int lane, int i) {
    const int l32 = lane & 31, h = lane >> 5;
    if constexpr (KC) {
      return *(const i32x4*)(buf + (w0 + l32) * KW + (((2 * S + h) ^ swz(l32)) << 4) + i * 32 * KW);
    } else if constexpr (ELT == 2) {
      const int q = lane >> 4, rr = (lane >> 2) & 3, aa = lane & 3;
      const int c = (w0 >> 3) + 4 * i + 2 * (q & 1) + (aa >> 1);
      const uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)buf +
                          (8 * (q >> 1) + rr) * (CH * 16) + (aa & 1) * 8 + ((c ^ swz(rr)) << 4);
      return Raw{read_across<16 * S * CH * 16>(at), read_across<(16 * S + 4) * CH * 16>(at)};
    } else {
      const int c = (w0 >> 2) + 8 * i + (l32 >> 2);
      const uint8_t* a = buf + (8 * S + 4 * h) * (CH * 16) + (l32 & 3) * 4 + ((c ^ swz(4 * h)) << 4);
      return i32x4{*(const int*)a, *(const int*)(a + CH * 16), *(const int*)(a + 2 * CH * 16),
                   *(const int*)(a + 3 * CH * 16)};
    }
  }
};

template <int ELT>
__device__ inline f32x16 block_mma(i32x4 b, i32x4 a, f32x16 c) {
  if constexpr (ELT == 2)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0,
                                                   0);
  const f32x4 fb = __builtin_bit_cast(f32x4, b), fa = __builtin_bit_cast(f32x4, a);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(fb[e], fa[e], c, 0, 0, 0);
  return c;
}

// Tile (mt, nt) of launch index b: every XCD takes a contiguous run of tiles,
// groups of kGroup tile rows walked along n, so the tiles an XCD works on at
// once share their operands in its L2.
constexpr int kGroup = 8;
__device__ inline void tile_of(int b, int nm, int nn, int* mt, int* nt) {
  const int nb = nm * nn, n_full = nb / kXcds * kXcds;
  const int L = b < n_full ? (b % kXcds) * (n_full / kXcds) + b / kXcds : b;
  const int g = L / (kGroup * nn), m_first = g * kGroup, gm = min(kGroup, nm - m_first);
  const int r = L - g * kGroup * nn;
  *mt = m_first + r % gm;
  *nt = r / gm;
}

// The end of a tile from row m0 and column n0: the waves' sums through LDS to the
// epilogue (OP kPartial: float32 sums to part, rows ld_part apart).  slab(j, wm):
// 32 rows of TN float32 for block column j of a row of waves; j and j + 1 may not
// share any, j and j + 2 may.
template <int OP, int ELT, int WM, int WN, int BM, int BN, class Slab>
__device__ DATTRI_INLINE inline void finish_tile(const GemmArgs& a, const f32x16 (&acc)[BN][BM], int m0, int n0,
                                                 float* __restrict__ part, int64_t ld_part, Slab slab) {
  constexpr int TM = WM * BM * 32, TN = WN * BN * 32, kThreads = WM * WN * 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  // Block column j of every wave as rows of TN float32, 16-byte chunks XORed by
  // row so that the lanes' writes (32 rows of one chunk) spread over the banks.
  const int l32 = lane & 31, h = lane >> 5;
  constexpr int LPR = TN / 4;  // lanes per row in the epilogue
  constexpr int kRows = 4;     // rows a thread takes at once (a slab holds whole rounds of them)
  static_assert(WM * 32 % (kThreads / LPR * kRows) == 0, "slab rows");
  const int c = tid % LPR;
#pragma unroll
  for (int j = 0; j < BM; ++j) {
    uint8_t *const y0 = slab(j, 0), *const y1 = slab(j, 1);  // of the rows of waves
    if (j == 0) stage_barrier();  // the last stage's reads are done; the buffers of j - 2 are by the barrier below
#pragma unroll
    for (int i = 0; i < BN; ++i)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int c = (wn * BN + i) * 8 + 2 * v + h;
        *(f32x4*)((wm ? y1 : y0) + l32 * (TN * 4) + ((c ^ (l32 & 15)) << 4)) =
            f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]};
      }
    stage_barrier();
    // row r of the slab is row (r / 32) * 32 BM + 32 j + r % 32 of the tile
    auto tile_row = [&](int row) { return (row >> 5) * (BM * 32) + 32 * j + (row & 31); };
    auto value = [&](int row) {
      return *(const f32x4*)((row & 32 ? y1 : y0) + (row & 31) * (TN * 4) + ((c ^ (row & 15)) << 4));
    };
    if constexpr (OP == kPartial) {
      const TileRows<4> out(part, ld_part, m0, n0, min(TM, a.M - m0),
                            min((int64_t)TN, ld_part - n0));
      if (n0 + 4 * c < ld_part)
#pragma unroll 4
        for (int row = tid / LPR; row < WM * 32; row += kThreads / LPR)
          buffer_store4<4, 1>(out.r, tile_row(row) * out.ld + 16 * c, value(row), 4);
    } else {
      const int rows = min(TM, a.M - m0), width = min(TN, a.N - n0);
      auto finish = [&](auto take, const auto& e, auto get) {  // `take` rows at once
        constexpr int U = decltype(take)::value;
#pragma unroll 1
        for (int row = tid / LPR; row < WM * 32; row += kThreads / LPR * U) {
          int at[U];
          f32x4 v[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            at[u] = tile_row(row + u * (kThreads / LPR));
            v[u] = get(row + u * (kThreads / LPR));
          }
          e.run(at, v);
        }
      };
      if (a.vec && width % 4 == 0) {  // four neighbours per lane
        if (4 * c < width)
          finish(std::integral_constant<int, kRows>{}, TileEpilogue<OP, ELT, kRows, 1>(a, m0, n0, rows, width, 4 * c), value);
      } else {  // rows on any element: every LPR-th column, so that lanes are neighbours
        auto apart = [&](int row) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int n = c + e * LPR;
            v[e] = *(const float*)((row & 32 ? y1 : y0) + (row & 31) * (TN * 4) + (((n >> 2) ^ (row & 15)) << 4) +
                                   (n & 3) * 4);
          }
          return v;
        };
        if (c < width)
          finish(std::integral_constant<int, 2>{}, TileEpilogue<OP, ELT, 2, LPR>(a, m0, n0, rows, width, c), apart);
      }
    }
  }
}

// The LDS of a tile: kBuffers arrays of kBytes.
template <bool AC, bool BC, int ELT, int KW, int WM, int WN, int BM, int BN>
struct TileBuffers {
  static constexpr int TM = WM * BM * 32, TN = WN * BN * 32, kBuffers = buffers_of(KW);
  static constexpr int kStage = Side<ELT, AC, TM, KW>::kBytes + Side<ELT, BC, TN, KW>::kBytes;
  static constexpr int kSlab = 32 * TN * 4;  // epilogue: one block column of a row of waves, four of them
  static constexpr int kBytes = std::max(kStage, kSlab * 4 / kBuffers);
};
#define DATTRI_TILE_BUFFERS(B)                                                                        \
  __shared__ __align__(1024) uint8_t x0[B::kBytes], x1[B::kBytes], x2[B::kBuffers == 4 ? B::kBytes : 16], \
      x3[B::kBuffers == 4 ? B::kBytes : 16]

// The tile from row m0 and column n0, rows and columns below a.M and a.N: stages
// s0 .. s0 + ns - 1 of k, up to k_end.  WM x WN waves; BM x BN blocks of 32 x 32
// each.  OP kPartial: float32 sums to part, rows ld_part apart.  x0 .. x3: arrays
// of TileBuffers, or larger ones (different arrays, so that the compiler can tell
// a read of one from the loads into another).
template <int OP, bool AC, bool BC, int ELT, int KW, int WM, int WN, int BM, int BN>
__device__ DATTRI_INLINE inline void tile_product(const GemmArgs& a, int m0, int n0, int s0, int ns, int k_end,
                                                  float* __restrict__ part, int64_t ld_part, uint8_t* x0, uint8_t* x1,
                                                  uint8_t* x2, uint8_t* x3) {
  static_assert(WM * WN == 4 && WM <= 2, "four waves");
  constexpr int TM = WM * BM * 32, TN = WN * BN * 32;
  typedef Side<ELT, AC, TM, KW> SA;
  typedef Side<ELT, BC, TN, KW> SB;
  constexpr int kBuffers = buffers_of(KW), kSteps = KW / 32, kSlab = 32 * TN * 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  SA sa;
  SB sb;
  sa.init(a.A, a.lda, m0, a.M, k_end, wave, lane);
  sb.init(a.B, a.ldb, n0, a.N, k_end, wave, lane);

  f32x16 acc[BN][BM];
#pragma unroll
  for (int i = 0; i < BN; ++i)
#pragma unroll
    for (int j = 0; j < BM; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  typename SB::Frag fb[2][BN];  // fragments of even and odd K steps
  typename SA::Frag fa[2][BM];
  // fragment J of K step S, A's first
  auto read = [&](auto S, auto J, const uint8_t* x) DATTRI_INLINE {
    constexpr int s = decltype(S)::value, j = decltype(J)::value;
    if constexpr (j < BM)
      fa[s & 1][j] = SA::template read<s>(x, wm * BM * 32, lane, j);
    else
      fb[s & 1][j - BM] = SB::template read<s>(x + SA::kBytes, wn * BN * 32, lane, j - BM);
  };
  constexpr int kLoads = SA::kLoads + SB::kLoads;
  constexpr int kHalf = kLoads / 2;  // in the step behind the barrier, the others in the next
  // loads From .. To - 1 of stage st, A's first
  auto issue = [&](int st, uint8_t* x, auto From, auto To) DATTRI_INLINE {
    const rsrc_t ra = sa.range(s0 + st), rb = sb.range(s0 + st);
    unrolled<kLoads>([&](auto J) DATTRI_INLINE {
      constexpr int j = decltype(J)::value;
      if constexpr (j >= decltype(From)::value && j < decltype(To)::value) {
        if constexpr (j < SA::kLoads)
          sa.load(ra, s0 + st, x, wave, j);
        else
          sb.load(rb, s0 + st, x + SA::kBytes, wave, j - SA::kLoads);
      }
    });
  };
  // K step S: its products, and between them the reads of the step after it
  // (from rx) and loads From .. To - 1 of stage lst.  One wave
  // has a SIMD to itself, so what stands between two MFMA delays the second once
  // it takes longer than the first: the order is fixed, a read or two at a time.
  auto step = [&](auto S, const uint8_t* rx, int lst, uint8_t* lx, auto From, auto To) DATTRI_INLINE {
    constexpr int s = decltype(S)::value & 1, kBlocks = BN * BM, kFirst = (7 * kBlocks + 7) / 8,
                  from = decltype(From)::value, to = decltype(To)::value;
    unrolled<kBlocks>([&](auto M) DATTRI_INLINE {
      constexpr int m = decltype(M)::value, i = m / BM, j = m % BM;
      unrolled<BM + BN>([&](auto J) DATTRI_INLINE {
        constexpr int q = decltype(J)::value;
        if constexpr (m < kFirst && q >= (BM + BN) * m / kFirst && q < (BM + BN) * (m + 1) / kFirst)
          read(std::integral_constant<int, (decltype(S)::value + 1) % kSteps>{}, J, rx);
      });
      issue(lst, lx, std::integral_constant<int, from + (to - from) * m / kBlocks>{},
            std::integral_constant<int, from + (to - from) * (m + 1) / kBlocks>{});
      acc[i][j] = block_mma<ELT>(operand(fb[s][i]), operand(fa[s][j]), acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    });
    landed(fa[1 - s]);
    landed(fb[1 - s]);
  };
  typedef std::integral_constant<int, 0> zero_t;
  typedef std::integral_constant<int, kHalf> half_t;
  typedef std::integral_constant<int, kLoads> all_t;
  if (ns > 0) {
    issue(0, x0, zero_t{}, all_t{});
    if constexpr (kBuffers == 4) {
      issue(1, x1, zero_t{}, all_t{});
      issue(2, x2, zero_t{}, all_t{});
      issue(3, x3, zero_t{}, half_t{});
    } else {
      issue(1, x1, zero_t{}, half_t{});
    }
    wait_vmcnt_dma<(kBuffers - 2) * kLoads + kHalf>();  // stage 0 has landed
    plain_barrier();
    unrolled<BM + BN>([&](auto J) DATTRI_INLINE { read(zero_t{}, J, x0); });
    landed(fa[0]);
    landed(fb[0]);
    // On entry step 0 of stage st (in cx) is in registers, and stages st + 1 ..
    // st + kBuffers - 1 are on their way, the last but for its second part.
    // Loads past the last stage fetch nothing (their k is past the sides' K) and
    // fill with zeros.
    auto stage = [&](int st, uint8_t* cx, const uint8_t* nx, uint8_t* px) DATTRI_INLINE {
      step(zero_t{}, cx, st + kBuffers - 1, px, half_t{}, all_t{});
      if constexpr (kSteps == 4) {
        step(std::integral_constant<int, 1>{}, cx, 0, cx, zero_t{}, zero_t{});
        step(std::integral_constant<int, 2>{}, cx, 0, cx, zero_t{}, zero_t{});
      }
      // stage st is in registers, st + 1 has landed: the stages after it may still be under way
      wait_vmcnt_dma<(kBuffers - 2) * kLoads>();
      stage_barrier();
      step(std::integral_constant<int, kSteps - 1>{}, nx, st + kBuffers, cx, zero_t{}, half_t{});
    };
    for (int st = 0; st < ns; st += kBuffers) {  // a last round that is not full ends in stages of zeros
      if constexpr (kBuffers == 4) {
        stage(st, x0, x1, x3);
        stage(st + 1, x1, x2, x0);
        stage(st + 2, x2, x3, x1);
        stage(st + 3, x3, x0, x2);
      } else {
        stage(st, x0, x1, x1);
        stage(st + 1, x1, x0, x0);
      }
    }
    wait_all();
  }

  finish_tile<OP, ELT, WM, WN, BM, BN>(a, acc, m0, n0, part, ld_part, [&](int j, int wm) {
    // the rows of waves: in one buffer each
    uint8_t* const y = kBuffers == 4 ? (j & 1 ? x2 : x0) : (j & 1 ? x1 : x0);
    return wm ? (kBuffers == 4 ? (j & 1 ? x3 : x1) : y + kSlab) : y;
  });
}

// Sums of a split product's partial tiles in split order, and the epilogue.
template <int OP, int ELT>
__global__ __launch_bounds__(256) void gemm_join_kernel(GemmArgs a, const float* __restrict__ part, int64_t ld_part,
                                                        int splits) {
  const int nv = (a.N + 3) / 4;
  const int64_t total = (int64_t)a.M * nv, step = (int64_t)a.M * ld_part;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int m = (int)(i / nv), n = (int)(i - (int64_t)m * nv) * 4;
    const float* p = part + m * ld_part + n;
    f32x4 s = *(const f32x4*)p;
    int y = 1;
    for (; y + 3 < splits; y += 4) {
      const f32x4 v0 = *(const f32x4*)(p + y * step), v1 = *(const f32x4*)(p + (y + 1) * step),
                  v2 = *(const f32x4*)(p + (y + 2) * step), v3 = *(const f32x4*)(p + (y + 3) * step);
      s = (((s + v0) + v1) + v2) + v3;
    }
    for (; y < splits; ++y) s += *(const f32x4*)(p + y * step);
    epilogue4<OP, ELT>(a, m, n, s);
  }
}

// Rows of `w` elements copied to rows of `ld_out` (a multiple of 16 bytes),
// zeros behind; both operands in one launch (rows 0: nothing).
struct Repack {
  const uint8_t* src;
  uint8_t* dst;
  int64_t ld, rows;
  int w, ld_out;
};
__device__ inline int64_t repack_at() {  // a wave per row
  return row_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}
template <int ELT>
__device__ DATTRI_INLINE inline void repack_row(const Repack& p, int64_t r) {
  constexpr int U = ELT == 1 ? 2 : 4;  // pieces per lane under way
  const int lane = threadIdx.x & 63;
  const uint8_t* const src = p.src + r * p.ld * ELT;
  uint8_t* const dst = p.dst + r * p.ld_out * ELT;
  const int width = p.w * ELT, out = p.ld_out * ELT;
  // 16 bytes per lane from the aligned words that hold them, shifted into place; a word is read only if some of its
  // bytes are the row's, and those behind the row become zeros
  const int shift = (int)((uintptr_t)src & 3);
  const rsrc_t words = make_rsrc(src - shift, (uint32_t)(width + shift + 3) / 4 * 4);
  for (int c0 = lane * 16; c0 < out; c0 += 1024 * U) {
    uint32_t v[U][5];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < (ELT == 4 ? 4 : 5); ++e) v[u][e] = load4(words, c0 + 1024 * u + 4 * e);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + 1024 * u;
      i32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (ELT == 4) {
          o[e] = (int)v[u][e];
        } else {
          const uint32_t x = __builtin_amdgcn_alignbyte(v[u][e + 1], v[u][e], shift);
          const int left = width - (c + 4 * e);  // bytes of the row in this word
          o[e] = (int)(left >= 4 ? x : left > 0 ? x & ((1u << 8 * left) - 1u) : 0u);
        }
      }
      if (c < out) *(i32x4*)(dst + c) = o;
    }
  }
}
template <int ELT>
__global__ __launch_bounds__(256) void repack_kernel(Repack a, Repack b) {
  const int64_t at = repack_at();
  if (at >= a.rows + b.rows) return;
  repack_row<ELT>(at < a.rows ? a : b, at < a.rows ? at : at - a.rows);
}

// Whether rows of `w` elements can be read in 16-byte pieces as they are.
inline bool on_chunks(const void* p, int64_t ld, int64_t w, int elt) {
  return (uintptr_t)p % 16 == 0 && ld * elt % 16 == 0 && w * elt % 16 == 0;
}

// An operand and where its repacked rows go; updates pointer and stride.
inline Repack repack_of(const void** src, int64_t* ld, int64_t w, int64_t rows, int elt, uint8_t* dst) {
  const int ld_out = (int)((w * elt + 15) / 16 * 16 / elt);
  const Repack r = {(const uint8_t*)*src, dst, *ld, rows, (int)w, ld_out};
  *src = dst;
  *ld = ld_out;
  return r;
}

}  // namespace tile
}  // namespace dattri
