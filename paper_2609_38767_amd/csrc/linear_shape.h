// How a product of the linear layers is cut (host only, no HIP): tile variant,
// splits of k, stages per split.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace dattri {

constexpr int buffers_of(int kw) { return 256 / kw; }  // stage buffers (and stages unrolled)

enum Variant { kBig, kMid, kSlim, kFew };  // 256 x 256, 128 x 128, 64 x 128, 32 x 128
struct GemmShape {
  Variant v;
  int kw;  // bytes of k per stage
  int64_t nm, nn;
  int splits, sps;
};

// Bytes of k per stage: 128 where both operands have k contiguous (whole cache
// lines) and nothing else hides the loads: bf16, one workgroup per CU.  Else 64,
// twice the buffers (128 x 128 tiles, 2048^3: 24 us, 27 with 128 bytes).
constexpr int stage_bytes(bool ac, bool bc, int elt, int tm) { return ac && bc && elt == 2 && tm == 256 ? 128 : 64; }

inline GemmShape gemm_shape(int64_t M, int64_t N, int64_t K, int elt, bool ac, bool bc) {
  auto cut = [&](Variant v, int64_t splits) {
    GemmShape g;
    const int tm = v == kBig ? 256 : v == kMid ? 128 : v == kSlim ? 64 : 32, tn = v == kBig ? 256 : 128;
    g.v = v;
    g.kw = stage_bytes(ac, bc, elt, tm);
    g.nm = (M + tm - 1) / tm;
    g.nn = (N + tn - 1) / tn;
    const int64_t stages = std::max<int64_t>(1, (K * elt + g.kw - 1) / g.kw), round = buffers_of(g.kw);
    splits = std::max<int64_t>(1, std::min(splits, stages * g.kw / 512));
    g.sps = (int)((stages + splits - 1) / splits);
    if (splits > 1) g.sps = (int)((g.sps + round - 1) / round * round);  // whole rounds of the buffers
    g.splits = (int)((stages + g.sps - 1) / g.sps);
    return g;
  };
  // Few rows: the other operand is what there is to read, by as many workgroups
  // as keep its loads in flight.
  if (ac && M <= 64) {
    const Variant v = M <= 32 ? kFew : kSlim;
    const int64_t tiles = (N + 127) / 128;
    return cut(v, std::min<int64_t>(64, (v == kFew ? 1024 : 768) / std::max<int64_t>(tiles, 1)));
  }
  // Else the cut with the least time as modelled, in us: the CU with most tiles
  // (FLOP at the rate one CU reaches on a large product, 12% less where it has one
  // workgroup of 128 x 128 only; plus what a tile costs besides), and the partial
  // tiles of a split written, read and joined.  1531 x 1024 -> 4096 float32: 128 x
  // 128 whole 123 us, in two splits 110, 256 x 256 244.
  const double rate[2] = {elt == 2 ? 5.2e6 : 0.58e6, elt == 2 ? 4.0e6 : 0.565e6}, fixed[2] = {12., 3.};
  const int64_t all = (K * elt + 63) / 64 * 64;
  GemmShape best = {};
  double best_us = 0.;
  for (int v = kBig; v <= kMid; ++v)
    for (int64_t splits = 1; splits <= 32; ++splits) {
      const GemmShape g = cut((Variant)v, splits);
      if (g.splits != splits) continue;
      // the CU with most tiles; the last split's may be short
      const double each = (double)g.nm * g.nn, last = splits > 1 ? (double)all / ((int64_t)g.sps * g.kw) - (splits - 1) : 1.;
      const bool alone = each * splits <= 256.;
      const double rounds = alone ? 1. : std::max(1. + last, std::ceil(each * (splits - 1 + last) / 256.));
      const int64_t side = v == kBig ? 256 : 128;
      const double flop = 2. * side * side * g.sps * (g.kw / elt);
      double us = rounds * (flop / (rate[v] * (alone && v == kMid ? 0.88 : 1.)) + fixed[v]);
      if (g.splits > 1) us += 3. + 8. * g.splits * M * N / 6.0e6;
      if (best_us == 0. || us < best_us) {
        best = g;
        best_us = us;
      }
    }
  return best;
}

}  // namespace dattri
