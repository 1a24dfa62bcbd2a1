// How an 8-bit product is cut (host only, no HIP): form, splits of k, groups of
// 128 k per split.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "linear_shape.h"

namespace dattri {

// kFew: the form without tiles; elt: bytes of a result.
struct Shape8 {
  Variant v;
  int64_t nm, nn;
  int splits, sps;
};

// Stage buffers: short stages have four.
inline int round_of(Variant v, int elt) { return v == kSlim || (v == kMid && elt == 2) ? 4 : 2; }

inline Shape8 shape8(int64_t M, int64_t N, int64_t K, int elt) {
  const int64_t stages = std::max<int64_t>(1, (K + 127) / 128);
  auto cut = [&](Variant v, int64_t splits) {
    Shape8 g = {};
    const int tm = v == kBig ? 256 : v == kMid ? 128 : 64, tn = v == kBig ? 256 : 128;
    g.v = v;
    g.nm = (M + tm - 1) / tm;
    g.nn = (N + tn - 1) / tn;
    splits = std::max<int64_t>(1, std::min(splits, stages / 4));
    g.sps = (int)((stages + splits - 1) / splits);
    if (splits > 1) g.sps = round_of(v, elt) * ((g.sps + round_of(v, elt) - 1) / round_of(v, elt));
    g.splits = (int)((stages + g.sps - 1) / g.sps);
    return g;
  };
  // Without tiles every 16 weight rows read all rows of X again.  us without and with tiles, weights out of the caches:
  // 4096 -> 14336 one row 14.4/16.3, four 16.3/16.3, seven 17.2/16.5 (float32 18.1/17.7), eight 17.8/16.5, sixteen
  // 22.4/16.7; 14336 -> 4096 seven 17.8/17.0 (float32 17.9/18.4), eight 18.0/16.9; 8192 -> 4096, 34M weights, eight
  // 11.1/13.3, sixteen 13.3/13.8; 4096 -> 4096 one row 6.2/10.7.
  if (M < 8 || (M <= 16 && N * K < 40000000)) return cut(kFew, 1);
  // One workgroup per CU, whose ring keeps 75 KB of loads under way (weights out of the caches): 64 x 4096 -> 14336 20.1
  // us in two splits, 25.0 whole, 26.5 in six; 64 x 14336 -> 4096 20.4 in eight, 26.2 in four, 69.6 whole.  With half
  // the CUs at work splits of eight groups of k or more do (64 x 4096 -> 4096 14.0 us in four, 14.9 in eight; 64 x
  // 8192 -> 2048 14.3 in eight, 15.3 in sixteen; but 64 x 4096 -> 1024 11.9 in four, 10.8 in eight), and eight groups
  // stay whole (64 x 1024 -> 4096 8.5, in two 9.7).
  if (M <= 64) {
    const int64_t strips = (N + 127) / 128;
    return cut(kSlim, stages <= 8 ? 1 : std::min<int64_t>({64, 256 / strips, std::max<int64_t>(128 / strips, stages / 8)}));
  }
  // The cut with the least modelled time, as for the other products (gemm_shape):
  // FLOP per us of a CU, us besides, and what a lone workgroup of 128 x 128 reaches
  // of the rate where two share a CU otherwise (float32 results).  1000 x 1000 ->
  // 1000: 64 x 128 12.3 us, 128 x 128 14.1; 1536 x 4096 -> 2304: 35.6 and 24.7.
  const double rate[3] = {8.8e6, elt == 2 ? 6.2e6 : 4.3e6, elt == 2 ? 4.8e6 : 3.e6}, fixed[3] = {12., 4., 3.5},
               lone = elt == 2 ? 1. : 0.85;
  Shape8 best = {};
  double best_us = 0.;
  for (int v = elt == 2 ? kBig : kMid; v <= kSlim; ++v)
    for (int64_t splits = 1; splits <= 32; ++splits) {
      const Shape8 g = cut((Variant)v, splits);
      if (g.splits != splits) continue;
      const double each = (double)g.nm * g.nn, last = splits > 1 ? (double)stages / g.sps - (splits - 1) : 1.;
      const bool alone = each * splits <= 256.;
      const double rounds = alone ? 1. : std::max(1. + last, std::ceil(each * (splits - 1 + last) / 256.));
      const double area = v == kBig ? 65536. : v == kMid ? 16384. : 8192.;
      double us = rounds * (2. * area * g.sps * 128 / (rate[v] * (alone && v == kMid ? lone : 1.)) + fixed[v]);
      if (g.splits > 1) us += 3. + 8. * g.splits * M * N / 6.0e6;
      if (best_us == 0. || us < best_us) {
        best = g;
        best_us = us;
      }
    }
  return best;
}

}  // namespace dattri
