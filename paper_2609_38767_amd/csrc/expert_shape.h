// How the experts' products are cut (no HIP; all but tile_rows host only): tiles, splits of k.
// Nothing of the boundaries is known here: the choice goes by the mean rows of an
// expert.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "linear_shape.h"

namespace dattri {

struct ExpertShape {
  Variant v;
  int kw;      // bytes of k per stage
  int splits;  // of k: an expert's rows (weight gradients), else all of it
};

// Which tile rows of tm rows each are counted of a segment of n rows: all that it
// meets; those that it fills to more than half; the one that it fills to half at
// most.  n goes up to the largest int32, so nothing is added to it.
enum Rows { kAll, kFull, kRest };
constexpr int tile_rows(Rows r, int n, int tm) {
  return r == kAll ? n / tm + (n % tm > 0) : r == kFull ? n / tm + (n % tm > tm / 2) : n % tm > 0 && n % tm <= tm / 2;
}

// Whether tiles are split along k at all: the largest have work enough, and float32
// ones of 64 x 128 lie too near to 32 x 128 whole.
constexpr bool expert_splits(Variant v, int elt) { return v != kBig && !(v == kSlim && elt == 4); }

// The cut with the least modelled time, in us: FLOP at the rate that a CU reaches
// with its tiles on many rows, what a tile costs besides, the rounds of tiles over
// the CUs (the largest tiles come one per CU, others share it), the partial tiles
// of a split written, read and joined, and the bytes of operands and weights met
// at 5 TB/s, of which the smaller part is hidden but for three tenths.
//   m, n, k as in GemmArgs; rows take the place of m in products over rows, and
//   the mean rows of an expert that of k in weight gradients.
// Measured, bf16, us with 256 x 256 / 128 x 128 / 64 x 128 / 32 x 128 tiles:
// forward 4096 -> 14336, eight experts: 16 rows 206/143/135/133, 256 rows
// 215/192/185/203, 1024 rows 242/263/309/485, 16384 rows 1692/2435/3498/6390; 64
// experts of 4096 -> 1024, 32768 rows 371/449/566/876.  float32, five experts of
// 769 -> 1030, 1531 rows: 284/75/50/50; one of 3232 -> 392, 28 rows, without a
// split: 64 in 32 x 128.
// float32 weight gradients leave out 256 x 256 (3% more at most) and take 64 x 128
// too; bf16 ones would gain little there (24 and 27) and lose elsewhere.  us in 128
// x 128 / 64 x 128, * the model's choice: 1531 rows, five experts of 769 -> 1030
// 67/49*, one 52/61*, 16 of 1536 -> 1536 96*/98; 6000 rows, five of 512 -> 2048
// 179/108*, one 112*/180, 32 153*/136, eight of 256 -> 300 30/48*; 300 rows, 32 of
// 1536 -> 1536 109*/121.  Of 108 sizes (1 to 32 experts, 300 to 6000 rows, six
// pairs of widths) it was within 6% of the better of the two in 91.
inline ExpertShape expert_shape(bool weight_grad, int64_t rows, int64_t experts, int64_t m, int64_t n, int64_t k,
                                int elt, bool bc) {
  const double rate[4] = {elt == 2 ? 5.2e6 : 0.58e6, elt == 2 ? 3.4e6 : 0.565e6, elt == 2 ? 2.4e6 : 0.5e6,
                          elt == 2 ? 1.4e6 : 0.45e6},
               fixed[4] = {12., 3., 2., 1.5};
  const int64_t met = std::max<int64_t>(1, std::min(experts, rows));
  const double mean = (double)rows / experts;
  const double bytes = weight_grad ? 4. * experts * m * n + (double)elt * rows * (m + n)
                                   : (double)elt * (met * n * k + rows * (n + k));
  ExpertShape best = {};
  double best_us = 0.;
  for (int v = weight_grad && elt == 4 ? kMid : kBig; v <= (!weight_grad ? kFew : elt == 4 ? kSlim : kMid); ++v) {
    const int64_t tm = v == kBig ? 256 : v == kMid ? 128 : v == kSlim ? 64 : 32, tn = v == kBig ? 256 : 128;
    const int kw = stage_bytes(!weight_grad, bc, elt, (int)tm);
    const double nn = (double)((n + tn - 1) / tn);
    // an expert's last tile is half empty on average, and none has less than one
    const double nm = weight_grad ? (double)experts * ((m + tm - 1) / tm)
                                  : std::max((double)met, (double)rows / tm + 0.5 * met);
    const double depth = weight_grad ? mean : (double)k;
    for (int splits = 1; splits <= (expert_splits((Variant)v, elt) ? 32 : 1); ++splits) {
      if (splits > 1 && depth * elt / splits < 512.) break;
      const double tiles = nm * nn * splits / 256.;
      // weight gradients: an expert of many rows makes long tiles, which many short ones even out
      const double rounds = weight_grad ? std::max(1., tiles + (v == kBig || (v == kMid && elt == 4) ? 1. : 0.5))
                            : v <= kMid ? std::max(1., std::ceil(tiles)) : std::max(1., tiles + 0.5);
      const double work = rounds * (2. * tm * tn * depth / splits / rate[v] + fixed[v]), read = bytes / 5.e6;
      double us = std::max(work, read) + 0.3 * std::min(work, read);
      if (splits > 1)  // and only where the gain is clear: 64 rows of 14336 <- 4096, eight experts, 137 us whole, 160 in five
        us = 1.1 * us + 4. + 8. * splits * (weight_grad ? (double)experts * m : (double)rows) * n / 5.e6;
      if (best_us == 0. || us < best_us) {
        best = ExpertShape{(Variant)v, kw, splits};
        best_us = us;
      }
    }
  }
  // Few rows whose tiles leave half the CUs without work read the weights slowly, and two splits of k give the others
  // some; `met` is the most experts that the rows can meet.  us whole and in two splits, 64 experts, weights out of the
  // caches, rows spread by chance:
  //   forward of 4096 -> 1024 bf16: 8 rows 38/26, 16 rows (128 tiles) 42/33, 18 rows (144) 44/48, 20 rows 45/52;
  //   of 16 rows and k -> 1024, bf16: k 768 12.4/12.8, 1024 14.1/14.0, 1280 18.1/15.7, 2048 23.8/19.0; float32: k 256
  //   10.7/11.6, 512 15.6/14.7, 768 21.2/17.7; input gradients of 1024 <- k bf16: 768 11.5/12.1, 1024 14.1/13.4, 1280
  //   15.6/14.6, 4096 38/29.
  // Below 2560 bytes of k a split has too few stages for what its join takes.
  if (!weight_grad && best.v == kFew && best.splits == 1 && k * elt >= 2560 &&
      std::max((double)met, (double)rows / 32 + 0.5 * met) * ((n + 127) / 128) <= 128.)
    best.splits = 2;
  if (best.splits > 1 && !weight_grad) {  // whole rounds of the buffers
    const int64_t stages = (k * elt + best.kw - 1) / best.kw, round = buffers_of(best.kw),
                  sps = ((stages + best.splits - 1) / best.splits + round - 1) / round * round;
    best.splits = (int)((stages + sps - 1) / sps);
  }
  return best;
}

}  // namespace dattri
