// loss_plan.h -- how the cross entropy's products are cut into tiles, splits, pieces of the
// vocabulary and of the rows, and what its workspace holds.  Plain C++: no HIP.
#pragma once

#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "sieve.h"

namespace sieve {
namespace loss {

constexpr int64_t kMaxRows = 1 << 24;      // of h, and of the table
constexpr int kMaxN = 65536;
constexpr int64_t kPieceValues = 1 << 27;  // of g, in 16 bits each
constexpr int64_t kMaxPiece = 65536;       // vectors
constexpr int64_t kRowChunk = 65536;       // rows of h in one launch of the forward pass

// The shapes of a work-group's tile (loss.hip): tiles of 128 x 128 at two a CU, the same with more
// loads on their way, 256 x 256, and those for values of three planes.
enum Size { kSmall, kDeep, kLarge, kTriple };
struct Measured {
  int bm, bn, places;
  double each;           // us a value of k and tile, where the chip is full
};
constexpr Measured kMeasured[] = {{128, 128, 512, 0.0175},
                                  {128, 128, 256, 0.0107},
                                  {256, 256, 256, 0.029},
                                  {128, 128, 256, 0.05}};
constexpr int kSmallest = 128;  // the lesser of the shapes' BM

// A part of a row's sum: the largest dot product of it, and the sum of
// exp(scale (dot product - largest)).
struct Part {
  float top, sum;
};

// What a row's g is divided by, inverse (0 where the row gives no gradient), and its factor.
struct Row {
  float inverse, factor;
};

// Up to so many rows, and of 16-bit values: each 16 vectors read the rows again, and tiles keep up
// from some rows on.  131,072 x 1,024 f16, tables from memory: one row 52 us, 4 rows 55, 16 rows
// 68; in tiles 56, whatever the rows.  fp32 has no planes to pack here: one row 126 us, 16 rows
// 137; in tiles 636 (17 to 32 rows), and no others than a matrix instruction's 16 fit here.
constexpr int kThinRows = 16, kThinRows16 = 4, kThinMost = 1024;

constexpr int kMostLargest = 1024;  // work-groups that each leave their largest factor

inline int64_t round256(int64_t n) { return (n + 255) & ~int64_t(255); }

inline int64_t tiles_of(int64_t m, int64_t n, const Measured& x) {
  return ((m + x.bm - 1) / x.bm) * ((n + x.bn - 1) / x.bn);
}

// The shape of a product's tiles that takes the shortest, by what was measured; 4 us go around
// each tile.
inline Size size_of(int64_t m, int64_t n, int64_t k, int planes) {
  if (planes == 3) return kTriple;
  Size best = kSmall;
  double least = INFINITY;
  for (const Size size : {kSmall, kDeep, kLarge}) {
    const Measured& x = kMeasured[size];
    const int64_t rounds = (tiles_of(m, n, x) + x.places - 1) / x.places;
    const double us = (double)rounds * (x.each * (double)k + 4.0);
    if (us < least) {
      least = us;
      best = size;
    }
  }
  return best;
}

// How the two gradients' products are spread over the chip: the shape of their tiles, and into how
// many splits of k each.
struct Spread {
  Size size;
  int splits_h, splits_w;
};

// dh is [mh, n] over kh values, dw [mw, n] over kw.  Splits are written, read and added at 4 TB/s.
inline Spread spread_of(int64_t mh, int64_t kh, int64_t mw, int64_t kw, int64_t n, int planes) {
  Spread best{kSmall, 1, 1};
  double least = INFINITY;
  const int options[] = {1, 2, 3, 4, 6, 8, 12, 16};
  for (const Size size : {kSmall, kDeep, kLarge, kTriple}) {
    if ((planes == 3) != (size == kTriple)) continue;
    const Measured& x = kMeasured[size];
    const int64_t th = tiles_of(mh, n, x), tw = tiles_of(mw, n, x);
    for (const int sh : options) {
      if (sh > 1 && kh / sh < 256) break;
      const double one_h = x.each * (double)kh / sh + 4.0;
      for (const int sw : options) {
        if (sw > 1 && kw / sw < 256) break;
        const double one_w = x.each * (double)kw / sw + 4.0;
        const double all = (double)(th * sh) * one_h + (double)(tw * sw) * one_w;
        const int64_t rounds = (th * sh + tw * sw + x.places - 1) / x.places;
        const double mean = all / (double)(th * sh + tw * sw);
        double us = std::max({(double)rounds * mean, one_h, one_w});
        if (sh > 1) us += 2.0 + (double)mh * n * 2e-6 * sh;
        if (sw > 1) us += 4.0 + (double)mw * n * 2e-6 * sw;
        if (us < least) {
          least = us;
          best = {size, sh, sw};
        }
      }
    }
  }
  return best;
}

struct Layout {
  int64_t piece;                 // vectors of a piece, a multiple of 256
  int64_t chunk;                 // rows that g is kept of at a time, in the backward pass
  int64_t k;                     // n, up to the next multiple of 8
  int planes;
  int weighed_planes;            // of h in dw's product
  Spread spread;
  bool sum_h, sum_w;             // sums of splits, and dh's over the pieces, dw's over the chunks:
                                 // else the products write the gradients themselves
  int64_t h, w, part, target, g, weighed, row, largest, dh, dw, power, bytes;
};

inline Layout layout_of(int64_t rows, int64_t vocab, int32_t n, int32_t dtype, bool backward) {
  Layout l{};
  l.planes = dtype == SIEVE_F32 ? 3 : 1;
  l.k = (n + 7) & ~7;
  // as many as leave a piece its 256 vectors
  l.chunk = std::min(std::max<int64_t>(rows, 1), kPieceValues / (l.planes * 256) & ~int64_t(255));
  const int64_t piece = std::min(kPieceValues / (l.planes * l.chunk), kMaxPiece);
  l.piece = std::min(piece & ~int64_t(255), round256(vocab));
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t was = at;
    at += round256(bytes);
    return was;
  };
  l.h = take(rows * l.k * 2 * l.planes);
  l.w = take(l.piece * l.k * 2 * l.planes);
  if (!backward) {
    const int64_t chunk = std::min(rows, kRowChunk);
    // of the tiles, or of the few rows' work-groups
    const int64_t parts = std::max<int64_t>((vocab + kSmallest - 1) / kSmallest,
                                            rows <= kThinRows ? kThinMost : 0);
    l.part = take(parts * chunk * (int64_t)sizeof(Part));
    l.target = take(chunk * 4);
  } else {
    const int64_t vs = std::min(l.piece, vocab);
    // h times its row's factor is rounded a second time: where dw's product takes a few us at the
    // most (2^31 products: 4 us), what that loses is a plane of its own
    const bool few = dtype != SIEVE_F32 && rows * vocab <= (int64_t(1) << 31) / n;
    l.weighed_planes = few ? 2 : l.planes;
    l.spread = spread_of(l.chunk, vs, vs, few ? 2 * l.chunk : l.chunk, n, l.planes);
    l.g = take(l.chunk * l.piece * 2 * l.planes);
    l.weighed = take(rows * l.k * 2 * l.weighed_planes);
    l.row = take(rows * (int64_t)sizeof(Row));
    l.largest = take(kMostLargest * 4);
    l.sum_h = l.piece < vocab || l.spread.splits_h > 1;
    l.sum_w = l.chunk < rows || l.spread.splits_w > 1;
    l.dh = take(l.sum_h ? l.spread.splits_h * rows * l.k * 4 : 0);
    l.dw = take(l.sum_w ? l.spread.splits_w * l.piece * l.k * 4 : 0);
    l.power = take(4);
  }
  l.bytes = at;
  return l;
}

}  // namespace loss
}  // namespace sieve
