// muon_tiles.h -- the tiles of the products, on the host.
#pragma once

#include <algorithm>
#include <vector>

#include "muon.h"
#include "optim.h"

namespace frk {

// A factor of a product: a matrix of the workspace by its rows or by its columns, S and P by either.
struct Factor {
  uint32_t block, col_blocks;
  bool by_columns, iterate;
  uint32_t first(uint32_t b) const { return block + (by_columns ? 2 * b : b * col_blocks); }
  // S and P: where the factor's 256 rows from block b on leave the tiles that exist, and what they meet there on the other side.
  uint32_t switch_at(uint32_t b, uint32_t depth) const { return iterate ? depth : std::min(depth, 2 * (b / 2 * 2 + 2)); }
  uint32_t after(uint32_t b, uint32_t col_block) const { return iterate ? 0 : block + (b / 2 * 2 + 2) * col_blocks + col_block; }
};

// A phase's product for a matrix.
struct ProductOf {
  Factor a, b;
  uint32_t depth, square;
  uint32_t out, rows, cols;  // rows and columns in blocks of 128

  ProductOf(int phase, const MuonDesc& d) {
    const uint32_t x = static_cast<uint32_t>(d.x[0] / kMuonBlockBytes), s = static_cast<uint32_t>(d.s / kMuonBlockBytes), p = static_cast<uint32_t>(d.p / kMuonBlockBytes);
    const uint32_t side = d.side_blocks;
    square = 2 * side;
    if (phase == kGram) {
      a = b = {x, d.col_blocks, d.tall != 0, true};
      depth = d.tall ? 2 * d.row_blocks : d.col_blocks;
    } else if (phase == kPolynomial) {
      a = b = {s, square, false, false};
      depth = square;
    } else {
      const Factor q = {p, square, false, false};
      a = d.tall ? Factor{x, d.col_blocks, false, true} : q;
      b = d.tall ? q : Factor{x, d.col_blocks, true, true};
      depth = square;
    }
    out = phase == kGram ? s : phase == kPolynomial ? p : x;
    rows = phase == kNext ? d.row_blocks : side;
    cols = phase == kNext ? d.col_blocks / 2 : side;
  }
  // Calls f(row, column, narrow) for every tile, of a symmetric result those on and below the diagonal.
  template <class F>
  void each(int phase, bool all_narrow, F f) const {
    auto columns = [&](uint32_t r, uint32_t end) {
      for (uint32_t c = 0; c < end; c += all_narrow ? 1 : 2) f(r, c, all_narrow || c + 1 == cols);
    };
    if (phase == kNext && !b.by_columns) {
      for (uint32_t r = 0; r < rows; r += 2) columns(r, cols);
    } else if (phase == kNext) {  // (tiles that share the long side's blocks one after the other)
      for (uint32_t c = 0; c < cols; c += all_narrow ? 1 : 2)
        for (uint32_t r = 0; r < rows; r += 2) f(r, c, all_narrow || c + 1 == cols);
    } else {
      for (uint32_t r = 0; r < rows; r += 2) columns(r, std::min(r + 2, cols));
    }
  }
  uint32_t tiles(int phase, bool all_narrow) const {
    uint32_t n = 0;
    each(phase, all_narrow, [&](uint32_t, uint32_t, bool) { ++n; });
    return n;
  }
  // Of blocks of rows r and r + 1, of columns c and, unless it is narrow, c + 1.
  MuonTile tile(int phase, uint32_t r, uint32_t c, bool narrow) const {
    MuonTile t = {};
    t.phase = static_cast<uint32_t>(phase);
    const bool second = r + 1 < rows;
    t.a[0] = a.first(r);
    // (beyond an odd number of blocks of rows: the last one again, its results are dropped)
    t.a[1] = a.first(second ? r + 1 : r);
    t.b[0] = b.first(c);
    // (a narrow tile's CTAs have 64 rows or columns each, of rows the halves of a block)
    t.b[1] = !narrow ? b.first(c + 1) : b.first(c) + (b.by_columns ? 1 : 0);
    t.a_switch = a.switch_at(r, depth);
    t.b_switch = b.switch_at(c, depth);
    for (uint32_t k = 0; k < 2; ++k) {
      t.a_after[k] = a.after(r, 2 * (second ? r + k : r));
      t.b_after[k] = b.after(c, narrow ? 2 * c + k : 2 * (c + k));
    }
    t.a_next = a.by_columns ? a.col_blocks : 1;
    t.b_next = b.by_columns ? b.col_blocks : 1;
    t.square = square;
    t.depth = depth;
    t.flags = (narrow ? kNarrow : 0) | (a.by_columns ? kAColumns : 0) | (b.by_columns ? kBColumns : 0) | (second ? kSecond : 0) |
              (a.iterate ? kAIterate : 0) | (b.iterate ? kBIterate : 0) | (phase != kNext && r == c && !narrow ? kSame : 0);
    t.across = 2 * cols;
    t.out = out + r * t.across + 2 * c;
    t.row = static_cast<uint16_t>(r);
    t.col = static_cast<uint16_t>(c);
    return t;
  }
};

// The tiles of an iteration over the matrices that are split, or those that are not: S of all, then P, then X, in each those with the longest
// contraction first.  ends: where each phase's end.  A phase that has so few tiles that narrow ones do not fill the SMs has narrow ones: their
// last 64 columns are done in half the time.  (Sums are the same.)
inline void plan_tiles(const std::vector<MuonDesc>& descs, bool split, std::vector<MuonTile>& tiles, uint32_t (&ends)[kPhases]) {
  std::vector<uint32_t> mine;
  for (uint32_t m = 0; m < descs.size(); ++m)
    if ((descs[m].split != 0) == split) mine.push_back(m);
  bool narrow[kPhases];
  for (int phase = 0; phase < kPhases; ++phase) {
    uint64_t n = 0;
    for (uint32_t m : mine) n += ProductOf(phase, descs[m]).tiles(phase, true);
    narrow[phase] = n <= kSms / 2;
  }
  for (int phase = 0; phase < kPhases; ++phase) {
    std::stable_sort(mine.begin(), mine.end(),
                     [&](uint32_t x, uint32_t y) { return ProductOf(phase, descs[x]).depth > ProductOf(phase, descs[y]).depth; });
    for (uint32_t m : mine) {
      const ProductOf q(phase, descs[m]);
      const int from = (phase + kPhases - 1) % kPhases;
      const uint32_t needs = m * kPhases + from, count = kSignals * ProductOf(from, descs[m]).tiles(from, narrow[from]);
      q.each(phase, narrow[phase], [&](uint32_t r, uint32_t c, bool is_narrow) {
        MuonTile t = q.tile(phase, r, c, is_narrow);
        t.done = m * kPhases + phase;
        t.needs = needs;
        t.count = count;
        tiles.push_back(t);
      });
    }
    ends[phase] = static_cast<uint32_t>(tiles.size());
  }
}

}  // namespace frk
