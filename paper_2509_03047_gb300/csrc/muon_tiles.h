// muon_tiles.h -- the tiles of the products, on the host.
#pragma once

#include <algorithm>
#include <vector>

#include "muon.h"

namespace frk {

// A factor of a product: a matrix of the workspace by its rows or by its columns, S and P by either.
struct Factor {
  uint32_t block, col_blocks;
  bool by_columns, iterate;
  uint32_t first(uint32_t b) const { return block + (by_columns ? 2 * b : b * col_blocks); }
  // S and P: where the factor's 256 rows from block b on leave the tiles that exist, and what they meet there on the other side.
  uint32_t switch_at(uint32_t b, uint32_t depth) const { return iterate ? depth : std::min(depth, 2 * (b + 2)); }
  uint32_t after(uint32_t b, uint32_t mine) const { return iterate ? 0 : block + (b + 2) * col_blocks + 2 * mine; }
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
  uint32_t tiles(int phase) const {  // symmetric results: on and below the diagonal
    const uint32_t r = (rows + 1) / 2, c = (cols + 1) / 2;
    return phase == kNext ? r * c : r * (r + 1) / 2;
  }
  MuonTile tile(int phase, uint32_t r, uint32_t c) const {
    MuonTile t = {};
    t.phase = static_cast<uint32_t>(phase);
    const bool narrow = c + 1 == cols, second = r + 1 < rows;
    t.a[0] = a.first(r);
    // (beyond an odd number of blocks of rows: the last one again, its results are dropped)
    t.a[1] = a.first(second ? r + 1 : r);
    t.b[0] = b.first(c);
    // (a narrow tile's CTAs have 64 rows or columns each, of rows the halves of a block)
    t.b[1] = !narrow ? b.first(c + 1) : b.first(c) + (b.by_columns ? 1 : 0);
    t.a_switch = a.switch_at(r, depth);
    t.b_switch = b.switch_at(c, depth);
    for (uint32_t k = 0; k < 2; ++k) {
      t.a_after[k] = a.after(r, second ? r + k : r);
      t.b_after[k] = b.after(c, c + k);  // (a narrow tile is the last one, whose blocks do not change sides)
    }
    t.a_next = a.by_columns ? a.col_blocks : 1;
    t.b_next = b.by_columns ? b.col_blocks : 1;
    t.square = square;
    t.depth = depth;
    t.flags = (narrow ? kNarrow : 0) | (a.by_columns ? kAColumns : 0) | (b.by_columns ? kBColumns : 0) | (second ? kSecond : 0) |
              (a.iterate ? kAIterate : 0) | (b.iterate ? kBIterate : 0);
    t.across = 2 * cols;
    t.out = out + r * t.across + 2 * c;
    t.row = static_cast<uint16_t>(r);
    t.col = static_cast<uint16_t>(c);
    return t;
  }
};

// The tiles of an iteration over the matrices that are split, or those that are not: S of all, then P, then X, in each those with the longest contraction first.  ends: where each phase's end.
inline void plan_tiles(const std::vector<MuonDesc>& descs, bool split, std::vector<MuonTile>& tiles, uint32_t (&ends)[kPhases]) {
  for (int phase = 0; phase < kPhases; ++phase) {
    std::vector<ProductOf> all;
    for (const MuonDesc& d : descs) all.emplace_back(phase, d);
    std::vector<uint32_t> order;
    for (uint32_t m = 0; m < descs.size(); ++m)
      if ((descs[m].split != 0) == split) order.push_back(m);
    std::stable_sort(order.begin(), order.end(), [&](uint32_t x, uint32_t y) { return all[x].depth > all[y].depth; });
    for (uint32_t m : order) {
      const ProductOf& q = all[m];
      const int from = (phase + kPhases - 1) % kPhases;
      const uint32_t needs = m * kPhases + from, count = kSignals * ProductOf(from, descs[m]).tiles(from);
      auto add = [&](uint32_t r, uint32_t c) {
        MuonTile t = q.tile(phase, r, c);
        t.done = m * kPhases + phase;
        t.needs = needs;
        t.count = count;
        tiles.push_back(t);
      };
      if (phase == kNext && !descs[m].tall) {  // (tiles that share the long side's blocks one after the other)
        for (uint32_t c = 0; c < q.cols; c += 2)
          for (uint32_t r = 0; r < q.rows; r += 2) add(r, c);
      } else {
        for (uint32_t r = 0; r < q.rows; r += 2)
          for (uint32_t c = 0; c < (phase == kNext ? q.cols : r + 1); c += 2) add(r, c);
      }
    }
    ends[phase] = static_cast<uint32_t>(tiles.size());
  }
}

}  // namespace frk
