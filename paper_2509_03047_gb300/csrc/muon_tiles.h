// muon_tiles.h -- the tiles of the products, on the host.
#pragma once

#include <algorithm>
#include <numeric>
#include <vector>

#include "muon.h"

namespace frk {

// The tiles of each phase's products, those with the longest contraction first, so that the last to be started are short.
inline void plan_tiles(const std::vector<MuonDesc>& descs, std::vector<MuonTile> (&tiles)[kPhases]) {
  for (int phase = 0; phase < kPhases; ++phase) {
    std::vector<uint32_t> order(descs.size());
    std::iota(order.begin(), order.end(), 0u);
    auto depth = [&](uint32_t t) {
      const MuonDesc& d = descs[t];
      return phase == kGram ? (d.tall ? d.row_blocks : d.col_blocks / 2) : d.side_blocks;
    };
    std::stable_sort(order.begin(), order.end(), [&](uint32_t a, uint32_t b) { return depth(a) > depth(b); });
    for (uint32_t t : order) {
      const MuonDesc& d = descs[t];
      const uint32_t rows = phase == kNext ? d.row_blocks : d.side_blocks, cols = phase == kNext ? d.col_blocks / 2 : d.side_blocks;
      // (tiles that share the long side's blocks one after the other)
      auto add = [&](uint32_t r, uint32_t c) {
        if (phase == kNext || c <= r) tiles[phase].push_back({t, static_cast<uint16_t>(r), static_cast<uint16_t>(c), c + 1 < cols});
      };
      if (phase == kNext && !d.tall) {
        for (uint32_t c = 0; c < cols; c += 2)
          for (uint32_t r = 0; r < rows; r += 2) add(r, c);
      } else {
        for (uint32_t r = 0; r < rows; r += 2)
          for (uint32_t c = 0; c < cols; c += 2) add(r, c);
      }
    }
  }
}

}  // namespace frk
