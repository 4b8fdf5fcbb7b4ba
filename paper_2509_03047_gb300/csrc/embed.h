// embed.h -- the embedding's plan and kernel launchers (internal to libflashrec).
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/flashrec.h"
#include "optim.h"

namespace frk {

// A batch's tokens: 4 or 8 bytes each.  Row of the slice, or rows and above.
struct Tokens {
  const void* at;
  uint64_t n;
  uint64_t first, rows;
  uint32_t wide;
#ifdef __CUDACC__
  __device__ __forceinline__ uint64_t row(uint64_t i) const {
    const int64_t t = wide ? static_cast<const int64_t*>(at)[i] : static_cast<const int32_t*>(at)[i];
    return static_cast<uint64_t>(t) - first;
  }
#endif
};

// ---- lookup

struct LookupParams {
  Tokens tokens;
  const void* table;
  void* out;
  uint64_t dim;
  float scale;
  uint32_t bf16_table, bf16_out;
};
cudaError_t launch_lookup(const LookupParams& p, cudaStream_t s);

// Elements that move together, so that a vector of `a` and one of `b` start on the boundaries of their loads and stores.
inline int vector_elems(uint64_t dim, const void* a, uint32_t a_bytes, const void* b, uint32_t b_bytes) {
  for (int v = 8; v > 1; v /= 2) {
    auto on = [&](const void* p, uint32_t bytes) { return reinterpret_cast<uintptr_t>(p) % (v * bytes < 16 ? v * bytes : 16) == 0; };
    if (dim % v == 0 && on(a, a_bytes) && on(b, b_bytes)) return v;
  }
  return 1;
}

// ---- the batch's tokens of the slice, sorted by row, in their order within a row

struct Met {  // a token of the batch
  uint32_t row, at;
};
constexpr int kSortThreads = 1024, kSortEach = 4, kSortTile = kSortThreads * kSortEach;
constexpr uint64_t kCompareTokens = 4096;  // a batch of up to this many is sorted by comparing each with all
constexpr uint32_t kSortCluster = 16;  // CTAs that sort a batch of up to a tile for each in one launch
constexpr uint64_t kClusterTokens = static_cast<uint64_t>(kSortCluster) * kSortTile;
constexpr uint32_t kSortCtas = 128;    // of a larger batch's launches
constexpr uint64_t kFillShare = 128 << 10;  // bytes per CTA
constexpr int kMostDigit = 9;          // bits of a pass

struct SortPlan {
  int passes, bits;  // bits of a pass
  uint32_t bins() const { return 1u << bits; }
};
inline SortPlan sort_plan(uint64_t rows) {
  int bits = 1;
  while (bits < 31 && (1ull << bits) < rows) ++bits;
  const int passes = (bits + kMostDigit - 1) / kMostDigit;
  return {passes, (bits + passes - 1) / passes};
}
struct SortParams {
  Tokens tokens;
  Met* sorted[2];   // the passes' results in turn
  uint32_t* counts; // per CTA and bin
  uint32_t* found;  // tokens of the slice
  uint32_t* n_long; // set to zero
  uint64_t share;   // tokens per CTA
  uint32_t ctas;
  uint8_t* fill;    // zeros go here, by CTAs of the first launch beyond the sort's: the gradient's rows before some are written
  uint64_t fill_bytes;
  int each;         // tokens per thread and tile
  int bits;
  int pass;
};
cudaError_t configure_sort();
// All passes; the result is sorted[last].
cudaError_t launch_sort(SortParams p, const SortPlan& plan, int* last, cudaStream_t s);

// ---- the gradient

// How a warp's lanes share a tile of columns.  Vectors of 8, 4, 2, 1 elements, 32 vectors apart; kOdd: rows that do not start on vectors'
// boundaries, by the 16-byte granules around them.  kWide: two vectors of 8.
constexpr int kOdd = 0, kWide = 16;
constexpr int vector_of(int v) { return v == kOdd ? 1 : v == kWide ? 8 : v; }
constexpr int lane_vectors(int v) { return v == kOdd ? 12 : v == kWide ? 2 : v == 8 ? 1 : v == 4 ? 2 : 4; }
constexpr int tile_width(int v) { return 32 * vector_of(v) * lane_vectors(v); }
// The granules around a row's columns from `first` on, `width` of them at most: 16 bytes at `begin` and so on, as many as `bytes` reaches into.
struct Granules {
  uint64_t begin;
  uint32_t bytes;
#ifdef __CUDACC__
  __host__ __device__ __forceinline__
#endif
  Granules(uint64_t base, uint64_t row, uint64_t dim, uint64_t first, uint32_t width, uint32_t size) {
    const uint64_t from = base + (row * dim + first) * size, left = dim - first;
    begin = from & ~15ull;
    bytes = (static_cast<uint32_t>(from) & 15) + static_cast<uint32_t>(left < width ? left : width) * size;
  }
};
// Whether they lie in a buffer of `rows` rows: those of its first and last row may reach beyond it, where memory is somebody else's.  (A row has
// more than kOddLeast elements, so no other row's do.)
#ifdef __CUDACC__
__host__ __device__ __forceinline__
#else
inline
#endif
bool by_granules(uint64_t row, uint64_t rows) { return row != 0 && row + 1 != rows; }
// The sorted tokens are cut into ranges of equal length, one for a warp per tile of columns; a multiple of what a CTA has.
constexpr uint32_t kSumWarps = 8;
// Ranges times column tiles, about.  A range has its fixed cost (the tokens at its borders, its part), some 5 us: one wave of them is best for odd
// rows and for wide ones that are added to, three where a token costs a warp little or rows' writes are spread unevenly.  GB300, per SM 16, 24,
// 32, 48, 72 warps, us: 500,001 tokens x 321 fp32 155, 159, 173, 182, 215; 32,768 x 768 accumulating 45.6, 48.3, 48.0, 48.5, 48.0; 300,000 x 8
// accumulating 88, -, -, 72, -; 65,536 x 4,096 137, 153, -, 129, 129.
constexpr uint32_t kFewRangeWarps = kSms * 16, kRangeWarps = kSms * 48;
constexpr uint32_t kLeastRange = 32, kShortRange = 8;  // tokens: of a range, of one where a wave of them is not full
// Rows of odd length up to this go element by element, a lane's four at most.
constexpr uint64_t kOddLeast = 128;
// From here on a warp takes 1 KiB or more of a row, not half of it: 65,536 tokens of 4,096 130 -> 123 us (of 768 45 -> 52).
constexpr uint64_t kWideLeast = 1024;
inline int kind_of(uint64_t dim, int vector) { return vector == 1 && dim > kOddLeast ? kOdd : vector == 8 && dim >= kWideLeast ? kWide : vector; }
inline uint32_t column_tiles(uint64_t dim, int v) { return static_cast<uint32_t>((dim + tile_width(v) - 1) / tile_width(v)); }
// (Of the sizes alone, not of the kind that a call's addresses allow: which tokens of a long row are added together depends on it.)
inline uint32_t ranges_of(uint64_t n, uint64_t dim, bool accumulate) {
  const int v = kind_of(dim, vector_elems(dim, nullptr, 2, nullptr, 2));
  const uint32_t tiles = column_tiles(dim, v);
  const bool few = v == kOdd || (accumulate && tiles > 1);
  auto share = [](uint64_t x, uint64_t of) { return (x + of - 1) / of; };
  const uint64_t wave = share(kFewRangeWarps, tiles), fill = few ? wave : share(kRangeWarps, tiles), whole = share(n, kLeastRange),
                 brief = share(n, kShortRange) < wave ? share(n, kShortRange) : wave;
  const uint64_t most = whole > brief ? whole : brief;
  const uint64_t ranges = share(most < fill ? most : fill, kSumWarps) * kSumWarps;
  return static_cast<uint32_t>(ranges > kSumWarps ? ranges : kSumWarps);
}
struct SumParams {
  const Met* sorted;
  const uint32_t* found;
  uint32_t* n_long;  // rows in several CTAs' parts
  uint32_t* longs;   // the CTA where each begins
  float* parts;      // two rows per CTA
  const void* out;
  void* grad;
  uint64_t dim, rows, n;  // n rows of out
  float scale;
  uint32_t ranges, tiles;
  uint32_t ctas, zero_ctas;
  uint32_t rows_per_zero_warp;
  uint32_t accumulate;
  uint32_t configure;  // 1: no launch, the kernel's shared-memory size is set
  uint32_t bf16_out, bf16_grad;
  int v;
};
cudaError_t configure_sum();
cudaError_t launch_sum(const SumParams& p, cudaStream_t s);

}  // namespace frk
