// Rows of odd length are copied by 16-byte granules (csrc/embed.h, as embed_sum.cu
// copies them): no granule of a row that goes that way lies outside its buffer, for
// buffers at any element's boundary, of one row to many, and every row's elements are
// covered.  Without a GPU.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "embed.h"

using namespace frk;

#define CHECK(x) do { if (!(x)) { std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)

int main() {
  std::mt19937_64 rng(6);
  auto below = [&](uint64_t n) { return rng() % n; };
  const uint32_t width = static_cast<uint32_t>(tile_width(kOdd));
  uint64_t by = 0, beyond = 0;
  for (int round = 0; round < 20000; ++round) {
    const uint32_t size = below(2) ? 2 : 4;
    const uint64_t dim = kOddLeast + 1 + below(below(2) ? 8 : 1200), rows = 1 + below(8), base = (1 << 20) + size * below(40);
    const uint64_t end = base + rows * dim * size;
    for (uint64_t row = 0; row < rows; ++row)
      for (uint64_t first = 0; first < dim; first += width) {
        const Granules g(base, row, dim, first, width, size);
        const uint64_t from = base + (row * dim + first) * size, last = g.begin + (g.bytes + 15) / 16 * 16;
        CHECK(g.begin % 16 == 0 && g.begin <= from && from - g.begin < 16);
        CHECK(g.begin + g.bytes == from + (dim - first < width ? dim - first : width) * size);
        const bool inside = g.begin >= base && last <= end;
        if (by_granules(row, rows)) {
          CHECK(inside);
          ++by;
        }
        beyond += !inside;
      }
  }
  CHECK(by > 1000 && beyond > 1000);  // both come up
  std::printf("embed_granules ok\n");
  return 0;
}
