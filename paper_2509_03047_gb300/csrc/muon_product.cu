// muon_product.cu -- the products of the orthogonalised update, all matrices of a
// list in one launch.
#include <cuda_runtime.h>

#include "kernels.h"
#include "muon_block.cuh"

namespace frk {

namespace {

// A product's factors as D[i][j] = sum over k of A(i, k) B(j, k): each a matrix of the workspace, read by its rows or by its columns.
struct Factor {
  const uint8_t* at;
  uint32_t col_blocks;
  bool by_columns;
  __device__ __forceinline__ float get(uint32_t i, uint32_t k) const {
    const uint32_t r = by_columns ? k : i, c = by_columns ? i : k;
    return __half2float(*reinterpret_cast<const __half*>(at + chunk_at(col_blocks, r, c / 8) + c % 8 * 2));
  }
};

template <int kPhase>
__global__ void __launch_bounds__(256) product_kernel(const __grid_constant__ MuonProduct p) {
  __shared__ float a[16][kTile + 1], b[16][kTile + 1];
  wait_for_kernel_before();
  if (p.clip != nullptr && p.clip->nonfinite != 0) return;
  const MuonTile t = p.tiles[blockIdx.x];
  const MuonDesc& d = p.tensors[t.tensor];
  const Factor x = {p.work + d.x[p.from], d.col_blocks, (kPhase == kGram) == (d.tall != 0)};
  Factor f = x, g = x;
  if (kPhase == kPoly) f = g = {p.work + d.s, 2 * d.side_blocks, false};
  if (kPhase == kNext) {
    const Factor q = {p.work + d.p, 2 * d.side_blocks, false};
    f = d.tall ? Factor{x.at, x.col_blocks, false} : q;
    g = d.tall ? q : Factor{x.at, x.col_blocks, true};
  }
  const uint32_t depth = kPhase == kGram ? (d.tall ? d.row_blocks * kBlockRows : d.col_blocks * kBlockCols) : d.side_blocks * 128;
  const uint32_t i0 = t.row * kTile, j0 = t.col * kTile;
  const int row = threadIdx.x / 8, col = threadIdx.x % 8;  // two rows, 32 apart, of eight columns
  float sum[2][8] = {};
  for (uint32_t k0 = 0; k0 < depth; k0 += 16) {
    for (int q = threadIdx.x; q < 16 * kTile; q += 256) {
      const int k = q % 16, i = q / 16;
      a[k][i] = f.get(i0 + i, k0 + k);
      b[k][i] = g.get(j0 + i, k0 + k);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sum[0][j] += a[k][row] * b[k][col * 8 + j];
        sum[1][j] += a[k][row + 32] * b[k][col * 8 + j];
      }
    __syncthreads();
  }
  finish_chunk<kPhase>(p, d, i0 + row, j0 / 8 + col, sum[0]);
  finish_chunk<kPhase>(p, d, i0 + row + 32, j0 / 8 + col, sum[1]);
}

}  // namespace

void plan_tiles(const std::vector<MuonDesc>& descs, std::vector<MuonTile> (&tiles)[kPhases]) {
  for (uint32_t t = 0; t < descs.size(); ++t) {
    const MuonDesc& d = descs[t];
    auto all = [&](int phase, uint32_t rows, uint32_t cols) {
      for (uint32_t r = 0; r < rows / kTile; ++r)
        for (uint32_t c = 0; c < cols / kTile; ++c) tiles[phase].push_back({t, static_cast<uint16_t>(r), static_cast<uint16_t>(c)});
    };
    all(kGram, d.side_blocks * 128, d.side_blocks * 128);
    all(kPoly, d.side_blocks * 128, d.side_blocks * 128);
    all(kNext, d.row_blocks * kBlockRows, d.col_blocks * kBlockCols);
  }
}

cudaError_t launch_muon_product(int phase, const MuonProduct& p, cudaStream_t s) {
  auto* const kernel = phase == kGram ? product_kernel<kGram> : phase == kPoly ? product_kernel<kPoly> : product_kernel<kNext>;
  return launch_chained(kernel, static_cast<int>(p.n_tiles), 256, 0, s, p);
}

}  // namespace frk
