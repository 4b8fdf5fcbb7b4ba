// embed_lookup.cu -- rows of the table for a batch of tokens.
//
// A thread has vectors of elements of the output, kEach of them a block's width
// apart: its tokens, then its table's vectors are on their way together.
//
// Bound by writing the output: 32,768 tokens of 4,096 in bf16, half of them in the
// slice of 16,032 rows, 44 us, 95% of the copy rate for what it needs.  (28 bytes per
// thread are spilled in the kernels of vectors of 8 bf16 elements, and of 4 fp32 ones to
// bf16, which keep 40 registers for six CTAs per SM: within these 5%.)
#include <cuda_runtime.h>

#include "embed.h"
#include "embed_vector.cuh"
#include "kernels.h"

namespace frk {

namespace {

constexpr int kThreads = 256, kEach = 4;

template <int V, bool Bf16Table, bool Bf16Out>
__global__ void __launch_bounds__(kThreads) lookup_kernel(const __grid_constant__ LookupParams p) {
  wait_for_kernel_before();
  const uint64_t across = p.dim / V, all = p.tokens.n * across;
  const uint64_t start = static_cast<uint64_t>(blockIdx.x) * (kThreads * kEach) + threadIdx.x;
  uint64_t row[kEach], column[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const uint64_t i = start + k * kThreads;
    // (a 64-bit division where the batch needs it)
    const uint64_t token = all >> 32 ? i / across : static_cast<uint32_t>(i) / static_cast<uint32_t>(across);
    column[k] = (i - token * across) * V;
    row[k] = i < all ? p.tokens.row(token) : p.tokens.rows;
  }
  Raw<V, Bf16Table> in[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k)
    if (row[k] < p.tokens.rows) in[k].load(p.table, row[k] * p.dim + column[k]);
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const uint64_t i = start + k * kThreads;
    if (i >= all) break;
    Raw<V, Bf16Out> out;
    if (row[k] < p.tokens.rows) {
      float x[V];
      in[k].get(x);
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] *= p.scale;
      out.set(x);
    } else {
      out.clear();
    }
    out.store(p.out, i * V);
  }
}

// Vectors of few elements: a warp has a row, so that no vector's place takes a division.  bf16, 100 million elements, rows of 101, 321, 1,001, 4,999
// elements, us: 74, 181, 179, 180 by flat vectors, 51, 76, 66, 83 by rows; of 37 elements 27 and 57 (few are on their way); by 12 or 16 at a time 72
// to 109.  Vectors of 4 or 8 are faster flat (rows of 256: 44, by rows 110).
constexpr int kRowEach = 6;
constexpr uint64_t kRowLeast = 64;
template <int V, bool Bf16Table, bool Bf16Out>
__global__ void __launch_bounds__(kThreads) row_kernel(const __grid_constant__ LookupParams p) {
  wait_for_kernel_before();
  const uint64_t i = static_cast<uint64_t>(blockIdx.x) * (kThreads / 32) + threadIdx.x / 32;
  if (i >= p.tokens.n) return;
  const uint64_t row = p.tokens.row(i), to = i * p.dim, from = row * p.dim;
  const bool there = row < p.tokens.rows;
  for (uint64_t first = threadIdx.x % 32 * V; first < p.dim; first += 32 * V * kRowEach) {
    Raw<V, Bf16Table> in[kRowEach];
#pragma unroll
    for (int k = 0; k < kRowEach; ++k)
      if (there && first + k * 32 * V < p.dim) in[k].load(p.table, from + first + k * 32 * V);
#pragma unroll
    for (int k = 0; k < kRowEach; ++k) {
      if (first + k * 32 * V >= p.dim) break;
      Raw<V, Bf16Out> out;
      if (there) {
        float x[V];
        in[k].get(x);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] *= p.scale;
        out.set(x);
      } else {
        out.clear();
      }
      out.store(p.out, to + first + k * 32 * V);
    }
  }
}

template <int V>
cudaError_t launch(const LookupParams& p, cudaStream_t s) {
  if constexpr (V <= 2) {
    if (p.dim / V > kRowLeast) {
      const uint64_t ctas = (p.tokens.n + kThreads / 32 - 1) / (kThreads / 32);
      auto* const kernel = p.bf16_table ? (p.bf16_out ? row_kernel<V, true, true> : row_kernel<V, true, false>)
                                        : (p.bf16_out ? row_kernel<V, false, true> : row_kernel<V, false, false>);
      return launch_chained(kernel, static_cast<int>(ctas), kThreads, 0, s, p);
    }
  }
  const uint64_t all = p.tokens.n * (p.dim / V), ctas = (all + kThreads * kEach - 1) / (kThreads * kEach);
  if (ctas > 0x7FFFFFFF) return cudaErrorInvalidValue;
  auto* const kernel = p.bf16_table ? (p.bf16_out ? lookup_kernel<V, true, true> : lookup_kernel<V, true, false>)
                                    : (p.bf16_out ? lookup_kernel<V, false, true> : lookup_kernel<V, false, false>);
  return launch_chained(kernel, static_cast<int>(ctas), kThreads, 0, s, p);
}

}  // namespace

cudaError_t launch_lookup(const LookupParams& p, cudaStream_t s) {
  switch (vector_elems(p.dim, p.table, p.bf16_table ? 2 : 4, p.out, p.bf16_out ? 2 : 4)) {
    case 8: return launch<8>(p, s);
    case 4: return launch<4>(p, s);
    case 2: return launch<2>(p, s);
    default: return launch<1>(p, s);
  }
}

}  // namespace frk
