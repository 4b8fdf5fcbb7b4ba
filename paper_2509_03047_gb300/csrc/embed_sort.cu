// embed_sort.cu -- the tokens of a batch that fall into the slice, sorted by row
// and, within a row, in the batch's order.
//
// Counting sort by digits of up to 11 bits, the lowest first.  A pass counts each
// CTA's digits, then every CTA finds its places by adding up the counts of the
// CTAs before it, and a token's among its CTA's by warps in turn: a warp's tokens
// of one digit are found by a vote, those of the warps before by a table of counts
// per warp and digit.  Nothing depends on the order in which anything runs.
#include <cuda_runtime.h>

#include "embed.h"
#include "kernels.h"

namespace frk {

namespace {

constexpr int kWarps = kSortThreads / 32;
constexpr uint32_t kAll = 0xFFFFFFFFu;

// Exclusive sums over `n` (a power of two, at most 2 kSortThreads) counts in shared memory; every thread calls.
__device__ __forceinline__ uint32_t scan(uint32_t* x, uint32_t n, uint32_t* warps) {
  const uint32_t t = threadIdx.x, lane = t % 32;
  const uint32_t a = 2 * t < n ? x[2 * t] : 0, b = 2 * t + 1 < n ? x[2 * t + 1] : 0;
  uint32_t sum = a + b;
#pragma unroll
  for (int k = 1; k < 32; k *= 2) {
    const uint32_t y = __shfl_up_sync(kAll, sum, k);
    if (lane >= k) sum += y;
  }
  if (lane == 31) warps[t / 32] = sum;
  __syncthreads();
  if (t < 32) {
    uint32_t w = warps[t];
#pragma unroll
    for (int k = 1; k < 32; k *= 2) {
      const uint32_t y = __shfl_up_sync(kAll, w, k);
      if (lane >= k) w += y;
    }
    warps[t] = w;
  }
  __syncthreads();
  const uint32_t before = (t >= 32 ? warps[t / 32 - 1] : 0) + sum - a - b;
  if (2 * t < n) x[2 * t] = before;
  if (2 * t + 1 < n) x[2 * t + 1] = before + a;
  const uint32_t total = warps[kWarps - 1];
  __syncthreads();
  return total;
}

struct Shared {
  uint32_t* base;    // per digit: where the CTA's next token of it goes
  uint16_t* before;  // per warp and digit
  uint32_t* warps;
  __device__ Shared(uint8_t* at, uint32_t bins)
      : base(reinterpret_cast<uint32_t*>(at)), before(reinterpret_cast<uint16_t*>(at + bins * 4)),
        warps(reinterpret_cast<uint32_t*>(at + bins * (4 + kWarps * 2))) {}
};
size_t shared_bytes(uint32_t bins) { return bins * (4 + kWarps * 2) + kWarps * 4; }

// Each token's place among the tile's of its digit, and the tile's counts per warp, then sums over the warps before in their place; totals
// per digit by `add(digit, total)`.  digit >= bins: no token.  A warp's tokens are consecutive, the lanes' in turn.
template <class Add>
__device__ __forceinline__ void rank_tile(const Shared& sh, uint32_t bins, const uint32_t (&digit)[kSortEach], uint32_t (&rank)[kSortEach], Add add) {
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  uint16_t* mine = sh.before + warp * bins;
  for (uint32_t i = lane; i < bins; i += 32) mine[i] = 0;
  __syncwarp();
#pragma unroll
  for (int k = 0; k < kSortEach; ++k) {
    const uint32_t same = __match_any_sync(kAll, digit[k]);
    const uint32_t earlier = digit[k] < bins ? mine[digit[k]] : 0;
    rank[k] = earlier + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (digit[k] < bins && lane == 31 - __clz(same)) mine[digit[k]] = static_cast<uint16_t>(rank[k] + 1);
    __syncwarp();
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < bins; i += kSortThreads) {
    uint32_t sum = 0;
#pragma unroll 8
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t n = sh.before[w * bins + i];
      sh.before[w * bins + i] = static_cast<uint16_t>(sum);
      sum += n;
    }
    add(i, sum);
  }
  __syncthreads();
}

// The token of place i in a tile as a thread has it: warps take 32 * kSortEach consecutive ones.
__device__ __forceinline__ uint32_t tile_index(int k) { return (threadIdx.x / 32 * kSortEach + k) * 32 + threadIdx.x % 32; }

template <bool First>
__device__ __forceinline__ Met get(const SortParams& p, uint64_t i) {
  if (!First) return p.sorted[(p.pass + 1) % 2][i];
  const uint64_t row = p.tokens.row(i);
  return {row < p.tokens.rows ? static_cast<uint32_t>(row) : kAll, static_cast<uint32_t>(i)};
}
__device__ __forceinline__ uint32_t digit_of(const SortParams& p, int pass, uint32_t row) {
  return row == kAll ? kAll : row >> (pass * p.bits) & ((1u << p.bits) - 1);
}

template <bool First>
__global__ void __launch_bounds__(kSortThreads) count_kernel(const __grid_constant__ SortParams p) {
  __shared__ uint32_t counts[1 << kMostDigit];
  const uint32_t bins = 1u << p.bits;
  for (uint32_t i = threadIdx.x; i < bins; i += kSortThreads) counts[i] = 0;
  wait_for_kernel_before();
  __syncthreads();
  const uint64_t n = First ? p.tokens.n : *p.found, begin = blockIdx.x * p.share, end = min(begin + p.share, n);
  for (uint64_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
    const Met m = get<First>(p, i);
    if (m.row == kAll) continue;
    atomicAdd(counts + digit_of(p, p.pass, m.row), 1u);
    if (First && p.met != nullptr) p.met[m.row] = 1;
  }
  if (First && blockIdx.x == 0 && threadIdx.x == 0) *p.n_long = 0;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < bins; i += kSortThreads) p.counts[static_cast<uint64_t>(blockIdx.x) * bins + i] = counts[i];
}

template <bool First>
__global__ void __launch_bounds__(kSortThreads) place_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ __align__(16) uint8_t raw[];
  const uint32_t bins = 1u << p.bits;
  const Shared sh(raw, bins);
  wait_for_kernel_before();
  // (up to two digits per thread)
  uint32_t before[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t i = threadIdx.x + j * kSortThreads;
    if (i >= bins) break;
    uint32_t total = 0;
#pragma unroll 16
    for (uint32_t c = 0; c < p.ctas; ++c) {
      if (c == blockIdx.x) before[j] = total;
      total += p.counts[static_cast<uint64_t>(c) * bins + i];
    }
    sh.base[i] = total;
  }
  __syncthreads();
  const uint32_t found = scan(sh.base, bins, sh.warps);
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if (threadIdx.x + j * kSortThreads < bins) sh.base[threadIdx.x + j * kSortThreads] += before[j];
  if (First && blockIdx.x == 0 && threadIdx.x == 0) *p.found = found;
  __syncthreads();
  const uint64_t n = First ? p.tokens.n : *p.found, begin = blockIdx.x * p.share, end = min(begin + p.share, n);
  for (uint64_t at = begin; at < end; at += kSortTile) {
    Met m[kSortEach];
    uint32_t digit[kSortEach], rank[kSortEach], place[kSortEach];
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      const uint64_t i = at + tile_index(k);
      m[k] = i < end ? get<First>(p, i) : Met{kAll, 0};
      digit[k] = digit_of(p, p.pass, m[k].row);
    }
    uint32_t totals[2] = {0, 0};
    rank_tile(sh, bins, digit, rank, [&](uint32_t i, uint32_t total) { totals[i >= kSortThreads] = total; });
#pragma unroll
    for (int k = 0; k < kSortEach; ++k)
      place[k] = digit[k] != kAll ? sh.base[digit[k]] + sh.before[threadIdx.x / 32 * bins + digit[k]] + rank[k] : 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (threadIdx.x + j * kSortThreads < bins) sh.base[threadIdx.x + j * kSortThreads] += totals[j];
#pragma unroll
    for (int k = 0; k < kSortEach; ++k)
      if (digit[k] != kAll) p.sorted[p.pass % 2][place[k]] = m[k];
    // (rank_tile's barriers come between these sums and their next use)
  }
}

// A batch of one tile: all passes in one CTA.
__global__ void __launch_bounds__(kSortThreads) small_kernel(const __grid_constant__ SortParams p, int passes) {
  extern __shared__ __align__(16) uint8_t raw[];
  const uint32_t bins = 1u << p.bits;
  Met* const tile = reinterpret_cast<Met*>(raw);
  const Shared sh(raw + kSortTile * sizeof(Met), bins);
  wait_for_kernel_before();
  uint32_t n = static_cast<uint32_t>(p.tokens.n);
  for (int pass = 0; pass < passes; ++pass) {
    Met m[kSortEach];
    uint32_t digit[kSortEach], rank[kSortEach];
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      const uint32_t i = tile_index(k);
      m[k] = i < n ? (pass == 0 ? get<true>(p, i) : tile[i]) : Met{kAll, 0};
      digit[k] = digit_of(p, pass, m[k].row);
      if (pass == 0 && p.met != nullptr && m[k].row != kAll) p.met[m[k].row] = 1;
    }
    rank_tile(sh, bins, digit, rank, [&](uint32_t i, uint32_t total) { sh.base[i] = total; });
    n = scan(sh.base, bins, sh.warps);
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      if (digit[k] == kAll) continue;
      const uint32_t to = sh.base[digit[k]] + sh.before[threadIdx.x / 32 * bins + digit[k]] + rank[k];
      if (pass + 1 < passes)
        tile[to] = m[k];
      else
        p.sorted[0][to] = m[k];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    *p.found = n;
    *p.n_long = 0;
  }
}

}  // namespace

cudaError_t configure_sort() {
  const int big = static_cast<int>(shared_bytes(1u << kMostDigit));
  cudaError_t e = cudaFuncSetAttribute(place_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, big);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(place_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, big);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, big + kSortTile * static_cast<int>(sizeof(Met)));
  return e;
}

cudaError_t launch_sort(SortParams p, const SortPlan& plan, int* last, cudaStream_t s) {
  p.bits = plan.bits;
  if (p.tokens.n <= kSortTile) {
    *last = 0;
    return launch_chained(small_kernel, 1, kSortThreads, shared_bytes(plan.bins()) + kSortTile * sizeof(Met), s, p, plan.passes);
  }
  p.share = (p.tokens.n + kSortCtas - 1) / kSortCtas;
  p.share = p.share < kSortShare ? kSortShare : (p.share + kSortTile - 1) / kSortTile * kSortTile;
  p.ctas = static_cast<uint32_t>((p.tokens.n + p.share - 1) / p.share);
  for (p.pass = 0; p.pass < plan.passes; ++p.pass) {
    cudaError_t e = launch_chained(p.pass == 0 ? count_kernel<true> : count_kernel<false>, static_cast<int>(p.ctas), kSortThreads, 0, s, p);
    if (e == cudaSuccess)
      e = launch_chained(p.pass == 0 ? place_kernel<true> : place_kernel<false>, static_cast<int>(p.ctas), kSortThreads, shared_bytes(plan.bins()), s, p);
    if (e != cudaSuccess) return e;
  }
  *last = (plan.passes - 1) % 2;
  return cudaSuccess;
}

}  // namespace frk
