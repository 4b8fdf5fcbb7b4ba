// embed_sort.cu -- the tokens of a batch that fall into the slice, sorted by row
// and, within a row, in the batch's order.
//
// Counting sort by digits of up to 9 bits, the lowest first.  A pass counts each
// CTA's digits, then every CTA finds its places by adding up the counts of the
// CTAs before it, and a token's among its CTA's by warps in turn: a warp's tokens
// of one digit are found by a vote, those of the warps before by a table of counts
// per warp and digit.  Nothing depends on the order in which anything runs.
//
// A batch of up to 4,096 tokens is sorted by comparing each with all, one of up to
// 65,536 in one launch, by a cluster of CTAs that read each other's counts from shared
// memory; a larger one by two launches per pass.
//
// Bound by latencies (a pass: tokens, votes, the counts of all CTAs, the places, 8
// us): 32,768 tokens 18 us, 65,536 20, 500,001 of 259 rows 24.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "embed.h"
#include "kernels.h"

namespace frk {

namespace {

constexpr int kWarps = kSortThreads / 32;
constexpr uint32_t kAll = 0xFFFFFFFFu;

static_assert((1 << kMostDigit) <= kSortThreads, "a thread has a digit");

// Exclusive sums over `n` (at most kSortThreads) counts in shared memory; every thread calls.
__device__ __forceinline__ uint32_t scan(uint32_t* x, uint32_t n, uint32_t* warps) {
  const uint32_t t = threadIdx.x, lane = t % 32;
  const uint32_t a = t < n ? x[t] : 0;
  uint32_t sum = a;
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
  if (t < n) x[t] = (t >= 32 ? warps[t / 32 - 1] : 0) + sum - a;
  const uint32_t total = warps[kWarps - 1];
  __syncthreads();
  return total;
}

struct Shared {
  uint32_t* base;    // per digit: where the CTA's next token of it goes
  uint32_t* totals;  // per digit: of the tile
  uint32_t* warps;
  uint16_t* before;  // per warp and digit
  __device__ Shared(uint8_t* at, uint32_t bins)
      : base(reinterpret_cast<uint32_t*>(at)), totals(base + bins), warps(totals + bins), before(reinterpret_cast<uint16_t*>(warps + kWarps)) {}
};
size_t shared_bytes(uint32_t bins) { return bins * (8 + kWarps * 2) + kWarps * 4; }

// The lanes with this lane's digit (kAll: no token), for each of its tokens: a vote per bit, the tokens' votes side by side.
__device__ __forceinline__ void same_digit(const uint32_t (&digit)[kSortEach], int bits, uint32_t (&same)[kSortEach]) {
#pragma unroll
  for (int k = 0; k < kSortEach; ++k) {
    const uint32_t there = __ballot_sync(kAll, digit[k] != kAll);
    same[k] = digit[k] != kAll ? there : ~there;
  }
  for (int b = 0; b < bits; ++b) {
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      const bool set = digit[k] >> b & 1;
      const uint32_t ones = __ballot_sync(kAll, set);
      same[k] &= set ? ones : ~ones;
    }
  }
}

// Each token's place among the tile's of its digit, and the tile's counts per warp, then sums over the warps before in their place, and totals.
// digit >= bins: no token.  A warp's tokens are consecutive, the lanes' in turn.
__device__ __forceinline__ void rank_tile(const Shared& sh, uint32_t bins, int bits, int each, const uint32_t (&digit)[kSortEach], uint32_t (&rank)[kSortEach]) {
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  uint16_t* mine = sh.before + warp * bins;
  for (uint32_t i = lane; i < bins / 2; i += 32) reinterpret_cast<uint32_t*>(mine)[i] = 0;
  uint32_t same[kSortEach];
  same_digit(digit, bits, same);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < kSortEach; ++k) {
    if (k >= each) break;
    const uint32_t earlier = digit[k] < bins ? mine[digit[k]] : 0;
    rank[k] = earlier + __popc(same[k] & ((1u << lane) - 1));
    __syncwarp();
    if (digit[k] < bins && lane == 31 - __clz(same[k])) mine[digit[k]] = static_cast<uint16_t>(rank[k] + 1);
    __syncwarp();
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < bins; i += kSortThreads) {
    uint32_t sum = 0;
    for (int w = 0; w < kWarps; w += 8) {
      uint32_t n[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) n[j] = sh.before[(w + j) * bins + i];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sh.before[(w + j) * bins + i] = static_cast<uint16_t>(sum);
        sum += n[j];
      }
    }
    sh.totals[i] = sum;
  }
  __syncthreads();
}

// The place in a tile of a thread's token k: warps take 32 * each consecutive ones.
__device__ __forceinline__ uint32_t tile_index(int each, int k) { return (threadIdx.x / 32 * each + k) * 32 + threadIdx.x % 32; }

template <bool First>
__device__ __forceinline__ Met get(const SortParams& p, int pass, uint64_t i) {
  if (!First) return p.sorted[(pass + 1) % 2][i];
  const uint64_t row = p.tokens.row(i);
  return {row < p.tokens.rows ? static_cast<uint32_t>(row) : kAll, static_cast<uint32_t>(i)};
}
__device__ __forceinline__ uint32_t digit_of(const SortParams& p, int pass, uint32_t row) {
  return row == kAll ? kAll : row >> (pass * p.bits) & ((1u << p.bits) - 1);
}

// Tokens [begin, end) of a tile, their digits and ranks.
template <bool First>
__device__ __forceinline__ void take_tile(const SortParams& p, const Shared& sh, uint32_t bins, int pass, uint64_t begin, uint64_t end, Met (&m)[kSortEach],
                                          uint32_t (&digit)[kSortEach], uint32_t (&rank)[kSortEach]) {
#pragma unroll
  for (int k = 0; k < kSortEach; ++k) {
    const uint64_t i = begin + tile_index(p.each, k);
    m[k] = k < p.each && i < end ? get<First>(p, pass, i) : Met{kAll, 0};
    digit[k] = digit_of(p, pass, m[k].row);
  }
  rank_tile(sh, bins, p.bits, p.each, digit, rank);
}
__device__ __forceinline__ void put_tile(const SortParams& p, const Shared& sh, uint32_t bins, int pass, const Met (&m)[kSortEach],
                                         const uint32_t (&digit)[kSortEach], const uint32_t (&rank)[kSortEach]) {
#pragma unroll
  for (int k = 0; k < kSortEach; ++k)
    if (digit[k] != kAll) p.sorted[pass % 2][sh.base[digit[k]] + sh.before[threadIdx.x / 32 * bins + digit[k]] + rank[k]] = m[k];
}

// Zeros: share `index` of the bytes.  (While the sort waits for latencies on some SMs, the others write.)
__device__ __forceinline__ void fill_share(const SortParams& p, uint64_t index) {
  const uint64_t begin = index * kFillShare, end = min(begin + kFillShare, p.fill_bytes);
  if (begin >= end) return;
  uint8_t* const to = p.fill + begin;
  const uint32_t head = static_cast<uint32_t>(min((16 - reinterpret_cast<uint64_t>(to) % 16) % 16, end - begin));
  const uint32_t whole = static_cast<uint32_t>((end - begin - head) / 16), tail = static_cast<uint32_t>(end - begin - head) % 16;
  for (uint32_t i = threadIdx.x; i < whole; i += kSortThreads) reinterpret_cast<uint4*>(to + head)[i] = make_uint4(0, 0, 0, 0);
  if (threadIdx.x < head / 2) reinterpret_cast<uint16_t*>(to)[threadIdx.x] = 0;
  if (threadIdx.x < tail / 2) reinterpret_cast<uint16_t*>(to + head + 16ull * whole)[threadIdx.x] = 0;
}

template <bool First>
__global__ void __launch_bounds__(kSortThreads) count_kernel(const __grid_constant__ SortParams p) {
  __shared__ uint32_t counts[1 << kMostDigit];
  const uint32_t bins = 1u << p.bits;
  for (uint32_t i = threadIdx.x; i < bins; i += kSortThreads) counts[i] = 0;
  wait_for_kernel_before();
  if (First && blockIdx.x >= p.ctas) return fill_share(p, blockIdx.x - p.ctas);
  __syncthreads();
  const uint64_t n = First ? p.tokens.n : *p.found, begin = blockIdx.x * p.share, end = min(begin + p.share, n);
  for (uint64_t at = begin; at < end; at += kSortTile) {
    uint32_t digit[kSortEach];
#pragma unroll
    for (int k = 0; k < kSortEach; ++k) {
      const uint64_t i = at + k * kSortThreads + threadIdx.x;
      digit[k] = digit_of(p, p.pass, i < end ? get<First>(p, p.pass, i).row : kAll);
    }
    // (one addition for a warp's tokens of one digit: a third of a batch may be the same)
    uint32_t same[kSortEach];
    same_digit(digit, p.bits, same);
#pragma unroll
    for (int k = 0; k < kSortEach; ++k)
      if (digit[k] != kAll && threadIdx.x % 32 == 31 - __clz(same[k])) atomicAdd(counts + digit[k], static_cast<uint32_t>(__popc(same[k])));
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
  uint32_t before = 0;
  if (threadIdx.x < bins) {
    uint32_t total = 0;
#pragma unroll 16
    for (uint32_t c = 0; c < p.ctas; ++c) {
      if (c == blockIdx.x) before = total;
      total += p.counts[static_cast<uint64_t>(c) * bins + threadIdx.x];
    }
    sh.base[threadIdx.x] = total;
  }
  __syncthreads();
  const uint32_t found = scan(sh.base, bins, sh.warps);
  if (threadIdx.x < bins) sh.base[threadIdx.x] += before;
  if (First && blockIdx.x == 0 && threadIdx.x == 0) *p.found = found;
  __syncthreads();
  const uint64_t n = First ? p.tokens.n : *p.found, begin = blockIdx.x * p.share, end = min(begin + p.share, n);
  for (uint64_t at = begin; at < end; at += kSortTile) {
    Met m[kSortEach];
    uint32_t digit[kSortEach], rank[kSortEach];
    take_tile<First>(p, sh, bins, p.pass, at, end, m, digit, rank);
    put_tile(p, sh, bins, p.pass, m, digit, rank);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < bins; i += kSortThreads) sh.base[i] += sh.totals[i];
    // (the next tile's barriers come between these sums and their use)
  }
}

// All passes of a batch of a tile per CTA of the cluster.
__global__ void __launch_bounds__(kSortThreads) cluster_kernel(const __grid_constant__ SortParams p, int passes) {
  extern __shared__ __align__(16) uint8_t raw[];
  namespace cg = cooperative_groups;
  const cg::cluster_group cluster = cg::this_cluster();
  const uint32_t bins = 1u << p.bits, me = cluster.block_rank();
  const Shared sh(raw, bins);
  wait_for_kernel_before();
  if (blockIdx.x >= p.ctas) return fill_share(p, blockIdx.x - p.ctas);  // (other clusters than the first)
  uint64_t n = p.tokens.n;
  for (int pass = 0; pass < passes; ++pass) {
    Met m[kSortEach];
    uint32_t digit[kSortEach], rank[kSortEach];
    const uint64_t begin = me * p.share, end = min(begin + p.share, n);
    if (pass == 0)
      take_tile<true>(p, sh, bins, pass, begin, end, m, digit, rank);
    else
      take_tile<false>(p, sh, bins, pass, begin, end, m, digit, rank);
    cluster.sync();
    uint32_t before = 0;
    if (threadIdx.x < bins) {
      uint32_t total = 0;
#pragma unroll 16
      for (uint32_t c = 0; c < p.ctas; ++c) {
        if (c == me) before = total;
        total += *cluster.map_shared_rank(sh.totals + threadIdx.x, c);
      }
      sh.base[threadIdx.x] = total;
    }
    __syncthreads();
    n = scan(sh.base, bins, sh.warps);
    if (threadIdx.x < bins) sh.base[threadIdx.x] += before;
    __syncthreads();
    put_tile(p, sh, bins, pass, m, digit, rank);
    // the tokens for the next pass; and no CTA changes or leaves counts that others read
    cluster.sync();
  }
  if (me == 0 && threadIdx.x == 0) {
    *p.found = static_cast<uint32_t>(n);
    *p.n_long = 0;
  }
}

// A small batch: a token's place is the number of tokens of lower rows, and of its row before it.  16 threads count for each.
constexpr uint32_t kCompareEach = 16, kCompareShare = kSortThreads / kCompareEach;
__global__ void __launch_bounds__(kSortThreads) compare_kernel(const __grid_constant__ SortParams p) {
  __shared__ __align__(16) uint32_t rows[kCompareTokens];
  wait_for_kernel_before();
  if (blockIdx.x >= p.ctas) return fill_share(p, blockIdx.x - p.ctas);
  const uint32_t n = static_cast<uint32_t>(p.tokens.n), whole = (n + 3) / 4;
  uint32_t found = 0;
  for (uint32_t i = threadIdx.x; i < 4 * whole; i += kSortThreads) {
    rows[i] = i < n ? get<true>(p, 0, i).row : kAll;
    found += rows[i] != kAll;
  }
  if (blockIdx.x == 0) {
    __shared__ uint32_t all;
    if (threadIdx.x == 0) all = 0;
    __syncthreads();
    found = __reduce_add_sync(kAll, found);
    if (threadIdx.x % 32 == 0) atomicAdd(&all, found);
    __syncthreads();
    if (threadIdx.x == 0) {
      *p.found = all;
      *p.n_long = 0;
    }
  }
  __syncthreads();
  const uint32_t i = blockIdx.x * kCompareShare + threadIdx.x / kCompareEach, row = i < n ? rows[i] : kAll;
  uint32_t place = 0;
#pragma unroll 4
  for (uint32_t v = threadIdx.x % kCompareEach; v < whole; v += kCompareEach) {
    const uint4 r = reinterpret_cast<const uint4*>(rows)[v];
    const uint32_t least = row + (4 * v < i);  // below it: of a lower row, or of this one and before
    if (v == i / 4) {
      place += (r.x < row + (4 * v < i)) + (r.y < row + (4 * v + 1 < i)) + (r.z < row + (4 * v + 2 < i)) + (r.w < row);
    } else {
      place += (r.x < least) + (r.y < least) + (r.z < least) + (r.w < least);
    }
  }
#pragma unroll
  for (uint32_t k = kCompareEach / 2; k > 0; k /= 2) place += __shfl_xor_sync(kAll, place, k);
  if (threadIdx.x % kCompareEach == 0 && row != kAll) p.sorted[0][place] = {row, i};
}

uint32_t fill_ctas(const SortParams& p) { return static_cast<uint32_t>((p.fill_bytes + kFillShare - 1) / kFillShare); }

cudaError_t launch_cluster(const SortParams& p, int passes, size_t shared, cudaStream_t s) {
  cudaLaunchAttribute a[2] = {};
  a[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  a[0].val.programmaticStreamSerializationAllowed = 1;
  a[1].id = cudaLaunchAttributeClusterDimension;
  a[1].val.clusterDim.x = p.ctas;
  a[1].val.clusterDim.y = a[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3((fill_ctas(p) + p.ctas - 1) / p.ctas * p.ctas + p.ctas);
  c.blockDim = dim3(kSortThreads);
  c.dynamicSmemBytes = shared;
  c.stream = s;
  c.attrs = a;
  c.numAttrs = 2;
  cudaLaunchKernelEx(&c, cluster_kernel, p, passes);
  return cudaGetLastError();
}

}  // namespace

cudaError_t configure_sort() {
  const int big = static_cast<int>(shared_bytes(1u << kMostDigit));
  cudaError_t e = cudaFuncSetAttribute(place_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, big);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(place_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, big);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(cluster_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, big);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(cluster_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  return e;
}

cudaError_t launch_sort(SortParams p, const SortPlan& plan, int* last, cudaStream_t s) {
  p.bits = plan.bits;
  *last = (plan.passes - 1) % 2;
  const uint64_t n = p.tokens.n;
  if (n <= kCompareTokens) {
    *last = 0;
    p.ctas = n == 0 ? 1 : static_cast<uint32_t>((n + kCompareShare - 1) / kCompareShare);
    return launch_chained(compare_kernel, static_cast<int>(p.ctas + fill_ctas(p)), kSortThreads, 0, s, p);
  }
  if (n <= kClusterTokens) {
    p.ctas = 1;
    while (p.ctas < kSortCluster && p.ctas * static_cast<uint64_t>(kSortThreads) < n) p.ctas *= 2;
    p.each = static_cast<int>((n + p.ctas * kSortThreads - 1) / (p.ctas * kSortThreads));
    p.share = static_cast<uint64_t>(p.each) * kSortThreads;
    return launch_cluster(p, plan.passes, shared_bytes(plan.bins()), s);
  }
  p.each = kSortEach;
  p.share = ((n + kSortCtas - 1) / kSortCtas + kSortTile - 1) / kSortTile * kSortTile;
  p.ctas = static_cast<uint32_t>((n + p.share - 1) / p.share);
  for (p.pass = 0; p.pass < plan.passes; ++p.pass) {
    cudaError_t e = launch_chained(p.pass == 0 ? count_kernel<true> : count_kernel<false>, static_cast<int>(p.ctas + (p.pass == 0 ? fill_ctas(p) : 0)),
                                   kSortThreads, 0, s, p);
    if (e == cudaSuccess)
      e = launch_chained(p.pass == 0 ? place_kernel<true> : place_kernel<false>, static_cast<int>(p.ctas), kSortThreads, shared_bytes(plan.bins()), s, p);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace frk
