// embed_sum.cu -- the table's gradient: per row the sum of its tokens' gradients.
//
// The tokens, sorted by row, are cut into ranges of equal length whatever the rows
// are, so that a token that is a third of the batch costs no more than others: a
// warp takes a range, and a tile of columns of it, a CTA eight ranges of a tile.  A
// warp adds row by row in fp32, in the tokens' order, and writes a row at its last
// token.  A range's border inside a row moves to the row's start if the row has no
// more tokens than a range.  A longer row's parts are added in the ranges' order by
// the CTA where it ends, or, if it began in another, by a second launch, from the
// workspace, where a warp adds every eighth CTA's and then the warps' sums are added.
// Rows that no token meets are filled with zeros by CTAs of their own, or have been,
// beside the sort.  Ranges follow from the batch and the sizes alone, so a repeated
// call gives the same bits, at any addresses.
//
// Bound by gathering rows: 65,536 tokens of 4,096 in bf16 94 us, 5.4 TB/s (HBM 69%;
// latencies, three batches of a range on their way); by instructions with odd rows:
// 500,001 tokens of 321 in fp32 115 us, 5.7 TB/s.
#include <cuda_runtime.h>

#include "embed.h"
#include "embed_vector.cuh"
#include "kernels.h"

namespace frk {

namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;
constexpr int kThreads = kSumWarps * 32;
constexpr int kJoinThreads = 256;

__device__ __forceinline__ uint32_t span_of(uint32_t found, uint32_t ranges) {
  const uint32_t share = (found + ranges - 1) / ranges;
  return share < kShortRange ? kShortRange : share;
}

// The first place in [lo, hi) whose row is `row` or above, or hi; 32 places are looked at together.
__device__ __forceinline__ uint32_t first_at_least(const Met* sorted, uint32_t lo, uint32_t hi, uint32_t row, uint32_t lane) {
  while (lo < hi) {
    const uint32_t step = (hi - lo + 31) / 32, i = lo + lane * step;
    const uint32_t below = __popc(__ballot_sync(kAll, i < hi && sorted[i].row < row));
    if (below == 0) return lo;
    hi = min(hi, lo + below * step);
    lo += (below - 1) * step + 1;
  }
  return lo;
}

// Where the range that would start at b does, and whether that is inside a long row.
struct Border {
  uint32_t at;
  bool inside;
};
__device__ __forceinline__ Border border(const Met* sorted, uint32_t found, uint32_t span, uint64_t b, uint32_t lane) {
  if (b == 0) return {0, false};
  if (b >= found) return {found, false};
  const uint32_t at = static_cast<uint32_t>(b);
  // the 32 tokens on either side, by one latency
  const uint32_t left = at >= lane + 1 ? sorted[at - 1 - lane].row : kAll, right = at + lane < found ? sorted[at + lane].row : kAll;
  const uint32_t row = __shfl_sync(kAll, right, 0);
  const uint32_t other_left = ~__ballot_sync(kAll, left == row), other_right = ~__ballot_sync(kAll, right == row);
  uint32_t before = other_left ? __ffs(other_left) - 1 : 32, after = other_right ? __ffs(other_right) - 1 : 32;
  if (before == 0) return {at, false};
  if (span > 32 && before == 32) before = at - first_at_least(sorted, at > span ? at - span : 0, at, row, lane);
  if (span > 32 && after == 32) after = first_at_least(sorted, at, static_cast<uint32_t>(min(b + span, static_cast<uint64_t>(found))), row + 1, lane) - at;
  // (a count cut off at a span, or at 32 of a span of up to 32, is of a long row)
  return before + after > span ? Border{at, true} : Border{at - before, false};
}

template <int V>
__device__ __forceinline__ void add(float (&sum)[V], const float (&x)[V]) {
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = __fadd_rn(sum[j], x[j]);
}

// scale * sum, and what is there already, rounded once.
template <int V, bool Bf16, bool Add>
__device__ __forceinline__ void finish(void* grad, uint64_t element, float scale, const float (&sum)[V], const Raw<V, Bf16>& old) {
  float x[V];
  if (Add) {
    old.get(x);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = __fmaf_rn(scale, sum[j], x[j]);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = __fmul_rn(scale, sum[j]);
  }
  Raw<V, Bf16> w;
  w.set(x);
  w.store(grad, element);
}

// The rows that no token meets: zeros.  A lane looks one row up.
template <int V, bool Bf16>
__device__ __forceinline__ void clear_rows(const SumParams& p, uint32_t found, uint32_t warp, uint32_t lane) {
  const uint64_t row = static_cast<uint64_t>(warp) * p.rows_per_zero_warp + lane;
  uint32_t lo = 0, hi = found;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (p.sorted[mid].row < row)
      lo = mid + 1;
    else
      hi = mid;
  }
  const bool there = lane < p.rows_per_zero_warp && row < p.rows;
  const bool met = there && lo < found && p.sorted[lo].row == row;
  const uint64_t across = p.dim / V;
  Raw<V, Bf16> zero;
  zero.clear();
  for (uint32_t left = __ballot_sync(kAll, there && !met); left != 0; left &= left - 1) {
    const uint64_t at = (static_cast<uint64_t>(warp) * p.rows_per_zero_warp + __ffs(left) - 1) * p.dim;
    for (uint64_t c = lane; c < across; c += 32) zero.store(p.grad, at + c * V);
  }
}

// A warp's ring in shared memory: the tokens whose vectors, and where they are added to, rows, are on their way.  kRing: tokens, in four
// batches, three of them under way while one is added.  A lane copies what it reads, or with kOdd the warp the granules around a tile's row.
template <int Kind, bool Bf16Out, bool Bf16Grad, bool Add>
struct Ring {
  static constexpr int V = vector_of(Kind), kVectors = lane_vectors(Kind), kWidth = tile_width(Kind);
  static constexpr int kSpare = Kind == kOdd ? 16 : 0;
  static constexpr int kIn = kWidth * (Bf16Out ? 2 : 4) + kSpare, kOld = Add ? kWidth * (Bf16Grad ? 2 : 4) + kSpare : 0;
  static constexpr int kMost = Kind == kOdd ? 13 << 10 : Add ? 6 << 10 : 8 << 10;
  static constexpr int kRing = 16 * (kIn + kOld) <= kMost ? 16 : 8 * (kIn + kOld) <= kMost ? 8 : 4, kBatch = kRing / 4;
  static constexpr int kBytes = kRing * (kIn + kOld);
  // a CTA's, and what its warps hand on
  static constexpr int kParts = 2 * kSumWarps * kWidth * 4;
  static constexpr int kShared = kSumWarps * kBytes > kParts ? kSumWarps * kBytes : kParts;
  uint8_t* at;
  uint32_t lane;
  uint64_t first, dim;  // column of the tile, columns of a row

  __device__ __forceinline__ uint64_t column(int c) const { return first + (c * 32 + lane) * V; }
  __device__ __forceinline__ bool mine(int c) const { return column(c) < dim; }
  __device__ __forceinline__ uint8_t* in_slot(uint32_t token) const { return at + token % kRing * kIn; }
  __device__ __forceinline__ uint8_t* old_slot(uint32_t token) const { return at + kRing * kIn + token % kRing * kOld; }

  // Row `row` of a buffer of `rows`.
  template <bool Bf16>
  __device__ __forceinline__ void copy(uint8_t* slot, const void* base, uint64_t row, uint64_t rows) const {
    constexpr int kSize = Bf16 ? 2 : 4;
    if constexpr (Kind == kOdd) {
      const Granules g(reinterpret_cast<uint64_t>(base), row, dim, first, kWidth, kSize);
      if (by_granules(row, rows)) {
        const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(slot)) + lane * 16;
        const uint8_t* const begin = reinterpret_cast<const uint8_t*>(g.begin) + lane * 16;
#pragma unroll
        for (int k = 0; k < (kWidth * kSize + 16 + 511) / 512; ++k)
          if (lane * 16 + k * 512 < g.bytes) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + k * 512), "l"(begin + k * 512) : "memory");
      } else {
        using T = typename Words<kSize>::T;
        const uint64_t from = reinterpret_cast<uint64_t>(base) + (row * dim + first) * kSize;
        T* const to = reinterpret_cast<T*>(slot + (from & 15));
        const uint64_t width = min(static_cast<uint64_t>(kWidth), dim - first);
        for (uint32_t i = lane; i < width; i += 32) to[i] = reinterpret_cast<const T*>(from)[i];
      }
    } else {
#pragma unroll
      for (int c = 0; c < kVectors; ++c)
        if (mine(c)) Raw<V, Bf16>::copy(slot + (c * 32 + lane) * V * kSize, base, row * dim + column(c));
    }
  }
  template <bool Bf16>
  __device__ __forceinline__ Raw<V, Bf16> get(const uint8_t* slot, const void* base, uint64_t row, int c) const {
    constexpr int kSize = Bf16 ? 2 : 4;
    // (where it starts in its granule: of the address's low bits alone)
    const uint32_t shift =
        Kind == kOdd ? (static_cast<uint32_t>(reinterpret_cast<uint64_t>(base)) + (static_cast<uint32_t>(row) * static_cast<uint32_t>(dim) + static_cast<uint32_t>(first)) * kSize) & 15u : 0;
    Raw<V, Bf16> r;
    r.load(slot + shift + (c * 32 + lane) * V * kSize, 0);
    return r;
  }
  // Other lanes' copies, and reads before the next copies.
  __device__ __forceinline__ void together() const {
    if constexpr (Kind == kOdd) __syncwarp();
  }
};

// (CTAs per SM: with three a wide row's registers spill, 124 -> 144 us; with them odd rows go from 138 to 125.)
template <int Kind, bool Bf16Out, bool Bf16Grad, bool Add>
__global__ void __launch_bounds__(kThreads, Kind == kWide ? 2 : 3) sum_kernel(const __grid_constant__ SumParams p) {
  using R = Ring<Kind, Bf16Out, Bf16Grad, Add>;
  constexpr int V = R::V, kVectors = R::kVectors, kWidth = R::kWidth, kBatch = R::kBatch;
  extern __shared__ __align__(16) uint8_t raw[];
  // What each warp has of the row that it starts in, if that ends there, and of the one that goes on after it: in the ring's place, after it.
  auto heads = reinterpret_cast<float(*)[kWidth]>(raw), tails = heads + kSumWarps;
  __shared__ uint32_t ended[kSumWarps], from_inside[kSumWarps], to_inside[kSumWarps];
  wait_for_kernel_before();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, found = *p.found;
  if (blockIdx.x >= p.ctas) {
    if (!Add) clear_rows<V, Bf16Grad>(p, found, (blockIdx.x - p.ctas) * kSumWarps + warp, lane);
    return;
  }
  const uint32_t span = span_of(found, p.ranges), cta = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles;
  const uint64_t b = (static_cast<uint64_t>(cta) * kSumWarps + warp) * span;
  const Border from = border(p.sorted, found, span, b, lane), to = border(p.sorted, found, span, b + span, lane);
  auto place = [&](int c, int j) { return (c * V + j) * 32 + lane; };
  const R ring = {raw + warp * R::kBytes, lane, static_cast<uint64_t>(tile) * kWidth, p.dim};
  bool head = from.inside;  // the row at hand started in a range before
  uint32_t head_row = kAll;
  float sum[kVectors][V] = {}, head_sum[kVectors][V] = {};
  // 32 tokens, those after them, and on their way the next ones
  struct Group {
    Met m;
    uint32_t after;
  };
  auto fetch = [&](uint32_t i) {
    i += lane;
    return Group{i < to.at ? p.sorted[i] : Met{kAll, 0}, i + 1 < found && i < to.at ? p.sorted[i + 1].row : kAll};
  };
  auto ends_of = [&](const Group& g) { return __ballot_sync(kAll, g.m.row != kAll && g.m.row != g.after); };
  const uint32_t count = to.at - from.at;
  Group now = fetch(from.at), next = fetch(from.at + 32), later = fetch(from.at + 64);
  uint32_t ends = ends_of(now), next_ends = ends_of(next);
  // the copies of batch k + ... of this group, or the next
  auto issue = [&](uint32_t base, uint32_t k) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const uint32_t j = k + u, i = j % 32;
      const uint32_t token = __shfl_sync(kAll, j < 32 ? now.m.at : next.m.at, i);
      const uint32_t row = Add ? __shfl_sync(kAll, j < 32 ? now.m.row : next.m.row, i) : 0;
      if (base + j >= count) continue;
      ring.template copy<Bf16Out>(ring.in_slot(base + j), p.out, token, p.n);
      if (Add && (j < 32 ? ends : next_ends) >> i & 1) ring.template copy<Bf16Grad>(ring.old_slot(base + j), p.grad, row, p.rows);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int k = 0; k < 3; ++k) issue(0, k * kBatch);
  for (uint32_t base = 0; base < count; base += 32) {
    for (uint32_t k = 0; k < 32 && base + k < count; k += kBatch) {
      ring.together();
      issue(base, k + 3 * kBatch);
      asm volatile("cp.async.wait_group 3;" ::: "memory");
      ring.together();
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (base + k + u >= count) break;
        const uint32_t token = Kind == kOdd ? __shfl_sync(kAll, now.m.at, k + u) : 0;
#pragma unroll
        for (int c = 0; c < kVectors; ++c) {
          float x[V];
          ring.template get<Bf16Out>(ring.in_slot(base + k + u), p.out, token, c).get(x);
          add(sum[c], x);
        }
        if (!(ends >> (k + u) & 1)) continue;
        const uint32_t row = __shfl_sync(kAll, now.m.row, k + u);
#pragma unroll
        for (int c = 0; c < kVectors; ++c) {
          if (head) {
#pragma unroll
            for (int j = 0; j < V; ++j) head_sum[c][j] = sum[c][j];
          } else if (ring.mine(c)) {
            Raw<V, Bf16Grad> old;
            if (Add) old = ring.template get<Bf16Grad>(ring.old_slot(base + k + u), p.grad, row, c);
            finish<V, Bf16Grad, Add>(p.grad, row * p.dim + ring.column(c), p.scale, sum[c], old);
          }
#pragma unroll
          for (int j = 0; j < V; ++j) sum[c][j] = 0.0f;
        }
        if (head) head_row = row;
        head = false;
      }
    }
    now = next;
    next = later;
    later = fetch(from.at + base + 96);
    ends = next_ends;
    next_ends = ends_of(next);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  if (from.inside && !head) {
#pragma unroll
    for (int c = 0; c < kVectors; ++c)
#pragma unroll
      for (int j = 0; j < V; ++j) heads[warp][place(c, j)] = head_sum[c][j];
  }
  if (to.inside) {
#pragma unroll
    for (int c = 0; c < kVectors; ++c)
#pragma unroll
      for (int j = 0; j < V; ++j) tails[warp][place(c, j)] = sum[c][j];
  }
  if (lane == 0) {
    ended[warp] = from.inside && !head;
    from_inside[warp] = from.inside;
    to_inside[warp] = to.inside;
  }
  __syncthreads();
  // A row that ends in a warp after the one where it began, and one that goes on after the CTA, is added up by that warp.
  const bool last = warp == kSumWarps - 1 && to_inside[warp];
  for (int end = 0; end < 2; ++end) {  // 0: the row that ends here, 1: the one that goes on
    if (end == 0 ? !ended[warp] : !last) continue;
    // the warp where the row begins in this CTA: back over those that are all inside it
    int w = static_cast<int>(warp);
    if (end == 0 || (from_inside[w] && !ended[w])) {
      for (--w; w >= 0 && from_inside[w] && !ended[w]; --w) {
      }
    }
    const bool before = w < 0;  // it began in an earlier CTA
#pragma unroll
    for (int c = 0; c < kVectors; ++c) {
      float total[V] = {};
      for (int k = before ? 0 : w; k < static_cast<int>(warp) + end; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) total[j] = __fadd_rn(total[j], tails[k][place(c, j)]);
      if (end == 0)
#pragma unroll
        for (int j = 0; j < V; ++j) total[j] = __fadd_rn(total[j], heads[warp][place(c, j)]);
      if (!ring.mine(c)) continue;
      if (end == 0 && !before) {
        const uint64_t at = static_cast<uint64_t>(head_row) * p.dim + ring.column(c);
        Raw<V, Bf16Grad> old;
        if (Add) old.load(p.grad, at);
        finish<V, Bf16Grad, Add>(p.grad, at, p.scale, total, old);
      } else {
        Raw<V, false> part;
        part.set(total);
        part.store(p.parts, (2ull * cta + !before) * p.dim + ring.column(c));
      }
    }
    if (end == 1 && !before && tile == 0 && lane == 0) p.longs[atomicAdd(p.n_long, 1u)] = cta;
  }
}

// A long row's parts: the second of the CTA where it begins, the first of the CTAs after it that begin inside it.  (The list's order is any;
// each row has its place.)
template <int Kind, bool Bf16Grad, bool Add>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ SumParams p) {
  constexpr int V = vector_of(Kind), kVectors = lane_vectors(Kind), kWarps = kJoinThreads / 32, kWidth = tile_width(Kind);
  __shared__ float sums[kWarps][kWidth];
  wait_for_kernel_before();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t found = *p.found, span = span_of(found, p.ranges) * kSumWarps;  // of a CTA
  const uint64_t items = static_cast<uint64_t>(*p.n_long) * p.tiles;
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t g = p.longs[item / p.tiles];
    const uint32_t row = p.sorted[static_cast<uint64_t>(g + 1) * span].row;
    uint32_t more = 0;  // parts after the first one
    for (;;) {
      const uint64_t at = static_cast<uint64_t>(g + 1 + more + threadIdx.x) * span;
      const uint32_t n = __syncthreads_count(at < found && p.sorted[at < found ? at : 0].row == row);
      more += n;
      if (n < kJoinThreads) break;
    }
    const uint64_t first = item % p.tiles * kWidth;
    float sum[kVectors][V] = {};
#pragma unroll 4
    for (uint32_t k = warp; k <= more; k += kWarps) {
#pragma unroll
      for (int c = 0; c < kVectors; ++c) {
        const uint64_t column = first + (c * 32 + lane) * V;
        if (column >= p.dim) continue;
        Raw<V, false> w;
        w.load(p.parts, (2ull * (g + k) + (k == 0)) * p.dim + column);
        float x[V];
        w.get(x);
        add(sum[c], x);
      }
    }
#pragma unroll
    for (int c = 0; c < kVectors; ++c)
#pragma unroll
      for (int j = 0; j < V; ++j) sums[warp][(c * V + j) * 32 + lane] = sum[c][j];
    __syncthreads();
    for (int c = warp; c < kVectors; c += kWarps) {  // a vector of columns each
      const uint64_t column = first + (c * 32 + lane) * V;
      if (column < p.dim) {
        float total[V] = {};
        for (int w = 0; w < kWarps; ++w)
#pragma unroll
          for (int j = 0; j < V; ++j) total[j] = __fadd_rn(total[j], sums[w][(c * V + j) * 32 + lane]);
        Raw<V, Bf16Grad> old;
        if (Add) old.load(p.grad, row * p.dim + column);
        finish<V, Bf16Grad, Add>(p.grad, row * p.dim + column, p.scale, total, old);
      }
    }
    __syncthreads();
  }
}

template <int Kind, bool Bf16Out, bool Bf16Grad, bool Add>
cudaError_t launch(const SumParams& p, cudaStream_t s) {
  constexpr int kShared = Ring<Kind, Bf16Out, Bf16Grad, Add>::kShared;
  if (p.configure) return cudaFuncSetAttribute(sum_kernel<Kind, Bf16Out, Bf16Grad, Add>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared);
  cudaError_t e = launch_chained(sum_kernel<Kind, Bf16Out, Bf16Grad, Add>, static_cast<int>(p.ctas + p.zero_ctas), kThreads, kShared, s, p);
  if (e == cudaSuccess) e = launch_chained(join_kernel<Kind, Bf16Grad, Add>, static_cast<int>(kSms * 2), kJoinThreads, 0, s, p);
  return e;
}
template <int Kind, bool Bf16Out>
cudaError_t launch_typed(const SumParams& p, cudaStream_t s) {
  if (p.accumulate) return p.bf16_grad ? launch<Kind, Bf16Out, true, true>(p, s) : launch<Kind, Bf16Out, false, true>(p, s);
  return p.bf16_grad ? launch<Kind, Bf16Out, true, false>(p, s) : launch<Kind, Bf16Out, false, false>(p, s);
}
template <int Kind>
cudaError_t launch_wide(const SumParams& p, cudaStream_t s) {
  return p.bf16_out ? launch_typed<Kind, true>(p, s) : launch_typed<Kind, false>(p, s);
}

}  // namespace

cudaError_t configure_sum() {
  SumParams p = {};
  p.configure = 1;
  for (int k = 0; k < 48; ++k) {
    p.v = k / 8 == 5 ? kOdd : 1 << k / 8;
    p.bf16_out = k & 1;
    p.bf16_grad = k >> 1 & 1;
    p.accumulate = k >> 2 & 1;
    const cudaError_t e = launch_sum(p, nullptr);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_sum(const SumParams& p, cudaStream_t s) {
  switch (p.v) {
    case 8: return launch_wide<8>(p, s);
    case 4: return launch_wide<4>(p, s);
    case 2: return launch_wide<2>(p, s);
    case kOdd: return launch_wide<kOdd>(p, s);
    case kWide: return launch_wide<kWide>(p, s);
    default: return launch_wide<1>(p, s);
  }
}

}  // namespace frk
