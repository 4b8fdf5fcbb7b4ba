// embed_sum.cu -- the table's gradient: per row the sum of its tokens' gradients.
//
// The tokens, sorted by row, are cut into ranges of equal length whatever the rows
// are, so that a token that is a third of the batch costs no more than others: a
// warp takes a range, and a tile of columns of it, a CTA eight ranges of a tile.  A
// warp adds row by row in fp32, in the tokens' order, and writes a row at its last
// token.  A range's border inside a row moves to the row's start if the row has no
// more tokens than a range.  A longer row's parts are added in the ranges' order by
// the CTA where it ends, or, if it began in another, by a second launch, from the
// workspace.  Ranges follow from the batch alone, so a repeated call gives the same bits.
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
  return share < kLeastRange ? kLeastRange : share;
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

// Tokens whose vectors are on their way together: what 32 registers hold of them and, where they are added to, of the rows.
constexpr int tokens_ahead(int elems, bool bf16_out, bool bf16_grad, bool add) {
  const int words = (elems * (bf16_out ? 2 : 4) + (add ? elems * (bf16_grad ? 2 : 4) : 0) + 3) / 4;
  return 32 / words >= 8 ? 8 : 32 / words >= 4 ? 4 : 2;
}

template <int V, bool Bf16Out, bool Bf16Grad, bool Add>
__global__ void __launch_bounds__(kThreads, 3) sum_kernel(const __grid_constant__ SumParams p) {
  constexpr int kVectors = lane_vectors(V), kWidth = 32 * V * kVectors;
  constexpr int kAhead = tokens_ahead(V * kVectors, Bf16Out, Bf16Grad, Add);
  // What each warp has of the row that it starts in, if that ends there, and of the one that goes on after it.
  __shared__ float heads[kSumWarps][kWidth], tails[kSumWarps][kWidth];
  __shared__ uint32_t ended[kSumWarps], from_inside[kSumWarps], to_inside[kSumWarps];
  wait_for_kernel_before();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, found = *p.found;
  if (blockIdx.x >= p.sum_ctas) {
    if (!Add) clear_rows<V, Bf16Grad>(p, found, (blockIdx.x - p.sum_ctas) * kSumWarps + warp, lane);
    return;
  }
  const uint32_t span = span_of(found, p.ranges), cta = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles;
  const uint64_t b = (static_cast<uint64_t>(cta) * kSumWarps + warp) * span;
  const Border from = border(p.sorted, found, span, b, lane), to = border(p.sorted, found, span, b + span, lane);
  const uint64_t first = static_cast<uint64_t>(tile) * kWidth + lane * V;
  auto column = [&](int c) { return first + c * (32 * V); };
  auto mine = [&](int c) { return column(c) < p.dim; };
  auto place = [&](int c, int j) { return (c * V + j) * 32 + lane; };
  bool head = from.inside;  // the row at hand started in a range before
  uint32_t head_row = kAll;
  float sum[kVectors][V] = {};
  // (the next 32 tokens are on their way while these are added)
  auto tokens = [&](uint32_t i) { return i < to.at ? p.sorted[i] : Met{kAll, 0}; };
  auto row_after = [&](uint32_t i) { return i + 1 < found && i < to.at ? p.sorted[i + 1].row : kAll; };
  Met m = tokens(from.at + lane);
  uint32_t after = row_after(from.at + lane);
  for (uint32_t i = from.at; i < to.at; i += 32) {
    const uint32_t here = min(to.at - i, 32u);
    const uint32_t ends = __ballot_sync(kAll, lane < here && m.row != after);
    const Met now = m;
    m = tokens(i + 32 + lane);
    after = row_after(i + 32 + lane);
    for (uint32_t k = 0; k < here; k += kAhead) {
      Raw<V, Bf16Out> in[kAhead][kVectors];
      Raw<V, Bf16Grad> old[Add ? kAhead : 1][kVectors];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint64_t at = static_cast<uint64_t>(__shfl_sync(kAll, now.at, k + u)) * p.dim;
        const uint64_t row = Add ? static_cast<uint64_t>(__shfl_sync(kAll, now.row, k + u)) * p.dim : 0;
        if (k + u >= here) continue;
#pragma unroll
        for (int c = 0; c < kVectors; ++c)
          if (mine(c)) in[u][c].load(p.out, at + column(c));
        if (!Add || !(ends >> (k + u) & 1)) continue;
#pragma unroll
        for (int c = 0; c < kVectors; ++c)
          if (mine(c)) old[u][c].load(p.grad, row + column(c));
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (k + u >= here) break;
#pragma unroll
        for (int c = 0; c < kVectors; ++c) {
          float x[V];
          in[u][c].get(x);
          add(sum[c], x);
        }
        if (!(ends >> (k + u) & 1)) continue;
        const uint32_t row = __shfl_sync(kAll, now.row, k + u);
#pragma unroll
        for (int c = 0; c < kVectors; ++c) {
          if (head) {
#pragma unroll
            for (int j = 0; j < V; ++j) heads[warp][place(c, j)] = sum[c][j];
          } else if (mine(c)) {
            finish<V, Bf16Grad, Add>(p.grad, static_cast<uint64_t>(row) * p.dim + column(c), p.scale, sum[c], old[Add ? u : 0][c]);
          }
#pragma unroll
          for (int j = 0; j < V; ++j) sum[c][j] = 0.0f;
        }
        if (head) head_row = row;
        head = false;
      }
    }
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
      if (!mine(c)) continue;
      if (end == 0 && !before) {
        const uint64_t at = static_cast<uint64_t>(head_row) * p.dim + column(c);
        Raw<V, Bf16Grad> old;
        if (Add) old.load(p.grad, at);
        finish<V, Bf16Grad, Add>(p.grad, at, p.scale, total, old);
      } else {
        Raw<V, false> part;
        part.set(total);
        part.store(p.parts, (2ull * cta + !before) * p.dim + column(c));
      }
    }
    if (end == 1 && !before && tile == 0 && lane == 0) p.longs[atomicAdd(p.n_long, 1u)] = cta;
  }
}

// A long row's parts: the second of the CTA where it begins, the first of the CTAs after it that begin inside it.  (The list's order is any;
// each row has its place.)
template <int V, bool Bf16Grad, bool Add>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ SumParams p) {
  constexpr int kVectors = lane_vectors(V), kWarps = kJoinThreads / 32, kWidth = 32 * V * kVectors;
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
    if (warp < kVectors) {  // a vector of columns each
      const uint64_t column = first + (warp * 32 + lane) * V;
      if (column < p.dim) {
        float total[V] = {};
        for (int w = 0; w < kWarps; ++w)
#pragma unroll
          for (int j = 0; j < V; ++j) total[j] = __fadd_rn(total[j], sums[w][(warp * V + j) * 32 + lane]);
        Raw<V, Bf16Grad> old;
        if (Add) old.load(p.grad, row * p.dim + column);
        finish<V, Bf16Grad, Add>(p.grad, row * p.dim + column, p.scale, total, old);
      }
    }
    __syncthreads();
  }
}

template <int V, bool Bf16Out, bool Bf16Grad, bool Add>
cudaError_t launch(const SumParams& p, cudaStream_t s) {
  cudaError_t e = launch_chained(sum_kernel<V, Bf16Out, Bf16Grad, Add>, static_cast<int>(p.sum_ctas + p.zero_ctas), kThreads, 0, s, p);
  if (e == cudaSuccess) e = launch_chained(join_kernel<V, Bf16Grad, Add>, static_cast<int>(kSms * 2), kJoinThreads, 0, s, p);
  return e;
}
template <int V, bool Bf16Out>
cudaError_t launch_typed(const SumParams& p, cudaStream_t s) {
  if (p.accumulate) return p.bf16_grad ? launch<V, Bf16Out, true, true>(p, s) : launch<V, Bf16Out, false, true>(p, s);
  return p.bf16_grad ? launch<V, Bf16Out, true, false>(p, s) : launch<V, Bf16Out, false, false>(p, s);
}
template <int V>
cudaError_t launch_wide(const SumParams& p, cudaStream_t s) {
  return p.bf16_out ? launch_typed<V, true>(p, s) : launch_typed<V, false>(p, s);
}

}  // namespace

cudaError_t launch_sum(const SumParams& p, cudaStream_t s) {
  switch (p.v) {
    case 8: return launch_wide<8>(p, s);
    case 4: return launch_wide<4>(p, s);
    case 2: return launch_wide<2>(p, s);
    default: return launch_wide<1>(p, s);
  }
}

}  // namespace frk
