// optim_clip.cu -- the norm of all gradients, the count of non-finite ones, and
// the factor that clips them, in one launch.
//
// A lane squares the eight elements that it has of each block into two fp32
// sums, which a float pair takes up error-free every kClipSeg blocks: 64
// squares are added in fp32 at a time, at most.  A segment whose fp32 sum is
// not finite (a NaN or Inf, or an overflow) or so small that squares may have
// lost bits to underflow is added again by the lanes concerned, element by
// element in fp64, the non-finite ones counted and left out.  Warps, then CTAs,
// then the partial sums of all CTAs are added in fp64 in a fixed order; the CTA
// that is last to finish adds those.
#include <cmath>

#include "kernels.h"
#include "optim.h"

namespace frk {

namespace {

constexpr uint32_t kClipSeg = 16;

template <bool Bf16>
__device__ __forceinline__ float element(const void* p, uint64_t i) {
  return Bf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(p)[i]) << 16) : static_cast<const float*>(p)[i];
}

struct LaneSums {
  float hi = 0.0f, lo = 0.0f;  // of segments added in fp32
  double exact = 0.0;          // of segments added in fp64
  uint32_t nonfinite = 0;
};

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return r;
}

// Blocks [first, first + count) of one tensor, count <= kClipSeg.
template <bool Bf16>
__device__ __forceinline__ void add_segment(const OptDesc& d, uint32_t first, uint32_t count, int lane, LaneSums& s) {
  float2 sum = make_float2(0.0f, 0.0f);
  uint32_t any = 0;  // a bit set: some element is not +0
  for (uint32_t k = 0; k < count; ++k) {
    const uint64_t at = static_cast<uint64_t>(first + k) * kOptBlock + lane * kOptLane;
    if (d.aligned && at + kOptLane <= d.n) {
      if (Bf16) {
        const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(d.grad) + at);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u));
          sum = fma2(x, x, sum);
          any |= w[j];
        }
      } else {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(d.grad) + at);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float4 a = q[j];
          const float2 x = make_float2(a.x, a.y), y = make_float2(a.z, a.w);
          sum = fma2(x, x, sum);
          sum = fma2(y, y, sum);
          any |= __float_as_uint(a.x) | __float_as_uint(a.y) | __float_as_uint(a.z) | __float_as_uint(a.w);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < kOptLane; j += 2) {
        float2 x;
        x.x = at + j < d.n ? element<Bf16>(d.grad, at + j) : 0.0f;
        x.y = at + j + 1 < d.n ? element<Bf16>(d.grad, at + j + 1) : 0.0f;
        sum = fma2(x, x, sum);
        any |= __float_as_uint(x.x) | __float_as_uint(x.y);
      }
    }
  }
  const float t = __fadd_rn(sum.x, sum.y);
  // A square below 2^-126 is off by 2^-150 at most: nothing beside 2^-90.  (At
  // 2^96 a segment the pair does not overflow: a lane has fewer than 2^31.)
  if (!(t < 0x1p96f) || (t < 0x1p-90f && any != 0)) {
    for (uint32_t k = 0; k < count; ++k) {
      const uint64_t at = static_cast<uint64_t>(first + k) * kOptBlock + lane * kOptLane;
      for (int j = 0; j < kOptLane && at + j < d.n; ++j) {
        const float x = element<Bf16>(d.grad, at + j);
        if ((__float_as_uint(x) & 0x7F800000u) == 0x7F800000u)
          ++s.nonfinite;
        else
          s.exact += static_cast<double>(x) * static_cast<double>(x);
      }
    }
    return;
  }
  // TwoSum of hi and each half
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const float x = half ? sum.y : sum.x;
    const float r = __fadd_rn(s.hi, x), back = __fsub_rn(r, s.hi);
    s.lo = __fadd_rn(s.lo, __fadd_rn(__fsub_rn(s.hi, __fsub_rn(r, back)), __fsub_rn(x, back)));
    s.hi = r;
  }
}

// Sums over a CTA, in thread 0, in an order that the thread count fixes.
__device__ __forceinline__ ClipPartial cta_sum(double sum, uint64_t count, ClipPartial* warps) {
#pragma unroll
  for (int k = 16; k > 0; k /= 2) {
    sum += __shfl_down_sync(0xFFFFFFFFu, sum, k);
    count += __shfl_down_sync(0xFFFFFFFFu, count, k);
  }
  if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = {sum, count};
  __syncthreads();
  ClipPartial all = {0.0, 0};
  if (threadIdx.x == 0)
    for (int k = 0; k < kOptWarps; ++k) {
      all.sumsq += warps[k].sumsq;
      all.nonfinite += warps[k].nonfinite;
    }
  return all;
}

__global__ void __launch_bounds__(32 * kOptWarps) clip_kernel(const ClipParams p) {
  __shared__ ClipPartial warps[kOptWarps];
  __shared__ bool last;
  wait_for_kernel_before();
  const int lane = threadIdx.x % 32;
  const uint32_t w = blockIdx.x * kOptWarps + threadIdx.x / 32;
  uint32_t b = opt_range(p.work.n_blocks, p.work.n_warps, w);
  const uint32_t end = opt_range(p.work.n_blocks, p.work.n_warps, w + 1);
  LaneSums s;
  if (b < end) {
    for (uint32_t t = p.work.start[w]; b < end; ++t) {
      const OptDesc d = p.work.tensors[t];
      const uint32_t stop = min(end, d.first + d.n_blocks);
      for (; b < stop; b += min(kClipSeg, stop - b)) {
        const uint32_t count = min(kClipSeg, stop - b);
        if (d.bf16_grad)
          add_segment<true>(d, b - d.first, count, lane, s);
        else
          add_segment<false>(d, b - d.first, count, lane, s);
      }
    }
  }
  const ClipPartial mine = cta_sum(static_cast<double>(s.hi) + static_cast<double>(s.lo) + s.exact, s.nonfinite, warps);
  if (threadIdx.x == 0) {
    p.partials[blockIdx.x] = mine;
    __threadfence();
    last = atomicInc(p.done, gridDim.x - 1) == gridDim.x - 1;  // wraps to zero with the last
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  double sum = 0.0;
  uint64_t count = 0;
  for (uint32_t i = threadIdx.x; i < gridDim.x; i += 32 * kOptWarps) {
    sum += __ldcg(&p.partials[i].sumsq);
    count += __ldcg(&p.partials[i].nonfinite);
  }
  const ClipPartial all = cta_sum(sum, count, warps);
  if (threadIdx.x == 0) {
    const double norm = p.grad_scale * sqrt(all.sumsq);
    fr_clip r;
    r.norm = static_cast<float>(norm);
    r.scale = all.nonfinite ? 0.0f : static_cast<float>(p.grad_scale * (norm > p.max_norm ? p.max_norm / norm : 1.0));
    r.nonfinite = all.nonfinite;
    *p.out = r;
  }
}

}  // namespace

cudaError_t launch_clip(const ClipParams& p, int n_ctas, cudaStream_t s) {
  return launch_chained(clip_kernel, n_ctas, 32 * kOptWarps, 0, s, p);
}

}  // namespace frk
