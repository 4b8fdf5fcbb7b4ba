// optim_clip.cu -- the norm of all gradients, the count of non-finite ones, and
// the factor that clips them, in one launch.
//
// A lane squares the eight elements that it has of each block into two fp32
// sums, which a float pair takes up error-free after the warp's blocks of a
// segment: at most 64 squares are added in fp32 at a time.  A sum that is
// not finite (a NaN or Inf, or an overflow) or so small that squares may have
// lost bits to underflow is added again by the lanes concerned, element by
// element in fp64, the non-finite ones counted and left out.  Lanes, warps and
// CTAs are added as float pairs in a fixed order, by the CTA that is last to
// finish at the end.
//
// Which lane has which element does not depend on the address (the order of the
// sums must not): off the 16-byte boundary a lane loads the granules around its
// elements and shifts them out.  (Each granule that it loads holds one of them.)
//
// Bound by reading: one pass, up to eight 16-byte loads per lane in flight with
// 32 warps per SM.  GB300: 2.0 GB of bf16 278 us (7.2 TB/s; a plain read of 8 GB
// reaches 7.4), 247 MB 38 us, 400 views at odd places in 108 MB 25 us (a tensor's
// end inside a warp's blocks costs it two latencies), 2 MB of 51 tensors in L2 6.1
// us, of one tensor 4.6.  Of these a launch is 2, the loads, behind the tensor's
// descriptor, 1, and the last CTA's sum, behind the others' counts, 1.6.
#include "kernels.h"
#include "optim_block.cuh"

namespace frk {

namespace {

static_assert(kClipMost * kOptLane / 2 <= 64, "squares in one fp32 sum");

template <bool Bf16>
__device__ __forceinline__ float element(const void* p, uint64_t i) {
  return Bf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(p)[i]) << 16) : static_cast<const float*>(p)[i];
}

// (hi, lo) += (h, l), error-free in hi (Knuth's TwoSum), to 2^-44 in all.
__device__ __forceinline__ void add_to_pair(float& hi, float& lo, float h, float l) {
  const float s = __fadd_rn(hi, h), back = __fsub_rn(s, hi);
  const float e = __fadd_rn(__fadd_rn(__fsub_rn(hi, __fsub_rn(s, back)), __fsub_rn(h, back)), __fadd_rn(lo, l));
  hi = __fadd_rn(s, e);
  lo = __fsub_rn(e, __fsub_rn(hi, s));
}

// Granules of 16 bytes around a lane's eight elements.
template <bool Bf16, bool Shifted>
struct Granules {
  static constexpr int kWords = Bf16 ? 4 : 8, kLoaded = kWords / 4 + Shifted;
  uint4 g[kLoaded];
  // at: address of the first element, floored to a granule's
  __device__ __forceinline__ void load(uint64_t at) {
#pragma unroll
    for (int k = 0; k < kLoaded; ++k) g[k] = load_16(reinterpret_cast<const uint4*>(at) + k);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < kLoaded; ++k) g[k] = make_uint4(0, 0, 0, 0);
  }
  // shift: bytes from there to the first element
  __device__ __forceinline__ void words(uint32_t shift, uint32_t (&w)[kWords]) const {
    uint32_t a[4 * kLoaded];
#pragma unroll
    for (int k = 0; k < kLoaded; ++k) a[4 * k] = g[k].x, a[4 * k + 1] = g[k].y, a[4 * k + 2] = g[k].z, a[4 * k + 3] = g[k].w;
    if constexpr (Shifted) {
      // by 8 bytes, then 4, then 2
#pragma unroll
      for (int i = 0; i < kWords + 2; ++i) a[i] = shift & 8 ? a[i + 2 < 4 * kLoaded ? i + 2 : i] : a[i];
#pragma unroll
      for (int i = 0; i < kWords + 1; ++i) a[i] = shift & 4 ? a[i + 1] : a[i];
      if (Bf16)
#pragma unroll
        for (int i = 0; i < kWords; ++i) a[i] = shift & 2 ? __funnelshift_r(a[i], a[i + 1], 16) : a[i];
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = a[i];
  }
};

template <bool Bf16>
__device__ __forceinline__ void add_words(const uint32_t (&w)[Bf16 ? 4 : 8], Pair& sum, uint32_t& any) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    Pair x;
    if (Bf16) {
      x = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u));
      any |= w[j];
    } else {
      x = make_float2(__uint_as_float(w[Bf16 ? 0 : 2 * j]), __uint_as_float(w[Bf16 ? 0 : 2 * j + 1]));
      any |= w[Bf16 ? 0 : 2 * j] | w[Bf16 ? 0 : 2 * j + 1];
    }
    sum = fma2(x, x, sum);
  }
}

// The warp's blocks [block, stop) of one tensor.
template <bool Bf16, bool Shifted>
__device__ __forceinline__ void add_blocks(const void* grad, uint64_t n, uint32_t block, uint32_t stop, int lane, ClipPartial& s) {
  constexpr int kAhead = (Bf16 ? 8 : 4) / (Shifted ? 2 : 1);  // blocks loaded at a time
  constexpr int kBytes = Bf16 ? 2 : 4;
  Pair sum = pair(0.0f);
  uint32_t any = 0;  // a bit set: some element is not +0
  const uint32_t shift = Shifted ? static_cast<uint32_t>(reinterpret_cast<uint64_t>(grad)) % 16 : 0;
  const uint64_t base = reinterpret_cast<uint64_t>(grad) - shift + lane * kOptLane * kBytes;
  const uint32_t whole = static_cast<uint32_t>(min(n / kOptBlock, static_cast<uint64_t>(stop)));
  uint32_t b = block;
  for (; b < whole; b += kAhead) {
    Granules<Bf16, Shifted> r[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (b + k < whole)
        r[k].load(base + static_cast<uint64_t>(b + k) * kOptBlock * kBytes);
      else
        r[k].clear();
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      uint32_t w[Bf16 ? 4 : 8];
      r[k].words(shift, w);
      add_words<Bf16>(w, sum, any);
    }
  }
  // the tensor's last block, where it is not whole and this warp's
  const uint32_t last = static_cast<uint32_t>(n / kOptBlock);
  if (last < stop && n % kOptBlock && last >= block) {
    const uint64_t at = static_cast<uint64_t>(last) * kOptBlock + lane * kOptLane;
#pragma unroll
    for (int j = 0; j < kOptLane; j += 2) {
      Pair x;
      x.x = at + j < n ? element<Bf16>(grad, at + j) : 0.0f;
      x.y = at + j + 1 < n ? element<Bf16>(grad, at + j + 1) : 0.0f;
      sum = fma2(x, x, sum);
      any |= __float_as_uint(x.x) | __float_as_uint(x.y);
    }
  }
  const float t = __fadd_rn(sum.x, sum.y);
  // A square below 2^-126 is off by 2^-150 at most: nothing beside 2^-90.  (Sums
  // below 2^80 do not overflow the pairs: a plan has fewer than 2^40 elements.)
  if (!(t < 0x1p80f) || (t < 0x1p-90f && any != 0)) {
    for (b = block; b < stop; ++b) {
      const uint64_t at = static_cast<uint64_t>(b) * kOptBlock + lane * kOptLane;
      for (int j = 0; j < kOptLane && at + j < n; ++j) {
        const float x = element<Bf16>(grad, at + j);
        if ((__float_as_uint(x) & 0x7F800000u) == 0x7F800000u)
          ++s.nonfinite;
        else
          s.exact += static_cast<double>(x) * static_cast<double>(x);
      }
    }
    return;
  }
  add_to_pair(s.hi, s.lo, sum.x, 0.0f);
  add_to_pair(s.hi, s.lo, sum.y, 0.0f);
}

// The sum over a warp, in lane 0.  The fp64 pipe is narrow (a conversion and an
// addition in each of an SM's warps take 0.7 us): it is left out where no lane
// has a sum in fp64.
__device__ __forceinline__ void warp_sum(ClipPartial& s) {
#pragma unroll
  for (int k = 16; k > 0; k /= 2) {
    const float h = __shfl_down_sync(0xFFFFFFFFu, s.hi, k), l = __shfl_down_sync(0xFFFFFFFFu, s.lo, k);
    add_to_pair(s.hi, s.lo, h, l);
  }
  if (!__any_sync(0xFFFFFFFFu, s.exact != 0.0 || s.nonfinite != 0)) return;
#pragma unroll
  for (int k = 16; k > 0; k /= 2) {
    s.exact += __shfl_down_sync(0xFFFFFFFFu, s.exact, k);
    s.nonfinite += __shfl_down_sync(0xFFFFFFFFu, s.nonfinite, k);
  }
}

// The record of a sum.
__device__ __forceinline__ fr_clip record(const ClipPartial& s, float grad_scale, float max_norm) {
  fr_clip r;
  r.nonfinite = s.nonfinite;
  r.norm = 0.0f;
  if (s.hi > 0.0f) {
    // the root by a step of Newton's from an approximation, its residual exact: 0.6 us less than in fp64
    const float y = rsqrtf(s.hi), x = __fmul_rn(s.hi, y), xx = __fmul_rn(x, x);
    const float e = __fadd_rn(__fsub_rn(__fsub_rn(s.hi, xx), __fmaf_rn(x, x, -xx)), s.lo);
    r.norm = __fmul_rn(grad_scale, __fmaf_rn(__fmul_rn(0.5f, y), e, x));
  }
  const float part = r.norm > max_norm ? __fdiv_rn(max_norm, r.norm) : 1.0f;
  r.scale = __fmul_rn(grad_scale, part);
  // in fp64 too where fp32 holds the norm or the quotient, and with it perhaps the factor, with fewer bits
  if (s.exact != 0.0 || r.norm == INFINITY || (s.hi > 0.0f && r.norm < 0x1p-126f) || part < 0x1p-126f) {
    const double norm = grad_scale * sqrt(static_cast<double>(s.hi) + static_cast<double>(s.lo) + s.exact);
    r.norm = static_cast<float>(norm);
    r.scale = norm > max_norm ? static_cast<float>(grad_scale * (max_norm / norm)) : grad_scale;
  }
  if (s.nonfinite) r.scale = 0.0f;
  return r;
}

// What the norm needs of a tensor.
struct Tensor {
  const void* grad;
  uint64_t n;
  uint32_t first, n_blocks, bf16;
};
__device__ __forceinline__ Tensor tensor(const ClipParams& p, uint32_t t) {
  const OptDesc& d = p.work.tensors[t];
  return {d.grad, d.n, d.first, d.n_blocks, d.bf16_grad};
}

__global__ void __launch_bounds__(32 * kClipWarps, 1) clip_kernel(const __grid_constant__ ClipParams p) {
  __shared__ ClipPartial warps[kClipWarps];
  const int lane = threadIdx.x % 32;
  const uint32_t warp = threadIdx.x / 32, per_warp = p.work.per_warp;
  uint32_t t = 0, b = (blockIdx.x * kClipWarps + warp) * per_warp;
  Tensor d = {};
  if (b < p.work.n_blocks) d = tensor(p, t = first_tensor(p.work, blockIdx.x, warp, kClipWarps, b));  // (the plan's tables: nothing writes them)
  wait_for_kernel_before();
  ClipPartial s = {0.0f, 0.0f, 0.0, 0};
  for (uint32_t k = blockIdx.x; k < p.work.n_groups; k += gridDim.x) {
    b = (k * kClipWarps + warp) * per_warp;
    const uint32_t end = min(b + per_warp, p.work.n_blocks);
    if (b >= end) break;
    if (k != blockIdx.x) {
      const uint32_t now = first_tensor(p.work, k, warp, kClipWarps, b);
      if (now != t) d = tensor(p, t = now);
    }
    for (;;) {
      const uint32_t from = b - d.first, to = min(end - d.first, d.n_blocks);
      b += to - from;
      const bool shifted = reinterpret_cast<uint64_t>(d.grad) % 16 != 0;
      if (d.bf16)
        shifted ? add_blocks<true, true>(d.grad, d.n, from, to, lane, s) : add_blocks<true, false>(d.grad, d.n, from, to, lane, s);
      else
        shifted ? add_blocks<false, true>(d.grad, d.n, from, to, lane, s) : add_blocks<false, false>(d.grad, d.n, from, to, lane, s);
      if (b >= end) break;
      d = tensor(p, ++t);  // a warp's blocks are side by side: so are their tensors
    }
  }
  warp_sum(s);
  if (lane == 0) warps[warp] = s;
  __syncthreads();
  if (warp != 0) return;
  static_assert(kClipWarps == 32, "one lane for each");
  s = warps[lane];
  warp_sum(s);
  uint32_t before = 0;
  if (lane == 0) {
    p.partials[blockIdx.x] = s;
    // releases the partial sum, and acquires the others' for the last; wraps to zero with it
    asm volatile("atom.inc.acq_rel.gpu.global.u32 %0, [%1], %2;" : "=r"(before) : "l"(p.done), "r"(gridDim.x - 1) : "memory");
  }
  if (__shfl_sync(0xFFFFFFFFu, before, 0) != gridDim.x - 1) return;
  __syncwarp();
  s = {0.0f, 0.0f, 0.0, 0};
  constexpr int kEach = (kClipCtas + 31) / 32;
  ClipPartial q[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const uint32_t i = k * 32 + lane;
    q[k] = {0.0f, 0.0f, 0.0, 0};
    if (i < gridDim.x) {
      const ClipPartial* at = p.partials + i;
      q[k] = {__ldcg(&at->hi), __ldcg(&at->lo), __ldcg(&at->exact), __ldcg(&at->nonfinite)};
    }
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    add_to_pair(s.hi, s.lo, q[k].hi, q[k].lo);
    if (q[k].exact != 0.0) s.exact += q[k].exact;
    s.nonfinite += q[k].nonfinite;
  }
  warp_sum(s);
  if (lane == 0) *p.out = record(s, p.grad_scale, p.max_norm);
}

}  // namespace

cudaError_t launch_clip(const ClipParams& p, cudaStream_t s) {
  const uint32_t n_ctas = p.work.n_groups < 1 ? 1 : p.work.n_groups < kClipCtas ? p.work.n_groups : kClipCtas;
  return launch_chained(clip_kernel, static_cast<int>(n_ctas), 32 * kClipWarps, 0, s, p);
}

}  // namespace frk
