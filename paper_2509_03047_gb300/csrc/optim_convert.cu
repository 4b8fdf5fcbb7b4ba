// optim_convert.cu -- moments from 32 bits to 8 and back.
#include "kernels.h"
#include "optim.h"
#include "optim_block.cuh"

namespace frk {

namespace {

template <bool Aligned, bool ToEight>
__device__ __forceinline__ void convert_block(const OptDesc& s, const OptDesc& d, uint32_t block, RandomKey key, bool random,
                                              int lane) {
  const uint64_t first = static_cast<uint64_t>(block) * kOptBlock;
  const int left = static_cast<int>(min(s.n - first, static_cast<uint64_t>(kOptBlock)));
  float m[kOptLane], v[kOptLane];
  if (ToEight) {
    load<Aligned>(static_cast<const float*>(s.m) + first, lane, left, m);
    load<Aligned>(static_cast<const float*>(s.v) + first, lane, left, v);
    uint32_t rm[kOptLane], rv[kOptLane], rw[kOptLane];
    if (random) random_bits<Aligned>(key, first, lane, rm, rw);
#pragma unroll
    for (int j = 0; j < kOptLane; ++j) {
      rv[j] = rm[j] >> 16;
      v[j] = v[j] < 0.0f ? 0.0f : v[j];
    }
    store_moments<Aligned, true>(m, rm, random, static_cast<uint8_t*>(d.m) + first, d.m_exp + block, lane, left);
    store_moments<Aligned, false>(v, rv, random, static_cast<uint8_t*>(d.v) + first, d.v_exp + block, lane, left);
  } else {
    uint32_t a[kOptLane], c[kOptLane];
    load<Aligned>(static_cast<const uint8_t*>(s.m) + first, lane, left, a);
    load<Aligned>(static_cast<const uint8_t*>(s.v) + first, lane, left, c);
    const uint32_t em = s.m_exp[block], ev = s.v_exp[block];
#pragma unroll
    for (int j = 0; j < kOptLane; ++j) {
      m[j] = decode_m(a[j], em);
      v[j] = decode_v(c[j], ev);
    }
    store<Aligned>(static_cast<float*>(d.m) + first, lane, left, m);
    store<Aligned>(static_cast<float*>(d.v) + first, lane, left, v);
  }
}

__global__ void __launch_bounds__(32 * kOptWarps) convert_kernel(const ConvertParams p) {
  wait_for_kernel_before();
  const int lane = threadIdx.x % 32;
  const uint32_t w = blockIdx.x * kOptWarps + threadIdx.x / 32;
  uint32_t b = opt_range(p.src.n_blocks, p.src.n_warps, w);
  const uint32_t end = opt_range(p.src.n_blocks, p.src.n_warps, w + 1);
  if (b >= end) return;
  for (uint32_t t = p.src.start[w]; b < end; ++t) {
    const OptDesc s = p.src.tensors[t], d = p.dst.tensors[t];
    const RandomKey key = random_key(p.key, s.tensor);
    const uint32_t stop = min(end, s.first + s.n_blocks);
    const bool aligned = s.aligned && d.aligned;
    for (; b < stop; ++b) {
      if (p.to_eight) {
        if (aligned)
          convert_block<true, true>(s, d, b - s.first, key, p.random, lane);
        else
          convert_block<false, true>(s, d, b - s.first, key, p.random, lane);
      } else {
        if (aligned)
          convert_block<true, false>(s, d, b - s.first, key, p.random, lane);
        else
          convert_block<false, false>(s, d, b - s.first, key, p.random, lane);
      }
    }
  }
}

}  // namespace

cudaError_t launch_convert(const ConvertParams& p, int n_ctas, cudaStream_t s) {
  return launch_chained(convert_kernel, n_ctas, 32 * kOptWarps, 0, s, p);
}

}  // namespace frk
