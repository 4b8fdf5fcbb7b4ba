// optim_convert.cu -- moments from 32 bits to 8 and back.
#include "kernels.h"
#include "optim.h"
#include "optim_block.cuh"

namespace frk {

namespace {

// A negative second moment counts as zero, a NaN stays one.
__device__ __forceinline__ float not_negative(float x) { return x < 0.0f ? 0.0f : fabsf(x); }

template <bool ToEight, bool Random>
__device__ __forceinline__ void convert_whole(const OptDesc& s, const OptDesc& d, uint32_t block, RandomKey key, int lane) {
  const uint64_t first = static_cast<uint64_t>(block) * kOptBlock;
  Pair m[4], v[4];
  if constexpr (ToEight) {
    RawF32 raw_m, raw_v;
    raw_m.load(static_cast<const float*>(s.m) + first, lane);
    raw_v.load(static_cast<const float*>(s.v) + first, lane);
    raw_m.get(m);
    raw_v.get(v);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = make_float2(not_negative(v[j].x), not_negative(v[j].y));
    uint32_t u[4];
    if (Random) random_pairs(key, first, lane, u);
    store_codes<true, Random>(m, u, static_cast<uint8_t*>(d.m) + first, d.m_exp + block, lane);
    store_codes<false, Random>(v, u, static_cast<uint8_t*>(d.v) + first, d.v_exp + block, lane);
  } else {
    RawCodes raw_m, raw_v;
    raw_m.load(static_cast<const uint8_t*>(s.m) + first, lane);
    raw_v.load(static_cast<const uint8_t*>(s.v) + first, lane);
    const uint32_t em = s.m_exp[block], ev = s.v_exp[block];
    decode4<true>(raw_m.a.x, em, m[0], m[1]);
    decode4<true>(raw_m.a.y, em, m[2], m[3]);
    decode4<false>(raw_v.a.x, ev, v[0], v[1]);
    decode4<false>(raw_v.a.y, ev, v[2], v[3]);
    const Pair nan = pair(__uint_as_float(0x7FC00000u));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (em == 255) m[j] = nan;
      if (ev == 255) v[j] = nan;
    }
    store_f32(static_cast<float*>(d.m) + first, lane, m);
    store_f32(static_cast<float*>(d.v) + first, lane, v);
  }
}

template <bool ToEight, bool Random>
__device__ __noinline__ void convert_any(const OptDesc* from, const OptDesc* to, uint32_t block, RandomKey key, int lane) {
  const OptDesc s = *from, d = *to;
  const uint64_t first = static_cast<uint64_t>(block) * kOptBlock;
  const int left = static_cast<int>(min(s.n - first, static_cast<uint64_t>(kOptBlock)));
  float m[kOptLane], v[kOptLane];
  if (ToEight) {
    load_any<float>(static_cast<const float*>(s.m) + first, lane, left, m);
    load_any<float>(static_cast<const float*>(s.v) + first, lane, left, v);
#pragma unroll
    for (int j = 0; j < kOptLane; ++j) v[j] = not_negative(v[j]);
    store_codes_any<true>(m, Random, key, first, static_cast<uint8_t*>(d.m) + first, d.m_exp + block, lane, left);
    store_codes_any<false>(v, Random, key, first, static_cast<uint8_t*>(d.v) + first, d.v_exp + block, lane, left);
  } else {
    load_codes_any<true>(static_cast<const uint8_t*>(s.m) + first, s.m_exp[block], lane, left, m);
    load_codes_any<false>(static_cast<const uint8_t*>(s.v) + first, s.v_exp[block], lane, left, v);
    store_any<float>(static_cast<float*>(d.m) + first, lane, left, m);
    store_any<float>(static_cast<float*>(d.v) + first, lane, left, v);
  }
}

template <bool ToEight, bool Random>
__global__ void __launch_bounds__(32 * kOptWarps, 4) convert_kernel(const __grid_constant__ ConvertParams p) {
  wait_for_kernel_before();
  const int lane = threadIdx.x % 32;
  const uint32_t b = blockIdx.x * kOptWarps + threadIdx.x / 32;
  if (b >= p.src.n_blocks) return;
  const uint32_t t = tensor_of(p.src, p.src.start[blockIdx.x], b);
  const OptDesc s = p.src.tensors[t], d = p.dst.tensors[t];
  RandomKey key = {0, 0};
  if (Random) key = random_key(p.key, s.tensor);
  const uint32_t block = b - s.first;
  if (s.aligned && d.aligned && block < s.n / kOptBlock)
    convert_whole<ToEight, Random>(s, d, block, key, lane);
  else
    convert_any<ToEight, Random>(p.src.tensors + t, p.dst.tensors + t, block, key, lane);
}

}  // namespace

cudaError_t launch_convert(const ConvertParams& p, cudaStream_t s) {
  const int n_ctas = static_cast<int>(p.src.n_units);
  if (!p.to_eight) return launch_chained(convert_kernel<false, false>, n_ctas, 32 * kOptWarps, 0, s, p);
  if (p.random) return launch_chained(convert_kernel<true, true>, n_ctas, 32 * kOptWarps, 0, s, p);
  return launch_chained(convert_kernel<true, false>, n_ctas, 32 * kOptWarps, 0, s, p);
}

}  // namespace frk
