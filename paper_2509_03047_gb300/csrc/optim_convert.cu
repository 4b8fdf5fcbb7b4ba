// optim_convert.cu -- moments from 32 bits to 8 and back.
//
// Bound by memory, 10 bytes per element: GPT-2 small (1.24 GB) to 8 bits 181 us
// (6.8 TB/s), back 181 us (6.8); 18 million elements in 2,000 tensors 34 and 31 us,
// 8 of them what a launch and its first and last blocks take.  Not near its floor,
// element by element: 10,000 tensors of 1 to 2,000 elements (26 MB) 12 and 8.4 us;
// buffers off the vectors' boundaries, 134 million elements 342 and 271 to 288 us
// (194 and 197 aligned).
#include <type_traits>

#include "kernels.h"
#include "optim.h"
#include "optim_block.cuh"

namespace frk {

namespace {

// A negative second moment counts as zero, a NaN stays one.
__device__ __forceinline__ float not_negative(float x) { return x < 0.0f ? 0.0f : fabsf(x); }

// A whole block's loads.
template <bool ToEight>
struct Raw {
  std::conditional_t<ToEight, RawF32, RawCodes> m, v;
  uint32_t em, ev;
  __device__ __forceinline__ void load(const OptDesc& s, uint32_t block, int lane) {
    m.load(lane_at<ToEight ? 4 : 1>(s.m, block, lane), kOptLane);
    v.load(lane_at<ToEight ? 4 : 1>(s.v, block, lane), kOptLane);
    if (!ToEight) em = read_exponent(s.m_exp[block], kSpanM), ev = read_exponent(s.v_exp[block], kSpanV);
  }
};

template <bool ToEight, bool Random>
__device__ __forceinline__ void convert_whole(const Raw<ToEight>& r, const OptDesc& d, uint32_t block, RandomKey key, int lane) {
  const uint64_t first = static_cast<uint64_t>(block) * kOptBlock;
  Pair m[4], v[4];
  if constexpr (ToEight) {
    r.m.get(m);
    r.v.get(v);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = make_float2(not_negative(v[j].x), not_negative(v[j].y));
    uint32_t u[4];
    if (Random) random_pairs(key, random_counter(key, (first >> 1) + 4 * lane), u);
    const uint32_t em = store_codes<true, Random>(m, u, lane_at<1>(d.m, block, lane), kOptLane);
    const uint32_t ev = store_codes<false, Random>(v, u, lane_at<1>(d.v, block, lane), kOptLane);
    if (lane == 0) d.m_exp[block] = stored_exponent(em), d.v_exp[block] = stored_exponent(ev);
  } else {
    decode4<true>(r.m.a[0], r.em, m[0], m[1]);
    decode4<true>(r.m.a[1], r.em, m[2], m[3]);
    decode4<false>(r.v.a[0], r.ev, v[0], v[1]);
    decode4<false>(r.v.a[1], r.ev, v[2], v[3]);
    const Pair nan = pair(__uint_as_float(0x7FC00000u));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (r.em == 255) m[j] = nan;
      if (r.ev == 255) v[j] = nan;
    }
    store_f32(lane_at<4>(d.m, block, lane), kOptLane, m);
    store_f32(lane_at<4>(d.v, block, lane), kOptLane, v);
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
__global__ void __launch_bounds__(32 * kOptWarps) convert_kernel(const __grid_constant__ ConvertParams p) {
  constexpr uint32_t kBlocks = kConvertBlocks;
  const int lane = threadIdx.x % 32;
  uint32_t b = (blockIdx.x * kOptWarps + threadIdx.x / 32) * kBlocks;
  const uint32_t end = min(b + kBlocks, p.src.n_blocks);
  if (b >= end) return;
  uint32_t t = first_tensor(p.src, blockIdx.x, threadIdx.x / 32, kOptWarps, b);
  OptDesc s = p.src.tensors[t], d = p.dst.tensors[t];  // (the plans' tables: nothing writes them)
  wait_for_kernel_before();
#pragma unroll 1
  for (;;) {
    RandomKey key = {0, 0};
    if (Random) key = random_key(p.key, s.tensor);
    const uint32_t block = b - s.first, whole = s.aligned && d.aligned ? static_cast<uint32_t>(s.n / kOptBlock) : 0;
    if (b + kBlocks == end && block + kBlocks <= whole) {
      Raw<ToEight> r[kBlocks];
#pragma unroll
      for (uint32_t k = 0; k < kBlocks; ++k) r[k].load(s, block + k, lane);
#pragma unroll
      for (uint32_t k = 0; k < kBlocks; ++k) convert_whole<ToEight, Random>(r[k], d, block + k, key, lane);
      return;
    }
    if (block < whole) {
      Raw<ToEight> r;
      r.load(s, block, lane);
      convert_whole<ToEight, Random>(r, d, block, key, lane);
    } else {
      convert_any<ToEight, Random>(p.src.tensors + t, p.dst.tensors + t, block, key, lane);
    }
    if (++b == end) return;
    t = tensor_of(p.src, t, b);
    s = p.src.tensors[t], d = p.dst.tensors[t];
  }
}

}  // namespace

cudaError_t launch_convert(const ConvertParams& p, cudaStream_t s) {
  const int n_ctas = static_cast<int>(p.src.n_groups);
  if (!p.to_eight) return launch_chained(convert_kernel<false, false>, n_ctas, 32 * kOptWarps, 0, s, p);
  if (p.random) return launch_chained(convert_kernel<true, true>, n_ctas, 32 * kOptWarps, 0, s, p);
  return launch_chained(convert_kernel<true, false>, n_ctas, 32 * kOptWarps, 0, s, p);
}

}  // namespace frk
