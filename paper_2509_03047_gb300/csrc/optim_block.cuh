// optim_block.cuh -- a warp's block of 256 elements: loads, stores, random bits,
// coding of 8-bit moments.
#pragma once

#include "optim.h"
#include "optim_math.cuh"

namespace frk {

// The eight elements of a lane, in an aligned tensor lane * 8 + j, else j * 32
// + lane (single elements, coalesced).
template <bool Aligned>
__device__ __forceinline__ int place(int lane, int j) {
  return Aligned ? lane * kOptLane + j : j * 32 + lane;
}

// Loads and stores of a lane's elements [0, left) of a block; elements past the
// end read as zero.
template <bool Aligned>
__device__ __forceinline__ void load(const float* p, int lane, int left, float (&x)[kOptLane]) {
  if (Aligned && left >= (lane + 1) * kOptLane) {
    const float4 a = reinterpret_cast<const float4*>(p)[lane * 2], b = reinterpret_cast<const float4*>(p)[lane * 2 + 1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) x[j] = place<Aligned>(lane, j) < left ? p[place<Aligned>(lane, j)] : 0.0f;
}
template <bool Aligned>
__device__ __forceinline__ void store(float* p, int lane, int left, const float (&x)[kOptLane]) {
  if (Aligned && left >= (lane + 1) * kOptLane) {
    reinterpret_cast<float4*>(p)[lane * 2] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[lane * 2 + 1] = make_float4(x[4], x[5], x[6], x[7]);
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    if (place<Aligned>(lane, j) < left) p[place<Aligned>(lane, j)] = x[j];
}
template <bool Aligned>
__device__ __forceinline__ void load(const uint16_t* p, int lane, int left, float (&x)[kOptLane]) {
  if (Aligned && left >= (lane + 1) * kOptLane) {
    const uint4 a = reinterpret_cast<const uint4*>(p)[lane];
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    x[j] = place<Aligned>(lane, j) < left ? __uint_as_float(static_cast<uint32_t>(p[place<Aligned>(lane, j)]) << 16) : 0.0f;
}
template <bool Aligned>
__device__ __forceinline__ void store(uint16_t* p, int lane, int left, const uint16_t (&x)[kOptLane]) {
  if (Aligned && left >= (lane + 1) * kOptLane) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = x[2 * j] | static_cast<uint32_t>(x[2 * j + 1]) << 16;
    reinterpret_cast<uint4*>(p)[lane] = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    if (place<Aligned>(lane, j) < left) p[place<Aligned>(lane, j)] = x[j];
}
template <bool Aligned>
__device__ __forceinline__ void load(const uint8_t* p, int lane, int left, uint32_t (&x)[kOptLane]) {
  if (Aligned && left >= (lane + 1) * kOptLane) {
    const uint2 a = reinterpret_cast<const uint2*>(p)[lane];
#pragma unroll
    for (int j = 0; j < kOptLane; ++j) x[j] = ((j < 4 ? a.x : a.y) >> (8 * (j & 3))) & 0xFFu;
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) x[j] = place<Aligned>(lane, j) < left ? p[place<Aligned>(lane, j)] : 0u;
}
template <bool Aligned>
__device__ __forceinline__ void store(uint8_t* p, int lane, int left, const uint32_t (&x)[kOptLane]) {
  if (Aligned && left >= (lane + 1) * kOptLane) {
    reinterpret_cast<uint2*>(p)[lane] = make_uint2(x[0] | x[1] << 8 | x[2] << 16 | x[3] << 24, x[4] | x[5] << 8 | x[6] << 16 | x[7] << 24);
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    if (place<Aligned>(lane, j) < left) p[place<Aligned>(lane, j)] = static_cast<uint8_t>(x[j]);
}

// The random bits of a lane's elements: for the moments, and for a bf16 weight.
template <bool Aligned>
__device__ __forceinline__ void random_bits(RandomKey key, uint64_t first, int lane, uint32_t (&moments)[kOptLane],
                                            uint32_t (&weights)[kOptLane]) {
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) {
    const uint64_t i = first + place<Aligned>(lane, j);
    const int odd = static_cast<int>(i & 1);
    const uint32_t u = random_pair(key, i >> 1), w = random_weights(u);
    moments[j] = random_moments(u, odd);
    weights[j] = odd ? w & 0xFFFFu : w >> 16;
  }
}

__device__ __forceinline__ uint32_t warp_max(uint32_t x) { return __reduce_max_sync(0xFFFFFFFFu, x); }

// Codes a block's moments and stores them; rnd: the lane's random bits, shifted so that the low half counts.
template <bool Aligned, bool Signed>
__device__ __forceinline__ void store_moments(const float (&x)[kOptLane], const uint32_t (&rnd)[kOptLane], bool random,
                                              uint8_t* codes, uint8_t* exponent, int lane, int left) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  const uint32_t e = block_exponent(warp_max(top), Signed ? kSpanM : kSpanV);
  uint32_t c[kOptLane];
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) {
    const uint32_t r = random ? (rnd[j] & 0xFFFFu) << 4 : round_nearest(__float_as_uint(x[j]));
    c[j] = Signed ? encode_m(x[j], r, e) : encode_v(x[j], r, e);
  }
  store<Aligned>(codes, lane, left, c);
  if (lane == 0) *exponent = static_cast<uint8_t>(e);
}

}  // namespace frk
