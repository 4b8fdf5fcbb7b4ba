// muon_block.cuh -- an iterate's blocks: places of chunks of eight elements,
// halves of a number, what a product's sum becomes.
#pragma once

#include <cuda_fp16.h>

#include "muon.h"

namespace frk {

// Byte offset of the 16-byte chunk of columns 8 c ... 8 c + 7 of row r in a matrix of `col_blocks` blocks per block row.
__device__ __forceinline__ uint64_t chunk_at(uint32_t col_blocks, uint32_t r, uint32_t c) {
  const uint64_t block = static_cast<uint64_t>(r / kBlockRows) * col_blocks + c / 8;
  return block * kBlockBytes + (r % kBlockRows) * 128 + (((c % 8) ^ (r % 8)) * 16);
}

__device__ __forceinline__ uint32_t half2_bits(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return reinterpret_cast<const uint32_t&>(h);
}
__device__ __forceinline__ float2 half2_floats(uint32_t w) { return __half22float2(reinterpret_cast<const __half2&>(w)); }

// The two fp16 numbers of each of eight: the nearest one, and the nearest one to what is left.
__device__ __forceinline__ void split(const float (&x)[8], uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    h[j] = half2_bits(x[2 * j], x[2 * j + 1]);
    const float2 f = half2_floats(h[j]);
    l[j] = half2_bits(x[2 * j] - f.x, x[2 * j + 1] - f.y);
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void floats(const uint4& w, float (&x)[8]) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = half2_floats(v[j]);
    x[2 * j] = f.x;
    x[2 * j + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 halves(const float (&x)[8]) {
  return make_uint4(half2_bits(x[0], x[1]), half2_bits(x[2], x[3]), half2_bits(x[4], x[5]), half2_bits(x[6], x[7]));
}

// What eight sums of a product, of row r and the columns 8 c ..., become.
//   S = X X^T            sums in X's scale twice
//   P = a I + b S + c S^2
//   X = P X1 + a X2      X1, X2 the halves of the old X; a I in P has the first one's part
template <int kPhase>
__device__ __forceinline__ void finish_chunk(const MuonProduct& p, const MuonDesc& d, uint32_t r, uint32_t c, float (&v)[8]) {
  if (kPhase == kGram) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= kScaleS / (kScaleX * kScaleX);
    *reinterpret_cast<uint4*>(p.work + d.s + chunk_at(2 * d.side_blocks, r, c)) = halves(v);
  } else if (kPhase == kPoly) {
    const uint64_t at = chunk_at(2 * d.side_blocks, r, c);
    float s[8];
    floats(*reinterpret_cast<const uint4*>(p.work + d.s + at), s);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float own = r == 8 * c + j ? p.a * kScaleP : 0.0f;
      v[j] = own + s[j] * (p.b * (kScaleP / kScaleS)) + v[j] * (p.c * (kScaleP / (kScaleS * kScaleS)));
    }
    *reinterpret_cast<uint4*>(p.work + d.p + at) = halves(v);
  } else {
    const uint64_t at = chunk_at(d.col_blocks, r, c);
    float x[8];
    floats(*reinterpret_cast<const uint4*>(p.work + d.low + at), x);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = v[j] * (1.0f / kScaleP) + p.a * x[j];
    uint4 hi, lo;
    split(v, hi, lo);
    *reinterpret_cast<uint4*>(p.work + d.x[p.from ^ 1] + at) = hi;
    *reinterpret_cast<uint4*>(p.work + d.low + at) = lo;
  }
}

}  // namespace frk
