// muon_block.cuh -- an iterate's blocks: places of chunks of eight elements,
// halves of a number.
#pragma once

#include <cuda_fp16.h>

#include "muon.h"

namespace frk {

// Byte offset of the 16-byte chunk of columns 8 c ... 8 c + 7 of row r in a matrix of `col_blocks` blocks per block row.
__device__ __forceinline__ uint64_t chunk_at(uint32_t col_blocks, uint32_t r, uint32_t c) {
  const uint64_t block = static_cast<uint64_t>(r / kBlockRows) * col_blocks + c / 8;
  return block * kMuonBlockBytes + (r % kBlockRows) * 128 + (((c % 8) ^ (r % 8)) * 16);
}

// The same of the second halves.
__device__ __forceinline__ uint64_t low_at(uint32_t col_blocks, uint32_t r, uint32_t c) {
  const uint64_t block = static_cast<uint64_t>(r / kBlockRows) * col_blocks + c / 8;
  return block * kMuonBlockBytes + ((c % 8) * kBlockRows + r % kBlockRows) * 16;
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

}  // namespace frk
