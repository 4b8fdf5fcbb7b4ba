// embed_vector.cuh -- V consecutive elements of a row, in bf16 or fp32, as fp32 numbers.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>
#include <cstring>

namespace frk {

template <int Bytes>
struct Words;
template <>
struct Words<2> { using T = uint16_t; };
template <>
struct Words<4> { using T = uint32_t; };
template <>
struct Words<8> { using T = uint2; };
template <>
struct Words<16> { using T = uint4; };

// As they lie in memory: one load of up to 16 bytes, or two.
template <int V, bool Bf16>
struct Raw {
  static constexpr int kBytes = V * (Bf16 ? 2 : 4), kPiece = kBytes < 16 ? kBytes : 16, kPieces = kBytes / kPiece;
  using T = typename Words<kPiece>::T;
  T w[kPieces];
  __device__ __forceinline__ void load(const void* base, uint64_t element) {
    const T* at = reinterpret_cast<const T*>(static_cast<const uint8_t*>(base) + element * (Bf16 ? 2 : 4));
#pragma unroll
    for (int k = 0; k < kPieces; ++k) w[k] = at[k];
  }
  // To shared memory, asynchronously where a piece has four bytes or more.
  static __device__ __forceinline__ void copy(void* shared, const void* base, uint64_t element) {
    const T* at = reinterpret_cast<const T*>(static_cast<const uint8_t*>(base) + element * (Bf16 ? 2 : 4));
    T* const to = static_cast<T*>(shared);
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(to + k));
      if constexpr (kPiece == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(a), "l"(at + k) : "memory");
      else if constexpr (kPiece >= 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(a), "l"(at + k), "n"(kPiece) : "memory");
      else
        to[k] = at[k];
    }
  }
  __device__ __forceinline__ void store(void* base, uint64_t element) const {
    T* at = reinterpret_cast<T*>(static_cast<uint8_t*>(base) + element * (Bf16 ? 2 : 4));
#pragma unroll
    for (int k = 0; k < kPieces; ++k) at[k] = w[k];
  }
  __device__ __forceinline__ void clear() { memset(w, 0, sizeof w); }
  __device__ __forceinline__ void get(float (&x)[V]) const {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if constexpr (Bf16) {
        const uint32_t word = V == 1 ? reinterpret_cast<const uint16_t*>(w)[0] : reinterpret_cast<const uint32_t*>(w)[j / 2];
        x[j] = __uint_as_float(j % 2 ? word & 0xFFFF0000u : word << 16);
      } else {
        x[j] = __uint_as_float(reinterpret_cast<const uint32_t*>(w)[j]);
      }
    }
  }
  __device__ __forceinline__ void set(const float (&x)[V]) {
    if constexpr (Bf16) {
#pragma unroll
      for (int j = 0; j < V; ++j) reinterpret_cast<__nv_bfloat16*>(w)[j] = __float2bfloat16_rn(x[j]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) reinterpret_cast<float*>(w)[j] = x[j];
    }
  }
};

}  // namespace frk
