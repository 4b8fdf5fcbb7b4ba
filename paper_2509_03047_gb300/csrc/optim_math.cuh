// optim_math.cuh -- arithmetic of the optimizer step that its kernels share:
// the update, the 8-bit moments' code, the random bits of a rounding.
//
// Every operation is written as the one rounding that it is (no contraction
// is left to the compiler), so all kernels and paths give the same bits.
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

#include "optim.h"

namespace frk {

// ---- 8-bit moments (the format is described in flashrec.h)

constexpr int kSpanM = 15, kSpanV = 31;  // binades below a block's top

// A block's exponent from the largest bit pattern of |x| in it (256 for some
// NaNs, stored as 255).  The largest code is reached whichever way its element
// is rounded: 0xFFFFF is the most that a rounding adds.
__device__ __forceinline__ uint32_t block_exponent(uint32_t top, int span) { return max((top + 0xFFFFFu) >> 23, static_cast<uint32_t>(span + 1)); }
__device__ __forceinline__ uint8_t stored_exponent(uint32_t e) { return static_cast<uint8_t>(min(e, 255u)); }
// An exponent byte as it is read: written by somebody else it may be below its floor.
__device__ __forceinline__ uint32_t read_exponent(uint32_t e, int span) { return max(e, static_cast<uint32_t>(span + 1)); }
__device__ __forceinline__ uint32_t code_base(uint32_t e, int span) { return (e - span) * 8; }

__device__ __forceinline__ uint32_t round_nearest(uint32_t bits) { return 0x7FFFFu + ((bits >> 20) & 1u); }

// r: what the rounding adds below bit 20.
__device__ __forceinline__ uint32_t encode_m(float x, uint32_t r, uint32_t e) {
  const uint32_t bits = __float_as_uint(x);
  const int c = static_cast<int>(((bits & 0x7FFFFFFFu) + r) >> 20) - static_cast<int>(code_base(e, kSpanM));
  return c < 1 || e >= 255 ? 0u : static_cast<uint32_t>(c) | ((bits >> 24) & 0x80u);
}
__device__ __forceinline__ uint32_t encode_v(float x, uint32_t r, uint32_t e) {
  const uint32_t bits = __float_as_uint(x) & 0x7FFFFFFFu;
  const int c = static_cast<int>((bits + r) >> 20) - static_cast<int>(code_base(e, kSpanV));
  return bits == 0 || e >= 255 ? 0u : static_cast<uint32_t>(max(c, 1));
}
__device__ __forceinline__ float decode_m(uint32_t code, uint32_t e) {
  const uint32_t c = code & 0x7Fu;
  const uint32_t bits = c ? ((c + code_base(e, kSpanM)) << 20) | ((code & 0x80u) << 24) : 0u;
  return e == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(bits);
}
__device__ __forceinline__ float decode_v(uint32_t code, uint32_t e) {
  const uint32_t bits = code ? (code + code_base(e, kSpanV)) << 20 : 0u;
  return e == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(bits);
}

// ---- random bits
//
// A counter-based generator: two rounds of multiplication and shift over the
// index of a pair of elements, keyed by 64 bits per tensor, then one product
// for each number that is taken.  The factors are, from L'Ecuyer, "Tables of
// linear congruential generators of different sizes and good lattice structure"
// (1999) and its successors, multipliers modulo 2^32; the golden ratio's in 64
// bits; and two odd 32-bit numbers of many scattered bits for a counter's low
// and high word, of which nothing is asked but that (the first a prime near the
// golden ratio's; the tests measure what comes out).
struct RandomKey {
  uint32_t lo, hi;
};
__device__ __forceinline__ RandomKey random_key(uint64_t key, uint32_t tensor) {
  const uint64_t k = mix64(key + tensor * 0x9E3779B97F4A7C15ull);
  return {static_cast<uint32_t>(k), static_cast<uint32_t>(k >> 32)};
}
constexpr uint32_t kRandomStep = 0x9E3779B1u;  // from a pair's counter to the next one's
__device__ __forceinline__ uint32_t random_counter(RandomKey k, uint64_t pair) {
  return static_cast<uint32_t>(pair) * kRandomStep + (k.lo ^ (static_cast<uint32_t>(pair >> 32) * 0x85EBCA77u));
}
__device__ __forceinline__ uint32_t random_mix(RandomKey k, uint32_t u) {
  u ^= u >> 16;
  u = u * 2891336453u + k.hi;
  return u ^ (u >> 15);
}
__device__ __forceinline__ uint32_t random_pair(RandomKey k, uint64_t pair) { return random_mix(k, random_counter(k, pair)); }
// 32 bits of the pair's first or second element: the high half rounds v, the low half m.
__device__ __forceinline__ uint32_t random_moments(uint32_t u, int odd) { return u * (odd ? 741103597u : 1597334677u); }
// The pair's weights: 16 bits each, the high half for the first.
__device__ __forceinline__ uint32_t random_weights(uint32_t u) { return u * 747796405u; }

// ---- pairs: two fp32 products per instruction, each rounded as a single one

__device__ __forceinline__ Pair pair(float x) { return make_float2(x, x); }
#define FR_PAIR(x) reinterpret_cast<const uint64_t&>(x)
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(FR_PAIR(a)), "l"(FR_PAIR(b)));
  return r;
}
// (add.rn.f32x2 of a product is contracted to a fused multiply-add by CUDA 13.0's
// assembler, with and without -fmad=false; two single additions are not.)
__device__ __forceinline__ Pair add2(Pair a, Pair b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(FR_PAIR(a)), "l"(FR_PAIR(b)), "l"(FR_PAIR(c)));
  return r;
}
#undef FR_PAIR

// ---- the update

// What a step's numbers are multiplied in as: the launch's, twice each so that
// the pairs come from constant memory, and the tensor's own.
struct Hyper {
  const StepNumbers& n;
  float scale, lr, decay;  // scale: of the gradient
};

// New moments, each product and sum rounded by itself.
__device__ __forceinline__ void update_moments(const Hyper& h, Pair grad, Pair& m, Pair& v) {
  const Pair g = mul2(grad, pair(h.scale));
  m = add2(mul2(m, h.n.b1), mul2(g, h.n.c1));
  v = add2(mul2(v, h.n.b2), mul2(mul2(g, g), h.n.c2));
}

// The parameter from the new moments.  The square root and the reciprocal are
// the hardware's approximations, 2^-23 off at most: under lr they are nothing
// beside the parameter's own rounding, and the correctly rounded ones take 20
// more instructions per element.  Subnormal second moments count as zero there,
// which is under 2^-63 v_fix of a denominator of at least eps; an eps too small for that
// (below 2^-39 v_fix) takes the correctly rounded ones.
__device__ __forceinline__ float approx_sqrt(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float approx_reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ Pair update_param(const Hyper& h, Pair p, Pair m, Pair v) {
  const Pair below = fma2(make_float2(approx_sqrt(v.x), approx_sqrt(v.y)), h.n.v_fix, h.n.eps);
  const Pair u = mul2(m, make_float2(approx_reciprocal(below.x), approx_reciprocal(below.y)));
  return fma2(fma2(u, h.n.m_fix, mul2(p, pair(h.decay))), pair(-h.lr), p);
}
__device__ __forceinline__ Pair update_param_exactly(const Hyper& h, Pair p, Pair m, Pair v) {
  const Pair below = fma2(make_float2(__fsqrt_rn(v.x), __fsqrt_rn(v.y)), h.n.v_fix, h.n.eps);
  const Pair u = make_float2(__fdiv_rn(m.x, below.x), __fdiv_rn(m.y, below.y));
  return fma2(fma2(u, h.n.m_fix, mul2(p, pair(h.decay))), pair(-h.lr), p);
}

}  // namespace frk
