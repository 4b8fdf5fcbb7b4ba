// optim_block.cuh -- a warp's block of 256 elements: finding its tensor, loads,
// stores, random bits, coding of 8-bit moments.
//
// Where a tensor's buffers are aligned a block moves as vectors: lane l has the
// elements 8 l ... 8 l + 7.  Else (and a conversion's last block of a tensor)
// it moves element by element, lane l with the elements l, l + 32, ...  What lies
// past the tensor's end reads as zero.  Both give the same bits.  (The step
// brings whole blocks from any place to the vectors' order: fetch_odd, take_odd,
// copy_out.)
#pragma once

#include <type_traits>

#include "optim.h"
#include "optim_math.cuh"

namespace frk {

// The tensor of block b of a launch (b the same in the whole warp), from one, t,
// that is not after it.  The lanes look at 32 tensors at a time: of many small
// ones, one after the other cost 0.3 us each.
__device__ __forceinline__ uint32_t tensor_of(const OptWork& w, uint32_t t, uint32_t b) {
  if (b - w.tensors[t].first < w.tensors[t].n_blocks) return t;
  const uint32_t lane = threadIdx.x % 32;
  for (++t;; t += 32) {
    const bool after = t + lane >= w.n_tensors || w.tensors[t + lane].first > b;
    const uint32_t m = __ballot_sync(0xFFFFFFFFu, after);
    if (m) return t + __ffs(m) - 2;  // the one before the first that starts after b
  }
}

// The tensor of a warp's first block, b.
__device__ __forceinline__ uint32_t first_tensor(const OptWork& w, uint32_t group, uint32_t warp, int warps, uint32_t b) {
  return w.start_of_warps ? w.start[group * warps + warp] : tensor_of(w, w.start[group], b);
}

// ---- vectors

__device__ __forceinline__ uint4 load_16(const void* p) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}

__device__ __forceinline__ void copy_16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_8(uint32_t to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_4(uint32_t to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ uint32_t shared_4(uint32_t at) {
  uint32_t q;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(q) : "r"(at));
  return q;
}
__device__ __forceinline__ uint4 shared_16(uint32_t at) {
  uint4 q;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(at));
  return q;
}

// Bytes of the word before an address in it.
__device__ __forceinline__ uint32_t odd_bytes(const void* p) { return static_cast<uint32_t>(reinterpret_cast<uint64_t>(p)) & 3; }

// A lane's eight elements as they lie in memory, p: its place in the block.
// load() brings them to registers; `left` of them are in the tensor, in its last
// block fewer than eight, or none, and these go one by one.  fetch() starts the
// whole block's way to shared memory, each copy of the warp 512 or 256
// consecutive bytes, from where take() has them.
// fetch_odd() and take_odd(): the same at any alignment.  A block off the boundary
// that fetch() needs goes by the 4-byte words that hold its elements (of the first
// and last one the neighbours' bytes too, which are dropped); if it starts inside
// a word there is one more than it fills, which goes to `extra`.
// (32 bytes go by one instruction: two of 16 bytes, each lane's beside one
// another, write at 4.7 TB/s where this does at 7.0.)
struct RawF32 {
  static constexpr int kBytes = 4;
  uint32_t a[8];
  static __device__ __forceinline__ void fetch(uint32_t to, const void* p, int lane) {
    const uint8_t* q = static_cast<const uint8_t*>(p) - 16 * lane;  // (of 32 bytes a lane, copies of 16)
    copy_16(to + 16 * lane, q);
    copy_16(to + 512 + 16 * lane, q + 512);
  }
  __device__ __forceinline__ void take(uint32_t from, int lane) {
    const uint4 x = shared_16(from + 32 * lane), y = shared_16(from + 32 * lane + 16);
    a[0] = x.x, a[1] = x.y, a[2] = x.z, a[3] = x.w, a[4] = y.x, a[5] = y.y, a[6] = y.z, a[7] = y.w;
  }
  static __device__ __forceinline__ void fetch_odd(uint32_t to, uint32_t, const void* p, int lane) {
    if (reinterpret_cast<uint64_t>(p) % 16 == 0) return fetch(to, p, lane);
    const uint8_t* q = static_cast<const uint8_t*>(p) - 28 * lane;
#pragma unroll
    for (int j = 0; j < 8; ++j) copy_4(to + 128 * j + 4 * lane, q + 128 * j);
  }
  __device__ __forceinline__ void take_odd(uint32_t from, uint32_t, const void*, int lane) { take(from, lane); }
  __device__ __forceinline__ void load(const void* p, int left) {
    if (left >= kOptLane) {
      asm volatile("ld.global.L1::no_allocate.v8.u32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]), "=r"(a[4]), "=r"(a[5]), "=r"(a[6]), "=r"(a[7])
                   : "l"(p));
      return;
    }
#pragma unroll
    for (int j = 0; j < kOptLane; ++j) a[j] = j < left ? static_cast<const uint32_t*>(p)[j] : 0u;
  }
  __device__ __forceinline__ void get(Pair (&x)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = make_float2(__uint_as_float(a[2 * j]), __uint_as_float(a[2 * j + 1]));
  }
};
struct RawBf16 {
  static constexpr int kBytes = 2;
  uint32_t a[4];
  static __device__ __forceinline__ void fetch(uint32_t to, const void* p, int lane) { copy_16(to + 16 * lane, p); }
  __device__ __forceinline__ void take(uint32_t from, int lane) {
    const uint4 q = shared_16(from + 16 * lane);
    a[0] = q.x, a[1] = q.y, a[2] = q.z, a[3] = q.w;
  }
  static __device__ __forceinline__ void fetch_odd(uint32_t to, uint32_t extra, const void* p, int lane) {
    if (reinterpret_cast<uint64_t>(p) % 16 == 0) return fetch(to, p, lane);
    const uint32_t shift = odd_bytes(p);
    const uint8_t* q = static_cast<const uint8_t*>(p) - shift - 12 * lane;
#pragma unroll
    for (int j = 0; j < 4; ++j) copy_4(to + 128 * j + 4 * lane, q + 128 * j);
    if (shift && lane == 0) copy_4(extra, q + 512);
  }
  __device__ __forceinline__ void take_odd(uint32_t from, uint32_t extra, const void* p, int lane) {
    take(from, lane);
    const uint32_t shift = 8 * odd_bytes(p), more = shared_4(lane < 31 ? from + 16 * lane + 16 : extra);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __funnelshift_r(a[i], i < 3 ? a[i + 1] : more, shift);
  }
  __device__ __forceinline__ void load(const void* p, int left) {
    if (left >= kOptLane) {
      const uint4 q = load_16(p);
      a[0] = q.x, a[1] = q.y, a[2] = q.z, a[3] = q.w;
      return;
    }
#pragma unroll
    for (int j = 0; j < kOptLane; ++j) {
      const uint32_t x = j < left ? static_cast<const uint16_t*>(p)[j] : 0u;
      a[j / 2] = j & 1 ? a[j / 2] | x << 16 : x;
    }
  }
  __device__ __forceinline__ void get(Pair (&x)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = make_float2(__uint_as_float(a[j] << 16), __uint_as_float(a[j] & 0xFFFF0000u));
  }
};
struct RawCodes {
  static constexpr int kBytes = 1;
  uint32_t a[2];
  static __device__ __forceinline__ void fetch(uint32_t to, const void* p, int lane) { copy_8(to + 8 * lane, p); }
  __device__ __forceinline__ void take(uint32_t from, int lane) {
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(a[0]), "=r"(a[1]) : "r"(from + 8 * lane));
  }
  static __device__ __forceinline__ void fetch_odd(uint32_t to, uint32_t extra, const void* p, int lane) {
    if (reinterpret_cast<uint64_t>(p) % 8 == 0) return fetch(to, p, lane);
    const uint32_t shift = odd_bytes(p);
    const uint8_t* q = static_cast<const uint8_t*>(p) - shift - 4 * lane;
    copy_4(to + 4 * lane, q);
    copy_4(to + 128 + 4 * lane, q + 128);
    if (shift && lane == 0) copy_4(extra, q + 256);
  }
  __device__ __forceinline__ void take_odd(uint32_t from, uint32_t extra, const void* p, int lane) {
    take(from, lane);
    const uint32_t shift = 8 * odd_bytes(p), more = shared_4(lane < 31 ? from + 8 * lane + 8 : extra);
    a[0] = __funnelshift_r(a[0], a[1], shift);
    a[1] = __funnelshift_r(a[1], more, shift);
  }
  __device__ __forceinline__ void load(const void* p, int left) {
    if (left >= kOptLane) {
      asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(a[0]), "=r"(a[1]) : "l"(p));
      return;
    }
    a[0] = a[1] = 0;
#pragma unroll
    for (int j = 0; j < kOptLane; ++j)
      if (j < left) a[j / 4] |= static_cast<uint32_t>(static_cast<const uint8_t*>(p)[j]) << 8 * (j & 3);
  }
};
__device__ __forceinline__ void store_f32(void* p, int left, const Pair (&x)[4]) {
  if (left >= kOptLane) {
    asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"f"(x[0].x), "f"(x[0].y), "f"(x[1].x), "f"(x[1].y),
                 "f"(x[2].x), "f"(x[2].y), "f"(x[3].x), "f"(x[3].y), "l"(p)
                 : "memory");
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    if (j < left) static_cast<float*>(p)[j] = j & 1 ? x[j / 2].y : x[j / 2].x;
}
__device__ __forceinline__ void store_bf16(void* p, int left, const uint32_t (&w)[4]) {
  if (left >= kOptLane) {
    *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    if (j < left) static_cast<uint16_t*>(p)[j] = static_cast<uint16_t>(j & 1 ? w[j / 2] >> 16 : w[j / 2]);
}
__device__ __forceinline__ void store_bytes(uint8_t* p, int left, const uint32_t (&w)[2]) {
  if (left >= kOptLane) {
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    return;
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    if (j < left) p[j] = static_cast<uint8_t>(w[j / 4] >> 8 * (j & 3));
}
// A whole block from shared memory, as the lanes have put it there at their
// places: by vectors where it starts on their boundary, else element by element,
// in each store of the warp 32 consecutive ones.  (By 4-byte words shifted
// together, the first and the last by bytes: 2% slower.)
template <class T>
__device__ __forceinline__ void copy_out(void* block, const uint8_t* staged, int lane) {
  using V = std::conditional_t<sizeof(T) == 1, uint2, uint4>;
  constexpr int kVectors = kOptLane * sizeof(T) / sizeof(V);
  if (reinterpret_cast<uint64_t>(block) % sizeof(V) == 0) {
    V x[kVectors];
#pragma unroll
    for (int j = 0; j < kVectors; ++j) x[j] = reinterpret_cast<const V*>(staged)[32 * j + lane];
#pragma unroll
    for (int j = 0; j < kVectors; ++j) static_cast<V*>(block)[32 * j + lane] = x[j];
    return;
  }
  T x[kOptLane];
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) x[j] = reinterpret_cast<const T*>(staged)[32 * j + lane];
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) static_cast<T*>(block)[32 * j + lane] = x[j];
}
// Of a lane's elements of a block of a tensor of n.
__device__ __forceinline__ int elements_left(uint64_t n, uint32_t block, int lane) {
  const uint64_t first = static_cast<uint64_t>(block) * kOptBlock;
  return n - first >= kOptBlock ? kOptLane : min(max(static_cast<int>(n - first) - lane * kOptLane, 0), kOptLane);
}

// A lane's place in a block of a buffer.
template <int Bytes>
__device__ __forceinline__ uint8_t* lane_at(const void* buffer, uint32_t block, int lane) {
  return static_cast<uint8_t*>(const_cast<void*>(buffer)) + (static_cast<uint64_t>(block) * kOptBlock + lane * kOptLane) * Bytes;
}

// Four codes of a block of exponent e (span < e < 255) as values: two at a time
// as bf16 patterns (a code's three fraction bits fit), zero codes without the
// base.
template <bool Signed>
__device__ __forceinline__ void decode4(uint32_t w, uint32_t e, Pair& x, Pair& y) {
  const uint32_t base = code_base(e, Signed ? kSpanM : kSpanV) * 16;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t h;
    if (Signed) {  // the bytes in the high halves' places: the sign is where it belongs
      const uint32_t two = __byte_perm(w, 0, k ? 0x3424 : 0x1404), c = (two >> 4) & 0x07F007F0u;
      h = (c + __vminu2(c, 0x00010001u) * base) | (two & 0x80008000u);
    } else {
      const uint32_t two = __byte_perm(w, 0, k ? 0x4342 : 0x4140);
      h = two * 16 + __vminu2(two, 0x00010001u) * base;
    }
    (k ? y : x) = make_float2(__uint_as_float(h << 16), __uint_as_float(h & 0xFFFF0000u));
  }
}

// Two values' patterns rounded and cut at bit 20, in 12 bits each with the sign.
template <bool Random>
__device__ __forceinline__ uint32_t cut2(Pair x, uint32_t r) {
  const uint32_t a = __float_as_uint(x.x), b = __float_as_uint(x.y);
  if (!Random) return (__byte_perm(a + round_nearest(a), b + round_nearest(b), 0x7632) >> 4) & 0x0FFF0FFFu;
  // r: 16 random bits for each.  Four bits down, the cut is where a conversion to
  // bf16 that rounds by given bits has it, and the patterns are small numbers.
  uint32_t h;
  asm("cvt.rs.bf16x2.f32 %0, %1, %2, %3;" : "=r"(h) : "f"(__uint_as_float(b >> 4)), "f"(__uint_as_float(a >> 4)), "r"(r));
  return h;
}

// Codes of four values of a block of exponent e, from their cut patterns.
// Unsigned: code 1 at least, so zeros are left to the caller.
template <bool Signed>
__device__ __forceinline__ uint32_t encode4(uint32_t h0, uint32_t h1, uint32_t e) {
  const uint32_t base = code_base(e, Signed ? kSpanM : kSpanV) * 0x00010001u;
  if (!Signed) return __byte_perm(__vmaxu2(h0, base + 0x00010001u) - base, __vmaxu2(h1, base + 0x00010001u) - base, 0x6420);
  const uint32_t c = __byte_perm(__vmaxu2(h0 & 0x07FF07FFu, base) - base, __vmaxu2(h1 & 0x07FF07FFu, base) - base, 0x6420);
  return c | ((__byte_perm(h0, h1, 0x7531) * 16) & (c + 0x7F7F7F7Fu) & 0x80808080u);  // no zero has a sign
}

// Largest bit pattern of |x| over the warp; a NaN's is above all others.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t warp_max(uint32_t x) { return __reduce_max_sync(0xFFFFFFFFu, x); }
__device__ __forceinline__ uint32_t block_top(const Pair (&x)[4]) {
  const float a = max3(x[0].x, x[0].y, x[1].x), b = max3(x[1].y, x[2].x, x[2].y);
  return warp_max(__float_as_uint(max3(max3(a, b, x[3].x), x[3].y, 0.0f)));
}

// A lane's random bits of a whole block: those of its four pairs of elements, from the first one's counter.
__device__ __forceinline__ void random_pairs(RandomKey key, uint32_t counter, uint32_t (&u)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) u[j] = random_mix(key, counter + j * kRandomStep);
}

__device__ __forceinline__ float min3(float a, float b, float c) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Codes a whole block's moments and stores them at the lane's place; returns the
// exponent.  u: the lane's random_pairs.
template <bool Signed, bool Random>
__device__ __forceinline__ uint32_t store_codes(const Pair (&x)[4], const uint32_t (&u)[4], uint8_t* codes, int left) {
  const uint32_t e = block_exponent(block_top(x), Signed ? kSpanM : kSpanV);
  uint32_t h[4], w[2];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    h[j] = cut2<Random>(x[j], Random ? __byte_perm(random_moments(u[j], 0), random_moments(u[j], 1), Signed ? 0x5410 : 0x7632) : 0u);
  w[0] = encode4<Signed>(h[0], h[1], e);
  w[1] = encode4<Signed>(h[2], h[3], e);
  if (!Signed) {  // second moments that are zero: whole rows, or none
    if (min3(min3(x[0].x, x[0].y, x[1].x), min3(x[1].y, x[2].x, x[2].y), fminf(x[3].x, x[3].y)) == 0.0f)
#pragma unroll
      for (int j = 0; j < kOptLane; ++j)
        if ((j & 1 ? x[j / 2].y : x[j / 2].x) == 0.0f) w[j / 4] &= ~(0xFFu << 8 * (j & 3));
  }
  if (e >= 255) w[0] = w[1] = 0;
  store_bytes(codes, left, w);
  return e;
}

// The exponents of a warp's consecutive blocks, one per lane: read before the
// first block's stores, written after the last's.  (A load from a sector with a
// store under way waits for it, and 32 blocks share a sector: block by block,
// four blocks a warp took twice the time of one.)
struct Exponents {
  uint32_t m, v;
  __device__ __forceinline__ void load(const uint8_t* me, const uint8_t* ve, int count, int lane) {
    m = v = 0;
    if (lane < count) m = me[lane], v = ve[lane];
    m = read_exponent(m, kSpanM), v = read_exponent(v, kSpanV);
  }
  __device__ __forceinline__ void store(uint8_t* me, uint8_t* ve, int count, int lane) const {
    if (lane < count) me[lane] = stored_exponent(m), ve[lane] = stored_exponent(v);
  }
  __device__ __forceinline__ uint32_t of_m(int k) const { return __shfl_sync(0xFFFFFFFFu, m, k); }
  __device__ __forceinline__ uint32_t of_v(int k) const { return __shfl_sync(0xFFFFFFFFu, v, k); }
  __device__ __forceinline__ void set(int k, int lane, uint32_t em, uint32_t ev) {
    if (lane == k) m = em, v = ev;
  }
};

// ---- element by element

template <class T>
__device__ __forceinline__ float to_float(T x) {
  if constexpr (sizeof(T) == 2)
    return __uint_as_float(static_cast<uint32_t>(x) << 16);
  else
    return x;
}
template <class T>
__device__ __forceinline__ void load_any(const void* block, int lane, int left, float (&x)[kOptLane]) {
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) x[j] = j * 32 + lane < left ? to_float(static_cast<const T*>(block)[j * 32 + lane]) : 0.0f;
}
template <class T>
__device__ __forceinline__ void store_any(T* block, int lane, int left, const T (&x)[kOptLane]) {
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    if (j * 32 + lane < left) block[j * 32 + lane] = x[j];
}
template <bool Signed>
__device__ __forceinline__ void load_codes_any(const uint8_t* block, uint32_t exponent, int lane, int left, float (&x)[kOptLane]) {
  const uint32_t e = read_exponent(exponent, Signed ? kSpanM : kSpanV);
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) {
    const uint32_t c = j * 32 + lane < left ? block[j * 32 + lane] : 0u;
    x[j] = Signed ? decode_m(c, e) : decode_v(c, e);
    if (j * 32 + lane >= left) x[j] = 0.0f;
  }
}
// random: the tensor's key counts
template <bool Signed>
__device__ __forceinline__ void store_codes_any(const float (&x)[kOptLane], bool random, RandomKey key, uint64_t first, uint8_t* codes,
                                                uint8_t* exponent, int lane, int left) {
  uint32_t top = 0, c[kOptLane];
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  const uint32_t e = block_exponent(warp_max(top), Signed ? kSpanM : kSpanV);
#pragma unroll
  for (int j = 0; j < kOptLane; ++j) {
    const uint64_t i = first + j * 32 + lane;
    uint32_t r = round_nearest(__float_as_uint(x[j]));
    if (random) {
      const uint32_t q = random_moments(random_pair(key, i >> 1), static_cast<int>(i & 1));
      r = (Signed ? q & 0xFFFFu : q >> 16) << 4;
    }
    c[j] = Signed ? encode_m(x[j], r, e) : encode_v(x[j], r, e);
  }
#pragma unroll
  for (int j = 0; j < kOptLane; ++j)
    if (j * 32 + lane < left) codes[j * 32 + lane] = static_cast<uint8_t>(c[j]);
  if (lane == 0) *exponent = stored_exponent(e);
}

}  // namespace frk
