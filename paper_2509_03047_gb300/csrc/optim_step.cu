// optim_step.cu -- the AdamW step over a list of tensors.
//
// One launch per class of tensors (parameter type, gradient type, moments in
// 32 or 8 bits).
#include <type_traits>

#include "kernels.h"
#include "optim.h"
#include "optim_block.cuh"

namespace frk {

namespace {

// Rounding of a bf16 weight that has no master: two elements, rnd of their pair.
__device__ __forceinline__ uint32_t random_bf16x2(Pair x, uint32_t u) {
  const uint32_t w = random_weights(u);
  uint32_t r;  // (the upper element takes the high half: the pair's first goes there, and back)
  asm("cvt.rs.bf16x2.f32 %0, %1, %2, %3;" : "=r"(r) : "f"(x.x), "f"(x.y), "r"(w));
  return __byte_perm(r, 0, 0x1032);
}
__device__ __forceinline__ uint32_t nearest_bf16x2(Pair x) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(x.y), "f"(x.x));
  return r;
}

template <int Weight, bool Bf16Grad, bool Eight, bool Random>
struct Step {
  using RawGrad = std::conditional_t<Bf16Grad, RawBf16, RawF32>;
  using RawParam = std::conditional_t<Weight == kWeightBf16, RawBf16, RawF32>;
  using RawMoment = std::conditional_t<Eight, RawCodes, RawF32>;
  static constexpr int kGradBytes = Bf16Grad ? 2 : 4, kMomentBytes = Eight ? 1 : 4;

  static __device__ __forceinline__ void whole(const Hyper& h, const OptDesc& d, uint32_t block, RandomKey key, int lane) {
    const uint64_t first = static_cast<uint64_t>(block) * kOptBlock;
    uint8_t* const m_at = static_cast<uint8_t*>(d.m) + first * kMomentBytes;
    uint8_t* const v_at = static_cast<uint8_t*>(d.v) + first * kMomentBytes;
    RawGrad raw_g;
    RawParam raw_p;
    RawMoment raw_m, raw_v;
    raw_g.load(static_cast<const uint8_t*>(d.grad) + first * kGradBytes, lane);
    raw_m.load(m_at, lane);
    raw_v.load(v_at, lane);
    raw_p.load(Weight == kWeightMaster ? static_cast<const void*>(d.master + first)
                                       : static_cast<const uint8_t*>(d.weight) + first * (Weight == kWeightBf16 ? 2 : 4), lane);
    Pair g[4], p[4], m[4], v[4];
    if constexpr (Eight) {
      const uint32_t em = d.m_exp[block], ev = d.v_exp[block];
      __syncwarp();  // every lane has read the exponents before one writes them
      decode4<true>(raw_m.a.x, em, m[0], m[1]);
      decode4<true>(raw_m.a.y, em, m[2], m[3]);
      decode4<false>(raw_v.a.x, ev, v[0], v[1]);
      decode4<false>(raw_v.a.y, ev, v[2], v[3]);
      if (em == 255 || ev == 255) {  // (rare) a block that has lost its moments
        const float nan = __uint_as_float(0x7FC00000u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (em == 255) m[j] = pair(nan);
          if (ev == 255) v[j] = pair(nan);
        }
      }
    } else {
      raw_m.get(m);
      raw_v.get(v);
    }
    raw_g.get(g);
    raw_p.get(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      update_moments(h, g[j], m[j], v[j]);
      p[j] = update_param(h, p[j], m[j], v[j]);
    }
    uint32_t u[4];
    if (Random) random_pairs(key, first, lane, u);
    if (Weight == kWeightMaster) store_f32(d.master + first, lane, p);
    if (Weight == kWeightF32) {
      store_f32(static_cast<float*>(d.weight) + first, lane, p);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = Random && Weight == kWeightBf16 ? random_bf16x2(p[j], u[j]) : nearest_bf16x2(p[j]);
      store_bf16(static_cast<uint16_t*>(d.weight) + first, lane, w);
    }
    if constexpr (Eight) {
      store_codes<true, Random>(m, u, m_at, d.m_exp + block, lane);
      store_codes<false, Random>(v, u, v_at, d.v_exp + block, lane);
    } else {
      store_f32(reinterpret_cast<float*>(m_at), lane, m);
      store_f32(reinterpret_cast<float*>(v_at), lane, v);
    }
  }

  static __device__ __noinline__ void any(const Hyper h, const OptDesc* tensor, uint32_t block, RandomKey key, int lane) {
    const OptDesc d = *tensor;
    const uint64_t first = static_cast<uint64_t>(block) * kOptBlock;
    const int left = static_cast<int>(min(d.n - first, static_cast<uint64_t>(kOptBlock)));
    uint8_t* const m_at = static_cast<uint8_t*>(d.m) + first * kMomentBytes;
    uint8_t* const v_at = static_cast<uint8_t*>(d.v) + first * kMomentBytes;
    float g[kOptLane], p[kOptLane], m[kOptLane], v[kOptLane];
    load_any<std::conditional_t<Bf16Grad, uint16_t, float>>(static_cast<const uint8_t*>(d.grad) + first * kGradBytes, lane, left, g);
    if (Weight == kWeightMaster)
      load_any<float>(d.master + first, lane, left, p);
    else if (Weight == kWeightBf16)
      load_any<uint16_t>(static_cast<const uint16_t*>(d.weight) + first, lane, left, p);
    else
      load_any<float>(static_cast<const float*>(d.weight) + first, lane, left, p);
    if (Eight) {
      const uint32_t em = d.m_exp[block], ev = d.v_exp[block];
      __syncwarp();
      load_codes_any<true>(m_at, em, lane, left, m);
      load_codes_any<false>(v_at, ev, lane, left, v);
    } else {
      load_any<float>(m_at, lane, left, m);
      load_any<float>(v_at, lane, left, v);
    }
#pragma unroll
    for (int j = 0; j < kOptLane; j += 2) {
      Pair a = make_float2(m[j], m[j + 1]), b = make_float2(v[j], v[j + 1]);
      update_moments(h, make_float2(g[j], g[j + 1]), a, b);
      const Pair q = update_param(h, make_float2(p[j], p[j + 1]), a, b);
      m[j] = a.x, m[j + 1] = a.y, v[j] = b.x, v[j + 1] = b.y, p[j] = q.x, p[j + 1] = q.y;
    }
    if (Weight == kWeightMaster) store_any<float>(d.master + first, lane, left, p);
    if (Weight == kWeightF32) {
      store_any<float>(static_cast<float*>(d.weight) + first, lane, left, p);
    } else {
      uint16_t w[kOptLane];
#pragma unroll
      for (int j = 0; j < kOptLane; ++j) {
        const uint64_t i = first + j * 32 + lane;
        const Pair twice = pair(p[j]);  // (the pair's half that counts)
        const uint32_t both = Random && Weight == kWeightBf16 ? random_bf16x2(twice, random_pair(key, i >> 1)) : nearest_bf16x2(twice);
        w[j] = static_cast<uint16_t>(i & 1 ? both >> 16 : both);
      }
      store_any<uint16_t>(static_cast<uint16_t*>(d.weight) + first, lane, left, w);
    }
    if (Eight) {
      store_codes_any<true>(m, Random, key, first, m_at, d.m_exp + block, lane, left);
      store_codes_any<false>(v, Random, key, first, v_at, d.v_exp + block, lane, left);
    } else {
      store_any<float>(reinterpret_cast<float*>(m_at), lane, left, m);
      store_any<float>(reinterpret_cast<float*>(v_at), lane, left, v);
    }
  }
};

template <int Weight, bool Bf16Grad, bool Eight, bool Random>
__global__ void __launch_bounds__(32 * kOptWarps, 4) step_kernel(const __grid_constant__ StepParams p) {
  wait_for_kernel_before();
  using S = Step<Weight, Bf16Grad, Eight, Random>;
  const int lane = threadIdx.x % 32;
  const uint32_t b = blockIdx.x * kOptWarps + threadIdx.x / 32;
  if (b >= p.work.n_blocks) return;
  const uint32_t t = tensor_of(p.work, p.work.start[blockIdx.x], b);
  const OptDesc d = p.work.tensors[t];
  Hyper h;
  h.scale = 1.0f;
  if (p.clip != nullptr) {
    if (p.clip->nonfinite != 0) return;
    h.scale = p.clip->scale;
  }
  h.b1 = p.b1, h.c1 = p.c1, h.b2 = p.b2, h.c2 = p.c2, h.eps = p.eps, h.m_fix = p.m_fix, h.v_fix = p.v_fix, h.exact = p.exact;
  h.lr = __fmul_rn(p.lr, d.lr_scale);
  h.decay = __fmul_rn(p.decay, d.decay_scale);
  RandomKey key = {0, 0};
  if (Random) key = random_key(p.key, d.tensor);
  const uint32_t block = b - d.first;
  if (d.aligned && block < d.n / kOptBlock)
    S::whole(h, d, block, key, lane);
  else
    S::any(h, p.work.tensors + t, block, key, lane);
}

template <class F>
auto for_class(const StepClass& c, bool random, F&& f) {
  auto with = [&](auto weight, auto grad, auto eight) {
    // random rounding concerns codes, and bf16 weights without a master
    if constexpr (decltype(eight)::value || decltype(weight)::value == kWeightBf16)
      if (random) return f(step_kernel<decltype(weight)::value, decltype(grad)::value, decltype(eight)::value, true>);
    return f(step_kernel<decltype(weight)::value, decltype(grad)::value, decltype(eight)::value, false>);
  };
  auto with_types = [&](auto weight) {
    if (c.bf16_grad)
      return c.eight ? with(weight, std::true_type(), std::true_type()) : with(weight, std::true_type(), std::false_type());
    return c.eight ? with(weight, std::false_type(), std::true_type()) : with(weight, std::false_type(), std::false_type());
  };
  if (c.weight == kWeightMaster) return with_types(std::integral_constant<int, kWeightMaster>());
  if (c.weight == kWeightBf16) return with_types(std::integral_constant<int, kWeightBf16>());
  return with_types(std::integral_constant<int, kWeightF32>());
}

}  // namespace

cudaError_t launch_step(const StepClass& c, const StepParams& p, cudaStream_t s) {
  return for_class(c, p.random != 0, [&](auto kernel) { return launch_chained(kernel, p.work.n_units, 32 * kOptWarps, 0, s, p); });
}

}  // namespace frk
