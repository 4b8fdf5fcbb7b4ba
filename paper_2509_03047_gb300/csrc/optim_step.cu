// optim_step.cu -- the AdamW step over a list of tensors.
//
// One launch per class of tensors (parameter type, gradient type, moments in
// 32 or 8 bits, on the vectors' boundaries or off them); one pass over each buffer, every element read, updated and
// written where it lies.  Bound by memory, and for 8-bit moments under bf16
// weights without a master, at 10 bytes per element, by instructions too.
//
// 32-bit moments: one block of 256 elements per warp, no loop.  The hardware's
// own order of many short CTAs reaches 7.1 TB/s (28 GB of a Llama-8B rank 3.97
// ms; GPT-2 small, 3.7 GB, 522 us; 0.77 GB in 10,000 tensors of 1 to 28,183
// elements 114 us, 6.7 TB/s; a copy moves 6.8 TB/s), warps that loop over
// the blocks at most 6.6, in any order: contiguous ranges, units side by side or
// a grid's stride, with 1 to 6 CTAs per SM, with and without eviction hints.
//
// 8-bit moments: a block is 2.5 to 4 KB and 380 instructions of a warp, so up
// to 8 consecutive blocks share what a warp does once (its tensor, its random
// key, its exponents), and the next ones come to shared memory meanwhile, by
// asynchronous copies that take no registers.  One block per warp: GPT-2 small in
// bf16 307 us, a Llama-8B rank with masters 2.77 ms; runs with the next block in
// registers 207 us and 2.38 ms; so 190 us (6.5 TB/s) and 2.31 ms (7.0).  At the
// former's 10 bytes per element warps issue in four of five cycles.  Lists of
// many small tensors wait for latencies, a tensor's last block, out of line,
// above all: 10,000 with masters, of 1 to 28,183 elements 91 us (4.8 TB/s), of 1
// to 2,000, 42 MB, 19.5 us (2.2).
//
// Tensors whose buffers lie off the vectors' boundaries in different ways: whole
// blocks come and go through shared memory, each buffer by vectors where it can.
// 134 million elements (aligned; only the gradient off; every buffer, each in its
// own way; and the gradient alone element by element, by Step::any): bf16 with
// 32-bit moments 421, 460, 537 and 568 us, with 8-bit ones 203, 278, 342 and 818;
// with masters 535, 564, 663 and 679, and 313, 327, 459 and 861.  (8-bit without
// the choice for each buffer 301 and 316, with masters 407 and 439: flat groups
// of gradients beside states of their own are the more usual.)
//
// An eps too small for the approximations (optim_math.cuh) takes Step::any for
// every block: GPT-2 small with masters 674 us (522), in bf16 with 8-bit moments
// 808 (190); a Llama-8B rank 5.39 ms (3.97), with 8-bit moments 7.10 (2.31).
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

__device__ __forceinline__ Hyper hyper(const StepParams& p, float scale, const OptDesc& d) {
  return {p.numbers, scale, __fmul_rn(p.lr, d.lr_scale), __fmul_rn(p.decay, d.decay_scale)};
}

template <int Weight, bool Bf16Grad, bool Eight, bool Odd, bool Random>
struct Step {
  using RawGrad = std::conditional_t<Bf16Grad, RawBf16, RawF32>;
  using RawParam = std::conditional_t<Weight == kWeightBf16, RawBf16, RawF32>;
  using RawMoment = std::conditional_t<Eight, RawCodes, RawF32>;
  static constexpr int kGradBytes = RawGrad::kBytes, kMomentBytes = RawMoment::kBytes;

  // Of a block in shared memory (Odd: and the four buffers' extra words, see
  // fetch_odd), and how many (a CTA's stay under 48 KiB).
  static constexpr int kSlot = kOptBlock * (kGradBytes + RawParam::kBytes + 2 * kMomentBytes), kSlotSize = kSlot + (Odd ? 16 : 0),
                       kSlots = !Eight ? 1 : kSlot <= 1536 ? 3 : 2;
  // The lane's places in a block.
  struct Places {
    const uint8_t* g;
    uint8_t *p, *w, *m, *v;  // w: the weight, where it is not the parameter
    __device__ __forceinline__ Places(const OptDesc& d, uint32_t block, int lane) {
      g = lane_at<kGradBytes>(d.grad, block, lane);
      p = lane_at<RawParam::kBytes>(Weight == kWeightMaster ? d.master : d.weight, block, lane);
      w = lane_at<2>(d.weight, block, lane);
      m = lane_at<kMomentBytes>(d.m, block, lane);
      v = lane_at<kMomentBytes>(d.v, block, lane);
    }
    __device__ __forceinline__ void next() {
      g += kOptBlock * kGradBytes;
      p += kOptBlock * RawParam::kBytes;
      w += kOptBlock * 2;
      m += kOptBlock * kMomentBytes;
      v += kOptBlock * kMomentBytes;
    }
  };
  // A block's loads.
  struct Raw {
    RawGrad g;
    RawParam p;
    RawMoment m, v;
    __device__ __forceinline__ void load(const Places& at, int left) {
      g.load(at.g, left);
      m.load(at.m, left);
      v.load(at.v, left);
      p.load(at.p, left);
    }
  };
  static __device__ __forceinline__ void put_f32(uint8_t* at, int left, const Pair (&x)[4]) {
    if constexpr (Odd) {
      reinterpret_cast<float4*>(at)[0] = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
      reinterpret_cast<float4*>(at)[1] = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
    } else {
      store_f32(at, left, x);
    }
  }
  // The rest of it; em and ev: its exponents, old and new.  Odd: stores go to the
  // lane's places in shared memory, `at` points there.
  static __device__ __forceinline__ void finish(const Hyper& h, const Places& at, int left, uint32_t counter, RandomKey key, const Raw& r,
                                                uint32_t& em, uint32_t& ev) {
    Pair g[4], p[4], m[4], v[4];
    if constexpr (Eight) {
      decode4<true>(r.m.a[0], em, m[0], m[1]);
      decode4<true>(r.m.a[1], em, m[2], m[3]);
      decode4<false>(r.v.a[0], ev, v[0], v[1]);
      decode4<false>(r.v.a[1], ev, v[2], v[3]);
      if (em == 255 || ev == 255) {  // (rare) a block that has lost its moments
        const float nan = __uint_as_float(0x7FC00000u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (em == 255) m[j] = pair(nan);
          if (ev == 255) v[j] = pair(nan);
        }
      }
    } else {
      r.m.get(m);
      r.v.get(v);
    }
    r.g.get(g);
    r.p.get(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      update_moments(h, g[j], m[j], v[j]);
      p[j] = update_param(h, p[j], m[j], v[j]);
    }
    uint32_t u[4];
    if (Random) random_pairs(key, counter, u);
    if (Weight == kWeightBf16) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = Random ? random_bf16x2(p[j], u[j]) : nearest_bf16x2(p[j]);
      store_bf16(at.p, left, w);
    } else {
      put_f32(at.p, left, p);
      if (Weight == kWeightMaster) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = nearest_bf16x2(p[j]);
        store_bf16(at.w, left, w);
      }
    }
    if constexpr (Eight) {
      em = store_codes<true, Random>(m, u, at.m, left);
      ev = store_codes<false, Random>(v, u, at.v, left);
    } else {
      put_f32(at.m, left, m);
      put_f32(at.v, left, v);
    }
  }

  // One block of an aligned tensor, whole or its last.
  static __device__ __forceinline__ void one(const Hyper& h, const OptDesc& d, uint32_t block, RandomKey key, int lane) {
    const Places at(d, block, lane);
    const int left = elements_left(d.n, block, lane);
    const uint32_t counter = random_counter(key, (static_cast<uint64_t>(block) * kOptBlock + d.skipped) / 2 + 4 * lane);
    Raw r;
    r.load(at, left);
    Exponents e = {0, 0};
    if (Eight) e.load(d.m_exp + block, d.v_exp + block, 1, lane);
    uint32_t em = e.of_m(0), ev = e.of_v(0);
    finish(h, at, left, counter, key, r, em, ev);
    e = {em, ev};
    if (Eight) e.store(d.m_exp + block, d.v_exp + block, 1, lane);
  }
  static __device__ __noinline__ void last(const StepParams& p, float scale, uint32_t t) {
    const OptDesc d = p.work.tensors[t];
    RandomKey key = {0, 0};
    if (Random) key = random_key(p.key, d.tensor);
    one(hyper(p, scale, d), d, d.n_blocks - 1, key, threadIdx.x % 32);
  }

  // `count` whole blocks of a tensor one after the other, the next one or two on
  // their way through shared memory.  Not unrolled: the code must stay in the
  // instruction cache.  Odd: off the vectors' boundaries; results leave by way of
  // the slot that their block came to.
  static __device__ __forceinline__ void run(const Hyper& h, const OptDesc& d, uint32_t block, int count, RandomKey key, int lane) {
    __shared__ __align__(16) uint8_t slots[kOptWarps * kSlots * kSlotSize];
    uint8_t* const my_slots = slots + (threadIdx.x / 32) * (kSlots * kSlotSize);
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(my_slots));
    Places at(d, block, lane);
    // (a run does not pass a multiple of 2^32 pairs: see run_length)
    uint32_t counter = random_counter(key, static_cast<uint64_t>(block) * (kOptBlock / 2) + 4 * lane);
    constexpr int kAtP = kOptBlock * kGradBytes, kAtM = kAtP + kOptBlock * RawParam::kBytes, kAtV = kAtM + kOptBlock * kMomentBytes;
    auto fetch = [&](int ahead, int slot) {
      const uint32_t to = mine + slot * kSlotSize;
      auto one = [&](auto raw, int offset, int extra, const uint8_t* p) {
        using R = decltype(raw);
        p += ahead * (kOptBlock * R::kBytes);
        Odd ? R::fetch_odd(to + offset, to + kSlot + extra, p, lane) : R::fetch(to + offset, p, lane);
      };
      one(RawGrad(), 0, 0, at.g);
      one(RawParam(), kAtP, 4, at.p);
      one(RawMoment(), kAtM, 8, at.m);
      one(RawMoment(), kAtV, 12, at.v);
    };
#pragma unroll
    for (int k = 0; k < kSlots - 1; ++k) {
      if (k < count) fetch(k, k);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    uint32_t em, ev;
    Exponents e = {0, 0};
    if (Eight) e.load(d.m_exp + block, d.v_exp + block, count, lane);
#pragma unroll 1
    for (int k = 0, slot = 0;;) {
      // into the slot that the block before has left
      if (k + kSlots - 1 < count) fetch(kSlots - 1, slot == 0 ? kSlots - 1 : slot - 1);
      asm volatile("cp.async.commit_group;" ::: "memory");  // (of nothing too: the wait counts groups)
      asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 1) : "memory");
      __syncwarp();  // what the other lanes fetched is there
      Raw r;
      const uint32_t from = mine + slot * kSlotSize;
      auto take = [&](auto& raw, int offset, int extra, const uint8_t* p) {
        Odd ? raw.take_odd(from + offset, from + kSlot + extra, p, lane) : raw.take(from + offset, lane);
      };
      take(r.g, 0, 0, at.g);
      take(r.p, kAtP, 4, at.p);
      take(r.m, kAtM, 8, at.m);
      take(r.v, kAtV, 12, at.v);
      __syncwarp();  // and taken, before the next turn fetches into the slot
      em = e.of_m(k), ev = e.of_v(k);
      if constexpr (Odd) {
        constexpr int kP = 0, kW = kOptBlock * RawParam::kBytes, kM = kW + (Weight == kWeightMaster ? kOptBlock * 2 : 0), kV = kM + kOptBlock * kMomentBytes;
        static_assert(kV + kOptBlock * kMomentBytes <= kSlot, "a block's results in its slot");
        uint8_t* const out = my_slots + slot * kSlotSize;
        Places to = at;
        to.p = out + kP + lane * kOptLane * RawParam::kBytes;
        to.w = out + kW + lane * kOptLane * 2;
        to.m = out + kM + lane * kOptLane * kMomentBytes;
        to.v = out + kV + lane * kOptLane * kMomentBytes;
        finish(h, to, kOptLane, counter, key, r, em, ev);
        __syncwarp();
        copy_out<std::conditional_t<Weight == kWeightBf16, uint16_t, float>>(at.p - lane * kOptLane * RawParam::kBytes, out + kP, lane);
        if (Weight == kWeightMaster) copy_out<uint16_t>(at.w - lane * kOptLane * 2, out + kW, lane);
        using Moment = std::conditional_t<Eight, uint8_t, float>;
        copy_out<Moment>(at.m - lane * kOptLane * kMomentBytes, out + kM, lane);
        copy_out<Moment>(at.v - lane * kOptLane * kMomentBytes, out + kV, lane);
        __syncwarp();  // as above
      } else {
        finish(h, at, kOptLane, counter, key, r, em, ev);
      }
      e.set(k, lane, em, ev);
      if (++k == count) break;
      slot = slot == kSlots - 1 ? 0 : slot + 1;
      counter += kOptBlock / 2 * kRandomStep;
      at.next();
    }
    if (Eight) e.store(d.m_exp + block, d.v_exp + block, count, lane);
  }

  // Any block of tensor t, element by element: a tensor's last one, or a head of
  // less than a block, off the vectors' boundaries; all for an eps that is too small.
  static __device__ __noinline__ void any(const StepParams& p, float scale, uint32_t t, uint32_t block) {
    const OptDesc d = p.work.tensors[t];
    const int lane = threadIdx.x % 32;
    const Hyper h = hyper(p, scale, d);
    RandomKey key = {0, 0};
    if (Random) key = random_key(p.key, d.tensor);
    const uint64_t first = static_cast<uint64_t>(block) * kOptBlock;
    const int left = static_cast<int>(min(d.n - first, static_cast<uint64_t>(kOptBlock)));
    uint8_t* const m_at = static_cast<uint8_t*>(d.m) + first * kMomentBytes;
    uint8_t* const v_at = static_cast<uint8_t*>(d.v) + first * kMomentBytes;
    float g[kOptLane], x[kOptLane], m[kOptLane], v[kOptLane];
    load_any<std::conditional_t<Bf16Grad, uint16_t, float>>(static_cast<const uint8_t*>(d.grad) + first * kGradBytes, lane, left, g);
    if (Weight == kWeightMaster)
      load_any<float>(d.master + first, lane, left, x);
    else if (Weight == kWeightBf16)
      load_any<uint16_t>(static_cast<const uint16_t*>(d.weight) + first, lane, left, x);
    else
      load_any<float>(static_cast<const float*>(d.weight) + first, lane, left, x);
    if (Eight) {
      const uint32_t em = d.m_exp[block], ev = d.v_exp[block];
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
      const Pair old = make_float2(x[j], x[j + 1]), q = p.exact ? update_param_exactly(h, old, a, b) : update_param(h, old, a, b);
      m[j] = a.x, m[j + 1] = a.y, v[j] = b.x, v[j + 1] = b.y, x[j] = q.x, x[j + 1] = q.y;
    }
    if (Weight == kWeightMaster) store_any<float>(d.master + first, lane, left, x);
    if (Weight == kWeightF32) {
      store_any<float>(static_cast<float*>(d.weight) + first, lane, left, x);
    } else {
      uint16_t w[kOptLane];
#pragma unroll
      for (int j = 0; j < kOptLane; ++j) {
        const uint64_t i = first + d.skipped + j * 32 + lane;
        const Pair twice = pair(x[j]);  // (the pair's half that counts)
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

// Blocks from `block` on whose pairs' indices have the same high word.
__device__ __forceinline__ uint32_t run_length(uint32_t block) {
  constexpr uint32_t kBlocks = (1ull << 33) / kOptBlock;
  return kBlocks - block % kBlocks;
}

template <int Weight, bool Bf16Grad, bool Eight, bool Odd, bool Random>
__global__ void __launch_bounds__(32 * kOptWarps, step_ctas(Eight, Weight, Bf16Grad, Odd)) step_kernel(const __grid_constant__ StepParams p) {
  using S = Step<Weight, Bf16Grad, Eight, Odd, Random>;
  const uint32_t per_warp = Eight ? p.work.per_warp : 1, warp = threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  uint32_t b = (blockIdx.x * kOptWarps + warp) * per_warp;
  const uint32_t end = min(b + per_warp, p.work.n_blocks);
  if (b >= end) return;
  uint32_t t = first_tensor(p.work, blockIdx.x, warp, kOptWarps, b);
  OptDesc d = p.work.tensors[t];  // (the plan's tables: nothing writes them)
  wait_for_kernel_before();
  float scale = 1.0f;
  if (p.clip != nullptr) {
    if (p.clip->nonfinite != 0) return;
    scale = p.clip->scale;
  }
#pragma unroll 1
  for (;;) {
    const uint32_t block = b - d.first;
    uint32_t count = 1;
    const uint32_t whole = static_cast<uint32_t>(d.n / kOptBlock);
    if (Odd ? !p.exact && block < whole : d.aligned && !p.exact) {
      RandomKey key = {0, 0};
      if (Random) key = random_key(p.key, d.tensor);
      if constexpr (!Eight && !Odd) {
        S::one(hyper(p, scale, d), d, block, key, lane);
      } else if (block < whole) {
        if (Eight) count = min(min(end - b, whole - block), run_length(block));
        S::run(hyper(p, scale, d), d, block, static_cast<int>(count), key, lane);
      } else if (!Odd) {
        S::last(p, scale, t);
      }
    } else {
      S::any(p, scale, t, block);
    }
    b += count;
    if (b >= end) return;
    t = tensor_of(p.work, t, b);
    d = p.work.tensors[t];
  }
}

template <class F>
auto for_class(const StepClass& c, bool random, F&& f) {
  auto with = [&](auto weight, auto grad, auto eight, auto odd) {
    // random rounding concerns codes, and bf16 weights without a master
    constexpr int kWeight = decltype(weight)::value;
    constexpr bool kGrad = decltype(grad)::value, kEight = decltype(eight)::value, kOdd = decltype(odd)::value;
    if constexpr (kEight || kWeight == kWeightBf16)
      if (random) return f(step_kernel<kWeight, kGrad, kEight, kOdd, true>);
    return f(step_kernel<kWeight, kGrad, kEight, kOdd, false>);
  };
  const std::true_type yes;
  const std::false_type no;
  auto with_moments = [&](auto weight, auto grad) {
    if (c.odd) return c.eight ? with(weight, grad, yes, yes) : with(weight, grad, no, yes);
    return c.eight ? with(weight, grad, yes, no) : with(weight, grad, no, no);
  };
  auto with_types = [&](auto weight) { return c.bf16_grad ? with_moments(weight, yes) : with_moments(weight, no); };
  if (c.weight == kWeightMaster) return with_types(std::integral_constant<int, kWeightMaster>());
  if (c.weight == kWeightBf16) return with_types(std::integral_constant<int, kWeightBf16>());
  return with_types(std::integral_constant<int, kWeightF32>());
}

}  // namespace

cudaError_t launch_step(const StepClass& c, const StepParams& p, cudaStream_t s) {
  return for_class(c, p.random != 0, [&](auto kernel) { return launch_chained(kernel, static_cast<int>(p.work.n_groups), 32 * kOptWarps, 0, s, p); });
}

}  // namespace frk
