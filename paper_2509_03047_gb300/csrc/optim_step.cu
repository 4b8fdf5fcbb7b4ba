// optim_step.cu -- the AdamW step over a list of tensors.
//
// One launch per class of tensors (parameter type, gradient type, moments in
// 32 or 8 bits, alignment).  A warp walks its range of blocks; in a block of
// 256 elements each lane has eight.
#include "kernels.h"
#include "optim.h"
#include "optim_block.cuh"

namespace frk {

namespace {

template <int Weight, bool Bf16Grad, bool Eight, bool Aligned>
__global__ void __launch_bounds__(32 * kOptWarps) step_kernel(const StepParams p) {
  wait_for_kernel_before();
  Hyper h;
  h.scale = 1.0f;
  if (p.clip != nullptr) {
    if (p.clip->nonfinite != 0) return;
    h.scale = p.clip->scale;
  }
  h.b1 = p.b1, h.c1 = p.c1, h.b2 = p.b2, h.c2 = p.c2, h.eps = p.eps, h.m_fix = p.m_fix, h.v_fix = p.v_fix;
  const int lane = threadIdx.x % 32;
  const uint32_t w = blockIdx.x * kOptWarps + threadIdx.x / 32;
  uint32_t b = opt_range(p.work.n_blocks, p.work.n_warps, w);
  const uint32_t end = opt_range(p.work.n_blocks, p.work.n_warps, w + 1);
  if (b >= end) return;
  for (uint32_t t = p.work.start[w]; b < end; ++t) {
    const OptDesc d = p.work.tensors[t];
    h.lr = __fmul_rn(p.lr, d.lr_scale);
    h.decay = __fmul_rn(p.decay, d.decay_scale);
    const RandomKey key = random_key(p.key, d.tensor);
    const uint32_t stop = min(end, d.first + d.n_blocks);
    for (; b < stop; ++b) {
      const uint64_t first = static_cast<uint64_t>(b - d.first) * kOptBlock;
      const int left = static_cast<int>(min(d.n - first, static_cast<uint64_t>(kOptBlock)));
      float g[kOptLane], x[kOptLane], m[kOptLane], v[kOptLane];
      if (Bf16Grad)
        load<Aligned>(static_cast<const uint16_t*>(d.grad) + first, lane, left, g);
      else
        load<Aligned>(static_cast<const float*>(d.grad) + first, lane, left, g);
      if (Weight == kWeightMaster)
        load<Aligned>(d.master + first, lane, left, x);
      else if (Weight == kWeightBf16)
        load<Aligned>(static_cast<const uint16_t*>(d.weight) + first, lane, left, x);
      else
        load<Aligned>(static_cast<const float*>(d.weight) + first, lane, left, x);
      uint8_t *cm = static_cast<uint8_t*>(d.m) + first, *cv = static_cast<uint8_t*>(d.v) + first;
      float *fm = static_cast<float*>(d.m) + first, *fv = static_cast<float*>(d.v) + first;
      if (Eight) {
        uint32_t a[kOptLane], c[kOptLane];
        load<Aligned>(cm, lane, left, a);
        load<Aligned>(cv, lane, left, c);
        const uint32_t em = d.m_exp[b - d.first], ev = d.v_exp[b - d.first];
        __syncwarp();  // every lane has read the exponents before one writes them
#pragma unroll
        for (int j = 0; j < kOptLane; ++j) {
          m[j] = decode_m(a[j], em);
          v[j] = decode_v(c[j], ev);
          if (place<Aligned>(lane, j) >= left) m[j] = v[j] = 0.0f;
        }
      } else {
        load<Aligned>(fm, lane, left, m);
        load<Aligned>(fv, lane, left, v);
      }
      uint32_t rm[kOptLane], rv[kOptLane], rw[kOptLane];
      if ((Eight || Weight == kWeightBf16) && p.random) {
        random_bits<Aligned>(key, first, lane, rm, rw);
#pragma unroll
        for (int j = 0; j < kOptLane; ++j) rv[j] = rm[j] >> 16;
      }
#pragma unroll
      for (int j = 0; j < kOptLane; ++j) {
        update_moments(h, g[j], m[j], v[j]);
        x[j] = update_param(h, x[j], m[j], v[j]);
      }
      if (Weight == kWeightMaster) store<Aligned>(d.master + first, lane, left, x);
      if (Weight == kWeightF32) {
        store<Aligned>(static_cast<float*>(d.weight) + first, lane, left, x);
      } else {
        uint16_t y[kOptLane];
#pragma unroll
        for (int j = 0; j < kOptLane; ++j) {
          if (Weight == kWeightBf16 && p.random && isfinite(x[j]))
            y[j] = static_cast<uint16_t>((__float_as_uint(x[j]) + rw[j]) >> 16);
          else
            y[j] = __bfloat16_as_ushort(__float2bfloat16_rn(x[j]));
        }
        store<Aligned>(static_cast<uint16_t*>(d.weight) + first, lane, left, y);
      }
      if (Eight) {
        store_moments<Aligned, true>(m, rm, p.random, cm, d.m_exp + (b - d.first), lane, left);
        store_moments<Aligned, false>(v, rv, p.random, cv, d.v_exp + (b - d.first), lane, left);
      } else {
        store<Aligned>(fm, lane, left, m);
        store<Aligned>(fv, lane, left, v);
      }
    }
  }
}

template <int W, bool G, bool E>
cudaError_t launch_aligned(bool aligned, const StepParams& p, int n_ctas, cudaStream_t s) {
  return aligned ? launch_chained(step_kernel<W, G, E, true>, n_ctas, 32 * kOptWarps, 0, s, p)
                 : launch_chained(step_kernel<W, G, E, false>, n_ctas, 32 * kOptWarps, 0, s, p);
}
template <int W>
cudaError_t launch_weight(const StepClass& c, const StepParams& p, int n_ctas, cudaStream_t s) {
  if (c.bf16_grad)
    return c.eight ? launch_aligned<W, true, true>(c.aligned, p, n_ctas, s) : launch_aligned<W, true, false>(c.aligned, p, n_ctas, s);
  return c.eight ? launch_aligned<W, false, true>(c.aligned, p, n_ctas, s) : launch_aligned<W, false, false>(c.aligned, p, n_ctas, s);
}

}  // namespace

cudaError_t launch_step(const StepClass& c, const StepParams& p, int n_ctas, cudaStream_t s) {
  return c.weight == kWeightMaster ? launch_weight<kWeightMaster>(c, p, n_ctas, s)
         : c.weight == kWeightBf16 ? launch_weight<kWeightBf16>(c, p, n_ctas, s)
                                   : launch_weight<kWeightF32>(c, p, n_ctas, s);
}

int step_ctas_per_sm(const StepClass&) { return 4; }

}  // namespace frk
