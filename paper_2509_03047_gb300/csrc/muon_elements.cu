// muon_elements.cu -- what the orthogonalised update does element by element:
// momentum and norm, the first iterate, the weights.
//
// Every operation is written as the one rounding that it is, as in
// optim_math.cuh, so both passes over the momentum see the same G.
//
// Bound by memory, at two thirds of its rate: 88 million elements in bf16 with their
// momenta, norm 165 us (10 bytes an element, 5.3 TB/s; each CTA waits for its stores
// before it is counted), X from it 169 (10), weights 106 (6).  More loads at a time, shorter and longer CTAs,
// and lists cut into parts that L2 holds are slower or equal.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "kernels.h"
#include "muon_block.cuh"
#include "optim_math.cuh"

namespace frk {

namespace {

constexpr int kWarps = kElementThreads / 32;

__device__ __forceinline__ bool skipped(const MuonParams& p) { return p.clip != nullptr && p.clip->nonfinite != 0; }
__device__ __forceinline__ bool is_split(const MuonParams& p, const MuonDesc& d) { return d.split && !p.one; }
__device__ __forceinline__ float grad_scale(const MuonParams& p) { return p.clip != nullptr ? p.clip->scale : 1.0f; }

// Eight consecutive elements of an fp32 or bf16 buffer from element i, `left` of them there; zeros after them.
__device__ __forceinline__ void load_f32(const float* at, uint64_t i, int left, float (&x)[8]) {
  at += i;
  if (left >= 8 && reinterpret_cast<uint64_t>(at) % 16 == 0) {
    const float4 u = *reinterpret_cast<const float4*>(at), v = *reinterpret_cast<const float4*>(at + 4);
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? at[j] : 0.0f;
  }
}
__device__ __forceinline__ void load_bf16(const __nv_bfloat16* at, uint64_t i, int left, float (&x)[8]) {
  at += i;
  if (left >= 8 && reinterpret_cast<uint64_t>(at) % 16 == 0) {
    const uint4 w = *reinterpret_cast<const uint4*>(at);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(v[j] << 16);
      x[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? __bfloat162float(at[j]) : 0.0f;
  }
}
__device__ __forceinline__ void load(const void* at, bool bf16, uint64_t i, int left, float (&x)[8]) {
  if (bf16)
    load_bf16(static_cast<const __nv_bfloat16*>(at), i, left, x);
  else
    load_f32(static_cast<const float*>(at), i, left, x);
}
__device__ __forceinline__ void store_f32(float* at, uint64_t i, int left, const float (&x)[8]) {
  at += i;
  if (left >= 8 && reinterpret_cast<uint64_t>(at) % 16 == 0) {
    *reinterpret_cast<float4*>(at) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(at + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) at[j] = x[j];
  }
}
__device__ __forceinline__ void store_bf16(__nv_bfloat16* at, uint64_t i, int left, const __nv_bfloat16 (&x)[8]) {
  at += i;
  if (left >= 8 && reinterpret_cast<uint64_t>(at) % 16 == 0) {
    *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(&x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) at[j] = x[j];
  }
}

// beta x + (1 - beta) h, each operation rounded.
__device__ __forceinline__ float mix(const MuonParams& p, float x, float h) { return __fadd_rn(__fmul_rn(x, p.beta), __fmul_rn(h, p.beta_rest)); }

// G from the gradient and (with momentum) the new momentum.
__device__ __forceinline__ void matrix_of(const MuonParams& p, float scale, const float (&grad)[8], const float (&m)[8], float (&g)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] = !p.momentum ? grad[j] : p.nesterov ? mix(p, m[j], __fmul_rn(grad[j], scale)) : m[j];
}

// New momenta, and per unit the sum of squares of G, scaled by a power of two that
// brings the unit's largest to [1, 2), so that no square over- or underflows.  The
// last unit of a matrix adds its units' sums, in their order, in fp64.
__global__ void __launch_bounds__(kElementThreads) norm_kernel(const __grid_constant__ MuonParams p) {
  __shared__ uint32_t tops[kWarps];
  __shared__ float sums[kWarps];
  __shared__ double wide[kWarps];
  __shared__ int exponents[kWarps];
  __shared__ uint32_t last;
  const uint32_t t = p.units[blockIdx.x], lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const MuonDesc& d = p.tensors[t];
  wait_for_kernel_before();
  // (after a wait that was given up momenta stay too, as long as nobody has asked)
  const bool stopped = p.momentum && *p.status != 0;
  if (skipped(p) || stopped) return;
  const float scale = grad_scale(p);
  const uint64_t n = d.rows * d.cols, first = static_cast<uint64_t>(blockIdx.x - d.first_unit) * kUnit;
  constexpr int kEach = kUnit / (8 * kElementThreads);
  float g[kEach][8];
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const uint64_t i = first + (k * kElementThreads + threadIdx.x) * 8;
    const int left = i < n ? static_cast<int>(min(n - i, uint64_t{8})) : 0;
    float m[8] = {}, grad[8];
    load(d.grad, d.bf16_grad, i, left, grad);
    if (p.momentum) {
      load_f32(d.momentum, i, left, m);
#pragma unroll
      for (int j = 0; j < 8; ++j) m[j] = mix(p, m[j], __fmul_rn(grad[j], scale));
      store_f32(d.momentum, i, left, m);
    }
    matrix_of(p, scale, grad, m, g[k]);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(g[k][j]) & 0x7FFFFFFFu);
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (lane == 0) tops[warp] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) top = max(top, tops[w]);
  // (a subnormal largest counts as 2^-126; Inf and NaN give NaN below)
  const int exponent = static_cast<int>(max(top >> 23, 1u)) - 127;
  const float to_one = ldexpf(1.0f, -min(exponent, 127));
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < kEach; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float y = g[k][j] * to_one;
      sum = __fmaf_rn(y, y, sum);
    }
#pragma unroll
  for (int k = 16; k > 0; k /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, k);
  if (lane == 0) sums[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0f;
    for (int w = 0; w < kWarps; ++w) sum += sums[w];
    if (top >= 0x7F800000u) sum = __uint_as_float(0x7FC00000u);
    p.partials[blockIdx.x] = {sum, exponent};
    uint32_t before;
    // releases the partial sum, and acquires the others' for the last; wraps to zero with it
    asm volatile("atom.inc.acq_rel.gpu.global.u32 %0, [%1], %2;" : "=r"(before) : "l"(&p.norms[t].done), "r"(d.n_units - 1) : "memory");
    last = before == d.n_units - 1;
  }
  __syncthreads();
  if (!last) return;
  const MuonPartial* q = p.partials + d.first_unit;
  int most = -1000;
  for (uint32_t i = threadIdx.x; i < d.n_units; i += kElementThreads) most = max(most, __ldcg(&q[i].exponent));
  most = __reduce_max_sync(0xFFFFFFFFu, most);
  if (lane == 0) exponents[warp] = most;
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) most = max(most, exponents[w]);
  double total = 0.0;
  for (uint32_t i = threadIdx.x; i < d.n_units; i += kElementThreads)
    total += ldexp(static_cast<double>(__ldcg(&q[i].sum)), 2 * (__ldcg(&q[i].exponent) - most));
#pragma unroll
  for (int k = 16; k > 0; k /= 2) total += __shfl_xor_sync(0xFFFFFFFFu, total, k);
  if (lane == 0) wide[warp] = total;
  __syncthreads();
  if (threadIdx.x != 0) return;
  total = 0.0;
  for (int w = 0; w < kWarps; ++w) total += wide[w];
  p.norms[t].to_one = ldexpf(1.0f, -min(most, 127));
  p.norms[t].factor = total == 0.0 ? 0.0f : static_cast<float>(kScaleX / sqrt(total));
}

// A block's chunks, four per thread: warps take rows, so that a warp's chunks are 512 consecutive bytes of the block.
struct Chunks {
  uint32_t block, row0, chunk;
  uint32_t first_col;
  __device__ __forceinline__ Chunks(const MuonDesc& d, uint32_t index) {
    block = index - d.first_block;
    row0 = block / d.col_blocks * kBlockRows + threadIdx.x / 8;
    chunk = block % d.col_blocks * 8 + threadIdx.x % 8;
    first_col = chunk * 8;
  }
  __device__ __forceinline__ uint32_t row(int k) const { return row0 + k * (kElementThreads / 8); }
};
constexpr int kChunks = kBlockRows * 8 / kElementThreads;

// X, in two halves, of a block: G scaled, zeros outside the matrix.
__global__ void __launch_bounds__(kElementThreads) iterate_kernel(const __grid_constant__ MuonParams p) {
  const uint32_t t = p.blocks[blockIdx.x];
  const MuonDesc& d = p.tensors[t];
  wait_for_kernel_before();
  if (skipped(p)) return;
  const float scale = grad_scale(p), to_one = p.norms[t].to_one, factor = p.norms[t].factor;
  const Chunks at(d, blockIdx.x);
  if (at.block == 0 && threadIdx.x < kPhases) p.done[t * kPhases + threadIdx.x] = 0;
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    const uint32_t r = at.row(k);
    const int left = r < d.rows && at.first_col < d.cols ? static_cast<int>(min(d.cols - at.first_col, uint64_t{8})) : 0;
    const uint64_t i = left ? r * d.cols + at.first_col : 0;
    float grad[8] = {}, m[8] = {}, x[8];
    if (!p.momentum || p.nesterov) load(d.grad, d.bf16_grad, i, left, grad);
    if (p.momentum) load_f32(d.momentum, i, left, m);
    matrix_of(p, scale, grad, m, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? (x[j] * to_one) * factor : 0.0f;
    uint4 hi, lo;
    split(x, hi, lo);
    *reinterpret_cast<uint4*>(p.work + d.x[0] + chunk_at(d.col_blocks, r, at.chunk)) = hi;
    if (is_split(p, d))
      *reinterpret_cast<uint4*>(p.work + d.low[0] + chunk_at(d.col_blocks, r, at.chunk)) = lo;
    else if (p.low)
      *reinterpret_cast<uint4*>(p.work + d.low[0] + low_at(d.col_blocks, r, at.chunk)) = lo;
  }
}

// (without products of them the last iterate has no second halves)
__device__ __forceinline__ void last_iterate(const MuonParams& p, const MuonDesc& d, uint32_t r, uint32_t c, float (&o)[8]) {
  const uint64_t at = chunk_at(d.col_blocks, r, c);
  floats(*reinterpret_cast<const uint4*>(p.work + d.x[p.last] + at), o);
  if (is_split(p, d)) {
    float lo[8];
    floats(*reinterpret_cast<const uint4*>(p.work + d.low[p.last] + at), lo);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] += lo[j];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] *= 1.0f / kScaleX;
}

// p - lr (update_scale O + decay p)
__global__ void __launch_bounds__(kElementThreads) apply_kernel(const __grid_constant__ MuonParams p) {
  const uint32_t t = p.blocks[blockIdx.x];
  const MuonDesc& d = p.tensors[t];
  wait_for_kernel_before();
  if (skipped(p) || *p.status != 0) return;
  const Chunks at(d, blockIdx.x);
  const float lr = __fmul_rn(p.lr, d.lr_scale), decay = __fmul_rn(p.decay, d.decay_scale);
  const RandomKey key = random_key(p.key, d.tensor);
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    const uint32_t r = at.row(k);
    if (r >= d.rows || at.first_col >= d.cols) continue;
    const int left = static_cast<int>(min(d.cols - at.first_col, uint64_t{8}));
    const uint64_t i = r * d.cols + at.first_col;
    float o[8], w[8];
    last_iterate(p, d, r, at.chunk, o);
    if (d.master != nullptr)
      load_f32(d.master, i, left, w);
    else
      load(d.weight, d.bf16_weight, i, left, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __fmaf_rn(__fmaf_rn(d.update_scale, o[j], __fmul_rn(decay, w[j])), -lr, w[j]);
    if (!d.bf16_weight) {
      store_f32(static_cast<float*>(d.weight), i, left, w);
      continue;
    }
    __nv_bfloat16 b[8];
    if (d.master != nullptr || !p.random) {
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = __float2bfloat16_rn(w[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t u = random_weights(random_pair(key, (i + j) / 2)), bits = __float_as_uint(w[j]);
        const uint32_t up = (i + j) % 2 ? u & 0xFFFFu : u >> 16;
        // (an Inf or NaN keeps its exponent, a NaN of low bits alone would not stay one)
        b[j] = (bits & 0x7F800000u) == 0x7F800000u ? __float2bfloat16_rn(w[j]) : __ushort_as_bfloat16(static_cast<uint16_t>((bits + up) >> 16));
      }
    }
    if (d.master != nullptr) store_f32(d.master, i, left, w);
    store_bf16(static_cast<__nv_bfloat16*>(d.weight), i, left, b);
  }
}

__global__ void __launch_bounds__(kElementThreads) update_kernel(const __grid_constant__ MuonParams p) {
  const uint32_t t = p.blocks[blockIdx.x];
  const MuonDesc& d = p.tensors[t];
  wait_for_kernel_before();
  if (*p.status != 0) return;
  const Chunks at(d, blockIdx.x);
#pragma unroll
  for (int k = 0; k < kChunks; ++k) {
    const uint32_t r = at.row(k);
    if (r >= d.rows || at.first_col >= d.cols) continue;
    const int left = static_cast<int>(min(d.cols - at.first_col, uint64_t{8}));
    const uint64_t i = r * d.cols + at.first_col;
    float o[8];
    last_iterate(p, d, r, at.chunk, o);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] *= d.update_scale;
    if (!d.bf16_update) {
      store_f32(static_cast<float*>(d.update), i, left, o);
      continue;
    }
    __nv_bfloat16 b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = __float2bfloat16_rn(o[j]);
    store_bf16(static_cast<__nv_bfloat16*>(d.update), i, left, b);
  }
}

}  // namespace

cudaError_t launch_muon_norm(const MuonParams& p, cudaStream_t s) { return launch_chained(norm_kernel, static_cast<int>(p.n_units), kElementThreads, 0, s, p); }
cudaError_t launch_muon_iterate(const MuonParams& p, cudaStream_t s) { return launch_chained(iterate_kernel, static_cast<int>(p.n_blocks), kElementThreads, 0, s, p); }
cudaError_t launch_muon_apply(const MuonParams& p, cudaStream_t s) { return launch_chained(apply_kernel, static_cast<int>(p.n_blocks), kElementThreads, 0, s, p); }
cudaError_t launch_muon_update(const MuonParams& p, cudaStream_t s) { return launch_chained(update_kernel, static_cast<int>(p.n_blocks), kElementThreads, 0, s, p); }

}  // namespace frk
