// optim.h -- the optimizer step's plan tables and kernel launchers (internal
// to libflashrec).
//
// Work is counted in blocks of kOptBlock elements from each tensor's start, a
// warp's unit: eight elements per lane.  A launch cuts the concatenated blocks
// of its tensors into one contiguous range per warp, so the warps take equal
// times whatever the tensor sizes.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/flashrec.h"

namespace frk {

constexpr int kOptBlock = FR_OPT_BLOCK;
constexpr int kOptLane = kOptBlock / 32;  // elements of a block per lane
static_assert(kOptBlock == 256, "eight elements per lane");

struct OptDesc {        // 96 bytes: one tensor that has elements
  void* weight;
  const void* grad;
  float* master;
  void* m;
  void* v;
  uint8_t* m_exp;
  uint8_t* v_exp;
  uint64_t n;           // elements
  uint32_t first;       // blocks of the tensors before it in its list
  uint32_t n_blocks;
  uint32_t tensor;      // index in the plan
  uint32_t bf16_grad;
  float lr_scale;
  float decay_scale;
  uint32_t aligned;     // every buffer that it has starts at a vector's boundary
  uint32_t unused;
};
static_assert(sizeof(OptDesc) == 96, "OptDesc layout");

// Tensors in order, and for each warp of a launch the tensor that its range
// starts in: warp w of n_warps takes the blocks [n_blocks * w / n_warps,
// n_blocks * (w + 1) / n_warps).
struct OptWork {
  const OptDesc* tensors;
  const uint32_t* start;
  uint32_t n_blocks;
  uint32_t n_warps;
};
__host__ __device__ inline uint32_t opt_range(uint32_t n_blocks, uint32_t n_warps, uint32_t w) {
  return static_cast<uint32_t>(static_cast<uint64_t>(n_blocks) * w / n_warps);
}

constexpr int kOptWarps = 8;  // per CTA, in every kernel here

// ---- the norm

// A launch's sums are added in an order that the warps' ranges decide, so how
// many there are follows from the sizes alone, not from the GPU: four blocks
// per warp at least, and 8 CTAs for each of a GB300's 152 SMs at most.
constexpr uint32_t kClipCtas = 8 * 152;
inline uint32_t clip_ctas(uint64_t n_blocks) {
  const uint64_t c = (n_blocks + 4 * kOptWarps - 1) / (4 * kOptWarps);
  return c < 1 ? 1 : c < kClipCtas ? static_cast<uint32_t>(c) : kClipCtas;
}
struct ClipPartial {  // of one CTA
  double sumsq;
  uint64_t nonfinite;
};
struct ClipParams {
  OptWork work;
  ClipPartial* partials;
  uint32_t* done;  // CTAs that have written theirs; zero before a launch and after it
  double grad_scale, max_norm;
  fr_clip* out;
};
cudaError_t launch_clip(const ClipParams& p, int n_ctas, cudaStream_t s);

// ---- the step

// Tensors of one launch have one type of everything.
enum : int { kWeightF32 = 0, kWeightBf16 = 1, kWeightMaster = 2 };  // the parameter: fp32 weight, bf16 weight, master
struct StepClass {
  int weight;
  bool bf16_grad, eight, aligned;
  int index() const { return ((weight * 2 + bf16_grad) * 2 + eight) * 2 + aligned; }
};
constexpr int kStepClasses = 3 * 2 * 2 * 2;

struct StepParams {
  OptWork work;
  const fr_clip* clip;         // may be null
  float b1, c1, b2, c2;        // beta1, 1 - beta1, beta2, 1 - beta2
  float lr, decay, eps;
  float m_fix, v_fix;          // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  uint32_t random;             // 1: FR_ROUND_RANDOM
  uint64_t key;                // of the random bits: mix64(mix64(seed) + step)
};
cudaError_t launch_step(const StepClass& c, const StepParams& p, int n_ctas, cudaStream_t s);
int step_ctas_per_sm(const StepClass& c);

// ---- conversion

struct ConvertParams {
  OptWork src, dst;  // the same blocks
  uint32_t to_eight;
  uint32_t random;
  uint64_t key;
};
constexpr int kConvertCtasPerSm = 4;
cudaError_t launch_convert(const ConvertParams& p, int n_ctas, cudaStream_t s);

// splitmix64's output function (Steele, Lea, Flood, "Fast splittable
// pseudorandom number generators", OOPSLA 2014).
__host__ __device__ inline uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

}  // namespace frk
