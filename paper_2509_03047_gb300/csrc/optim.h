// optim.h -- the optimizer step's plan tables and kernel launchers (internal
// to libflashrec).
//
// Work is counted in blocks of kOptBlock elements from each tensor's start:
// what a warp takes at a time, eight elements per lane.  A launch's blocks are
// those of its tensors one after the other, in units of consecutive blocks.
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

// Tensors in order, and for each unit the tensor that it starts in.
struct OptWork {
  const OptDesc* tensors;
  const uint32_t* start;
  uint32_t n_blocks, n_units, unit_blocks;
};

constexpr int kOptWarps = 8;  // per CTA, in every kernel here

// ---- the norm

// A launch's sums are added in an order that units and CTAs decide, so both
// follow from the sizes alone, not from the GPU: at most 4 CTAs for each of a
// GB300's 152 SMs, about four units for each, of 2 to 16 blocks per warp.
constexpr uint32_t kClipUnit = 16 * kOptWarps;
constexpr uint32_t kClipCtas = 4 * 152;
inline uint32_t clip_unit(uint64_t n_blocks) {
  const uint64_t per_warp = n_blocks / (4 * kClipCtas * kOptWarps);
  return static_cast<uint32_t>(per_warp < 2 ? 2 : per_warp < 16 ? per_warp : 16) * kOptWarps;
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
cudaError_t launch_clip(const ClipParams& p, cudaStream_t s);

// ---- the step

// Tensors of one launch have one type of everything.
enum : int { kWeightF32 = 0, kWeightBf16 = 1, kWeightMaster = 2 };  // the parameter: fp32 weight, bf16 weight, master
struct StepClass {
  int weight;
  bool bf16_grad, eight;
  int index() const { return (weight * 2 + bf16_grad) * 2 + eight; }
};
constexpr int kStepClasses = 3 * 2 * 2;

struct StepParams {
  OptWork work;
  const fr_clip* clip;         // may be null
  float b1, c1, b2, c2;        // beta1, 1 - beta1, beta2, 1 - beta2
  float lr, decay, eps;
  float m_fix, v_fix;          // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  uint32_t exact;              // 1: eps is too small for the approximations of update_param (optim_math.cuh)
  uint32_t random;             // 1: FR_ROUND_RANDOM
  uint64_t key;                // of the random bits: mix64(mix64(seed) + step)
};
cudaError_t launch_step(const StepClass& c, const StepParams& p, cudaStream_t s);

// ---- conversion

struct ConvertParams {
  OptWork src, dst;  // the same blocks
  uint32_t to_eight;
  uint32_t random;
  uint64_t key;
};
cudaError_t launch_convert(const ConvertParams& p, cudaStream_t s);

// splitmix64's output function (Steele, Lea, Flood, "Fast splittable
// pseudorandom number generators", OOPSLA 2014).
__host__ __device__ inline uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

}  // namespace frk
