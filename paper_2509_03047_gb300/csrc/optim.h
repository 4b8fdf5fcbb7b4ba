// optim.h -- the optimizer step's plan tables and kernel launchers (internal
// to libflashrec).
//
// Work is counted in blocks of kOptBlock elements from each tensor's start:
// what a warp takes at a time, eight elements per lane.  A launch's blocks are
// those of its tensors one after the other.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/flashrec.h"

namespace frk {

constexpr int kOptBlock = FR_OPT_BLOCK;
constexpr int kOptLane = kOptBlock / 32;  // elements of a block per lane
static_assert(kOptBlock == 256, "eight elements per lane");

struct OptDesc {        // 96 bytes: one tensor that has elements, or a part of it
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
  uint32_t skipped;     // elements of the plan's tensor before this one's first
};
static_assert(sizeof(OptDesc) == 96, "OptDesc layout");

// Tensors in order, cut into groups of `warps` times `per_warp` consecutive
// blocks, one for a CTA (the norm: one of a CTA's segments).  start: the tensor of
// each group's first block, or where the table stays small, of each warp's first
// one, which spares the way from there (10,000 tensors of up to 2,000 elements,
// 32-bit step 11.1 us, so 9.8; 20,000 larger ones alike).
struct OptWork {
  const OptDesc* tensors;
  const uint32_t* start;
  uint32_t n_tensors, n_blocks, n_groups, per_warp, start_of_warps;
};
constexpr uint64_t kMostWarpStarts = 1u << 18;

constexpr int kOptWarps = 8;  // per CTA of the step and the conversion
constexpr uint32_t kSms = 152;  // of a GB300

// ---- the norm

// A launch's sums are added in an order that segments and CTAs decide, so both
// follow from the sizes alone, not from the GPU: segments of 1 to 16 blocks per
// warp, one CTA per SM at most; CTA c of g takes the segments c, c + g, ...  (One CTA of 32 warps, not four of 8: each
// that ends costs the last one's count; the norm of 1 million elements 4.6 us,
// 8.6 with four.  One range of blocks per CTA: an 8B rank's 2 GB 287 us, so 276.)
constexpr int kClipWarps = 32;
constexpr uint32_t kClipCtas = kSms;
constexpr uint32_t kClipMost = 16;  // blocks per warp
inline uint32_t clip_blocks(uint64_t n_blocks) {  // per warp, so that every CTA has the same number of segments
  constexpr uint64_t kRound = static_cast<uint64_t>(kClipCtas) * kClipWarps;
  const uint64_t rounds = (n_blocks + kRound * kClipMost - 1) / (kRound * kClipMost);
  return rounds ? static_cast<uint32_t>((n_blocks + kRound * rounds - 1) / (kRound * rounds)) : 1;
}
struct ClipPartial {  // a sum of squares, of a lane, a warp or a CTA: hi + lo + exact
  float hi, lo;       // of what was added in fp32
  double exact;       // of what was added in fp64
  uint64_t nonfinite;
};
struct ClipParams {
  OptWork work;
  ClipPartial* partials;  // one per CTA
  uint32_t* done;  // CTAs that have written theirs; zero before a launch and after it
  float grad_scale, max_norm;
  fr_clip* out;
};
cudaError_t launch_clip(const ClipParams& p, cudaStream_t s);

// ---- the step

// Tensors of one launch have one type of everything.  Those that are odd (not all
// buffers on the vectors' boundaries, and a whole block) have launches of their
// own: in one kernel with the others they cost these up to 1% with 8-bit moments
// (10,000 tensors of 1 to 28,000 elements 3%).
enum : int { kWeightF32 = 0, kWeightBf16 = 1, kWeightMaster = 2 };  // the parameter: fp32 weight, bf16 weight, master
struct StepClass {
  int weight;
  bool bf16_grad, eight, odd;
  int index() const { return ((weight * 2 + bf16_grad) * 2 + eight) * 2 + odd; }
};
constexpr int kStepClasses = 3 * 2 * 2 * 2;

using Pair = float2;

struct StepNumbers {
  Pair b1, c1, b2, c2;  // beta1, 1 - beta1, beta2, 1 - beta2
  Pair m_fix, v_fix;    // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  Pair eps;
};
struct StepParams {
  OptWork work;
  const fr_clip* clip;         // may be null
  StepNumbers numbers;
  float lr, decay;
  uint32_t exact;              // 1: eps is too small for the approximations of update_param (optim_math.cuh)
  uint32_t random;             // 1: FR_ROUND_RANDOM
  uint64_t key;                // of the random bits: mix64(mix64(seed) + step)
};
// CTAs of eight warps per SM, what the registers of a lane's elements allow.  (Of
// the 8-bit classes the one that loads least gains by a fourth: GPT-2 small 193 us,
// 200 with three; with masters 299 with four, 290 with three.  Odd ones with every
// buffer off: 345 with four, 332 with three.)
constexpr int step_ctas(bool eight, int weight, bool bf16_grad, bool odd) { return eight && (odd || !(weight == kWeightBf16 && bf16_grad)) ? 3 : 4; }
// Consecutive blocks per warp.
inline uint32_t step_blocks(bool eight, uint64_t n_blocks) {
  if (!eight) return 1;
  const uint64_t warps = kSms * 3 * kOptWarps, b = n_blocks / (2 * warps);
  return static_cast<uint32_t>(b < 1 ? 1 : b < 8 ? b : 8);
}
cudaError_t launch_step(const StepClass& c, const StepParams& p, cudaStream_t s);

// ---- conversion

struct ConvertParams {
  OptWork src, dst;  // the same blocks
  uint32_t to_eight;
  uint32_t random;
  uint64_t key;
};
// Blocks per warp, loaded together (one, two, three, four of GPT-2 small: to 8
// bits 239, 193, 192, 202 us, back 185, 179, 180, 180; of 18 million elements in
// 2,000 tensors 40, 36, 38, 43 and 33 for each).
constexpr int kConvertBlocks = 2;
cudaError_t launch_convert(const ConvertParams& p, cudaStream_t s);

// splitmix64's output function (Steele, Lea, Flood, "Fast splittable
// pseudorandom number generators", OOPSLA 2014).
__host__ __device__ inline uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

}  // namespace frk
