// optim_api.cu -- the C ABI of the optimizer step (declared in
// include/flashrec.h) and its planner: the tensors of each launch in one list,
// with the tensors that its CTAs or warps start in.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <new>
#include <vector>

#include "../../include/flashrec.h"
#include "host.h"
#include "kernels.h"
#include "optim.h"

using namespace frk;

namespace {

// One launch's tensors, on the host and in the plan's device memory.
struct WorkList {
  std::vector<OptDesc> tensors;
  std::vector<uint32_t> start;
  uint64_t n_blocks = 0;
  uint32_t n_tensors = 0, n_groups = 0, per_warp = 1;
  bool start_of_warps = true;
  OptDesc* d_tensors = nullptr;
  uint32_t* d_start = nullptr;

  void add(OptDesc d) {
    d.first = static_cast<uint32_t>(n_blocks);
    n_blocks += d.n_blocks;
    tensors.push_back(d);
    ++n_tensors;
  }
  // For CTAs of `warps` warps.
  void cut(uint32_t blocks_per_warp, int warps) {
    per_warp = blocks_per_warp;
    const uint64_t per_group = static_cast<uint64_t>(per_warp) * warps, n_warps = (n_blocks + per_warp - 1) / per_warp;
    n_groups = static_cast<uint32_t>((n_blocks + per_group - 1) / per_group);
    start_of_warps = n_warps <= kMostWarpStarts;
    const uint64_t step = start_of_warps ? per_warp : per_group;
    start.resize(start_of_warps ? n_warps : n_groups);
    size_t t = 0;
    for (size_t i = 0; i < start.size(); ++i) {
      while (t + 1 < tensors.size() && tensors[t + 1].first <= i * step) ++t;
      start[i] = static_cast<uint32_t>(t);
    }
  }
  void place(PlanMemory& mem) {
    mem.table(&d_tensors, tensors);
    mem.table(&d_start, start);
  }
  OptWork work() const { return {d_tensors, d_start, n_tensors, static_cast<uint32_t>(n_blocks), n_groups, per_warp, start_of_warps}; }
};

}  // namespace

struct fr_opt_s {
  int device = 0;
  void* d_memory = nullptr;
  uint64_t n_elems = 0, n_blocks = 0;
  std::vector<uint64_t> sizes;  // of every tensor
  bool grads = true, params = true, moments = true;  // every tensor with elements has them
  bool eight = false, thirty_two = false;            // some tensor's moments have 8, 32 bits
  float most_lr = 0.0f, most_decay = 0.0f;           // the largest |lr_scale| and |decay_scale| of a step's tensors
  WorkList clip, convert;
  WorkList step[kStepClasses];
  StepClass classes[kStepClasses];
  ClipPartial* d_partials = nullptr;
  uint32_t* d_done = nullptr;
};

namespace {

Pair twice(double x) { return make_float2(static_cast<float>(x), static_cast<float>(x)); }
bool on(const void* p, uint64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
uint64_t type_bytes(uint32_t dtype) { return dtype == FR_DT_F32 ? 4 : dtype == FR_DT_BF16 ? 2 : 1; }
// The boundary on which a lane's eight elements move as one vector.
uint64_t vector_bytes(uint32_t dtype) { return kOptLane * type_bytes(dtype); }

// A tensor's descriptor, or why it has none.
const char* check(const fr_opt_tensor& x, bool& misaligned) {
  misaligned = false;
  if (x.flags != 0) return "tensor flags must be 0";
  if (x.n >= (1ull << 47)) return "tensor too large";
  if (!std::isfinite(x.lr_scale) || !std::isfinite(x.decay_scale)) return "a tensor's factors must be finite";
  const bool eight = x.state_dtype == FR_DT_BYTES;
  if (x.weight && x.weight_dtype != FR_DT_BF16 && x.weight_dtype != FR_DT_F32) return "weights are bf16 or fp32";
  if (x.grad && x.grad_dtype != FR_DT_BF16 && x.grad_dtype != FR_DT_F32) return "gradients are bf16 or fp32";
  if (x.master && (x.weight == nullptr || x.weight_dtype != FR_DT_BF16)) return "a master belongs to a bf16 weight";
  if ((x.m == nullptr) != (x.v == nullptr)) return "one of two moments is null";
  if (x.m && !eight && x.state_dtype != FR_DT_F32) return "moments are fp32 or bytes";
  const bool codes = x.m && eight;
  if ((x.m_exp != nullptr) != codes || (x.v_exp != nullptr) != codes) return "8-bit moments, and they alone, have exponents";
  misaligned = (x.weight && !on(x.weight, type_bytes(x.weight_dtype))) || (x.grad && !on(x.grad, type_bytes(x.grad_dtype))) ||
               !on(x.master, 4) || (x.m && (!on(x.m, type_bytes(x.state_dtype)) || !on(x.v, type_bytes(x.state_dtype))));
  return nullptr;
}

OptDesc describe(const fr_opt_tensor& x, uint64_t index) {
  OptDesc d = {};
  d.weight = x.weight;
  d.grad = x.grad;
  d.master = x.master;
  d.m = x.m;
  d.v = x.v;
  d.m_exp = x.m_exp;
  d.v_exp = x.v_exp;
  d.n = x.n;
  d.n_blocks = static_cast<uint32_t>((x.n + kOptBlock - 1) / kOptBlock);
  d.tensor = static_cast<uint32_t>(index);
  d.bf16_grad = x.grad && x.grad_dtype == FR_DT_BF16;
  d.lr_scale = x.lr_scale;
  d.decay_scale = x.decay_scale;
  d.aligned = (!x.weight || on(x.weight, vector_bytes(x.weight_dtype))) && (!x.grad || on(x.grad, vector_bytes(x.grad_dtype))) &&
              on(x.master, vector_bytes(FR_DT_F32)) && on(x.m, x.m ? vector_bytes(x.state_dtype) : 1) && on(x.v, x.v ? vector_bytes(x.state_dtype) : 1);
  return d;
}

// The elements of a tensor of the step before the first at which every buffer is
// on a vector's boundary, so that the rest of it moves as vectors: the views of
// flat groups start at any element, but at the same one in each.  0: none, or
// all are already, or the rest would not do: blocks of 8-bit moments start with
// the tensor, random bits of bf16 weights belong to pairs.
uint64_t head_elems(const fr_opt_tensor& x, const StepClass& c) {
  if (c.eight) return 0;
  auto to_boundary = [](const void* p, uint32_t dtype) {
    const uint64_t v = vector_bytes(dtype);
    return (v - reinterpret_cast<uintptr_t>(p) % v) % v / type_bytes(dtype);
  };
  const uint64_t head = to_boundary(x.weight, x.weight_dtype);
  if (to_boundary(x.grad, x.grad_dtype) != head || to_boundary(x.m, FR_DT_F32) != head || to_boundary(x.v, FR_DT_F32) != head) return 0;
  if (x.master && to_boundary(x.master, FR_DT_F32) != head) return 0;
  // (and a block's pairs must have one high word in their indices)
  return c.weight == kWeightBf16 && (head % 2 || x.n > 1ull << 33) ? 0 : head;
}

OptDesc part(const OptDesc& d, const fr_opt_tensor& x, uint64_t first, uint64_t n) {
  fr_opt_tensor y = x;
  auto advance = [&](const void* p, uint32_t dtype) {
    return const_cast<uint8_t*>(static_cast<const uint8_t*>(p)) + first * type_bytes(dtype);
  };
  y.weight = advance(x.weight, x.weight_dtype);
  y.grad = advance(x.grad, x.grad_dtype);
  if (x.master) y.master = reinterpret_cast<float*>(advance(x.master, FR_DT_F32));
  y.m = advance(x.m, FR_DT_F32);
  y.v = advance(x.v, FR_DT_F32);
  y.n = n;
  OptDesc r = describe(y, d.tensor);
  r.skipped = static_cast<uint32_t>(first);
  return r;
}

fr_status fill_opt(fr_opt p, const fr_opt_tensor* tensors, uint64_t n_tensors) {
  for (uint64_t t = 0; t < n_tensors; ++t) {
    const fr_opt_tensor& x = tensors[t];
    p->sizes.push_back(x.n);
    if (x.n == 0) continue;
    const OptDesc d = describe(x, t);
    p->n_elems += x.n;
    p->n_blocks += d.n_blocks;
    if (x.grad) p->clip.add(d);
    if (x.m) {
      OptDesc moments = d;
      moments.aligned = on(x.m, vector_bytes(x.state_dtype)) && on(x.v, vector_bytes(x.state_dtype));
      p->convert.add(moments);
    }
    if (x.weight && x.grad && x.m) {
      StepClass c;
      c.weight = x.master ? kWeightMaster : x.weight_dtype == FR_DT_BF16 ? kWeightBf16 : kWeightF32;
      c.bf16_grad = x.grad_dtype == FR_DT_BF16;
      c.eight = x.state_dtype == FR_DT_BYTES;
      p->most_lr = std::max(p->most_lr, std::fabs(x.lr_scale));
      p->most_decay = std::max(p->most_decay, std::fabs(x.decay_scale));
      const uint64_t head = head_elems(x, c);
      c.odd = !d.aligned && head == 0 && x.n >= kOptBlock;
      p->classes[c.index()] = c;
      if (head > 0 && head < x.n) {
        p->step[c.index()].add(part(d, x, 0, head));
        p->step[c.index()].add(part(d, x, head, x.n - head));
      } else {
        p->step[c.index()].add(d);
      }
    } else {
      p->params = false;
    }
    p->grads &= x.grad != nullptr;
    p->moments &= x.m != nullptr;
    if (x.m) (x.state_dtype == FR_DT_BYTES ? p->eight : p->thirty_two) = true;
  }
  PlanMemory mem;
  p->clip.cut(clip_blocks(p->clip.n_blocks), kClipWarps);
  p->clip.place(mem);
  if (p->moments) {
    p->convert.cut(kConvertBlocks, kOptWarps);
    p->convert.place(mem);
  }
  if (p->params)
    for (int c = 0; c < kStepClasses; ++c) {
      if (p->step[c].n_blocks == 0) continue;
      p->step[c].cut(step_blocks(p->classes[c].eight, p->step[c].n_blocks), kOptWarps);
      p->step[c].place(mem);
    }
  mem.table(&p->d_done, std::vector<uint32_t>(1, 0));
  mem.scratch(&p->d_partials, kClipCtas);
  const cudaError_t e = mem.commit(&p->d_memory);
  // The device has them now.
  auto drop = [](WorkList& l) {
    std::vector<OptDesc>().swap(l.tensors);
    std::vector<uint32_t>().swap(l.start);
  };
  drop(p->clip);
  drop(p->convert);
  for (WorkList& l : p->step) drop(l);
  return e == cudaSuccess ? FR_OK : report_cuda("plan device tables", e);
}

}  // namespace

extern "C" {

fr_status fr_opt_create(const fr_opt_tensor* tensors, uint64_t n_tensors, fr_opt* out) {
  CallRange nvtx("fr_opt_create");
  const char* const me = "fr_opt_create";
  if (out == nullptr) return report_invalid(me, "out is null");
  *out = nullptr;
  if (n_tensors > 0 && tensors == nullptr) return report_invalid(me, "tensors is null");
  if (n_tensors >= (1ull << 32)) return report_invalid(me, "too many tensors");
  uint64_t blocks = 0;
  for (uint64_t t = 0; t < n_tensors; ++t) {
    bool misaligned;
    if (const char* what = check(tensors[t], misaligned)) return report_invalid(me, what);
    if (misaligned) {
      report_invalid(me, "a buffer is not aligned to its element size");
      return FR_ERR_ALIGNMENT;
    }
    blocks += (tensors[t].n + kOptBlock - 1) / kOptBlock + 1;  // (a head may be a block of its own)
    if (blocks >= (1ull << 32) - 4096) return report_invalid(me, "too many elements");
  }

  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda("cudaGetDevice", e);

  fr_opt p = new (std::nothrow) fr_opt_s;
  if (p == nullptr) return report_invalid(me, "out of host memory");
  p->device = dev;
  fr_status st;
  try {
    st = fill_opt(p, tensors, n_tensors);
  } catch (const std::exception&) {  // std::bad_alloc, std::length_error
    st = report_invalid(me, "out of host memory");
  }
  if (st != FR_OK) {
    cudaFree(p->d_memory);
    delete p;
    return st;
  }
  *out = p;
  return FR_OK;
}

fr_status fr_opt_info(fr_opt p, uint64_t* n_tensors, uint64_t* n_elems, uint64_t* n_blocks) {
  if (p == nullptr) return report_invalid("fr_opt_info", "plan is null");
  if (n_tensors) *n_tensors = p->sizes.size();
  if (n_elems) *n_elems = p->n_elems;
  if (n_blocks) *n_blocks = p->n_blocks;
  return FR_OK;
}

void fr_opt_destroy(fr_opt p) {
  CallRange nvtx("fr_opt_destroy");
  if (p == nullptr) return;
  DeviceGuard g(p->device);
  cudaDeviceSynchronize();
  cudaFree(p->d_memory);
  delete p;
}

fr_status fr_grad_clip(fr_opt p, float max_norm, float grad_scale, fr_clip* out_dev, void* stream) {
  CallRange nvtx("fr_grad_clip");
  const char* const me = "fr_grad_clip";
  if (p == nullptr) return report_invalid(me, "plan is null");
  if (!p->grads) return report_invalid(me, "a tensor of the plan has no gradient");
  if (!(max_norm > 0.0f)) return report_invalid(me, "max_norm must be positive");
  if (!(grad_scale > 0.0f) || !std::isfinite(grad_scale)) return report_invalid(me, "grad_scale must be positive and finite");
  if (out_dev == nullptr || !on(out_dev, 8)) return report_invalid(me, "out_dev is null or not 8-byte aligned");
  DeviceGuard g(p->device);
  if (!g.ok) return report_cuda("select plan device", cudaGetLastError());
  ClipParams cp;
  cp.work = p->clip.work();
  cp.partials = p->d_partials;
  cp.done = p->d_done;
  cp.grad_scale = grad_scale;
  cp.max_norm = max_norm;
  cp.out = out_dev;
  const cudaError_t e = launch_clip(cp, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FR_OK : report_cuda("clip kernel launch", e);
}

fr_status fr_adamw_step(fr_opt p, const fr_adamw* h, const fr_clip* clip_dev, void* stream) {
  CallRange nvtx("fr_adamw_step");
  const char* const me = "fr_adamw_step";
  if (p == nullptr || h == nullptr) return report_invalid(me, "plan or hyper is null");
  if (!p->params) return report_invalid(me, "a tensor of the plan has no weight, gradient or moments");
  if (!(h->lr >= 0.0) || !std::isfinite(static_cast<float>(h->lr))) return report_invalid(me, "lr must be finite and not negative");
  if (!(h->weight_decay >= 0.0) || !std::isfinite(static_cast<float>(h->weight_decay)))
    return report_invalid(me, "weight_decay must be finite and not negative");
  if (!(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0))
    return report_invalid(me, "betas must be in [0, 1)");
  if (!(static_cast<float>(h->eps) > 0.0f) || !std::isfinite(static_cast<float>(h->eps))) return report_invalid(me, "eps must be positive and finite");
  if (!std::isfinite(static_cast<float>(h->lr) * p->most_lr)) return report_invalid(me, "lr times a tensor's lr_scale must be finite in fp32");
  if (!std::isfinite(static_cast<float>(h->weight_decay) * p->most_decay))
    return report_invalid(me, "weight_decay times a tensor's decay_scale must be finite in fp32");
  if (h->step == 0) return report_invalid(me, "step counts from 1");
  if (h->rounding > FR_ROUND_RANDOM) return report_invalid(me, "unknown rounding");
  if (h->reserved != 0) return report_invalid(me, "reserved must be 0");
  if (clip_dev != nullptr && !on(clip_dev, 8)) return report_invalid(me, "clip_dev is not 8-byte aligned");
  DeviceGuard g(p->device);
  if (!g.ok) return report_cuda("select plan device", cudaGetLastError());
  StepParams sp;
  sp.clip = clip_dev;
  sp.numbers.b1 = twice(h->beta1);
  sp.numbers.c1 = twice(1.0 - h->beta1);
  sp.numbers.b2 = twice(h->beta2);
  sp.numbers.c2 = twice(1.0 - h->beta2);
  sp.lr = static_cast<float>(h->lr);
  sp.decay = static_cast<float>(h->weight_decay);
  sp.numbers.eps = twice(h->eps);
  sp.numbers.m_fix = twice(1.0 / (1.0 - std::pow(h->beta1, static_cast<double>(h->step))));
  sp.numbers.v_fix = twice(1.0 / std::sqrt(1.0 - std::pow(h->beta2, static_cast<double>(h->step))));
  sp.exact = sp.numbers.eps.x < 0x1p-39f * sp.numbers.v_fix.x;
  sp.random = h->rounding == FR_ROUND_RANDOM;
  sp.key = mix64(mix64(h->seed) + h->step);
  for (int c = 0; c < kStepClasses; ++c) {
    if (p->step[c].n_blocks == 0) continue;
    sp.work = p->step[c].work();
    const cudaError_t e = launch_step(p->classes[c], sp, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return report_cuda("step kernel launch", e);
  }
  return FR_OK;
}

fr_status fr_opt_convert(fr_opt src, fr_opt dst, uint32_t rounding, uint64_t seed, void* stream) {
  CallRange nvtx("fr_opt_convert");
  const char* const me = "fr_opt_convert";
  if (src == nullptr || dst == nullptr) return report_invalid(me, "plan is null");
  if (!src->moments || !dst->moments) return report_invalid(me, "a tensor of the plans has no moments");
  if (rounding > FR_ROUND_RANDOM) return report_invalid(me, "unknown rounding");
  if (src->device != dst->device || src->sizes != dst->sizes) {
    report_invalid(me, "the two plans differ in device or sizes");
    return FR_ERR_PLAN_MISMATCH;
  }
  if (src->n_blocks == 0) return FR_OK;
  if ((src->eight && src->thirty_two) || (dst->eight && dst->thirty_two) || src->eight == dst->eight)
    return report_invalid(me, "one plan's moments are all fp32 and the other's all in 8 bits");
  DeviceGuard g(dst->device);
  if (!g.ok) return report_cuda("select plan device", cudaGetLastError());
  ConvertParams cp;
  cp.src = src->convert.work();
  cp.dst = dst->convert.work();
  cp.to_eight = dst->eight;
  cp.random = rounding == FR_ROUND_RANDOM;
  cp.key = mix64(mix64(seed));
  const cudaError_t e = launch_convert(cp, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FR_OK : report_cuda("convert kernel launch", e);
}

}  // extern "C"
