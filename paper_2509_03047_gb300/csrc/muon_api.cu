// muon_api.cu -- the C ABI of the orthogonalised update (declared in
// include/flashrec.h) and its planner: places of the iterates and of their
// squares in the plan's memory, units of the norm, blocks, tiles of the products.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <new>
#include <vector>

#include "../../include/flashrec.h"
#include "host.h"
#include "kernels.h"
#include "muon.h"
#include "muon_tiles.h"
#include "optim.h"

using namespace frk;

struct fr_muon_plan_s {
  int device = 0;
  void* d_memory = nullptr;
  uint64_t n_tensors = 0, n_elems = 0, device_bytes = 0;
  bool params = true, updates = true;       // every matrix with elements has what the step, fr_orthogonalize needs
  float most_lr = 0.0f, most_decay = 0.0f;  // the largest |lr_scale| and |decay_scale|
  uint32_t n_units = 0, n_blocks = 0, pairs = 0;  // pairs of CTAs that are resident together
  struct Part {                              // the matrices that are not split, and those that are
    uint64_t x_blocks = 0, p_blocks = 0;     // of all iterates, all squares
    uint32_t ends[kPhases] = {};             // of each phase's tiles
    uint32_t most_tiles = 0;                 // of a phase
    uint32_t deepest = 0;                    // steps of a contraction
    MuonTile* d_tiles = nullptr;
  } parts[2];
  MuonDesc* d_tensors = nullptr;
  uint32_t* d_units = nullptr;
  uint32_t* d_blocks = nullptr;
  uint32_t* d_done = nullptr;
  MuonPartial* d_partials = nullptr;
  MuonNorm* d_norms = nullptr;
  uint8_t* d_work = nullptr;
  uint8_t* d_sums = nullptr;                 // where a contraction is longer than a part
  uint32_t* d_status = nullptr;
  int64_t wait_clocks = kWaitClocks;
  MuonMaps maps;
};

namespace {

constexpr uint64_t kMostSide = FR_MUON_MOST_SIDE;
constexpr uint64_t kMostElems = 1ull << 35;  // filled up; copies' indices of blocks have 31 bits

bool on(const void* p, uint64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
uint64_t type_bytes(uint32_t dtype) { return dtype == FR_DT_F32 ? 4 : 2; }
bool is_float(uint32_t dtype) { return dtype == FR_DT_BF16 || dtype == FR_DT_F32; }

const char* check(const fr_muon_tensor& x, bool& misaligned) {
  misaligned = false;
  if ((x.flags & ~FR_MUON_BOTH_HALVES) != 0 || x.reserved != 0) return "unknown tensor flags, or reserved is not 0";
  if (x.rows > kMostSide || x.cols > kMostSide) return "a matrix has too many rows or columns";
  if (!std::isfinite(x.lr_scale) || !std::isfinite(x.decay_scale) || !std::isfinite(x.update_scale)) return "a matrix's factors must be finite";
  if (x.weight && !is_float(x.weight_dtype)) return "weights are bf16 or fp32";
  if (x.grad && !is_float(x.grad_dtype)) return "gradients are bf16 or fp32";
  if (x.update && !is_float(x.update_dtype)) return "updates are bf16 or fp32";
  if (x.master && (x.weight == nullptr || x.weight_dtype != FR_DT_BF16)) return "a master belongs to a bf16 weight";
  misaligned = (x.weight && !on(x.weight, type_bytes(x.weight_dtype))) || (x.grad && !on(x.grad, type_bytes(x.grad_dtype))) ||
               (x.update && !on(x.update, type_bytes(x.update_dtype))) || !on(x.master, 4) || !on(x.momentum, 4);
  return nullptr;
}

uint32_t pieces(uint64_t n, uint64_t of) { return static_cast<uint32_t>((n + of - 1) / of); }

// A matrix's descriptor but for its places in the workspace.
MuonDesc describe(const fr_muon_tensor& x, uint64_t index) {
  MuonDesc d = {};
  d.weight = x.weight;
  d.grad = x.grad;
  d.master = x.master;
  d.momentum = x.momentum;
  d.update = x.update;
  d.rows = x.rows;
  d.cols = x.cols;
  d.row_blocks = pieces(x.rows, kBlockRows);
  d.col_blocks = 2 * pieces(x.cols, 2 * kBlockCols);
  d.tall = x.rows > x.cols;
  d.side_blocks = d.tall ? d.col_blocks / 2 : d.row_blocks;
  d.n_units = pieces(x.rows * x.cols, kUnit);
  d.tensor = static_cast<uint32_t>(index);
  d.bf16_weight = x.weight && x.weight_dtype == FR_DT_BF16;
  d.bf16_grad = x.grad && x.grad_dtype == FR_DT_BF16;
  d.bf16_update = x.update && x.update_dtype == FR_DT_BF16;
  d.split = (x.flags & FR_MUON_BOTH_HALVES) || x.master || (x.weight && !d.bf16_weight) || (x.update && !d.bf16_update);
  d.lr_scale = x.lr_scale;
  d.decay_scale = x.decay_scale;
  d.update_scale = x.update_scale;
  return d;
}

uint64_t square_blocks(const MuonDesc& d) { return 2ull * d.side_blocks * d.side_blocks; }

cudaError_t make_maps(MuonMaps* maps, void* at, uint64_t bytes) {
  void* entry = nullptr;
  cudaDriverEntryPointQueryResult found;
  const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &entry, 12000, cudaEnableDefault, &found);
  if (e != cudaSuccess) return e;
  if (found != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
  const cuuint64_t sizes[4] = {kBlockCols, kBlockRows / 2, 2, bytes / kMuonBlockBytes}, strides[3] = {128, kMuonBlockBytes / 2, kMuonBlockBytes};
  const cuuint32_t steps[4] = {1, 1, 1, 1};
  auto make = [&](CUtensorMap* map, cuuint32_t halves, cuuint32_t blocks) {
    const cuuint32_t box[4] = {kBlockCols, kBlockRows / 2, halves, blocks};
    return reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(entry)(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, at, sizes, strides, box, steps,
                                                                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                                                                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  return make(&maps->rows, 2, 1) && make(&maps->columns, 1, 2) && make(&maps->half, 1, 1) ? cudaSuccess : cudaErrorInvalidValue;
}

fr_status fill_muon(fr_muon_plan p, const fr_muon_tensor* tensors, uint64_t n_tensors) {
  std::vector<MuonDesc> descs;
  std::vector<uint32_t> units, blocks;
  p->n_tensors = n_tensors;
  for (uint64_t t = 0; t < n_tensors; ++t) {
    const fr_muon_tensor& x = tensors[t];
    if (x.rows == 0 || x.cols == 0) continue;
    p->n_elems += x.rows * x.cols;
    p->params &= x.weight && x.grad && x.momentum;
    p->updates &= x.grad && x.update;
    p->most_lr = std::max(p->most_lr, std::fabs(x.lr_scale));
    p->most_decay = std::max(p->most_decay, std::fabs(x.decay_scale));
    MuonDesc d = describe(x, t);
    const uint64_t n = static_cast<uint64_t>(d.row_blocks) * d.col_blocks;
    auto& part = p->parts[d.split];
    d.x[0] = part.x_blocks * kMuonBlockBytes;
    d.p = part.p_blocks * kMuonBlockBytes;
    part.x_blocks += n;
    part.p_blocks += square_blocks(d);
    d.first_unit = static_cast<uint32_t>(units.size());
    d.first_block = static_cast<uint32_t>(blocks.size());
    const uint32_t me = static_cast<uint32_t>(descs.size());
    units.insert(units.end(), d.n_units, me);
    blocks.insert(blocks.end(), n, me);
    descs.push_back(d);
  }
  uint64_t bytes = 0;
  for (uint32_t k = 0; k < 2; ++k) {
    const auto& part = p->parts[k];
    const uint64_t x_bytes = part.x_blocks * kMuonBlockBytes, p_bytes = part.p_blocks * kMuonBlockBytes;
    for (MuonDesc& d : descs) {
      if (d.split != k) continue;
      d.x[0] += bytes;
      d.x[1] = d.x[0] + x_bytes;
      d.low[0] = d.x[1] + x_bytes;
      d.low[1] = d.low[0] + (k ? x_bytes : 0);
      d.p += bytes + (k ? 4 : 3) * x_bytes;
      d.s = d.p + p_bytes;
    }
    bytes += k ? 4 * (x_bytes + p_bytes) : 3 * x_bytes + 2 * p_bytes;
  }
  cudaError_t e = descs.empty() ? cudaSuccess : configure_muon_product();
  if (e == cudaSuccess && !descs.empty()) e = muon_pairs(&p->pairs);
  if (e != cudaSuccess) return report_cuda("the product kernels' shared memory", e);
  PlanMemory mem;
  mem.table(&p->d_tensors, descs);
  mem.table(&p->d_units, units);
  mem.table(&p->d_blocks, blocks);
  for (uint32_t k = 0; k < 2; ++k) {
    auto& part = p->parts[k];
    std::vector<MuonTile> tiles;
    plan_tiles(descs, k != 0, tiles, part.ends);
    for (int phase = 0; phase < kPhases; ++phase) part.most_tiles = std::max(part.most_tiles, part.ends[phase] - (phase ? part.ends[phase - 1] : 0));
    for (const MuonTile& t : tiles) part.deepest = std::max(part.deepest, t.depth);
    mem.table(&part.d_tiles, tiles);
  }
  mem.scratch(&p->d_done, descs.size() * kPhases);
  mem.table(&p->d_norms, std::vector<MuonNorm>(descs.size(), MuonNorm{}));
  mem.scratch(&p->d_partials, units.size());
  mem.table(&p->d_status, std::vector<uint32_t>(1, 0));
  mem.scratch(&p->d_work, bytes);
  // (products of one half for all have longer parts)
  if (p->parts[0].deepest > part_steps(false) || p->parts[1].deepest > part_steps(true)) mem.scratch(&p->d_sums, 2ull * p->pairs * kPartBytes);
  p->n_units = static_cast<uint32_t>(units.size());
  p->n_blocks = static_cast<uint32_t>(blocks.size());
  p->device_bytes = mem.bytes();
  e = mem.commit(&p->d_memory);
  if (e != cudaSuccess) return report_cuda("plan device tables", e);
  if (bytes == 0) return FR_OK;
  e = make_maps(&p->maps, p->d_work, bytes);
  return e == cudaSuccess ? FR_OK : report_cuda("tensor maps of the workspace", e);
}

// Largest |f| on [0, top] of an odd or even polynomial given by its values and the places where its derivative in s^2 vanishes.
template <class F>
double most(F f, double top, double q2, double q1, double q0) {
  double r = std::max(std::fabs(f(0.0)), std::fabs(f(top)));
  auto at = [&](double u) {  // a root u = s^2
    if (u > 0.0 && u < top * top) r = std::max(r, std::fabs(f(std::sqrt(u))));
  };
  if (q2 == 0.0) {
    if (q1 != 0.0) at(-q0 / q1);
  } else {
    const double disc = q1 * q1 - 4.0 * q2 * q0;
    if (disc >= 0.0) {
      at((-q1 + std::sqrt(disc)) / (2.0 * q2));
      at((-q1 - std::sqrt(disc)) / (2.0 * q2));
    }
  }
  return r;
}

const char* check_iterations(const fr_muon& h) {
  if (h.products > FR_MUON_ONE) return "unknown choice of products";
  if (h.iterations < 1 || h.iterations > FR_MUON_MOST) return "iterations must be 1 to FR_MUON_MOST";
  double top = 1.0;
  for (uint32_t i = 0; i < h.iterations; ++i) {
    const double a = h.coef[i][0], b = h.coef[i][1], c = h.coef[i][2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return "coefficients must be finite";
    auto p = [&](double s) { return a + s * s * (b + c * s * s); };
    auto next = [&](double s) { return s * p(s); };
    // (a hair more than the bound, for the roundings of X)
    const double reach = top * 1.01;
    // (P is rounded to fp16 as a whole; b S and c S^2 are fp32 numbers)
    if (!(most(p, reach, 0.0, 2.0 * c, b) <= kMostP)) return "a polynomial exceeds 15 on the singular values that it meets";
    top = most(next, reach, 5.0 * c, 3.0 * b, a);
    if (!(top <= kMostX)) return "an iteration takes a singular value above 2";
  }
  return nullptr;
}

// Lists of up to this many tiles per pair in a phase go through all iterations in one launch.  (In it pairs drift apart, and then share fewer blocks
// in L2.  24 layers of width 1024, 60 tiles per pair, 6.69 ms so and 5.96 by a launch per phase; 12 tiles per pair 2.84 and 2.81; 40 odd matrices, 3
// per pair, 343 and 466 us; three small ones 95 and 122.)
constexpr uint32_t kTogether = 4;

cudaError_t launch_products(fr_muon_plan p, const fr_muon& h, MuonProduct q, const fr_muon_plan_s::Part& part, cudaStream_t s) {
  q.x_blocks = static_cast<uint32_t>(part.x_blocks);
  q.p_blocks = static_cast<uint32_t>(part.p_blocks);
  q.parts = part.deepest > part_steps(q.split);
  if (part.most_tiles <= kTogether * p->pairs) {
    q.tiles = part.d_tiles;
    q.n_tiles = part.ends[kPhases - 1];
    q.iterations = h.iterations;
    q.waits = 1;
    return launch_muon_product(q, p->maps, std::min(p->pairs, part.most_tiles), s);
  }
  for (q.first = 0; q.first < h.iterations; ++q.first) {
    q.iterations = q.first + 1;
    for (int phase = 0; phase < kPhases; ++phase) {
      const uint32_t begin = phase ? part.ends[phase - 1] : 0;
      q.tiles = part.d_tiles + begin;
      q.n_tiles = part.ends[phase] - begin;
      const cudaError_t e = launch_muon_product(q, p->maps, p->pairs, s);
      if (e != cudaSuccess) return e;
    }
  }
  return cudaSuccess;
}

// X through all iterations, in the plan's workspace.
fr_status iterate(fr_muon_plan p, const fr_muon& h, MuonParams& mp, cudaStream_t s) {
  MuonProduct q = {};
  q.work = p->d_work;
  q.clip = mp.clip;
  q.status = p->d_status;
  q.wait_clocks = p->wait_clocks;
  q.done = p->d_done;
  q.sums = p->d_sums;
  // Of first halves alone: an iterate keeps its second ones if the iterations after it raise small singular values, and a rounding among them, by
  // more than 4.
  double gain = 1.0;
  for (uint32_t i = h.iterations; i-- > 0;) {
    for (int j = 0; j < 3; ++j) q.coef[i][j] = static_cast<float>(h.coef[i][j]);
    gain *= std::max(1.0, std::fabs(h.coef[i][0]));
    q.low |= static_cast<uint32_t>(gain > 4.0) << i;
  }
  mp.low = q.low & 1;
  mp.last = h.iterations % 2;
  mp.one = h.products == FR_MUON_ONE;
  cudaError_t e = launch_muon_norm(mp, s);
  if (e == cudaSuccess) e = launch_muon_iterate(mp, s);
  if (e != cudaSuccess) return report_cuda("element kernel launch", e);
  for (uint32_t k = 0; k < 2 && e == cudaSuccess; ++k) {
    q.split = k && !mp.one;
    if (p->parts[k].most_tiles > 0) e = launch_products(p, h, q, p->parts[k], s);
  }
  return e == cudaSuccess ? FR_OK : report_cuda("product kernel launch", e);
}

MuonParams params(fr_muon_plan p) {
  MuonParams mp = {};
  mp.tensors = p->d_tensors;
  mp.units = p->d_units;
  mp.blocks = p->d_blocks;
  mp.n_units = p->n_units;
  mp.n_blocks = p->n_blocks;
  mp.partials = p->d_partials;
  mp.norms = p->d_norms;
  mp.work = p->d_work;
  mp.status = p->d_status;
  mp.done = p->d_done;
  return mp;
}

}  // namespace

extern "C" {

fr_status fr_muon_create(const fr_muon_tensor* tensors, uint64_t n_tensors, fr_muon_plan* out) {
  CallRange nvtx("fr_muon_create");
  const char* const me = "fr_muon_create";
  if (out == nullptr) return report_invalid(me, "out is null");
  *out = nullptr;
  if (n_tensors > 0 && tensors == nullptr) return report_invalid(me, "tensors is null");
  if (n_tensors >= (1ull << 32)) return report_invalid(me, "too many tensors");
  uint64_t filled = 0;  // elements with the sides filled up
  for (uint64_t t = 0; t < n_tensors; ++t) {
    bool misaligned;
    if (const char* what = check(tensors[t], misaligned)) return report_invalid(me, what);
    if (misaligned) {
      report_invalid(me, "a buffer is not aligned to its element size");
      return FR_ERR_ALIGNMENT;
    }
    if (tensors[t].rows == 0 || tensors[t].cols == 0) continue;
    const MuonDesc d = describe(tensors[t], t);
    filled += 1ull * d.row_blocks * d.col_blocks * kBlockRows * kBlockCols + square_blocks(d) * kBlockRows * kBlockCols;
    if (filled >= kMostElems) return report_invalid(me, "too many elements");
  }

  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda("cudaGetDevice", e);

  fr_muon_plan p = new (std::nothrow) fr_muon_plan_s;
  if (p == nullptr) return report_invalid(me, "out of host memory");
  p->device = dev;
  fr_status st;
  try {
    st = fill_muon(p, tensors, n_tensors);
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

fr_status fr_muon_info(fr_muon_plan p, uint64_t* n_tensors, uint64_t* n_elems, uint64_t* device_bytes) {
  if (p == nullptr) return report_invalid("fr_muon_info", "plan is null");
  if (n_tensors) *n_tensors = p->n_tensors;
  if (n_elems) *n_elems = p->n_elems;
  if (device_bytes) *device_bytes = p->device_bytes;
  return FR_OK;
}

void fr_muon_destroy(fr_muon_plan p) {
  CallRange nvtx("fr_muon_destroy");
  if (p == nullptr) return;
  DeviceGuard g(p->device);
  cudaDeviceSynchronize();
  cudaFree(p->d_memory);
  delete p;
}

fr_status fr_muon_step(fr_muon_plan p, const fr_muon* h, const fr_clip* clip_dev, void* stream) {
  CallRange nvtx("fr_muon_step");
  const char* const me = "fr_muon_step";
  if (p == nullptr || h == nullptr) return report_invalid(me, "plan or hyper is null");
  if (!p->params) return report_invalid(me, "a matrix of the plan has no weight, gradient or momentum");
  if (!(h->lr >= 0.0) || !std::isfinite(static_cast<float>(h->lr))) return report_invalid(me, "lr must be finite and not negative");
  if (!(h->weight_decay >= 0.0) || !std::isfinite(static_cast<float>(h->weight_decay)))
    return report_invalid(me, "weight_decay must be finite and not negative");
  if (!(h->beta >= 0.0 && h->beta < 1.0)) return report_invalid(me, "beta must be in [0, 1)");
  if (!std::isfinite(static_cast<float>(h->lr) * p->most_lr)) return report_invalid(me, "lr times a matrix's lr_scale must be finite in fp32");
  if (!std::isfinite(static_cast<float>(h->weight_decay) * p->most_decay))
    return report_invalid(me, "weight_decay times a matrix's decay_scale must be finite in fp32");
  if (h->nesterov > 1) return report_invalid(me, "nesterov must be 0 or 1");
  if (h->step == 0) return report_invalid(me, "step counts from 1");
  if (h->rounding > FR_ROUND_RANDOM) return report_invalid(me, "unknown rounding");
  if (const char* what = check_iterations(*h)) return report_invalid(me, what);
  if (clip_dev != nullptr && !on(clip_dev, 8)) return report_invalid(me, "clip_dev is not 8-byte aligned");
  if (p->n_blocks == 0) return FR_OK;
  DeviceGuard g(p->device);
  if (!g.ok) return report_cuda("select plan device", cudaGetLastError());
  MuonParams mp = params(p);
  mp.clip = clip_dev;
  mp.beta = static_cast<float>(h->beta);
  mp.beta_rest = static_cast<float>(1.0 - h->beta);
  mp.lr = static_cast<float>(h->lr);
  mp.decay = static_cast<float>(h->weight_decay);
  mp.momentum = 1;
  mp.nesterov = h->nesterov;
  mp.random = h->rounding == FR_ROUND_RANDOM;
  mp.key = mix64(mix64(h->seed) + h->step);
  const fr_status st = iterate(p, *h, mp, static_cast<cudaStream_t>(stream));
  if (st != FR_OK) return st;
  const cudaError_t e = launch_muon_apply(mp, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FR_OK : report_cuda("weight kernel launch", e);
}

fr_status fr_muon_sync_status(fr_muon_plan p, void* stream) {
  CallRange nvtx("fr_muon_sync_status");
  if (p == nullptr) return report_invalid("fr_muon_sync_status", "plan is null");
  if (p->n_blocks == 0) return FR_OK;
  DeviceGuard g(p->device);
  if (!g.ok) return report_cuda("select plan device", cudaGetLastError());
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint32_t status = 0;
  cudaError_t e = cudaMemcpyAsync(&status, p->d_status, sizeof status, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && status != 0) {
    e = cudaMemsetAsync(p->d_status, 0, sizeof status, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess) return FR_ERR_DEVICE_TIMEOUT;
  }
  return e == cudaSuccess ? FR_OK : report_cuda("read the plan's status", e);
}

fr_status fr_orthogonalize(fr_muon_plan p, const fr_muon* h, void* stream) {
  CallRange nvtx("fr_orthogonalize");
  const char* const me = "fr_orthogonalize";
  if (p == nullptr || h == nullptr) return report_invalid(me, "plan or hyper is null");
  if (!p->updates) return report_invalid(me, "a matrix of the plan has no gradient or update");
  if (const char* what = check_iterations(*h)) return report_invalid(me, what);
  if (p->n_blocks == 0) return FR_OK;
  DeviceGuard g(p->device);
  if (!g.ok) return report_cuda("select plan device", cudaGetLastError());
  MuonParams mp = params(p);
  const fr_status st = iterate(p, *h, mp, static_cast<cudaStream_t>(stream));
  if (st != FR_OK) return st;
  const cudaError_t e = launch_muon_update(mp, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? FR_OK : report_cuda("update kernel launch", e);
}

}  // extern "C"
