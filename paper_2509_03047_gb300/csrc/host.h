// host.h -- what the C ABI's translation units share on the host: a profiler's
// range, the plan's device, a plan's device memory.
#pragma once

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <vector>

#include "layout.h"

namespace frk {

// A named NVTX range around each public call, so a profiler's timeline shows
// which call issued which kernels.  NVTX is header-only: with no profiler
// attached, push and pop return at once.
struct CallRange {
  explicit CallRange(const char* name) { nvtxRangePushA(name); }
  ~CallRange() { nvtxRangePop(); }
  CallRange(const CallRange&) = delete;
  CallRange& operator=(const CallRange&) = delete;
};

// Runs the calls on the plan's device and puts the caller's device back.
struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) {
      ok = false;
      return;
    }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
  }
};

// A plan's device memory: tables gathered on the host, then scratch, as one
// allocation and one copy.  (An allocation and a copy for each table, 40 of both
// for a batched plan, were half of the 2.6 ms that a plan over 8 tensors in 8
// batches took; it takes 0.6 ms now.)
class PlanMemory {
 public:
  template <class T>
  void table(T** at, const std::vector<T>& src) {
    if (src.empty()) return;
    const uint64_t off = align_up(tables_.size(), kAlign);
    tables_.resize(off + src.size() * sizeof(T));
    std::memcpy(tables_.data() + off, src.data(), src.size() * sizeof(T));
    places_.push_back({reinterpret_cast<void**>(at), off, false});
  }
  template <class T>
  void scratch(T** at, uint64_t count) {
    if (count == 0) return;
    places_.push_back({reinterpret_cast<void**>(at), scratch_, true});
    scratch_ = align_up(scratch_ + count * sizeof(T), kAlign);
  }
  uint64_t bytes() const { return std::max<uint64_t>(align_up(tables_.size(), kAlign) + scratch_, kAlign); }
  // Allocates, copies the tables and sets every pointer.  The wait is for the
  // copy's last part: one from pageable memory may return while that is still
  // on its way, on the legacy stream, and a call on a non-blocking stream is
  // not ordered after it.
  cudaError_t commit(void** memory) {
    const uint64_t first = align_up(tables_.size(), kAlign);
    cudaError_t e = cudaMalloc(memory, bytes());
    if (e != cudaSuccess) return e;
    if (!tables_.empty()) e = cudaMemcpy(*memory, tables_.data(), tables_.size(), cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);
    for (const Place& q : places_) *q.at = static_cast<uint8_t*>(*memory) + (q.scratch ? first : 0) + q.off;
    return e;
  }

 private:
  static constexpr uint64_t kAlign = 256;
  struct Place {
    void** at;
    uint64_t off;
    bool scratch;
  };
  std::vector<uint8_t> tables_;
  std::vector<Place> places_;
  uint64_t scratch_ = 0;
};

}  // namespace frk
