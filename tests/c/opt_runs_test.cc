// How many blocks in a row a warp of the 8-bit step takes (csrc/optim.h,
// csrc/optim_api.cu over fake_cuda.h): the lists that tests/test_gpu_optim_runs.py
// makes get the runs that it says, aligned and off the vectors' boundaries.
#include <cstdio>
#include <vector>

#include "fake_cuda.h"

#include "api.cu"
#include "optim_api.cu"

namespace {
std::vector<std::pair<StepClass, StepParams>> steps;
}

namespace frk {
cudaError_t launch_step(const StepClass& c, const StepParams& p, cudaStream_t) { steps.emplace_back(c, p); return cudaSuccess; }
cudaError_t launch_clip(const ClipParams&, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_convert(const ConvertParams&, cudaStream_t) { return cudaSuccess; }
}  // namespace frk

#define CHECK(x) do { if (!(x)) { std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)

int main() {
  constexpr uint64_t kRound = 7296;
  for (uint64_t run = 1; run <= 8; ++run) CHECK(step_blocks(true, run * kRound) == run && step_blocks(true, (run + 1) * kRound - 1) == run);
  CHECK(step_blocks(true, kRound - 1) == 1 && step_blocks(true, 100 * kRound) == 8);
  for (const uint64_t run : {3, 8})
    for (const uint64_t off : {0, 1}) {
      const uint64_t t = run * kRound * 256 * 101 / 1000;
      std::vector<fr_opt_tensor> list;
      uint64_t at = 1ull << 30;
      auto place = [&](uint64_t bytes) { void* p = reinterpret_cast<void*>(at); at += bytes / 512 * 512 + 1024; return p; };
      for (const uint64_t n : {4 * t + 3, uint64_t{255}, uint64_t{300}, 3 * t + 1, uint64_t{77}, uint64_t{256}, 2 * t - 1, t + 7}) {
        fr_opt_tensor x = {};
        x.n = n;
        x.weight = place(2 * n);
        x.grad = static_cast<uint8_t*>(place(2 * n)) + 2 * off;
        x.m = place(n), x.v = place(n);
        x.m_exp = static_cast<uint8_t*>(place(n / 256 + 1)), x.v_exp = static_cast<uint8_t*>(place(n / 256 + 1));
        x.weight_dtype = x.grad_dtype = FR_DT_BF16;
        x.state_dtype = FR_DT_BYTES;
        x.lr_scale = x.decay_scale = 1.0f;
        list.push_back(x);
      }
      fr_opt p = nullptr;
      CHECK(fr_opt_create(list.data(), list.size(), &p) == FR_OK);
      const fr_adamw h = {1e-3, 0.9, 0.95, 1e-8, 0.1, 1, 0, FR_ROUND_RANDOM, 0};
      steps.clear();
      CHECK(fr_adamw_step(p, &h, nullptr, nullptr) == FR_OK && steps.size() == 1 + off);
      for (auto& s : steps) CHECK(s.first.odd ? s.second.work.per_warp == run : off ? s.second.work.per_warp == 1 : s.second.work.per_warp == run);
      fr_opt_destroy(p);
    }
  std::printf("opt_runs ok\n");
  return 0;
}
