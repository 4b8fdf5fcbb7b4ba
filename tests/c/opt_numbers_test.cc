// Numbers of a step that fp32 holds one by one and not as the products that the
// kernels take (csrc/optim_api.cu over fake_cuda.h): refused, nothing launched.
#include <cmath>
#include <cstdio>
#include <vector>

#include "fake_cuda.h"

#include "api.cu"
#include "optim_api.cu"

namespace {
int launched = 0;
}

namespace frk {
cudaError_t launch_step(const StepClass&, const StepParams&, cudaStream_t) { ++launched; return cudaSuccess; }
cudaError_t launch_clip(const ClipParams&, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_convert(const ConvertParams&, cudaStream_t) { return cudaSuccess; }
}  // namespace frk

namespace {

#define CHECK(x) do { if (!(x)) { std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)

fr_opt_tensor tensor(uint64_t n, uint64_t at, float lr_scale, float decay_scale) {
  fr_opt_tensor x = {};
  x.n = n;
  x.weight = reinterpret_cast<void*>(at);
  x.grad = reinterpret_cast<void*>(at + (1 << 20));
  x.m = reinterpret_cast<void*>(at + (2 << 20));
  x.v = reinterpret_cast<void*>(at + (3 << 20));
  x.weight_dtype = x.grad_dtype = x.state_dtype = FR_DT_F32;
  x.lr_scale = lr_scale;
  x.decay_scale = decay_scale;
  return x;
}

// The status of a step of these tensors; it launches if and only if that is FR_OK.
fr_status step(const std::vector<fr_opt_tensor>& list, double lr, double decay) {
  fr_opt p = nullptr;
  CHECK(fr_opt_create(list.data(), list.size(), &p) == FR_OK);
  const fr_adamw h = {lr, 0.9, 0.95, 1e-8, decay, 1, 0, FR_ROUND_NEAREST, 0};
  launched = 0;
  const fr_status st = fr_adamw_step(p, &h, nullptr, nullptr);
  CHECK((st == FR_OK) == (launched > 0));
  fr_opt_destroy(p);
  return st;
}

}  // namespace

int main() {
  const uint64_t a = 1 << 30, b = 2ull << 30, c = 3ull << 30;
  const float one = 1.0f, big = 0x1p100f, most = 3.4028234663852886e38f;
  CHECK(step({tensor(1000, a, one, one)}, 1e-3, 0.1) == FR_OK);
  // products at the end of fp32's range, and past it
  CHECK(step({tensor(1000, a, big, one)}, 0x1p27, 0.1) == FR_OK);
  CHECK(step({tensor(1000, a, big, one)}, 0x1p28, 0.1) == FR_ERR_INVALID_ARG);
  CHECK(step({tensor(1000, a, one, big)}, 1e-3, 0x1p27) == FR_OK);
  CHECK(step({tensor(1000, a, one, big)}, 1e-3, 0x1p28) == FR_ERR_INVALID_ARG);
  CHECK(step({tensor(1000, a, most, most)}, 1.0, 1.0) == FR_OK);
  CHECK(step({tensor(1000, a, most, one)}, 1.0 + 0x1p-20, 1.0) == FR_ERR_INVALID_ARG);
  // of either sign, in any tensor that has elements
  CHECK(step({tensor(1000, a, -big, one)}, 0x1p28, 0.1) == FR_ERR_INVALID_ARG);
  CHECK(step({tensor(1000, a, one, -big)}, 1e-3, 0x1p28) == FR_ERR_INVALID_ARG);
  CHECK(step({tensor(1000, a, one, one), tensor(7, b, -big, one), tensor(500, c, 0.5f, one)}, 0x1p28, 0.1) == FR_ERR_INVALID_ARG);
  CHECK(step({tensor(1000, a, one, one), tensor(7, b, one, big), tensor(500, c, one, 0.0f)}, 1e-3, 0x1p28) == FR_ERR_INVALID_ARG);
  CHECK(step({tensor(1000, a, one, one), tensor(0, b, big, big)}, 0x1p28, 0x1p28) == FR_OK);
  // no factor, no product
  CHECK(step({tensor(1000, a, 0.0f, 0.0f)}, 3e38, 3e38) == FR_OK);
  std::printf("opt_numbers ok\n");
  return 0;
}
