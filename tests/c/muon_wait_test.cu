// muon_wait_test.cu -- a wait inside a product that never ends (a tile that asks for a
// count which nothing reaches) is given up after the plan's limit, here a few
// milliseconds: the step leaves weights, masters and updates as they were and its
// momenta advanced; later calls leave every byte; the status is told once; the next
// step after that is one like any other.  Linked with the library's objects but
// muon_api.o.  Exits 0 and prints "muon_wait ok".
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "muon_api.cu"

#define EXPECT(c)                                                    \
  do {                                                               \
    if (!(c)) {                                                      \
      std::fprintf(stderr, "%s:%d check failed: %s\n", __FILE__, __LINE__, #c); \
      std::exit(1);                                                  \
    }                                                                \
  } while (0)
#define CUDA(c) EXPECT((c) == cudaSuccess)

namespace {

uint32_t g_seed = 1;
uint32_t next_bits() { return (g_seed = g_seed * 1664525u + 1013904223u) >> 8; }

struct Sides {
  uint64_t rows, cols;
};

// A list's buffers, one after the other in one allocation: weights (fp32), gradients, momenta, updates of each matrix.
struct List {
  std::vector<Sides> sides;
  uint64_t n = 0;
  float* dev = nullptr;
  fr_muon_plan plan = nullptr;
  explicit List(const std::vector<Sides>& s) : sides(s) {
    for (const Sides& x : s) n += x.rows * x.cols;
    CUDA(cudaMalloc(reinterpret_cast<void**>(&dev), 4 * n * sizeof(float)));
    fill();
    std::vector<fr_muon_tensor> t;
    uint64_t at = 0;
    for (const Sides& x : s) {
      fr_muon_tensor y = {};
      y.weight = dev + at, y.grad = dev + n + at, y.momentum = dev + 2 * n + at, y.update = dev + 3 * n + at;
      y.rows = x.rows, y.cols = x.cols;
      y.weight_dtype = y.grad_dtype = y.update_dtype = FR_DT_F32;
      y.lr_scale = y.decay_scale = y.update_scale = 1.0f;
      t.push_back(y);
      at += x.rows * x.cols;
    }
    EXPECT(fr_muon_create(t.data(), t.size(), &plan) == FR_OK);
  }
  ~List() {
    fr_muon_destroy(plan);
    cudaFree(dev);
  }
  void fill() {
    g_seed = 1;
    std::vector<float> host(4 * n);
    for (float& x : host) x = static_cast<float>(static_cast<int>(next_bits() % 2001) - 1000) * 1e-3f;
    CUDA(cudaMemcpy(dev, host.data(), host.size() * sizeof(float), cudaMemcpyHostToDevice));
  }
  // Part 0: weights, 1: gradients, 2: momenta, 3: updates.
  std::vector<float> get(int part) const {
    std::vector<float> host(n);
    CUDA(cudaMemcpy(host.data(), dev + part * n, n * sizeof(float), cudaMemcpyDeviceToHost));
    return host;
  }
};
bool same(const std::vector<float>& a, const std::vector<float>& b) { return std::memcmp(a.data(), b.data(), a.size() * sizeof(float)) == 0; }

fr_muon numbers() {
  fr_muon h = {};
  h.lr = 1e-2, h.beta = 0.9, h.weight_decay = 0.1, h.step = 1, h.iterations = 5, h.nesterov = 1;
  for (auto& c : h.coef) c[0] = 3.4445, c[1] = -4.7750, c[2] = 2.0315;
  return h;
}

// Of a phase's tiles one asks for more than its counter reaches.
void check(const std::vector<Sides>& sides, int phase, uint32_t index) {
  const fr_muon h = numbers();
  List good(sides), bad(sides);
  EXPECT(fr_muon_step(good.plan, &h, nullptr, nullptr) == FR_OK && fr_muon_sync_status(good.plan, nullptr) == FR_OK);

  auto& part = bad.plan->parts[1];
  const uint32_t tile = part.ends[phase - 1] + index;
  EXPECT(part.most_tiles <= kTogether * bad.plan->pairs && tile < part.ends[phase]);
  MuonTile record;
  CUDA(cudaMemcpy(&record, part.d_tiles + tile, sizeof record, cudaMemcpyDeviceToHost));
  MuonTile never = record;
  never.count = 1u << 24;
  CUDA(cudaMemcpy(part.d_tiles + tile, &never, sizeof never, cudaMemcpyHostToDevice));
  bad.plan->wait_clocks = 20 << 20;
  const std::vector<float> weights = bad.get(0), updates = bad.get(3);

  // the step that gives up
  EXPECT(fr_muon_step(bad.plan, &h, nullptr, nullptr) == FR_OK);
  CUDA(cudaDeviceSynchronize());
  EXPECT(same(bad.get(0), weights) && same(bad.get(2), good.get(2)) && !same(good.get(0), weights));
  // those after it, also with the tile as it should be
  CUDA(cudaMemcpy(part.d_tiles + tile, &record, sizeof record, cudaMemcpyHostToDevice));
  for (int k = 0; k < 2; ++k) {
    EXPECT(fr_muon_step(bad.plan, &h, nullptr, nullptr) == FR_OK && fr_orthogonalize(bad.plan, &h, nullptr) == FR_OK);
    CUDA(cudaDeviceSynchronize());
    EXPECT(same(bad.get(0), weights) && same(bad.get(2), good.get(2)) && same(bad.get(3), updates));
  }
  EXPECT(fr_muon_sync_status(bad.plan, nullptr) == FR_ERR_DEVICE_TIMEOUT && fr_muon_sync_status(bad.plan, nullptr) == FR_OK);
  // restored, a step is a step
  bad.fill();
  EXPECT(fr_muon_step(bad.plan, &h, nullptr, nullptr) == FR_OK && fr_muon_sync_status(bad.plan, nullptr) == FR_OK);
  for (int k : {0, 2}) EXPECT(same(bad.get(k), good.get(k)));
}

}  // namespace

int main() {
  check({{64, 64}}, kPolynomial, 0);
  check({{64, 64}}, kNext, 0);
  const std::vector<Sides> several = {{300, 520}, {64, 64}, {200, 130}, {700, 700}, {90, 40}};
  check(several, kPolynomial, 3);
  check(several, kNext, 7);
  std::printf("muon_wait ok\n");
  return 0;
}
