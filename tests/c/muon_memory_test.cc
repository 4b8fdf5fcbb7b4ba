// The device memory of a plan of the orthogonalised update (csrc/muon_api.cu) without a
// GPU: a product whose contraction is longer than a part has a place for the sums of
// its parts, for each CTA of the launch, within the plan's allocation and beside
// everything else; one without has none; what fr_muon_info gives is the whole allocation.
#include <cstdio>
#include <random>

#include "fake_cuda.h"

#include "api.cu"
#include "muon_api.cu"

namespace {
struct Launch {
  MuonProduct p;
  uint32_t pairs;
};
std::vector<Launch> products;
uint32_t resident = 76;

CUresult fake_encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                     CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
  return CUDA_SUCCESS;
}
}  // namespace

extern "C" cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** f, unsigned, unsigned long long, cudaDriverEntryPointQueryResult* r) {
  *f = reinterpret_cast<void*>(fake_encode);
  *r = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}

namespace frk {
cudaError_t launch_muon_norm(const MuonParams&, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_muon_iterate(const MuonParams&, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_muon_apply(const MuonParams&, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_muon_update(const MuonParams&, cudaStream_t) { return cudaSuccess; }
cudaError_t configure_muon_product() { return cudaSuccess; }
cudaError_t muon_pairs(uint32_t* n) { *n = resident; return cudaSuccess; }
cudaError_t launch_muon_product(const MuonProduct& p, const MuonMaps&, uint32_t pairs, cudaStream_t) { products.push_back({p, pairs}); return cudaSuccess; }
}  // namespace frk

namespace {

#define CHECK(x) do { if (!(x)) { std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)

fr_muon_tensor matrix(uint64_t rows, uint64_t cols, bool fp32) {
  fr_muon_tensor x = {};
  x.rows = rows, x.cols = cols;
  x.grad = reinterpret_cast<void*>(1 << 21);
  x.update = reinterpret_cast<void*>(1 << 23);
  x.grad_dtype = FR_DT_BF16;
  x.update_dtype = fp32 ? FR_DT_F32 : FR_DT_BF16;
  x.lr_scale = x.decay_scale = x.update_scale = 1.0f;
  return x;
}

}  // namespace

int main() {
  std::mt19937_64 rng(5);
  auto below = [&](uint64_t n) { return rng() % n; };
  fr_muon h = {};
  h.iterations = 5;
  for (auto& c : h.coef) c[0] = 3.4445, c[1] = -4.7750, c[2] = 2.0315;
  uint32_t seen[2][2] = {};
  for (int round = 0; round < 120; ++round) {
    std::vector<fr_muon_tensor> list;
    const uint64_t n = below(4) + 1, longest = below(2) ? 9000 : 70000;
    for (uint64_t t = 0; t < n; ++t) {
      const uint64_t a = below(300) + 1, b = below(longest) + 1;
      list.push_back(below(2) ? matrix(a, b, below(2)) : matrix(b, a, below(2)));
    }
    resident = below(2) ? 76 : 3;
    fr_muon_plan p = nullptr;
    CHECK(fr_muon_create(list.data(), n, &p) == FR_OK);
    fake::finish_all();
    uint64_t bytes;
    CHECK(fr_muon_info(p, nullptr, nullptr, &bytes) == FR_OK);
    const uint8_t* const memory = static_cast<const uint8_t*>(p->d_memory);
    const uint64_t work = (3 * p->parts[0].x_blocks + 2 * p->parts[0].p_blocks + 4 * p->parts[1].x_blocks + 4 * p->parts[1].p_blocks) * kMuonBlockBytes;
    CHECK(p->d_work >= memory && p->d_work + work <= memory + bytes);
    CHECK(reinterpret_cast<uint8_t*>(p->d_partials + p->n_units) <= memory + bytes && reinterpret_cast<uint8_t*>(p->d_blocks + p->n_blocks) <= memory + bytes);
    for (uint32_t how : {FR_MUON_BY_TYPE, FR_MUON_ONE}) {
      products.clear();
      h.products = how;
      CHECK(fr_orthogonalize(p, &h, nullptr) == FR_OK);
      for (const Launch& l : products) {
        uint32_t deepest = 0;
        for (uint32_t i = 0; i < l.p.n_tiles; ++i) deepest = std::max(deepest, l.p.tiles[i].depth);
        const bool parts = l.p.parts;
        CHECK(l.p.parts == (deepest > part_steps(l.p.split)) || !l.p.waits);
        CHECK(parts || deepest <= part_steps(l.p.split));
        ++seen[l.p.split][parts];
        if (!parts) continue;
        CHECK(l.p.sums != nullptr && l.p.sums >= l.p.work + work && l.p.sums + 2ull * l.pairs * kPartBytes <= memory + bytes);
        CHECK(reinterpret_cast<uintptr_t>(l.p.sums) % 16 == reinterpret_cast<uintptr_t>(memory) % 16);
        // every byte of them is the plan's (the host's allocation takes the write)
        std::memset(l.p.sums, 0, 2ull * l.pairs * kPartBytes);
        CHECK(l.pairs <= p->pairs);
      }
    }
    bool longer = false;
    for (const fr_muon_tensor& x : list) longer |= (std::max(x.rows, x.cols) + 127) / 128 * 2 > part_steps(x.update_dtype == FR_DT_F32);
    CHECK((p->d_sums != nullptr) == longer);
    fr_muon_destroy(p);
  }
  // a matrix with bf16 outputs has products of both halves if its flag asks for them, and not with FR_MUON_ONE; other flags are refused
  resident = 76;
  for (uint32_t flags : {0u, 1u, FR_MUON_BOTH_HALVES, FR_MUON_BOTH_HALVES | 1, 4u, 0x80000000u}) {
    fr_muon_tensor x = matrix(100, 200, false);
    x.flags = flags;
    fr_muon_plan p = nullptr;
    const bool known = (flags & ~FR_MUON_BOTH_HALVES) == 0;
    CHECK(fr_muon_create(&x, 1, &p) == (known ? FR_OK : FR_ERR_INVALID_ARG) && (p != nullptr) == known);
    if (!known) continue;
    fake::finish_all();
    for (uint32_t how : {FR_MUON_BY_TYPE, FR_MUON_ONE}) {
      products.clear();
      h.products = how;
      CHECK(fr_orthogonalize(p, &h, nullptr) == FR_OK && products.size() == 1 && products[0].p.split == (flags != 0 && how == FR_MUON_BY_TYPE));
    }
    fr_muon_destroy(p);
  }
  for (int split = 0; split < 2; ++split)
    for (int parts = 0; parts < 2; ++parts) CHECK(seen[split][parts] > 5);
  std::printf("muon_memory ok\n");
  return 0;
}
