// The embedding's planner and refusals (csrc/embed_api.cu, csrc/embed.h) without a GPU.
#include <cstdio>
#include <random>

#include "fake_cuda.h"

#include "api.cu"
#include "embed_api.cu"

namespace {
std::vector<LookupParams> lookups;
std::vector<SortParams> sorts;
std::vector<SumParams> sums;
}  // namespace

namespace frk {
cudaError_t configure_sort() { return cudaSuccess; }
cudaError_t configure_sum() { return cudaSuccess; }
cudaError_t launch_lookup(const LookupParams& p, cudaStream_t) { lookups.push_back(p); return cudaSuccess; }
cudaError_t launch_sort(SortParams p, const SortPlan& plan, int* last, cudaStream_t) { sorts.push_back(p); *last = (plan.passes - 1) % 2; return cudaSuccess; }
cudaError_t launch_sum(const SumParams& p, cudaStream_t) { sums.push_back(p); return cudaSuccess; }
}  // namespace frk

namespace {
#define CHECK(x) do { if (!(x)) { std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)
void* place(uint64_t at) { return reinterpret_cast<void*>(at); }
}  // namespace

int main() {
  std::mt19937_64 rng(4);
  auto below = [&](uint64_t n) { return rng() % n; };
  for (int round = 0; round < 3000; ++round) {
    const uint64_t rows = below(3) ? below(200000) + 1 : below(20), dim = below(3) ? 8 * (below(600) + 1) : below(5000), most = below(2) ? below(300000) : below(50);
    fr_embed p = nullptr;
    CHECK(fr_embed_create(rows, dim, most, 7, &p) == FR_OK);
    uint64_t r, d, m, bytes;
    CHECK(fr_embed_info(p, &r, &d, &m, &bytes) == FR_OK && r == rows && d == dim && m == most && bytes <= 16 * most + (40 << 20));
    const uint64_t n = below(4) ? (most ? below(most + 1) : 0) : most;
    const uint32_t out_type = below(2) ? FR_DT_BF16 : FR_DT_F32, grad_type = below(2) ? FR_DT_BF16 : FR_DT_F32, accumulate = below(2);
    const uint64_t out = (1 << 20) + type_bytes(out_type) * below(9), grad = (1 << 21) + type_bytes(grad_type) * below(9);
    sorts.clear(), sums.clear(), lookups.clear();
    CHECK(fr_embed_grad(p, place(out), out_type, place(1 << 22), 4, n, 0.5f, place(grad), grad_type, accumulate, nullptr) == FR_OK);
    const bool runs = rows && dim && (n || !accumulate);
    CHECK(sorts.size() == (runs ? 1u : 0u) && sums.size() == (runs && n ? 1u : 0u));
    const bool fill = !accumulate && n < rows;
    if (runs) CHECK(sorts[0].fill_bytes == (fill ? rows * dim * type_bytes(grad_type) : 0) && (!fill || sorts[0].fill == place(grad)));
    if (runs && n) {
      const SumParams& q = sums[0];
      const int v = vector_of(q.v);
      CHECK(q.ranges == ranges_of(n, dim, accumulate));  // not of the addresses
      CHECK(dim % v == 0 && out % std::min<uint64_t>(16, v * type_bytes(out_type)) == 0 && grad % std::min<uint64_t>(16, v * type_bytes(grad_type)) == 0);
      CHECK(static_cast<uint64_t>(q.tiles) * tile_width(q.v) >= dim && static_cast<uint64_t>(q.tiles - 1) * tile_width(q.v) < dim);
      CHECK(q.ranges % kSumWarps == 0 && q.ranges >= kSumWarps && q.ranges <= p->ranges);
      CHECK(q.ctas == q.ranges / kSumWarps * q.tiles && (q.zero_ctas == 0) == (accumulate || fill));
      if (q.zero_ctas)
        CHECK(static_cast<uint64_t>(q.zero_ctas) * kSumWarps * q.rows_per_zero_warp >= rows && q.rows_per_zero_warp >= 1 && q.rows_per_zero_warp <= 32);
      CHECK(q.sorted == p->d_sorted[(p->sort.passes - 1) % 2] && q.sorted != nullptr);
      CHECK(sorts[0].counts != nullptr || n <= kClusterTokens);
    }
    CHECK(fr_embed_lookup(p, place(grad), grad_type, place(1 << 22), 8, n, 2.0f, place(out), out_type, nullptr) == FR_OK);
    CHECK(lookups.size() == (n && dim ? 1u : 0u));
    fr_embed_destroy(p);
  }
  // digits hold every row
  for (uint64_t rows : {1ull, 2ull, 3ull, 256ull, 512ull, 513ull, 50257ull, 262144ull, 262145ull, (1ull << 31) - 1}) {
    const SortPlan s = sort_plan(rows);
    CHECK(s.bits >= 1 && s.bits <= kMostDigit && (1ull << (s.bits * s.passes)) >= rows);
  }

  // refusals launch nothing
  lookups.clear(), sorts.clear(), sums.clear();
  fr_embed p = nullptr, none = nullptr;
  CHECK(fr_embed_create(1ull << 31, 8, 8, 0, &none) == FR_ERR_INVALID_ARG && fr_embed_create(8, 8, 1ull << 31, 0, &none) == FR_ERR_INVALID_ARG);
  CHECK(fr_embed_create(8, (1ull << 20) + 1, 8, 0, &none) == FR_ERR_INVALID_ARG && fr_embed_create(8, 8, 8, (1ull << 62) + 1, &none) == FR_ERR_INVALID_ARG);
  CHECK(fr_embed_create((1ull << 31) - 1, 1 << 20, 8, 0, &none) == FR_ERR_INVALID_ARG && none == nullptr);
  CHECK(fr_embed_create(8, 8, 8, 0, nullptr) == FR_ERR_INVALID_ARG && fr_embed_info(nullptr, nullptr, nullptr, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_embed_create(100, 16, 50, 0, &p) == FR_OK);
  void *const t = place(1 << 20), *const o = place(1 << 21), *const k = place(1 << 22);
  auto both = [&](fr_status want, const void* table, uint32_t table_type, const void* tokens, uint32_t token_bytes, uint64_t n, float scale, void* out,
                  uint32_t out_type) {
    return fr_embed_lookup(p, table, table_type, tokens, token_bytes, n, scale, out, out_type, nullptr) == want &&
           fr_embed_grad(p, out, out_type, tokens, token_bytes, n, scale, const_cast<void*>(table), table_type, 0, nullptr) == want;
  };
  CHECK(both(FR_ERR_INVALID_ARG, t, FR_DT_BYTES, k, 4, 5, 1.0f, o, FR_DT_F32) && both(FR_ERR_INVALID_ARG, t, FR_DT_F32, k, 4, 5, 1.0f, o, 7));
  CHECK(both(FR_ERR_INVALID_ARG, t, FR_DT_F32, k, 2, 5, 1.0f, o, FR_DT_F32) && both(FR_ERR_INVALID_ARG, t, FR_DT_F32, k, 4, 51, 1.0f, o, FR_DT_F32));
  CHECK(both(FR_ERR_INVALID_ARG, t, FR_DT_F32, k, 4, 5, INFINITY, o, FR_DT_F32) && both(FR_ERR_INVALID_ARG, t, FR_DT_F32, k, 4, 5, NAN, o, FR_DT_F32));
  CHECK(both(FR_ERR_INVALID_ARG, nullptr, FR_DT_F32, k, 4, 5, 1.0f, o, FR_DT_F32) && both(FR_ERR_INVALID_ARG, t, FR_DT_F32, nullptr, 4, 5, 1.0f, o, FR_DT_F32));
  CHECK(both(FR_ERR_INVALID_ARG, t, FR_DT_F32, k, 4, 5, 1.0f, nullptr, FR_DT_F32));
  CHECK(both(FR_ERR_ALIGNMENT, place(2), FR_DT_F32, k, 4, 5, 1.0f, o, FR_DT_F32) && both(FR_ERR_ALIGNMENT, t, FR_DT_F32, k, 4, 5, 1.0f, place(1), FR_DT_BF16));
  CHECK(both(FR_ERR_ALIGNMENT, t, FR_DT_F32, place(4), 8, 5, 1.0f, o, FR_DT_F32));
  CHECK(fr_embed_grad(p, o, FR_DT_F32, k, 4, 5, 1.0f, t, FR_DT_F32, 2, nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_embed_lookup(nullptr, t, FR_DT_F32, k, 4, 5, 1.0f, o, FR_DT_F32, nullptr) == FR_ERR_INVALID_ARG);
  CHECK(lookups.empty() && sorts.empty() && sums.empty());
  fr_embed_destroy(p);
  fr_embed_destroy(nullptr);
  std::printf("embed_plan ok\n");
  return 0;
}
