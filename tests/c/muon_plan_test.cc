// The orthogonalised update's planner (csrc/muon_api.cu, csrc/muon_tiles.h) without a
// GPU: over random lists of matrices, every tile's record is walked as the product
// kernel walks it, and must address, step by step, the blocks that the product needs,
// of those that exist; every block of a result comes up once; what a tile waits for is
// what counts; refusals launch nothing.
#include <cstdio>
#include <map>
#include <random>
#include <set>

#include "fake_cuda.h"

#include "api.cu"
#include "muon_api.cu"

namespace {
struct Launch {
  MuonProduct p;
  uint32_t pairs;
};
std::vector<Launch> products;
std::vector<MuonParams> norms, iterates, applies, updates;
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
cudaError_t launch_muon_norm(const MuonParams& p, cudaStream_t) { norms.push_back(p); return cudaSuccess; }
cudaError_t launch_muon_iterate(const MuonParams& p, cudaStream_t) { iterates.push_back(p); return cudaSuccess; }
cudaError_t launch_muon_apply(const MuonParams& p, cudaStream_t) { applies.push_back(p); return cudaSuccess; }
cudaError_t launch_muon_update(const MuonParams& p, cudaStream_t) { updates.push_back(p); return cudaSuccess; }
cudaError_t configure_muon_product() { return cudaSuccess; }
cudaError_t muon_pairs(uint32_t* n) { *n = resident; return cudaSuccess; }
cudaError_t launch_muon_product(const MuonProduct& p, const MuonMaps&, uint32_t pairs, cudaStream_t) { products.push_back({p, pairs}); return cudaSuccess; }
}  // namespace frk

namespace {

#define CHECK(x) do { if (!(x)) { std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); std::exit(1); } } while (0)

void clear() { products.clear(), norms.clear(), iterates.clear(), applies.clear(), updates.clear(); }

// A matrix's squares hold the tiles of 256 x 256 on and below the diagonal.
bool exists(uint32_t block_row, uint32_t block_col) { return block_row / 2 >= block_col / 4; }

// Step k of a factor as the kernel goes: the block and, by columns, which half of its rows.
struct At {
  uint32_t block, half;
  bool by_columns;
};
std::vector<At> walk(uint32_t first, uint32_t half, uint32_t next, bool by_columns, uint32_t at_switch, uint32_t after, uint32_t square, uint32_t depth) {
  std::vector<At> r;
  uint32_t block = first, flip = by_columns;
  for (uint32_t k = 0; k < depth; ++k) {
    if (k == at_switch) block = after, half = 0, next = square, flip = 1;
    r.push_back({block, half, flip != 0});
    block += (half & flip) || !flip ? next : 0;
    half ^= flip;
  }
  return r;
}

// The factor's 128 (a narrow tile's second: 64) rows from block b on, step k, must be this.
void check_factor(const std::vector<At>& got, uint32_t base, uint32_t col_blocks, bool columns_first, bool square, uint32_t b, uint32_t part, bool narrow) {
  for (uint32_t k = 0; k < got.size(); ++k) {
    const At& g = got[k];
    const uint32_t block_row = (g.block - base) / col_blocks, block_col = (g.block - base) % col_blocks;
    CHECK(g.block >= base);
    if (square) CHECK(exists(block_row, block_col));
    if (!g.by_columns) {
      CHECK(!columns_first || square);
      CHECK(block_row == b && block_col == k && g.half == (narrow ? part : 0));
    } else {
      CHECK(columns_first || square);
      CHECK(block_row == k / 2 && g.half == k % 2 && block_col == 2 * b + (narrow ? part : 0));
    }
  }
}

void check_tile(const MuonTile& t, const MuonDesc& d) {
  const uint32_t x = static_cast<uint32_t>(d.x[0] / kMuonBlockBytes), s = static_cast<uint32_t>(d.s / kMuonBlockBytes), q = static_cast<uint32_t>(d.p / kMuonBlockBytes);
  const uint32_t side = d.side_blocks, phase = t.phase;
  const bool narrow = t.flags & kNarrow, second = t.flags & kSecond;
  const uint32_t rows = phase == kNext ? d.row_blocks : side, cols = phase == kNext ? d.col_blocks / 2 : side;
  CHECK(t.row < rows && t.col < cols && second == (t.row + 1u < rows));
  CHECK(narrow || (t.col % 2 == 0 && t.col + 1u < cols));
  CHECK(t.row % 2 == 0);
  CHECK(t.depth == (phase == kGram ? (d.tall ? 2 * d.row_blocks : d.col_blocks) : 2 * side));
  const bool a_x = phase == kGram || (phase == kNext && d.tall), b_x = phase == kGram || (phase == kNext && !d.tall);
  CHECK(a_x == ((t.flags & kAIterate) != 0) && b_x == ((t.flags & kBIterate) != 0));
  const bool a_cols = phase == kGram && d.tall, b_cols = phase == kGram ? d.tall != 0 : phase == kNext && !d.tall;
  CHECK(a_cols == ((t.flags & kAColumns) != 0) && b_cols == ((t.flags & kBColumns) != 0));
  const uint32_t sq = phase == kPolynomial ? s : q;
  for (uint32_t rank = 0; rank < 2; ++rank) {
    const uint32_t row = t.row + (second ? rank : 0);
    check_factor(walk(t.a[rank], 0, t.a_next, a_cols, t.a_switch, t.a_after[rank], t.square, t.depth), a_x ? x : sq, a_x ? d.col_blocks : 2 * side,
                 a_cols, !a_x, row, 0, false);
    const uint32_t half = narrow && !b_cols ? rank : 0;
    check_factor(walk(t.b[rank], half, t.b_next, b_cols, t.b_switch, t.b_after[rank], t.square, t.depth), b_x ? x : sq,
                 b_x ? d.col_blocks : 2 * side, b_cols, !b_x, narrow ? t.col : t.col + rank, rank, narrow);
  }
  const bool same = t.flags & kSame;
  CHECK(same == (phase != kNext && t.row == t.col && !narrow));
  if (same)
    for (uint32_t rank = 0; rank < 2; ++rank)
      CHECK(t.a[rank] == t.b[rank] && t.a_after[rank] == t.b_after[rank] && t.a_switch == t.b_switch && t.a_next == t.b_next && a_cols == b_cols && second);
  CHECK(t.across == 2 * cols && t.out == (phase == kGram ? s : phase == kPolynomial ? q : x) + t.row * t.across + 2 * t.col);
}

fr_muon usual() {
  fr_muon h = {};
  h.lr = 1e-3, h.beta = 0.95, h.weight_decay = 0.1, h.step = 1, h.iterations = 5, h.nesterov = 1;
  for (auto& c : h.coef) c[0] = 3.4445, c[1] = -4.7750, c[2] = 2.0315;
  return h;
}

fr_muon_tensor matrix(uint64_t rows, uint64_t cols, bool fp32) {
  fr_muon_tensor x = {};
  x.rows = rows, x.cols = cols;
  x.weight = reinterpret_cast<void*>(1 << 20);
  x.grad = reinterpret_cast<void*>(1 << 21);
  x.momentum = reinterpret_cast<float*>(1 << 22);
  x.update = reinterpret_cast<void*>(1 << 23);
  x.weight_dtype = x.grad_dtype = x.update_dtype = FR_DT_BF16;
  if (fp32) x.master = reinterpret_cast<float*>(1 << 24);
  x.lr_scale = x.decay_scale = x.update_scale = 1.0f;
  return x;
}

}  // namespace

int main() {
  std::mt19937_64 rng(3);
  auto below = [&](uint64_t n) { return rng() % n; };
  const fr_muon h = usual();
  for (int round = 0; round < 150; ++round) {
    std::vector<fr_muon_tensor> list;
    const uint64_t n = below(9), most = below(2) ? 400 : 1500;
    for (uint64_t t = 0; t < n; ++t) list.push_back(matrix(below(8) ? below(most) + 1 : 0, below(8) ? below(most) + 1 : 1, below(2)));
    resident = below(2) ? 76 : 2;
    fr_muon_plan p = nullptr;
    CHECK(fr_muon_create(list.data(), n, &p) == FR_OK);
    fake::finish_all();
    clear();
    CHECK(fr_muon_step(p, &h, nullptr, nullptr) == FR_OK);
    std::set<uint32_t> with_elements;
    for (uint64_t t = 0; t < n; ++t)
      if (list[t].rows * list[t].cols) with_elements.insert(static_cast<uint32_t>(t));
    if (with_elements.empty()) {
      CHECK(norms.empty() && products.empty() && applies.empty());
      fr_muon_destroy(p);
      continue;
    }
    CHECK(norms.size() == 1 && iterates.size() == 1 && applies.size() == 1 && updates.empty());
    const MuonParams& mp = norms[0];
    // blocks and units: each matrix's, one after the other; places that do not overlap, within the plan's memory
    std::vector<std::pair<uint64_t, uint64_t>> places;
    uint32_t unit = 0, block = 0;
    for (uint32_t m = 0; m < with_elements.size(); ++m) {
      const MuonDesc& d = mp.tensors[m];
      const fr_muon_tensor& x = list[d.tensor];
      CHECK(with_elements.count(d.tensor) && d.rows == x.rows && d.cols == x.cols && d.tall == (x.rows > x.cols) && d.split == (x.master != nullptr));
      CHECK(d.first_unit == unit && d.first_block == block);
      for (uint64_t i = 0; i < (x.rows * x.cols + kUnit - 1) / kUnit; ++i) CHECK(mp.units[unit++] == m);
      const uint64_t bytes = 1ull * d.row_blocks * d.col_blocks * kMuonBlockBytes, square = 2ull * d.side_blocks * d.side_blocks * kMuonBlockBytes;
      for (uint64_t i = 0; i < bytes / kMuonBlockBytes; ++i) CHECK(mp.blocks[block++] == m);
      places.push_back({d.x[0], bytes}), places.push_back({d.x[1], bytes}), places.push_back({d.low[0], bytes});
      if (d.split) places.push_back({d.low[1], bytes});
      places.push_back({d.p, square}), places.push_back({d.s, square});
    }
    CHECK(unit == mp.n_units && block == mp.n_blocks);
    // the products: whichever launches they are, each round has each phase's tiles once
    uint32_t signals[2] = {0, 0};
    for (uint32_t k = 0; k < 2; ++k) {
      std::vector<Launch> mine;
      for (const Launch& l : products)
        if (l.p.split == k) mine.push_back(l);
      std::map<uint32_t, uint32_t> count;  // tiles per counter
      std::map<std::pair<uint32_t, uint32_t>, std::set<uint32_t>> out;  // blocks by matrix and phase
      uint32_t launches_of_round[3] = {0, 0, 0};
      for (const Launch& l : mine) {
        CHECK(l.pairs >= 1 && l.pairs <= resident);
        if (l.p.waits) {
          CHECK(mine.size() == 1 && l.p.first == 0 && l.p.iterations == h.iterations);
        } else {
          CHECK(l.p.iterations == l.p.first + 1 && mine.size() == 3 * h.iterations);
        }
        if (l.p.first != 0) continue;
        uint32_t phase = 0;
        for (uint32_t i = 0; i < l.p.n_tiles; ++i) {
          const MuonTile& t = l.p.tiles[i];
          const uint32_t m = t.done / kPhases;
          CHECK(t.done % kPhases == t.phase && t.needs == m * kPhases + (t.phase + 2) % 3 && t.phase >= phase);
          phase = t.phase;
          ++launches_of_round[phase];
          const MuonDesc& d = mp.tensors[m];
          CHECK(d.split == k);
          check_tile(t, d);
          count[t.done] += kSignals;
          for (uint32_t rank = 0; rank < (t.flags & kSecond ? 2u : 1u); ++rank)
            for (uint32_t q = 0; q < (t.flags & kNarrow ? 2u : 4u); ++q) CHECK((out[{m, t.phase}].insert(t.out + rank * t.across + q).second));
          // second halves and S lie where the kernel adds them
          CHECK(d.x[1] == d.x[0] + 1ull * l.p.x_blocks * kMuonBlockBytes && d.low[0] == d.x[0] + 2ull * l.p.x_blocks * kMuonBlockBytes);
          CHECK(d.s == d.p + 1ull * l.p.p_blocks * kMuonBlockBytes);
          if (k) {
            CHECK(d.low[1] == d.x[1] + 2ull * l.p.x_blocks * kMuonBlockBytes);
            if (t.row == 0 && t.col == 0 && t.phase == 0) {
              const uint64_t square = 2ull * d.side_blocks * d.side_blocks * kMuonBlockBytes;
              places.push_back({d.p + 2ull * l.p.p_blocks * kMuonBlockBytes, square}), places.push_back({d.s + 2ull * l.p.p_blocks * kMuonBlockBytes, square});
            }
          }
        }
      }
      for (const Launch& l : mine)
        for (uint32_t i = 0; i < l.p.n_tiles; ++i) CHECK(l.p.tiles[i].count == count[l.p.tiles[i].needs]);
      for (uint32_t m = 0; m < with_elements.size(); ++m) {
        const MuonDesc& d = mp.tensors[m];
        if (d.split != k) continue;
        ++signals[k];
        CHECK((out[{m, kNext}].size() == 1ull * d.row_blocks * d.col_blocks));
        for (uint32_t phase : {kGram, kPolynomial}) {
          uint64_t want = 0;
          for (uint32_t r = 0; r < d.side_blocks; ++r)
            for (uint32_t c = 0; c < 2 * d.side_blocks; ++c) want += exists(r, c);
          CHECK((out[{m, phase}].size() == want));
        }
      }
    }
    CHECK(signals[0] + signals[1] == with_elements.size());
    std::sort(places.begin(), places.end());
    uint64_t bytes;
    CHECK(fr_muon_info(p, nullptr, nullptr, &bytes) == FR_OK);
    for (size_t i = 0; i < places.size(); ++i) CHECK(places[i].first + places[i].second <= (i + 1 < places.size() ? places[i + 1].first : bytes));
    // one product for all: no launch with second halves
    clear();
    fr_muon one = h;
    one.products = FR_MUON_ONE;
    CHECK(fr_orthogonalize(p, &one, nullptr) == FR_OK && updates.size() == 1 && applies.empty() && norms[0].one == 1 && norms[0].momentum == 0);
    for (const Launch& l : products) CHECK(l.p.split == 0);
    fr_muon_destroy(p);
  }

  // which iterates keep their second halves: raised by more than 4 afterwards
  resident = 76;
  fr_muon_tensor x = matrix(100, 200, false);
  fr_muon_plan p = nullptr, none = nullptr;
  CHECK(fr_muon_create(&x, 1, &p) == FR_OK);
  fake::finish_all();
  clear();
  CHECK(fr_muon_step(p, &h, nullptr, nullptr) == FR_OK && products[0].p.low == 0x0F && iterates[0].low == 1 && applies[0].last == 1);

  // a wait that a kernel gave up is reported once
  CHECK(fr_muon_sync_status(p, nullptr) == FR_OK);
  *p->d_status = 1;
  CHECK(fr_muon_sync_status(p, nullptr) == FR_ERR_DEVICE_TIMEOUT && fr_muon_sync_status(p, nullptr) == FR_OK && *p->d_status == 0);

  // refusals launch nothing
  clear();
  auto refuses = [&](auto change) {
    fr_muon g = h;
    change(g);
    return fr_muon_step(p, &g, nullptr, nullptr) == FR_ERR_INVALID_ARG;
  };
  for (double bad : {1e300, -1.0, HUGE_VAL, static_cast<double>(NAN)}) {
    CHECK(refuses([&](fr_muon& g) { g.lr = bad; }));
    CHECK(refuses([&](fr_muon& g) { g.weight_decay = bad; }));
  }
  for (double bad : {-0.1, 1.0, static_cast<double>(NAN)}) CHECK(refuses([&](fr_muon& g) { g.beta = bad; }));
  CHECK(refuses([](fr_muon& g) { g.step = 0; }));
  CHECK(refuses([](fr_muon& g) { g.nesterov = 2; }));
  CHECK(refuses([](fr_muon& g) { g.rounding = 2; }));
  CHECK(refuses([](fr_muon& g) { g.products = 2; }));
  CHECK(refuses([](fr_muon& g) { g.iterations = 0; }));
  CHECK(refuses([](fr_muon& g) { g.iterations = FR_MUON_MOST + 1; }));
  CHECK(refuses([](fr_muon& g) { g.coef[4][1] = NAN; }));
  CHECK(refuses([](fr_muon& g) { g.coef[0][0] = 15.5; }));       // above 15 at a singular value of 0
  CHECK(refuses([](fr_muon& g) { g.coef[1][2] = 40.0; }));       // and elsewhere
  CHECK(refuses([](fr_muon& g) { g.coef[0][0] = 14.0, g.coef[0][1] = -20.0, g.coef[0][2] = 6.0; }));  // takes 0.5 above 2
  CHECK(!refuses([](fr_muon& g) { g.iterations = 1, g.coef[3][0] = NAN; }));  // not used
  clear();
  CHECK(fr_muon_step(p, &h, reinterpret_cast<fr_clip*>(4), nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_muon_step(nullptr, &h, nullptr, nullptr) == FR_ERR_INVALID_ARG && fr_muon_step(p, nullptr, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  CHECK(fr_orthogonalize(nullptr, &h, nullptr) == FR_ERR_INVALID_ARG && fr_muon_sync_status(nullptr, nullptr) == FR_ERR_INVALID_ARG);
  auto bad = [&](auto change, fr_status want) {
    fr_muon_tensor y = x;
    change(y);
    return fr_muon_create(&y, 1, &none) == want && none == nullptr;
  };
  CHECK(bad([](fr_muon_tensor& y) { y.flags = 1; }, FR_ERR_INVALID_ARG));
  CHECK(bad([](fr_muon_tensor& y) { y.reserved = 1; }, FR_ERR_INVALID_ARG));
  CHECK(bad([](fr_muon_tensor& y) { y.rows = FR_MUON_MOST_SIDE + 1; }, FR_ERR_INVALID_ARG));
  CHECK(bad([](fr_muon_tensor& y) { y.rows = y.cols = FR_MUON_MOST_SIDE; }, FR_ERR_INVALID_ARG));
  CHECK(bad([](fr_muon_tensor& y) { y.update_scale = INFINITY; }, FR_ERR_INVALID_ARG));
  CHECK(bad([](fr_muon_tensor& y) { y.weight_dtype = FR_DT_BYTES; }, FR_ERR_INVALID_ARG));
  CHECK(bad([](fr_muon_tensor& y) { y.weight_dtype = FR_DT_F32, y.master = reinterpret_cast<float*>(8); }, FR_ERR_INVALID_ARG));
  CHECK(bad([](fr_muon_tensor& y) { y.grad = reinterpret_cast<void*>(3); }, FR_ERR_ALIGNMENT));
  CHECK(bad([](fr_muon_tensor& y) { y.momentum = reinterpret_cast<float*>(6); }, FR_ERR_ALIGNMENT));
  CHECK(fr_muon_create(nullptr, 1, &none) == FR_ERR_INVALID_ARG && fr_muon_create(&x, 1, nullptr) == FR_ERR_INVALID_ARG);
  // parts of a list: what a call needs must be there
  fr_muon_tensor grads = x;
  grads.weight = nullptr, grads.momentum = nullptr, grads.master = nullptr;
  fr_muon_plan part = nullptr;
  CHECK(fr_muon_create(&grads, 1, &part) == FR_OK);
  fake::finish_all();
  CHECK(fr_muon_step(part, &h, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  CHECK(norms.empty() && iterates.empty() && products.empty() && applies.empty() && updates.empty());
  CHECK(fr_orthogonalize(part, &h, nullptr) == FR_OK);
  fr_muon_destroy(part);
  // factors times the step's numbers
  fr_muon_tensor large = x;
  large.lr_scale = 1e30f, large.decay_scale = 1e30f;
  CHECK(fr_muon_create(&large, 1, &part) == FR_OK);
  fake::finish_all();
  fr_muon g = h;
  g.lr = 1e10;
  CHECK(fr_muon_step(part, &g, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  g = h, g.weight_decay = 1e10;
  CHECK(fr_muon_step(part, &g, nullptr, nullptr) == FR_ERR_INVALID_ARG);
  fr_muon_destroy(part);
  fr_muon_destroy(p);
  fr_muon_destroy(nullptr);
  std::printf("muon_plan ok\n");
  return 0;
}
