// muon_product.cu -- the products of the orthogonalised update: X X^T, the polynomial
// in it, the next X, of all matrices of a list.
//
// D[i][j] = sum over k of A(i, k) B(j, k), tiles of 256 x 256 by pairs of CTAs, one
// pair per two SMs, each taking every n-th tile of the list.  A warp brings the
// factors' blocks, 64 of the contraction at a time; another multiplies; eight warps
// turn the sums into fp16 blocks, while the next tile's products fill the other half
// of tensor memory.  The blocks lie in memory as the tensor cores read them, by rows
// or by columns, so X X^T, X^T X and products from either side need no
// transposition.  Of the symmetric products the tiles on and below the diagonal are
// computed, and read both ways.  Sums of long contractions are put together from parts
// (muon.h), each CTA's in 128 KiB of its own: 14336 x 4096 in fp32 6,830 us, 128 x 2^20
// 41,400, off by 1.8e-4 and 4e-5.
//
// What bounds it, GB300:
//   products of first halves: the way from L2 to an SM.  A step is 512 clocks of
//     products and 32 KiB per SM, which take 570 (57 bytes a clock; a tile of 256 x
//     128, 24 KiB for 256 clocks, 404).  A tile has 500 to 1,000 clocks more before its
//     first step, a launch some 5 us.  Back to back the power limit counts: 14336 x
//     4096 five iterations 2.8 ms, 1,400 TFLOP/s of the needed work (half of a symmetric
//     product), 1,550 with the tiles' upper halves, at 1,550 MHz;
//   products of both halves: the tensor cores, three times the work for twice the
//     bytes: 1,670 TFLOP/s of it, at the power limit;
//   iterates of narrow matrices: HBM, 6 to 8 bytes an element each iteration;
//   small lists: 8,000 clocks a phase for its way through L2 (stores 1,900 until they
//     are seen, the wait 1,300, the first copies 1,000 to 3,000).
// Pairs of 256 x 256, not CTAs of 128 x 256 (22 TB/s from L2 at full rate) or 128 x
// 128 (29).  Six stages of 32 KiB and 4 KiB per finishing warp, not five and 8: 24
// layers of width 1024 6.44 -> 5.96 ms.  Second halves go past shared memory, each
// lane's own.  Ten warps leave 168 registers per thread, and 36 bytes of each thread's are
// spilled (132 and 56 where sums are put together).
#include <algorithm>

#include "kernels.h"
#include "muon_block.cuh"
#include "optim.h"
#include "tensor_core.cuh"

namespace frk {

namespace {

constexpr int kFactorBytes = 16384;  // 128 rows or columns of a factor, 64 of the contraction
constexpr int kHalf = 8192;
// The products of a step: first halves; or with second halves first times second and second times first as well, for 22 bits of each factor.
template <bool kSplit>
struct Stages {
  static constexpr int kCount = kSplit ? 3 : 6, kBytes = (kSplit ? 4 : 2) * kFactorBytes;
  static constexpr uint32_t kPart = part_steps(kSplit);
};
constexpr int kRingBytes = 12 * kFactorBytes, kMostStages = 6;
static_assert(Stages<true>::kCount * Stages<true>::kBytes == kRingBytes && Stages<false>::kCount * Stages<false>::kBytes == kRingBytes, "one size");
constexpr int kWarps = 8;            // that turn sums into blocks: a quarter of the rows, every other 64 columns
constexpr int kThreads = 64 + kWarps * 32;
constexpr int kStaging = kMuonBlockBytes / 4;  // per warp
constexpr int kTensorColumns = 512;
constexpr size_t kShared = 1024 + kRingBytes + kWarps * kStaging;
static_assert(kSignals == 2 * kWarps, "one per warp");

struct Control {
  uint64_t full[kMostStages], empty[kMostStages], sums_full[2], sums_empty[2];
  uint32_t tensor;
  uint32_t gave_up;
};

// A factor's place in the contraction, which goes from block to block of a row, or from half to half of a column's blocks.
struct Place {
  int32_t block, half, next, flip;
  __device__ __forceinline__ void advance() {
    block += half & flip || !flip ? next : 0;
    half ^= flip;
  }
};

// This pair's tiles in turn, each record read a tile ahead.
struct Tiles {
  const MuonProduct& p;
  uint32_t at, round, next_round;
  MuonTile now, next;
  __device__ __forceinline__ explicit Tiles(const MuonProduct& p) : p(p), at(blockIdx.x / 2), next_round(p.first) { read(); }
  __device__ __forceinline__ bool take() {
    if (next_round >= p.iterations) return false;
    now = next;
    round = next_round;
    at += gridDim.x / 2;
    read();
    return true;
  }
  // How often the counter that the tile needs must have been added to.
  __device__ __forceinline__ uint32_t count() const { return now.count * (now.phase == kGram ? round : round + 1); }
  // The place of the iterate before or after this iteration.
  __device__ __forceinline__ uint32_t iterate(uint32_t after) const { return (round + after) % 2 ? p.x_blocks : 0; }

 private:
  __device__ __forceinline__ void read() {
    while (at >= p.n_tiles && next_round < p.iterations) {
      at -= p.n_tiles;
      ++next_round;
    }
    if (next_round < p.iterations) next = p.tiles[at];
  }
};

// Where a stage and its phase stand.
template <bool kSplit>
struct Ring {
  uint32_t stage = 0, phase = 0;
  __device__ __forceinline__ void next() {
    if (++stage == Stages<kSplit>::kCount) {
      stage = 0;
      phase ^= 1;
    }
  }
};

template <bool kSplit>
__device__ __forceinline__ void bring(const MuonProduct& p, const MuonMaps& maps, uint32_t ring_at, Control& c, uint32_t rank) {
  constexpr int kStageBytes = Stages<kSplit>::kBytes;
  Ring<kSplit> r;
  const uint32_t full0 = shared_address(&c.full[0]), empty0 = shared_address(&c.empty[0]);
  for (Tiles tiles(p); tiles.take();) {
    const MuonTile& t = tiles.now;
    const bool narrow = t.flags & kNarrow, a_columns = t.flags & kAColumns, b_columns = t.flags & kBColumns;
    Place a = {static_cast<int32_t>((rank ? t.a[1] : t.a[0]) + (t.flags & kAIterate ? tiles.iterate(0) : 0)), 0, static_cast<int32_t>(t.a_next), a_columns};
    Place b = {static_cast<int32_t>((rank ? t.b[1] : t.b[0]) + (t.flags & kBIterate ? tiles.iterate(0) : 0)), narrow && !b_columns ? static_cast<int32_t>(rank) : 0,
               static_cast<int32_t>(t.b_next), b_columns};
    const CUtensorMap *a_map = a_columns ? &maps.columns : &maps.rows, *b_map = narrow ? &maps.half : b_columns ? &maps.columns : &maps.rows;
    if (p.waits) {
      if (!__all_sync(0xFFFFFFFFu, wait_count(p.done + t.needs, tiles.count(), p.wait_clocks, &c.gave_up))) return let_copies_land();
      before_reading_copies();
    }
    const bool same = t.flags & kSame;
    const uint32_t bytes = (kSplit ? 2 : 1) * (2 * kFactorBytes + (same ? 0 : narrow ? kFactorBytes : 2 * kFactorBytes));
    const int32_t a_low = 2 * static_cast<int32_t>(t.flags & kAIterate ? p.x_blocks : p.p_blocks),
                  b_low = 2 * static_cast<int32_t>(t.flags & kBIterate ? p.x_blocks : p.p_blocks);
    // (few instructions per step: one thread takes 4 to 6 clocks for each, and 512 clocks of products wait for it)
    for (uint32_t k = 0; k < t.depth; ++k) {
      if (k == t.a_switch) {
        a = {static_cast<int32_t>(rank ? t.a_after[1] : t.a_after[0]), 0, static_cast<int32_t>(t.square), 1};
        a_map = &maps.columns;
      }
      if (k == t.b_switch) {
        b = {static_cast<int32_t>(rank ? t.b_after[1] : t.b_after[0]), 0, static_cast<int32_t>(t.square), 1};
        b_map = narrow ? &maps.half : &maps.columns;
      }
      const uint32_t full = full0 + r.stage * 8, to = ring_at + r.stage * kStageBytes;
      if (!__all_sync(0xFFFFFFFFu, wait_phase(empty0 + r.stage * 8, r.phase ^ 1, p.wait_clocks, &c.gave_up))) return let_copies_land();
      if (one_lane()) {
        if (rank == 0) expect_bytes(full, bytes);
        load_blocks(to, a_map, a.half, a.block, full);
        if (!same) load_blocks(to + kFactorBytes, b_map, b.half, b.block, full);
        if (kSplit) {
          load_blocks(to + 2 * kFactorBytes, a_map, a.half, a.block + a_low, full);
          if (!same) load_blocks(to + 3 * kFactorBytes, b_map, b.half, b.block + b_low, full);
        }
      }
      __syncwarp();
      a.advance();
      b.advance();
      r.next();
    }
  }
}

template <bool kSplit, bool kParts>
__device__ __forceinline__ void multiply_tiles(const MuonProduct& p, uint32_t ring_at, Control& c) {
  constexpr int kStageBytes = Stages<kSplit>::kBytes;
  Ring<kSplit> r;
  const uint32_t full0 = shared_address(&c.full[0]), empty0 = shared_address(&c.empty[0]), tensor = c.tensor;
  uint32_t n = 0;
  for (Tiles tiles(p); tiles.take();) {
    const MuonTile& t = tiles.now;
    bool a_columns = t.flags & kAColumns, b_columns = t.flags & kBColumns;
    const uint32_t columns = t.flags & kNarrow ? 128 : 256, depth = t.depth, a_switch = t.a_switch, b_switch = t.b_switch;
    uint32_t kind, a_step, b_step;
    uint64_t a0, b0;
    auto set = [&] {
      kind = product_kind(a_columns, b_columns, columns);
      a_step = a_columns ? 2048 >> 4 : 32 >> 4;
      b_step = b_columns ? 2048 >> 4 : 32 >> 4;
      a0 = factor(ring_at, a_columns, kHalf);
      b0 = factor(ring_at + (t.flags & kSame ? 0 : kFactorBytes), b_columns, kHalf);
    };
    set();
    for (uint32_t k = 0; k < depth; ++n) {
      // a part, or all of it
      const uint32_t half = n % 2, begin = k, end = kParts ? min(begin + Stages<kSplit>::kPart, depth) : depth, sums = tensor + half * 256;
      if (!__all_sync(0xFFFFFFFFu, wait_phase(shared_address(&c.sums_empty[half]), (n / 2 + 1) % 2, p.wait_clocks, &c.gave_up))) return let_copies_land();
      tensor_fence_after();
      for (; k < end; ++k) {
        if (k == a_switch || k == b_switch) {
          a_columns |= k == a_switch;
          b_columns |= k == b_switch;
          set();
        }
        if (!__all_sync(0xFFFFFFFFu, wait_phase(full0 + r.stage * 8, r.phase, p.wait_clocks, &c.gave_up))) return let_copies_land();
        tensor_fence_after();
        const uint64_t a = a0 + r.stage * (kStageBytes >> 4), b = b0 + r.stage * (kStageBytes >> 4);
        if (one_lane()) {
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j) multiply(sums, a + j * a_step, b + j * b_step, kind, k > begin || j > 0);
          if (kSplit) {
            constexpr uint32_t kLow = 2 * kFactorBytes >> 4;
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) multiply(sums, a + j * a_step, b + kLow + j * b_step, kind, true);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) multiply(sums, a + kLow + j * a_step, b + j * b_step, kind, true);
          }
          arrive_after_products(empty0 + r.stage * 8);
        }
        __syncwarp();
        r.next();
      }
      if (one_lane()) arrive_after_products(shared_address(&c.sums_full[half]));
      __syncwarp();
    }
  }
}

// What is added to a row's 64 sums: of S, whose chunks lie as in the factors, or of second halves, whose chunks lie a block's rows apart.  (Not
// from this SM's first-level cache: other SMs have written it during this launch.)
struct Addend {
  uint4 x[8];
  // The warp's 32 rows as they lie, whole lines at a time; to_rows() afterwards.  (Each lane its row's chunks: 32 lines for a load, and the factors'
  // copies wait behind them, 3,000 clocks instead of 1,000.)
  __device__ __forceinline__ void of_square(const uint8_t* rows, uint32_t lane) {
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) x[k] = __ldcg(reinterpret_cast<const uint4*>(rows + k * 512 + lane * 16));
  }
  __device__ __forceinline__ void to_rows(uint8_t* staging, uint32_t lane) {
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) *reinterpret_cast<uint4*>(staging + k * 512 + lane * 16) = x[k];
    __syncwarp();
#pragma unroll
    for (uint32_t c = 0; c < 8; ++c) x[c] = *reinterpret_cast<const uint4*>(staging + lane * 128 + ((c ^ (lane % 8)) * 16));
    __syncwarp();
  }
  __device__ __forceinline__ void of_low(const uint8_t* block, uint32_t row) {
#pragma unroll
    for (uint32_t c = 0; c < 8; ++c) x[c] = __ldcg(reinterpret_cast<const uint4*>(block + (c * kBlockRows + row) * 16));
  }
};

// What sums of a product, the thread's row and 64 columns of it, become:
//   S = X X^T             sums in X's scale twice
//   P = a I + b S + c S^2
//   X = P X1 + a X2       X1, X2 the halves of the old X; a I in P has the first one's part.  (kSplit: X = P X, all of it)
// rounded to fp16, for the factors in shared memory; what the rounding leaves in `in_low` (kSplit), whose S has been used, or X's to `low` if that is
// not null.
template <int kPhase, bool kSplit>
__device__ __forceinline__ void finish_row(const float (&coef)[3], uint32_t diagonal, const float (&v)[64], const Addend& in, Addend& in_low, bool adds,
                                           uint8_t* staging, uint32_t row, uint8_t* low) {
#pragma unroll
  for (uint32_t c = 0; c < 8; ++c) {
    float x[8], y[8];
    if (kPhase == kPolynomial || (kPhase == kNext && !kSplit && adds)) floats(in.x[c], y);
    if (kPhase == kPolynomial && kSplit) {
      float z[8];
      floats(in_low.x[c], z);
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j) y[j] += z[j];
    }
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      const float sum = v[8 * c + j];
      if (kPhase == kGram) {
        x[j] = sum * (kScaleS / (kScaleX * kScaleX));
      } else if (kPhase == kPolynomial) {
        const float own = diagonal == 8 * c + j ? coef[0] * kScaleP : 0.0f;
        x[j] = own + y[j] * (coef[1] * (kScaleP / kScaleS)) + sum * (coef[2] * (kScaleP / (kScaleS * kScaleS)));
      } else {
        x[j] = sum * (1.0f / kScaleP);
        if (!kSplit && adds) x[j] += coef[0] * y[j];
      }
    }
    uint4* const to = reinterpret_cast<uint4*>(staging + row % 32 * 128 + ((c ^ (row % 8)) * 16));
    if (kSplit) {
      split(x, *to, in_low.x[c]);
    } else if (kPhase == kNext && low != nullptr) {
      uint4 lo;
      split(x, *to, lo);
      *reinterpret_cast<uint4*>(low + (c * kBlockRows + row) * 16) = lo;
    } else {
      *to = halves(x);
    }
  }
}

// The warp's rows from shared memory to their block.  Where tiles of a launch wait for one another, by ordinary stores, 512 bytes at a time: another
// SM sees them sooner.  Else by a bulk copy, which costs the warp nothing.
__device__ __forceinline__ void store_rows(uint8_t* to, const uint8_t* staging, uint32_t lane, bool soon) {
  if (soon) {
    __syncwarp();
#pragma unroll
    for (uint32_t k = 0; k < kStaging / 512; ++k)
      *reinterpret_cast<uint4*>(to + k * 512 + lane * 16) = *reinterpret_cast<const uint4*>(staging + k * 512 + lane * 16);
    __syncwarp();
    return;
  }
  before_copies();
  __syncwarp();
  if (lane == 0) {
    store_bytes(to, shared_address(staging), kStaging);
    end_stores();
  }
}

// A row's sums of a tile's parts so far, 64 columns of them: four at a time, where the row's neighbours have theirs beside them.
__device__ __forceinline__ float4* part_sums(const MuonProduct& p, uint32_t q, uint32_t row) {
  return reinterpret_cast<float4*>(p.sums + static_cast<uint64_t>(blockIdx.x) * kPartBytes) + q * 16 * kBlockRows + row;
}
__device__ __forceinline__ void add_parts(const float4* at, float (&v)[64]) {
#pragma unroll
  for (uint32_t c = 0; c < 16; ++c) {
    const float4 x = at[c * kBlockRows];
    v[4 * c] += x.x, v[4 * c + 1] += x.y, v[4 * c + 2] += x.z, v[4 * c + 3] += x.w;
  }
}

// One of the eight warps.  Each by itself: what it adds is on its way while the products run, its 32 rows of 64 columns leave together.
template <bool kSplit, bool kParts>
__device__ __forceinline__ void finish_tiles(const MuonProduct& p, uint8_t* staging, Control& c, uint32_t rank) {
  const uint32_t warp = threadIdx.x / 32 - 2, lane = threadIdx.x % 32;
  const uint32_t quarter = threadIdx.x / 32 % 4, row = quarter * 32 + lane;  // a warp reads the quarter of its index
  staging += warp * kStaging;
  const uint64_t to_low = 2ull * p.x_blocks * kMuonBlockBytes, to_square = static_cast<uint64_t>(p.p_blocks) * kMuonBlockBytes;
  uint32_t n = 0;
  for (Tiles tiles(p); tiles.take(); ++n) {
    const MuonTile& t = tiles.now;
    const uint32_t parts = t.flags & kNarrow ? 2 : 4;
    const bool mine = rank == 0 || t.flags & kSecond;
    const bool low_after = !kSplit && p.low >> (tiles.round + 1) & 1, adds = t.phase == kPolynomial || (!kSplit && t.phase == kNext && p.low >> tiles.round & 1);
    const float coef[3] = {p.coef[tiles.round][0], p.coef[tiles.round][1], p.coef[tiles.round][2]};
    uint8_t* const first = p.work + (static_cast<uint64_t>(t.out) + rank * t.across) * kMuonBlockBytes;
    Addend in, in_low;
    auto fetch = [&](uint32_t q) {
      if (t.phase == kPolynomial) {
        const uint8_t* const rows = first + q * kMuonBlockBytes + to_square + quarter * kStaging;
        in.of_square(rows, lane);
        if (kSplit) in_low.of_square(rows + 2 * to_square, lane);
      } else {
        in.of_low(first + q * kMuonBlockBytes + to_low, row);
      }
    };
    const bool several = kParts && t.depth > Stages<kSplit>::kPart;
    if (several) {
      for (uint32_t k = Stages<kSplit>::kPart; k < t.depth; k += Stages<kSplit>::kPart, ++n) {  // parts but the last
        if (!__all_sync(0xFFFFFFFFu, wait_phase(shared_address(&c.sums_full[n % 2]), n / 2 % 2, p.wait_clocks, &c.gave_up))) return let_copies_land();
        tensor_fence_after();
        for (uint32_t q = warp / 4; q < parts; q += 2) {
          float v[64];
          const uint32_t from = c.tensor + (quarter * 32 << 16) + n % 2 * 256 + q * 64;
          tensor_load(from, v);
          tensor_load(from + 32, v + 32);
          tensor_load_wait();
          if (!mine) continue;
          float4* const at = part_sums(p, q, row);
          if (k > Stages<kSplit>::kPart) add_parts(at, v);
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) at[i * kBlockRows] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        }
        tensor_fence_before();
        __syncwarp();
        if (lane == 0) arrive_in_first(shared_address(&c.sums_empty[n % 2]));
      }
    }
    const uint32_t half = n % 2;
    bool ok = true;
    if (mine && adds) {
      ok = !p.waits || wait_count(p.done + t.needs, tiles.count(), p.wait_clocks, &c.gave_up);
      fetch(warp / 4);
    }
    ok = wait_phase(shared_address(&c.sums_full[half]), n / 2 % 2, p.wait_clocks, &c.gave_up) && ok;
    if (!__all_sync(0xFFFFFFFFu, ok)) return let_copies_land();
    tensor_fence_after();
    for (uint32_t q = warp / 4; q < parts; q += 2) {
      float v[64];
      const uint32_t from = c.tensor + (quarter * 32 << 16) + half * 256 + q * 64;
      tensor_load(from, v);
      tensor_load(from + 32, v + 32);
      tensor_load_wait();
      if (q + 2 >= parts) tensor_fence_before();
      if (!mine) continue;
      if (several) add_parts(part_sums(p, q, row), v);
      if (lane == 0) wait_stores_read();  // of the rows before
      __syncwarp();
      if (t.phase == kPolynomial) {
        in.to_rows(staging, lane);
        if (kSplit) in_low.to_rows(staging, lane);
      }
      uint8_t* const block = first + q * kMuonBlockBytes;
      if (t.phase == kGram)
        finish_row<kGram, kSplit>(coef, 0, v, in, in_low, false, staging, row, nullptr);
      else if (t.phase == kPolynomial)  // (the diagonal's column of this row among the block's)
        finish_row<kPolynomial, kSplit>(coef, (t.row + rank) * kBlockRows + row - (2 * t.col + q) * kBlockCols, v, in, in_low, true, staging, row, nullptr);
      else
        finish_row<kNext, kSplit>(coef, 0, v, in, in_low, adds, staging, row, low_after ? block + to_low : nullptr);
      if (!kSplit && adds && q + 2 < parts) fetch(q + 2);
      uint8_t* const to = block + (t.phase == kNext ? static_cast<uint64_t>(tiles.iterate(1)) * kMuonBlockBytes : 0) + quarter * kStaging;
      store_rows(to, staging, lane, p.waits);
      if (kSplit) {
        if (lane == 0) wait_stores_read();
        __syncwarp();
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(staging + row % 32 * 128 + ((c ^ (row % 8)) * 16)) = in_low.x[c];
        if (adds && q + 2 < parts) fetch(q + 2);
        store_rows(to + (t.phase == kNext ? to_low : 2 * to_square), staging, lane, p.waits);
      }
    }
    __syncwarp();
    if (lane == 0) {
      if (p.waits) add_to_count(p.done + t.done);
      arrive_in_first(shared_address(&c.sums_empty[half]));
    }
  }
  if (lane == 0) wait_stores();
}

// kParts: some tile's contraction is longer than a part.  (Its code costs the others' tiles, in registers: 142 us instead of 136 for two small layers.)
template <bool kSplit, bool kParts>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    product_kernel(const __grid_constant__ MuonProduct p, const __grid_constant__ MuonMaps maps) {
  extern __shared__ uint8_t raw[];
  __shared__ Control c;
  const uint32_t ring_at = (shared_address(raw) + 1023) & ~1023u;
  uint8_t* const staging = raw + (ring_at - shared_address(raw)) + kRingBytes;
  const uint32_t rank = rank_in_pair(), warp = threadIdx.x / 32;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kMostStages; ++i) {
      barrier_init(shared_address(&c.full[i]), 1);
      barrier_init(shared_address(&c.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      barrier_init(shared_address(&c.sums_full[i]), 1);
      barrier_init(shared_address(&c.sums_empty[i]), 2 * kWarps);
    }
    c.gave_up = 0;
    barrier_init_done();
  }
  if (warp == 1) tensor_alloc(shared_address(&c.tensor), kTensorColumns);
  tensor_fence_before();
  __syncthreads();
  pair_sync();
  tensor_fence_after();
  wait_for_kernel_before();
  // (Once a product has given up a wait, those after it do nothing.  A pair whose CTAs disagree, because one of this launch gives up just now, ends by
  // its waits' limit.)
  const bool stopped = *static_cast<volatile uint32_t*>(p.status) != 0;
  if (!stopped && (p.clip == nullptr || p.clip->nonfinite == 0)) {
    if (warp == 0) {
      bring<kSplit>(p, maps, ring_at, c, rank);
    } else if (warp == 1) {
      if (rank == 0) multiply_tiles<kSplit, kParts>(p, ring_at, c);
    } else {
      finish_tiles<kSplit, kParts>(p, staging, c, rank);
    }
  }
  // Neither CTA frees or leaves while the other's products or arrivals may still reach it.
  __syncwarp();
  tensor_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && c.gave_up) *p.status = 1;
  pair_sync();
  tensor_fence_after();
  if (warp == 1) tensor_free(c.tensor, kTensorColumns);
}

cudaLaunchConfig_t config(uint32_t pairs, cudaStream_t s, cudaLaunchAttribute (&attrs)[1]) {
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(2 * pairs);
  c.blockDim = dim3(kThreads);
  c.dynamicSmemBytes = kShared;
  c.stream = s;
  attrs[0].id = cudaLaunchAttributeCooperative;
  attrs[0].val.cooperative = 1;
  c.attrs = attrs;
  c.numAttrs = 1;
  return c;
}

}  // namespace

namespace {
using Kernel = void (*)(const MuonProduct, const MuonMaps);
constexpr Kernel kKernels[2][2] = {{product_kernel<false, false>, product_kernel<false, true>}, {product_kernel<true, false>, product_kernel<true, true>}};
}  // namespace

cudaError_t configure_muon_product() {
  cudaError_t e = cudaSuccess;
  for (const auto& kernels : kKernels)
    for (Kernel kernel : kernels)
      if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kShared));
  return e;
}

cudaError_t muon_pairs(uint32_t* pairs) {
  cudaLaunchAttribute attrs[1] = {};
  cudaLaunchConfig_t c = config(kSms / 2, nullptr, attrs);
  c.numAttrs = 0;
  cudaError_t e = cudaSuccess;
  int least = kSms / 2, n = 0;
  for (const auto& kernels : kKernels)
    for (Kernel kernel : kernels) {
      if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&n, kernel, &c);
      least = std::min(least, n);
    }
  *pairs = static_cast<uint32_t>(least);
  return e != cudaSuccess ? e : *pairs > 0 ? cudaSuccess : cudaErrorLaunchOutOfResources;
}

cudaError_t launch_muon_product(const MuonProduct& p, const MuonMaps& maps, uint32_t pairs, cudaStream_t s) {
  const Kernel kernel = kKernels[p.split != 0][p.parts != 0];
  if (!p.waits) return launch_chained(kernel, static_cast<int>(2 * std::min(pairs, p.n_tiles)), kThreads, kShared, s, p, maps);
  cudaLaunchAttribute attrs[1] = {};
  const cudaLaunchConfig_t c = config(pairs, s, attrs);
  cudaLaunchKernelEx(&c, kernel, p, maps);
  return cudaGetLastError();
}

}  // namespace frk
