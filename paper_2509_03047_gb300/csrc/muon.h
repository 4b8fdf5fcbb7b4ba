// muon.h -- the orthogonalised update's plan tables and kernel launchers
// (internal to libflashrec).
//
// An iterate X of a matrix is held in blocks of 128 rows and 64 columns, 16 KiB
// each, block row after block row; sides are filled up with zeros to multiples of
// 128.  A block's row is 128 bytes, its eight 16-byte chunks permuted by the row
// (chunk c of row r lies at c ^ (r % 8)): the layout that the tensor cores read
// from shared memory, with the row as the contraction's index or the column, so a
// block goes there as it is and serves X X^T, X^T X, and products from
// either side without a transposition.  The square matrices of the smaller side,
// S = X X^T (or X^T X) and P = a I + b S + c S^2, are held alike, of them the tiles of
// 256 x 256 on and below the diagonal.  What X's rounding to fp16 leaves, which no
// product reads, has blocks of its own kind: chunk c of row r at c * 128 + r, so that
// a warp's 32 rows of a chunk are 512 bytes.
//
// A matrix with an fp32 output, or whose caller asks for it, (split) has second halves of everything, in blocks like
// the first ones, which enter the products too.  Its part of the workspace is apart:
// all x[0], x[1], second halves of either, P, S, second halves of either; the others'
// x[0], x[1], second halves, P, S.
//
// Scales: X 2^14, S 2^13, P 2^11, so that fp16 holds what the bounds on the
// polynomials (flashrec.h) allow: |X| <= 2, |S| <= 4, |P| <= 15 in the spectral
// norm, which no element exceeds; and elements down to 2^-28, 2^-27, 2^-25 of 1 are
// normal numbers.
#pragma once

#include <cstdint>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/flashrec.h"

namespace frk {

constexpr int kBlockRows = 128, kBlockCols = 64, kMuonBlockBytes = kBlockRows * kBlockCols * 2;
constexpr float kScaleX = 0x1p14f, kScaleS = 0x1p13f, kScaleP = 0x1p11f;
constexpr double kMostX = 2.0, kMostP = 15.0;

struct MuonDesc {        // one matrix that has elements
  void* weight;
  const void* grad;
  float* master;
  float* momentum;
  void* update;
  uint64_t rows, cols;
  uint64_t x[2];         // bytes in the workspace: the iterate's first halves, old and new
  uint64_t low[2];       // its second halves (split: a place for each, else one)
  uint64_t s, p;
  uint32_t row_blocks, col_blocks;  // of 128 rows, of 64 columns (an even number)
  uint32_t side_blocks;  // of 128, of the smaller side
  uint32_t tall;         // more rows than columns: S = X^T X, X <- X P
  uint32_t first_unit, n_units;     // of the norm
  uint32_t first_block;  // of all blocks of the plan's iterates
  uint32_t tensor;       // index in the plan
  uint32_t bf16_weight, bf16_grad, bf16_update;
  uint32_t split;        // products of both halves
  float lr_scale, decay_scale, update_scale;
};

// ---- elements: momentum and norm, X from G, the weights' update

constexpr int kUnit = 4096;       // elements of the norm that a CTA adds up
constexpr int kElementThreads = 256;

struct MuonPartial {  // a unit's sum of squares: sum * 4^exponent
  float sum;
  int exponent;
};
struct MuonNorm {     // a matrix's: X = (G * to_one) * factor, in X's scale
  float to_one, factor;
  uint32_t done;      // units that have been added; zero before a launch and after it
  uint32_t reserved;
};

struct MuonParams {
  const MuonDesc* tensors;
  const uint32_t* units;   // matrix of each unit
  const uint32_t* blocks;  // matrix of each block
  uint32_t n_units, n_blocks;
  MuonPartial* partials;
  MuonNorm* norms;
  uint8_t* work;
  const fr_clip* clip;     // may be null
  const uint32_t* status;  // not zero: a product gave up, no momentum, weight or update is written
  float beta, beta_rest;   // beta, 1 - beta
  float lr, decay;
  uint32_t momentum;       // 0: G is the gradient
  uint32_t nesterov;
  uint32_t random;
  uint64_t key;            // as in StepParams
  uint32_t last;           // which of x[] holds the last iterate
  uint32_t low;            // 1: the first iterate has second halves
  uint32_t one;            // 1: products of first halves for all
  uint32_t* done;          // the products' counters, set to zero
};
cudaError_t launch_muon_norm(const MuonParams& p, cudaStream_t s);
cudaError_t launch_muon_iterate(const MuonParams& p, cudaStream_t s);   // X, from G and the norm
cudaError_t launch_muon_apply(const MuonParams& p, cudaStream_t s);     // the step's weights
cudaError_t launch_muon_update(const MuonParams& p, cudaStream_t s);    // fr_orthogonalize's output

// ---- products

enum : int { kGram = 0, kPolynomial = 1, kNext = 2 };  // S, P, the next X
constexpr int kPhases = 3;

// D[i][j] = sum over k of A(i, k) B(j, k): a tile of it, 256 x 256 or 256 x 128, by a pair of CTAs.  All that a CTA needs of it in one record, so
// that the next tile's is there when its turn comes.  Numbers of blocks: of x[0]'s place where a factor or the result is an iterate.
// Of S and P only the tiles on and below the diagonal exist: from a step on a factor's blocks are those on the diagonal's other side, read the
// other way round.
struct __attribute__((aligned(16))) MuonTile {
  uint32_t a[2], b[2];              // first block of each CTA's part of the factors,
  uint32_t a_after[2], b_after[2];  // and the one at the step where the blocks change sides
  uint32_t a_switch, b_switch;      // that step
  uint32_t a_next, b_next;          // from a block to the next one of the contraction
  uint32_t square;                  // and, by columns, in S and P
  uint32_t depth;                   // steps of 64 of the contraction
  uint32_t flags;
  uint32_t phase;
  uint32_t out;                     // block of the result's first row and column
  uint32_t across;                  // the result's blocks per block of rows
  uint16_t row, col;                // of the tile, in blocks of 128
  uint32_t done;                    // the counter of the matrix and phase
  uint32_t needs;                   // the counter of the phase that this one reads from,
  uint32_t count;                   // and what that adds to it in an iteration
  uint32_t reserved[2];
};
static_assert(sizeof(MuonTile) == 96, "six loads of 16 bytes");
// kNarrow: 128 columns.  kAColumns, kBColumns: a factor is read by its columns, else its rows.  kSecond: there are rows for the second CTA.  kSame:
// on the diagonal, both factors are the same blocks.
enum : uint32_t { kNarrow = 1, kAColumns = 2, kBColumns = 4, kSecond = 8, kAIterate = 16, kBIterate = 32, kSame = 64 };
constexpr uint32_t kSignals = 16;  // of a tile: two CTAs, eight warps
constexpr int64_t kWaitClocks = 4ll << 30;  // some two seconds
// The tensor cores cut their sums off to fp32 with every 16 products, always towards zero: of long contractions that adds up.  So after this many steps of
// 64 the sums go to fp32 numbers in memory, and new ones begin in tensor memory.  (2^20 terms in one go: O off by 8e-3, with products of both halves
// as with one.)  Products of both halves lose up to 1.9e-4 by what a part of 4,096 terms is cut off; in one product a part of 32,768 is far below the
// factors' own rounding.
constexpr uint32_t part_steps(bool split) { return split ? 64 : 512; }
constexpr int kPartBytes = 128 * 256 * 4;  // of a CTA

// One launch takes a list through some iterations, or a phase of one: its tiles in order, iteration after iteration, each pair every n-th.  A tile waits until all
// those that it reads from have counted; they come before it in that order, and all CTAs are resident, so every wait ends.
struct MuonProduct {
  const MuonTile* tiles;
  uint32_t n_tiles;
  uint32_t first, iterations;  // this launch's: [first, iterations)
  uint8_t* work;
  const fr_clip* clip;
  uint32_t* status;         // set to 1 by a kernel that gave up a wait
  int64_t wait_clocks;      // after which it does
  uint32_t* done;           // counters, zero at the start
  uint32_t parts;           // 1: a tile's contraction is longer than a part
  uint8_t* sums;            // then kPartBytes for each CTA: of a tile's parts but the last
  uint32_t x_blocks;        // of all iterates: from x[0] to x[1], from either to its second halves twice as far
  uint32_t p_blocks;        // from P to S, the same
  uint32_t split;
  float coef[FR_MUON_MOST][3];
  uint32_t low;             // bit i: the iterate before iteration i has second halves
  uint32_t waits;           // 1: tiles of several phases
};
// Per device, before the first launch: opt the kernels in to their shared-memory size.
cudaError_t configure_muon_product();
// How many pairs are resident together.
cudaError_t muon_pairs(uint32_t* pairs);
// The workspace as blocks of two halves of 64 rows of 128 bytes.  A copy takes a block, the same half of two neighbouring blocks, or a half.
struct MuonMaps {
  CUtensorMap rows, columns, half;
};
cudaError_t launch_muon_product(const MuonProduct& p, const MuonMaps& maps, uint32_t pairs, cudaStream_t s);

}  // namespace frk
