// archead_head_loss, archead_head_loss_grad: sizes, workspace and the tile
// kernels' arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace archead {
namespace loss {

constexpr int kTileJ = 256;        // columns of a tile
constexpr int kStageK = 64;        // k of a stage
constexpr int kRowPad = 256;       // buffers hold this many tokens' rows or a multiple

// The products, out[i, j] = sum_k: 
//   kStats   i token, j vocabulary row, k of d: a tile's largest logit and sum of
//            exponentials per token, and the target's logit
//   kGrad    the same logits, as G = g (exp(l - lse) - [j = target]) in bf16, the operand
//            of the matrix units below, g in units of the largest: up to 2^-8 of each entry,
//            independent of one another, so less of a sum of many, and next to nothing at
//            the targets of tokens that count alike (fp32 entries would be two operands,
//            twice the products)
//   kHidden  i token, j of d, k vocabulary row: sums of G w into fp32
//   kHead    i vocabulary row, j of d, k token: rows of G^T x in bf16
enum Op { kStats, kGrad, kHidden, kHead };

struct TileArgs {
  const uint16_t* a;       // operand of i: [i][k], for kHead [k][i]
  const uint16_t* b;       // operand of j: [j][k], for kHidden and kHead [k][j]
  int64_t a_ld, b_ld;      // elements between rows
  int64_t rows;            // kHead: i; else of tokens at most (the device's count says)
  int64_t cols;            // j
  int64_t depth;           // k (kHead: at most, the device's count says)
  const int32_t* count;    // live tokens
  int64_t v0;              // first vocabulary row of the piece
  int64_t first_stages;    // kHidden: of the call's first piece
  // kStats
  float2* part;            // [token][n_part] (largest, sum)
  int64_t n_part, part0;   // tiles of the vocabulary; the piece's first one
  float* at_target;        // [token]
  // kGrad
  const int32_t* target;   // [token]
  const float* lse;        // [token]
  const float* g;          // [token], in units of the largest
  const float* unit;       // kHead: of g
  uint16_t* out;           // kGrad: G [token][out_ld]; kHead: dw
  int64_t out_ld;
  // kHidden
  float* sums;             // [part of k][row][sum_ld], all in sum_rows rows
  int64_t sum_ld, sum_rows;
  bool add;                // to what sums holds
};

// kHidden's parts of k: as many as bring its tiles to kTargetTiles and sums has rows
// for, by the number of live tokens (the same where they are added up; a shorter piece may
// add to the first of them only).
constexpr int kTargetTiles = 256;
constexpr int kPartStages = 8;     // stages of a part at least
__host__ __device__ inline int64_t padded_rows(int64_t live) { return (live + kRowPad - 1) / kRowPad * kRowPad; }
__host__ __device__ inline int splits_for(int64_t tiles, int64_t live, int64_t sum_rows, int64_t first_stages) {
  if (live <= 0) return 1;
  int64_t s = kTargetTiles / (tiles > 0 ? tiles : 1);
  const int64_t fit = sum_rows / padded_rows(live);
  s = s < fit ? s : fit;
  const int64_t parts = first_stages / kPartStages;
  s = s < parts ? s : parts;
  return s > 1 ? int(s) : 1;
}

// tiles of ti x 256, ti = 64, 128 or 256 (kHead: 128 or 256)
hipError_t launch_tiles(Op op, int ti, const TileArgs& g, hipStream_t s);

}  // namespace loss
}  // namespace archead
