// Launch interface of the kernels of scored attention (attn_scored*.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "layout.h"
#include "tokens.h"

namespace ca {

// What a tile's tokens have in common, over the tokens that are there (in the grid, with a document that is not negative).
struct TileLine {
  int32_t doc_min, doc_max;      // min > max: none is there
  float pos_min, pos_max, limit_min, limit_max;
  int32_t whole;                 // every slot holds one
  int32_t unused;
};

// Rows of `line` per tile, of B words each.
enum LineRow { kLinePosition = 0, kLineDocument = 1, kLineLimit = 2, kLineRows = 4 };

struct ScoredArgs : GridArgs {
  const void *q, *k, *v, *dout, *o;  // [batch, heads, N_pad, D] tile order, bf16
  void *out, *dq, *dk, *dv;
  const float* lse_in;         // backward: the forward call's
  float* lse;                  // forward: [batch, heads, N_pad]
  // the walk: for every row (head, tile) the tiles it visits; rows in launch order
  const int64_t* row_ptr;
  const int32_t* col_meta;     // tile id | padding class << 24 (bit 31 is not read)
  const int32_t* order;
  const int32_t* tile_class;   // [n]
  const SlotMask* class_mask;
  const uint8_t* class_perm;   // [num_classes * 128]
  int32_t batch, num_heads, D;
  int64_t n;
  float scale, cap;            // cap 0: none
  const float* slopes;         // [heads] or null
  // tokens as natural-order arrays [batch, N_real], null where not given
  const int32_t *positions, *limits, *documents;
  // workspace
  float* line;                 // [batch][n][kLineRows][B]: position, document (as an integer), limit; null where no array is given
  TileLine* tiles;             // [batch][n]
  float* rows;                 // backward: [batch * heads][n][2][B]: log-sum-exp in powers of two, delta
};

// bytes of the parts of the workspace, each a multiple of 256
inline int64_t line_bytes(int64_t batch, int64_t n, int64_t B) { return (batch * n * kLineRows * B * 4 + 255) / 256 * 256; }
inline int64_t tile_line_bytes(int64_t batch, int64_t n) { return (batch * n * (int64_t)sizeof(TileLine) + 255) / 256 * 256; }
inline int64_t row_stat_bytes(int64_t planes, int64_t n, int64_t B) { return planes * n * 2 * B * 4; }

// fills a.line and a.tiles
hipError_t launch_line(const ScoredArgs& a, hipStream_t stream);
hipError_t launch_scored_forward(const ScoredArgs& a, hipStream_t stream);
// fills a.rows
hipError_t launch_row_stats(const ScoredArgs& a, hipStream_t stream);
hipError_t launch_scored_dq(const ScoredArgs& a, hipStream_t stream);
// `a` holds the transposed walk
hipError_t launch_scored_dkv(const ScoredArgs& a, hipStream_t stream);

}  // namespace ca
