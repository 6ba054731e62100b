// Launch interface of the kernels of scored attention (attn_scored*.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <mutex>
#include <vector>

#include "layout.h"
#include "tokens.h"

namespace ca {

// What a tile's tokens have in common, over the tokens that are there (in the grid, with a document that is not negative).
struct TileLine {
  int32_t doc_min, doc_max;      // min > max: none is there
  float pos_min, pos_max, limit_min, limit_max;
  int32_t whole;                 // every token of the grid is there
  int32_t unused;
};

// Rows of `line` per tile, of B words each.
enum LineRow { kLinePosition = 0, kLineDocument = 1, kLineLimit = 2, kLineRows = 4 };

// The columns of a workgroup are a group: 128 tokens of one head, a tile of 128 or two neighbours of 64.  What they walk over, the union of the tiles' lists
// (rows of the layout for queries, columns for keys), is a run of steps of 64 tokens, one word each: tile id | half of the tile << 24 | its padding class << 25 (four
// bits) | 1 << 29 if pairs have to be compared | 1 << 30 if the first tile of the group keeps it | 1 << 31 if the second does.  Halves without a token are left out.
//
// Calls whose token arrays hide something are given runs of their own, made on the device from the arrays (visit_kernel): steps without a visible pair are
// left out, and those with nothing but visible pairs of tokens have bit 29 clear.
//
// A workgroup takes an item, a group's run or a part of it; where a group has several, each leaves its sums as a share, which a second kernel adds up in
// their order.
constexpr int kGroupTokens = 128;
constexpr float kLeastCap = 1.f / 65536, kMostCap = 4096.f;
struct ScoredItem {
  int64_t first;               // of its steps
  int32_t count, group, share; // share: -1 for a group that is one item
  int32_t batch;               // of items made on the device
};
struct ScoredMerge {
  int32_t group, first_share, shares, batch;
};
struct ScoredWalk {
  std::vector<uint32_t> steps;
  std::vector<int64_t> first;       // [groups + 1] runs
  // of calls that visit all of it: one batch entry
  std::vector<ScoredItem> items;    // longest first
  std::vector<ScoredMerge> merges;
  int64_t shares = 0;
  bool made = false;
  unsigned char* block = nullptr;   // device memory of all
  uint32_t* dev_steps = nullptr;
  int64_t* dev_first = nullptr;
  ScoredItem* dev_items = nullptr;
  ScoredMerge* dev_merges = nullptr;
};
struct ScoredState {
  std::mutex mutex;
  ScoredWalk rows, columns;  // of the layout
  ~ScoredState();
};
// Steps of 64 tokens that a workgroup's other work is worth (start, own tokens, results), and what a share adds, from launches of one run length: a run of
// no steps takes about 10 us, a step 1.0 to 2.0.
constexpr int64_t kItemSteps = 6, kShareSteps = 4, kMergeSteps = 4, kLeastSteps = 8;
// Workgroups that the device holds at a time: two per compute unit at head dim 128, three (gradients) or four (forward) at 64.
constexpr int64_t scored_places(int64_t D) { return D == 64 ? 768 : 512; }
// Items made on the device: runs longer than max(kLeastSteps, all steps / places) are cut, so there are fewer than `places` of them and at most twice as many shares.
constexpr int64_t most_merges(int64_t D) { return scored_places(D); }
constexpr int64_t most_shares(int64_t D) { return 2 * scored_places(D); }

// Sums of a share, per 32-token wave: four figures of every lane, and one (forward) or two (gradients) sums of D channels.
constexpr int64_t share_floats(int64_t D, int sums) { return kGroupTokens / 32 * (4 * 64 + sums * D * 32); }

// Runs and items made on the device, in the workspace.
struct VisitCounts {
  int32_t items, merges;
};
struct Visits {
  const uint32_t* from;        // the layout's steps
  const int64_t* first;        // [groups + 1]
  int64_t groups, total;       // of a batch entry: groups, steps
  int32_t keys;                // groups are of keys
  uint32_t* steps;             // [batch][total]
  int32_t* counts;             // [batch * groups]
  ScoredItem* items;           // [batch * groups + most_shares(D)]
  ScoredMerge* merges;         // [most_merges(D)]
  VisitCounts* header;
};

struct ScoredArgs : GridArgs {
  const void *q, *k, *v, *dout, *o;  // [batch, heads, N_pad, D] tile order, bf16
  void *out, *dq, *dk, *dv;
  const float* lse_in;         // backward: the forward call's
  float* lse;                  // forward: [batch, heads, N_pad]
  // the walk, see ScoredWalk
  const uint32_t* steps;
  const ScoredItem* items;
  const ScoredMerge* merges;
  const VisitCounts* header;   // where items were made on the device: how many there are; else null
  int64_t num_items, num_merges, shares;  // of one batch entry, or (header) most of all
  float* share_sums;           // workspace: [shares of all batch entries][sums of a share]
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
  float* rows;                 // backward: [batch * heads][n][2][B]: log-sum-exp in powers of two, minus delta (put right by dQ)
};

// bytes of the parts of the workspace, each a multiple of 256
inline int64_t line_bytes(int64_t batch, int64_t n, int64_t B) { return (batch * n * kLineRows * B * 4 + 255) / 256 * 256; }
inline int64_t tile_line_bytes(int64_t batch, int64_t n) { return (batch * n * (int64_t)sizeof(TileLine) + 255) / 256 * 256; }
inline int64_t row_stat_bytes(int64_t planes, int64_t n, int64_t B) { return planes * n * 2 * B * 4; }

// fills a.line and a.tiles
hipError_t launch_line(const ScoredArgs& a, hipStream_t stream);
// makes the runs and items of one or two walks
hipError_t launch_visits(const ScoredArgs& a, const Visits* visits, int count, hipStream_t stream);
hipError_t launch_scored_forward(const ScoredArgs& a, hipStream_t stream);
// fills a.rows
hipError_t launch_row_stats(const ScoredArgs& a, hipStream_t stream);
hipError_t launch_scored_dq(const ScoredArgs& a, hipStream_t stream);
// `a` holds the walk over the layout's columns
hipError_t launch_scored_dkv(const ScoredArgs& a, hipStream_t stream);

}  // namespace ca
