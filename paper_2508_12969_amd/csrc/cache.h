// Launch interface of the kernels over a paged cache of keys and values (cache.hip, attn_cache.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "rotary.h"

namespace ca {

constexpr int kMostDrafts = 64;  // of a sequence: the bits of a tree's word

struct CacheArgs {
  void *k, *v;                 // [num_pages][kv_heads][page_tokens][D]
  int64_t num_pages;
  int32_t page_tokens, kv_heads, sequences, table_width, tokens;
  int32_t frame_h, frame_w, span;  // span: tokens of a frame
  const int32_t *table, *lengths, *starts, *origins;
};

struct TokenStrides {
  int64_t token, head;  // elements
};

struct AppendArgs : CacheArgs, RowRule {
  const void *q, *k_new, *v_new;
  TokenStrides q_strides, k_strides, v_strides;
  void* q_out;
  int32_t heads;               // of q; 0: no queries
  const void *q_weight, *k_weight;
  int32_t origin[3];
  const int32_t* where;        // [tokens][3] or null
};

struct KeepArgs : CacheArgs {
  const int32_t *kept, *counts;
  int32_t width, row_bytes, heads_per_block;
};

// How a launch is shared out among workgroups, see Share.
enum CacheWay { kItems, kShares, kParts };

// An item (a tile of rows and a key head) that is cut.
struct CacheSplit {
  int32_t first;            // row of the packed tensors of its sequence's first new token
  int32_t key_head, first_row, rows;
  int32_t pieces;           // 0: there is none at this place
  int32_t fine;             // how its capped scores are held, see CacheRule
};

struct AttendArgs : CacheArgs {
  const void* q;
  TokenStrides q_strides;
  void* out;
  float* lse;
  int32_t heads, group, D;     // group: query heads of a key head
  float scale, cap;            // cap 0: none
  const float* slopes;         // [heads] or null
  int32_t causal, window;
  const uint64_t* tree;        // [tokens] or null
  bool many;                   // rows a sequence: tiles of kManyRows, else of kFewRows
  int64_t tiles;               // most row tiles that the sequences can have together
  CacheWay way;
  int32_t workgroups, least_steps;  // kShares: workgroups, least steps of a share
  int32_t part_steps, most_parts;   // kParts: items of more steps are cut
  CacheSplit* splits;          // workspace: [workgroups], or (kParts) [tiles * kv_heads]
  float* pieces;               // workspace: [workgroups][2], or [tiles * kv_heads][most_parts], of [rows of a tile][piece_row(D)]
};

// A few rows a sequence are taken in tiles of 32, which read their keys and values in steps of 32 tokens.
constexpr int kFewRows = 32, kFewStep = 32;
// Workgroups that the device holds at a time: one per compute unit at head dim 128 (its buffers fill the LDS), two at 64.
constexpr int few_workgroups(int D) { return D == 128 ? 256 : 512; }
// Many rows are taken in tiles of 128, with steps of 64 tokens that the waves of a workgroup share.
constexpr int kManyRows = 128, kManyStep = 64;
// Workgroups that the device holds at a time: with shares of a line, and of items or parts (many_waves).
constexpr int kManyWorkgroups = 512;
constexpr int many_places(int D) { return D == 64 ? 768 : 512; }
// Sums of a row: D, then the reference of the exponent and the sum of weights; rows begin at 16 bytes, and in different banks of LDS.
constexpr int piece_row(int D) { return D + 4; }

hipError_t launch_append(const AppendArgs& a, bool bf16, bool normed, hipStream_t stream);
hipError_t launch_keep(const KeepArgs& a, hipStream_t stream);
hipError_t launch_attend_few(const AttendArgs& a, hipStream_t stream);
hipError_t launch_attend_many(const AttendArgs& a, hipStream_t stream);
hipError_t launch_attend_f32(const AttendArgs& a, hipStream_t stream);

}  // namespace ca
