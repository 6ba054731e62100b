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
  int32_t width, row_bytes;
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
  int64_t tiles;               // most row tiles that the sequences can have together
};

hipError_t launch_append(const AppendArgs& a, bool bf16, bool normed, hipStream_t stream);
hipError_t launch_keep(const KeepArgs& a, hipStream_t stream);
hipError_t launch_attend(const AttendArgs& a, hipStream_t stream);

}  // namespace ca
