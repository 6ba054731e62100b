// New tokens into a paged cache of keys and values, with norm and rotation on the way, and moves within it.
//
//   k' = R(p) (w k r),  r = (mean(k^2) + eps)^-1/2,  v as it is: to slot j % page_tokens of page table[s][j / page_tokens];  q' likewise, to a tensor of its own.
//
// Bound: HBM, every row (token, head) is read once and written once.  As in rotary.hip a row lies in D / 8 lanes (bf16; D / 4 for fp32), a wave takes 64 / lanes tokens and walks over their
// heads, those of queries, keys and values one after the other, with angles and places made once per token.
#include <algorithm>

#include "cache_tokens.h"
#include "rows.h"

namespace ca {
namespace {

constexpr int kKeepThreads = 256, kKeepItems = 16, kKeepFewItems = 4;  // rows of a thread: 64 of 64 chunks are four at once

// The sequence that a row of the packed tensors belongs to: the last one that starts at or before it.  A wave's rows, first to last, follow each other: its lanes look at 64 sequences at a time
// for that of the first row, those of the others are among the next ones.
__device__ __forceinline__ int32_t sequence_of_row(const CacheArgs& a, int32_t first, int32_t last, int32_t row, int lane) {
  int32_t base = 0, count = a.sequences;  // starts[base] <= first, where starts ascends, and that of the sequence after these is past it
  while (true) {
    const int32_t stride = (count + 63) / 64, start = a.starts[base + min(lane * stride, count - 1)];
    const int found = 63 - (int)__builtin_clzll(__builtin_amdgcn_ballot_w64(start <= first) | 1);
    if (stride > 1) {
      const int32_t from = min(found * stride, count - 1);
      base += from;
      count = min(stride, count - from);
      continue;
    }
    int32_t s = base + min(found, count - 1), k = min(found, count - 1) + 1;
    for (; k < min(count, 64); ++k) {
      const int32_t next = __builtin_amdgcn_readlane(start, k);
      if (next > last) return s;
      if (next <= row) s = base + k;
    }
    for (k += base; k < a.sequences && a.starts[k] <= last; ++k)
      if (a.starts[k] <= row) s = k;
    return s;
  }
}

// Heads are walked in the order q, k, v; blockIdx.y takes heads_per_block of them.  kHeads of them are loaded while those before are computed, the first ones while the wave looks for its sequences.
template <class T, Pairing kPairing, bool kNorm>
__global__ __launch_bounds__(kRowThreads) void append_kernel(AppendArgs a, int heads_per_block) {
  constexpr int kVec = Row<T>::kVec, kHeads = 4;
  typedef typename Row<T>::Chunk Chunk;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Part p = part_of<T>(a, lane);
  const int64_t at = (((int64_t)blockIdx.x * kRowWaves + wave) << (6 - p.lanes_log2)) + p.row;
  const int32_t row = (int32_t)min(at, (int64_t)a.tokens - 1), first_row = (int32_t)min(at - p.row, (int64_t)a.tokens - 1);  // (first_row: of the wave)
  const int32_t last_row = (int32_t)min(at - p.row + ((1 << (6 - p.lanes_log2)) - 1), (int64_t)a.tokens - 1);
  const int h0 = blockIdx.y * heads_per_block, h1 = min(a.heads + 2 * a.kv_heads, h0 + heads_per_block);
  const int keys = a.heads, values = a.heads + a.kv_heads;  // where they begin
  const int64_t q_at = row * a.q_strides.token, k_at = row * a.k_strides.token, v_at = row * a.v_strides.token;
  auto source = [&](int h) {
    return h < keys     ? static_cast<const T*>(a.q) + q_at + h * a.q_strides.head
           : h < values ? static_cast<const T*>(a.k_new) + k_at + (h - keys) * a.k_strides.head
                        : static_cast<const T*>(a.v_new) + v_at + (h - values) * a.v_strides.head;
  };
  Chunk next[kHeads];
  auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (h + i < h1) next[i] = *reinterpret_cast<const Chunk*>(source(h + i) + p.first);
  };
  load(h0);
  Chunk q_weight, k_weight;
#pragma unroll
  for (int e = 0; e < kVec; ++e) q_weight[e] = k_weight[e] = (T)1.f;
  if (kNorm && a.q_weight && h0 < keys) q_weight = *reinterpret_cast<const Chunk*>(static_cast<const T*>(a.q_weight) + p.first);
  if (kNorm && a.k_weight && h0 < values && h1 > keys) k_weight = *reinterpret_cast<const Chunk*>(static_cast<const T*>(a.k_weight) + p.first);

  const int32_t s = sequence_of_row(a, __builtin_amdgcn_readfirstlane(first_row), __builtin_amdgcn_readfirstlane(last_row), row, lane);
  const Sequence seq = sequence_at(a, s);
  const bool live = p.live && at < a.tokens && row >= seq.first && row < seq.first + seq.count;
  const int32_t token = seq.base + (row - seq.first);
  const bool exists = live && token >= 0 && token < seq.length;
  const int32_t entry = exists ? divided(token, a.page_tokens) : 0, slot = exists ? token - entry * a.page_tokens : 0;
  const int32_t in_table = a.table[(int64_t)s * a.table_width + entry];  // (looked at when it is there)

  Turn<kVec> turn;
  no_turn(turn);
  if (a.angles && exists && h0 < values) {
    int where[3];
    if (a.where) {
#pragma unroll
      for (int i = 0; i < 3; ++i) where[i] = a.where[(int64_t)row * 3 + i];
    } else {
      const int32_t behind = token - seq.origin, line = behind < 0 ? 0 : divided(behind, a.frame_w), frame = divided(line, a.frame_h);
      const int32_t of[3] = {frame, line - frame * a.frame_h, behind - line * a.frame_w};
#pragma unroll
      for (int i = 0; i < 3; ++i) where[i] = behind < 0 ? -1 : (int)min((int64_t)a.origin[i] + of[i], (int64_t)0x7fffffff);
    }
    make_turn<T, kPairing != kNeighbours>(a, p, where[0], where[1], where[2], turn);
  }
  const Exchange<T> exchange(a, p, lane);
  // y = own_c x + other_c partner (times r), of queries and of keys
  float q_own[kVec], q_other[kVec], k_own[kVec], k_other[kVec];
  auto weigh = [&](const void* weight, const Chunk& w, float (&own_c)[kVec], float (&other_c)[kVec]) {
    Chunk wp;
    if constexpr (kPairing == kHalves) wp = exchange(w);
    if constexpr (kPairing == kApart) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) wp[e] = (T)1.f;
      if (kNorm && weight) wp = load_partner<T>(a, p, static_cast<const T*>(weight));
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      own_c[e] = turn.c[e], other_c[e] = turn.s[e];
      if (kNorm) own_c[e] *= (float)w[e], other_c[e] = from_partner(other_c[e], kPairing == kNeighbours ? (float)w[e ^ 1] : (float)wp[e]);
    }
  };
  weigh(a.q_weight, q_weight, q_own, q_other);
  weigh(a.k_weight, k_weight, k_own, k_other);
  const int32_t page = exists && in_table >= 0 && in_table < a.num_pages ? in_table : -1;
  T* const q_out = static_cast<T*>(a.q_out) + (int64_t)row * a.heads * a.D + p.first;
  const int64_t in_page = cache_row(a, max(page, 0), 0, slot) * a.D + p.first, page_head = (int64_t)a.page_tokens * a.D;

  for (int h = h0; h < h1; h += kHeads) {
    Chunk own[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) own[i] = next[i];
    load(h + kHeads);
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      const int head = h + i;
      if (head >= h1) break;
      if (head >= values) {
        if (page >= 0) __builtin_nontemporal_store(own[i], reinterpret_cast<Chunk*>(static_cast<T*>(a.v) + in_page + (head - values) * page_head));
        continue;
      }
      const bool key = head >= keys;
      Chunk other;
      if constexpr (kPairing == kHalves) other = exchange(own[i]);
      if constexpr (kPairing == kApart) other = load_partner<T>(a, p, source(head));
      float r = 1.f;
      if constexpr (kNorm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum += p.live ? (float)own[i][e] * (float)own[i][e] : 0.f;
        r = rsqrtf(row_sum(sum, p.lanes_log2) / a.D + a.eps);
      }
      Chunk y;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float x = (float)own[i][e], xp = kPairing == kNeighbours ? (float)own[i][e ^ 1] : (float)other[e];
        y[e] = (T)(r * ((key ? k_own[e] : q_own[e]) * x + from_partner(key ? k_other[e] : q_other[e], xp)));
      }
      if (key ? page >= 0 : live)
        __builtin_nontemporal_store(y, reinterpret_cast<Chunk*>(key ? static_cast<T*>(a.k) + in_page + (head - keys) * page_head : q_out + head * (int64_t)a.D));
    }
  }
}

// A workgroup moves the rows of some heads of one sequence, keys or values: where they go is looked up once, then all are loaded before the first is stored.  Bound: latency (counts, drafts, table
// and rows, one after the other).
template <int kItems>
__global__ __launch_bounds__(kKeepThreads) void keep_kernel(KeepArgs a) {
  __shared__ int64_t moves[kMostDrafts][2];  // rows of head 0: from, to; -1: this one stays
  const int32_t s = blockIdx.x, chunks = a.row_bytes / 16, rows_at_once = kKeepThreads / chunks, first_head = blockIdx.y * a.heads_per_block;
  const int32_t row = divided(threadIdx.x, chunks), chunk = threadIdx.x - row * chunks;
  char* const pages = static_cast<char*>(blockIdx.z ? a.v : a.k) + chunk * 16;
  const int32_t from = threadIdx.x < (unsigned)a.width ? a.kept[(int64_t)s * a.width + threadIdx.x] : -1;  // (asked for beside the counts)
  const Sequence seq = sequence_at(a, s);
  const int32_t count = max(0, min(min(a.counts[s], a.width), seq.count)), rows = min(a.heads_per_block, a.kv_heads - first_head) * count;
  if (count == 0) return;
  if (threadIdx.x < count) {
    const int32_t j = threadIdx.x;
    const bool moving = from >= 0 && from < seq.count && from != j && seq.base + j >= 0 && seq.base + from >= 0;
    const int32_t source = moving ? seq.base + from : 0, target = moving ? seq.base + j : 0;
    const int32_t source_page = page_at(a, s, source), target_page = page_at(a, s, target);
    const bool there = moving && source_page >= 0 && target_page >= 0;
    moves[j][0] = there ? cache_row(a, source_page, first_head, source - divided(source, a.page_tokens) * a.page_tokens) : -1;
    moves[j][1] = there ? cache_row(a, target_page, first_head, target - divided(target, a.page_tokens) * a.page_tokens) : -1;
  }
  __syncthreads();
  typedef __attribute__((ext_vector_type(4))) int intx4;
  intx4 held[kItems];
  char* to[kItems];
  int32_t head = divided(row, count), j = row - head * count;  // of the thread's row; the next one is rows_at_once further on
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    to[i] = nullptr;
    if (i * rows_at_once >= rows) continue;
    if (row < rows_at_once && row + i * rows_at_once < rows && moves[j][0] >= 0) {
      held[i] = *reinterpret_cast<const intx4*>(pages + (moves[j][0] + (int64_t)head * a.page_tokens) * a.row_bytes);
      to[i] = pages + (moves[j][1] + (int64_t)head * a.page_tokens) * a.row_bytes;
    }
    for (j += rows_at_once; j >= count; j -= count) ++head;
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i) asm volatile("" : "+v"(held[i]));  // (loaded before the barrier)
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kItems; ++i)
    if (to[i]) *reinterpret_cast<intx4*>(to[i]) = held[i];
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, bool bf16, bool normed, hipStream_t stream) {
  const int rows = kRowWaves << (6 - lanes_log2(a, bf16)), heads = a.heads + 2 * a.kv_heads;
  const int64_t blocks = ((int64_t)a.tokens + rows - 1) / rows;
  int split = 1;  // as rows_kernel: 2048 workgroups fill the card
  while (split < heads && blocks * split < 2048) split *= 2;
  const int per = (heads + std::min(split, heads) - 1) / std::min(split, heads);
  const dim3 grid((unsigned)blocks, (unsigned)((heads + per - 1) / per));
  if (blocks > 0xffffff || grid.y > 65535) return hipErrorInvalidValue;  // (2^32 threads in x)
  with_pairing(a, bf16, [&](auto type, auto pairing) {
    if (normed) append_kernel<decltype(type), decltype(pairing)::value, true><<<grid, kRowThreads, 0, stream>>>(a, per);
    else append_kernel<decltype(type), decltype(pairing)::value, false><<<grid, kRowThreads, 0, stream>>>(a, per);
  });
  return hipGetLastError();
}

hipError_t launch_keep(const KeepArgs& args, hipStream_t stream) {
  KeepArgs a = args;
  const int chunks = a.row_bytes / 16, rows_at_once = kKeepThreads / chunks;
  if (a.width > kMostDrafts || rows_at_once * kKeepItems < kMostDrafts || a.sequences > 0xffffff || a.kv_heads > 65535) return hipErrorInvalidValue;
  // four rows a thread, if all of the width is used: 256 sequences x 20 heads, one / eight heads a workgroup 19.6 / 8.4 us, 16 sequences x 8 heads 3.2 / 4.4
  a.heads_per_block = std::max(1, std::min(a.kv_heads, kKeepFewItems * rows_at_once / a.width));
  const dim3 grid((unsigned)a.sequences, (unsigned)((a.kv_heads + a.heads_per_block - 1) / a.heads_per_block), 2);
  // where four are all there are, more waves have registers: 256 sequences x 20 heads with room for sixteen / four 7.7 / 6.5 us
  if (a.heads_per_block * a.width <= kKeepFewItems * rows_at_once) keep_kernel<kKeepFewItems><<<grid, kKeepThreads, 0, stream>>>(a);
  else keep_kernel<kKeepItems><<<grid, kKeepThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ca
