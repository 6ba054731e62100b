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

constexpr int kKeepThreads = 256;

// The sequence that a row of the packed tensors belongs to: the last one that starts at or before it.
__device__ __forceinline__ int32_t sequence_of_row(const CacheArgs& a, int32_t row) {
  int32_t lo = 0, hi = a.sequences;  // starts[lo] <= row < starts[hi], where starts ascends
  while (hi - lo > 1) {
    const int32_t mid = (int32_t)(((uint32_t)lo + (uint32_t)hi) / 2);
    if (a.starts[mid] <= row) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Heads are walked in the order q, k, v; blockIdx.y takes heads_per_block of them.
template <class T, Pairing kPairing, bool kNorm>
__global__ __launch_bounds__(kRowThreads) void append_kernel(AppendArgs a, int heads_per_block) {
  constexpr int kVec = Row<T>::kVec, kHeads = 4;
  typedef typename Row<T>::Chunk Chunk;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Part p = part_of<T>(a, lane);
  const int64_t at = (((int64_t)blockIdx.x * kRowWaves + wave) << (6 - p.lanes_log2)) + p.row;
  const int32_t row = (int32_t)min(at, (int64_t)a.tokens - 1);
  const int32_t s = sequence_of_row(a, row);
  const Sequence seq = sequence_at(a, s);
  const bool live = p.live && at < a.tokens && row >= seq.first && row < seq.first + seq.count;
  const int32_t token = seq.base + (row - seq.first);
  const bool exists = live && token >= 0 && token < seq.length;
  const int32_t page = exists ? page_at(a, s, token) : -1, slot = exists ? token % a.page_tokens : 0;

  Turn<kVec> turn;
  no_turn(turn);
  if (a.angles && exists) {
    int where[3];
    if (a.where) {
#pragma unroll
      for (int i = 0; i < 3; ++i) where[i] = a.where[(int64_t)row * 3 + i];
    } else {
      const int32_t behind = token - seq.origin, line = behind / a.frame_w;
      const int32_t of[3] = {line / a.frame_h, line % a.frame_h, behind % a.frame_w};
#pragma unroll
      for (int i = 0; i < 3; ++i) where[i] = behind < 0 ? -1 : (int)min((int64_t)a.origin[i] + of[i], (int64_t)0x7fffffff);
    }
    make_turn<T, kPairing != kNeighbours>(a, p, where, turn);
  }
  const Exchange<T> exchange(a, p, lane);
  const int h0 = blockIdx.y * heads_per_block, h1 = min(a.heads + 2 * a.kv_heads, h0 + heads_per_block);

#pragma unroll
  for (int tensor = 0; tensor < 2; ++tensor) {
    const int first = tensor ? a.heads : 0, count = tensor ? a.kv_heads : a.heads, from = max(h0 - first, 0), to = min(h1 - first, count);
    if (from >= to) continue;
    const TokenStrides ss = tensor ? a.k_strides : a.q_strides;
    const T* __restrict__ src = static_cast<const T*>(tensor ? a.k_new : a.q) + row * ss.token;
    const bool store = tensor ? page >= 0 : live;
    const int64_t dst_head = tensor ? (int64_t)a.page_tokens * a.D : a.D;
    T* __restrict__ dst = static_cast<T*>(tensor ? a.k : a.q_out) + (tensor ? cache_row(a, max(page, 0), 0, slot) * a.D : (int64_t)row * a.heads * a.D) + p.first;
    float own_c[kVec], other_c[kVec];  // y = own_c x + other_c partner (times r)
#pragma unroll
    for (int e = 0; e < kVec; ++e) own_c[e] = turn.c[e], other_c[e] = turn.s[e];
    if constexpr (kNorm) {
      float w[kVec], wp[kVec];
      load_weights<T, kPairing>(a, p, tensor ? a.k_weight : a.q_weight, w, wp);
#pragma unroll
      for (int e = 0; e < kVec; ++e) own_c[e] *= w[e], other_c[e] = from_partner(other_c[e], wp[e]);
    }
    for (int h = from; h < to; h += kHeads) {
      Chunk own[kHeads], other[kHeads];
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        if (h + i < to && live) {
          const T* r = src + (h + i) * ss.head;
          own[i] = *reinterpret_cast<const Chunk*>(r + p.first);
          if constexpr (kPairing == kApart) other[i] = load_partner<T>(a, p, r);
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) own[i][e] = other[i][e] = (T)0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        if (h + i >= to) break;
        if constexpr (kPairing == kHalves) other[i] = exchange(own[i]);
        float r = 1.f;
        if constexpr (kNorm) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < kVec; ++e) sum += live ? (float)own[i][e] * (float)own[i][e] : 0.f;
          r = rsqrtf(row_sum(sum, p.lanes_log2) / a.D + a.eps);
        }
        Chunk y;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float x = (float)own[i][e], xp = kPairing == kNeighbours ? (float)own[i][e ^ 1] : (float)other[i][e];
          y[e] = (T)(r * (own_c[e] * x + from_partner(other_c[e], xp)));
        }
        if (store) *reinterpret_cast<Chunk*>(dst + (h + i) * dst_head) = y;
      }
    }
  }

  const int first = a.heads + a.kv_heads, from = max(h0 - first, 0), to = min(h1 - first, a.kv_heads);
  const T* __restrict__ src = static_cast<const T*>(a.v_new) + row * a.v_strides.token + p.first;
  T* __restrict__ dst = static_cast<T*>(a.v) + cache_row(a, max(page, 0), 0, slot) * a.D + p.first;
  for (int h = from; h < to; h += kHeads) {
    Chunk own[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (h + i < to && page >= 0) own[i] = *reinterpret_cast<const Chunk*>(src + (h + i) * a.v_strides.head);
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
      if (h + i < to && page >= 0) *reinterpret_cast<Chunk*>(dst + (int64_t)(h + i) * a.page_tokens * a.D) = own[i];
  }
}

// A workgroup moves the rows of one head of one sequence, keys or values: all of them are loaded before the first is stored.
__global__ __launch_bounds__(kKeepThreads) void keep_kernel(KeepArgs a) {
  constexpr int kItems = 16;  // 64 rows of at most 64 chunks
  const int32_t s = blockIdx.x, head = blockIdx.y, chunks = a.row_bytes / 16;
  char* const pages = static_cast<char*>(blockIdx.z ? a.v : a.k);
  const Sequence seq = sequence_at(a, s);
  const int count = max(0, min(min(a.counts[s], a.width), seq.count)), items = count * chunks;
  typedef __attribute__((ext_vector_type(4))) int intx4;
  intx4 held[kItems];
  char* to[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int item = i * kKeepThreads + threadIdx.x, j = item / chunks, chunk = item - j * chunks;
    to[i] = nullptr;
    if (item >= items) continue;
    const int32_t from = a.kept[(int64_t)s * a.width + j];
    if (from < 0 || from >= seq.count || from == j || seq.base + j < 0 || seq.base + from < 0) continue;
    const int32_t source = seq.base + from, target = seq.base + j;
    const int32_t source_page = page_at(a, s, source), target_page = page_at(a, s, target);
    if (source_page < 0 || target_page < 0) continue;
    held[i] = *reinterpret_cast<const intx4*>(pages + cache_row(a, source_page, head, source % a.page_tokens) * a.row_bytes + chunk * 16);
    to[i] = pages + cache_row(a, target_page, head, target % a.page_tokens) * a.row_bytes + chunk * 16;
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

hipError_t launch_keep(const KeepArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.sequences, (unsigned)a.kv_heads, 2);
  if (a.sequences > 0xffffff || a.kv_heads > 65535) return hipErrorInvalidValue;
  keep_kernel<<<grid, kKeepThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ca
