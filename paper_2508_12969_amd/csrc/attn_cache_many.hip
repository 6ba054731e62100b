// Attention over a paged cache for many rows a sequence: frames, prompts, trees of drafts with grouped heads.  See attn_cache.h.
#include "attn_cache.h"

namespace ca {
namespace {

constexpr int kManyWaves = kManyRows / 32, kManyThreads = kManyWaves * 64, kManySlices = kManyStep / kSlice;

template <class S>
struct ManyLds {
  static constexpr int kStepBytes = kManyStep * S::kRowBytes;
  char x[2][kStepBytes], y[2][kStepBytes];  // [buffer]
  float frames[kManyWaves][kManyStep];
};

// A part of a tile's steps.
struct ManyItem {
  int32_t sequence, key_head, part, parts;
  int64_t tile, slot;   // of the sequence; where its pieces lie
  Sequence q;
  Walk<kManyStep> walk;
  bool found;
  // entry: parts are outermost, then key heads, then tiles, the last of which come first (in a causal order they see most)
  __device__ __forceinline__ ManyItem(const AttendArgs& a, LineLds& lds, int64_t entry) {
    const int64_t item = entry % (a.tiles * a.kv_heads), index = a.tiles - 1 - item % a.tiles;
    part = (int32_t)(entry / (a.tiles * a.kv_heads));
    key_head = (int32_t)(item / a.tiles);
    slot = item * a.most_parts;
    const auto weight = [&](const Sequence& s) { return (int64_t)row_tiles(a, s, kManyRows); };
    const SequenceLine<kManyThreads> line(a, lds, weight);
    found = line.find(a, lds, index, sequence, tile, weight);
    if (!found) return;
    q = sequence_at(a, sequence);
    walk = walk_of<kManyStep>(a, q, (int32_t)(tile * kManyRows / a.group), (int32_t)((min((tile + 1) * kManyRows, (int64_t)q.count * a.group) - 1) / a.group));
    parts = max(1, min((walk.count + a.part_steps - 1) / a.part_steps, a.most_parts));
  }
};

// A workgroup takes a tile of 128 rows, 32 a wave, over steps of 64 tokens that the waves copy together, a slice each.  Tiles of a key head are neighbours in the launch order, on one XCD, so that its
// L2 serves their copies.
template <int D>
__global__ __attribute__((amdgpu_flat_work_group_size(kManyThreads, kManyThreads), amdgpu_waves_per_eu(2, 2))) void many_rows_kernel(AttendArgs a) {
  typedef CacheShape<D> S;
  constexpr int kBlocks = kManyStep / 32;
  __shared__ ManyLds<S> lds;
  __shared__ LineLds found;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, g = lane >> 5;
  const int64_t total = gridDim.x;
  const ManyItem item(a, found, xcd_launch_order(blockIdx.x, total, xcd_chunk(total)));
  if (!item.found || item.part >= item.parts) return;
  const Sequence q = item.q;
  const Walk<kManyStep> walk = item.walk;
  const CacheRule rule(a);
  const int32_t size = (walk.count + item.parts - 1) / item.parts, from = min(walk.count, item.part * size), to = min(walk.count, from + size);
  // the wave's rows, and what all of them, or any, see, in scalar registers
  const int64_t first_row = item.tile * kManyRows + wave * 32, all_rows = (int64_t)q.count * a.group;
  const int rows = (int)max((int64_t)0, min((int64_t)32, all_rows - first_row));
  CacheRow own(a, rule, q, item.key_head, first_row + i);
  const int32_t own_row = own.row >= 0 ? own.row : q.first, own_head = own.row >= 0 ? own.head : item.key_head * a.group;
  asm volatile("" : "+v"(own.slope), "+v"(own.drafts));  // (waited for here, not in the loop)
  const OwnOperand<S, S::kContraction> query(static_cast<const char*>(a.q) + (own_row * a.q_strides.token + own_head * a.q_strides.head) * 2, g, nullptr);
  const int32_t first_token = (int32_t)(first_row / a.group), last_token = (int32_t)((first_row + max(rows, 1) - 1) / a.group);
  const View least = view_at(a, q, max(a.tree ? q.base : q.base + first_token, 0)), most = view_at(a, q, max(a.tree ? q.length - 1 : q.base + last_token, 0));
  const int32_t sure_prompt = prompt_end(a, q), sure_hi = q.base < 0 ? 0 : a.tree ? q.base : least.hi, sure_lo = most.lo;
  const int32_t any_lo = a.tree ? min(least.lo, max(q.base, 0)) : least.lo, any_hi = a.tree ? q.length : most.hi;

  const SliceCopy<S> copy(lane);
  const Fragments<S> frag(lane);
  const uint32_t lds_x = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.x[0] + wave * S::kSliceBytes;
  const uint32_t lds_y = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.y[0] + wave * S::kSliceBytes;
  SlicePlaces<kManySlices, kManyStep> places;
  auto issue = [&](int32_t step) {
    places.at_step(a, q, item.sequence, item.key_head, walk, step, from, to, lane, S::kRowBytes);
    const int64_t at = places.at(step, wave);
    copy(static_cast<const char*>(a.k) + at, lds_x + (uint32_t)(step & 1) * ManyLds<S>::kStepBytes);
    copy(static_cast<const char*>(a.v) + at, lds_y + (uint32_t)(step & 1) * ManyLds<S>::kStepBytes);
  };

  floatx16 sum[S::kDBlocks];
#pragma unroll
  for (auto& t : sum) t = splat(0.f);
  Softmax soft;
  uint32_t there = 0;
  if (from < to) {
    issue(from);
    there = places.mask(from);
  }
  for (int32_t step = from; step < to; ++step) {
    const int buffer = step & 1;
    const int32_t token = walk.token(step);
    const bool full = there == (1u << kManySlices) - 1 && token + kManyStep <= q.length;
    WAIT_VMCNT(0);
    if (!full) clear_rows<S>(lds.y[buffer], (there >> wave) & 1u ? max(wave * kSlice, q.length - token) : wave * kSlice, (wave + 1) * kSlice, lane);
    WAIT_LGKMCNT0();
    BARRIER();  // the step is there, and nobody reads the other buffer any more
    const uint32_t here = there;
    if (step + 1 < to) {
      issue(step + 1);
      there = places.mask(step + 1);
    }
    const bool prompt = token < sure_prompt;
    if (rows == 0 || (!prompt && (token >= any_hi || token + kManyStep <= any_lo))) continue;
    const LdsTile x = (LdsTile)lds.x[buffer], y = (LdsTile)lds.y[buffer];
    floatx16 p[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) p[b] = block_product<S>(frag, x, b, query, splat(0.f));
    if (rule.capped)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) cap_scores(rule, p[b]);
    if (a.slopes) {
      lds.frames[wave][lane] = frame_of_token(a, q, token + lane);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) bias_scores(own, p[b], lds.frames[wave], b, g);
    }
    const bool sure = token + kManyStep <= sure_hi && (token >= sure_lo || token + kManyStep <= sure_prompt) && full;
    if (!sure)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) hide_tokens(a, q, own, p[b], token + b * 32, (here >> (2 * b)) & 3u, g);
    soften<kBlocks, S::kDBlocks>(rule, soft, p, sum);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      bf16x8 weights[2];
      rounded(p[b], weights);
      block_sums<S>(frag, y, b, weights, sum);
    }
  }

  const float total_weight = sum_with_partner(soft.sum);
  if (i >= rows) return;
  if (item.parts == 1) {
    const int64_t at = (int64_t)own.row * a.heads + own.head;
    const bool real = total_weight != 0.f;
    store_columns<S::kDBlocks>(static_cast<char*>(a.out) + at * S::kRowBytes, g, 0, sum, 1.f / total_weight, real);
    if (g == 0) a.lse[at] = real ? (__builtin_fmaf(soft.ref, rule.c2, rule.offset) + __builtin_amdgcn_logf(total_weight)) * 0.6931471805599453f : kMinusInf;
    return;
  }
  float* const piece = a.pieces + ((item.slot + item.part) * kManyRows + wave * 32 + i) * piece_row(D);
#pragma unroll
  for (int db = 0; db < S::kDBlocks; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<floatx4*>(piece + db * 32 + 8 * j + 4 * g) = floatx4{sum[db][4 * j], sum[db][4 * j + 1], sum[db][4 * j + 2], sum[db][4 * j + 3]};
  if (g == 0) *reinterpret_cast<float2*>(piece + D) = float2{soft.ref, total_weight};
}

// A workgroup takes some rows of a tile.
template <int D>
__global__ __launch_bounds__(kManyThreads) void many_rows_join_kernel(AttendArgs a) {
  __shared__ JoinLds<D, kManyThreads> lds;
  __shared__ LineLds found;
  const ManyItem item(a, found, blockIdx.x);
  if (!item.found || item.parts == 1) return;
  const int64_t first_row = item.tile * kManyRows;
  const int rows = (int)min((int64_t)kManyRows, (int64_t)item.q.count * a.group - first_row);
  for (int r = blockIdx.y; r < rows; r += gridDim.y)
    join_row<D>(a, item.q, item.key_head, first_row + r, item.parts, lds, [&](int k) { return a.pieces + ((item.slot + k) * kManyRows + r) * piece_row(D); });
}

template <int D>
hipError_t launch_many_rows(const AttendArgs& a, hipStream_t stream) {
  const int64_t items = a.tiles * a.kv_heads, workgroups = items * a.most_parts;
  if (workgroups < 1 || workgroups > 0xffffff) return hipErrorInvalidValue;  // (2^32 threads)
  many_rows_kernel<D><<<(unsigned)workgroups, kManyThreads, 0, stream>>>(a);
  if (a.most_parts > 1) many_rows_join_kernel<D><<<dim3((unsigned)items, 8), kManyThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_many(const AttendArgs& a, hipStream_t stream) { return a.D == 64 ? launch_many_rows<64>(a, stream) : launch_many_rows<128>(a, stream); }

}  // namespace ca
