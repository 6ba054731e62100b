// Attention over a paged cache for many rows a sequence: frames, prompts, trees of drafts with grouped heads.  See attn_cache.h.
#include "attn_cache.h"

namespace ca {
namespace {

constexpr int kManySlices = kManyStep / kSlice;
constexpr int kManyItemCost = 4;     // steps that a workgroup does in the time that it takes to begin an item; 16 trees with 2 / 3 / 4: 88 / 82 / 78 us
constexpr int kPlacedSteps = 128;    // whose slices are looked up together

template <class S, int kWaves, int kBuffers>
struct ManyLds {
  static constexpr int kStepBytes = kManyStep * S::kRowBytes;
  char x[kBuffers][kStepBytes], y[kBuffers][kStepBytes];
  float frames[kWaves][kManyStep];
  int64_t places[kPlacedSteps * kManySlices];  // where slices lie, -1: not there
};

// A workgroup takes a tile of rows, 32 a wave, over steps of 64 tokens that the waves copy together, some slices each.  Copies are kBuffers - 1 steps ahead.
template <int D, bool kLine, int kWaves, int kBuffers>
__global__ __attribute__((amdgpu_flat_work_group_size(kWaves * 64, kWaves * 64), amdgpu_waves_per_eu(2, 2))) void many_rows_kernel(AttendArgs a) {
  typedef CacheShape<D> S;
  typedef ManyLds<S, kWaves, kBuffers> Lds;
  constexpr int kRows = kWaves * 32, kThreads = kWaves * 64, kBlocks = kManyStep / 32, kAhead = kBuffers - 1;
  static_assert(kWaves == 4 || kWaves == 8, "a wave copies a slice of keys and one of values, or one of either");
  constexpr int kCopies = (kWaves == 4 ? 2 : 1) * S::kSliceLoads;  // of a step, a wave's
  __shared__ Lds lds;
  __shared__ LineLds found;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, g = lane >> 5;
  // Neighbours on the line, or tiles of one key head, are on one XCD (a frame of 13 tiles a head in chunks of 13 / as the ids come 391 / 418 us, 85 tiles in chunks of 64 / 8 4.90 / 5.09 ms).
  const int64_t total = gridDim.x, workgroup = a.way == kShares ? blockIdx.x % 8 * (total / 8) + blockIdx.x / 8 : xcd_launch_order(blockIdx.x, total, min(a.tiles, kXcdChunk));
  Share<kRows, kManyStep, kThreads, kManyItemCost> share;
  if (!share.begin(a, found, workgroup)) {
    share.leave(a, false);
    return;
  }
  const CacheRule rule(a);
  const SliceCopy<S> copy(lane);
  const Fragments<S> frag(lane);
  const int slice = wave % kManySlices;
  const uint32_t lds_x = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.x[0] + slice * S::kSliceBytes;
  const uint32_t lds_y = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.y[0] + slice * S::kSliceBytes;
  while (true) {
    const Sequence& q = share.q;
    const Walk<kManyStep> walk = share.walk;
    const int32_t from = min(walk.count, share.done), to = min(walk.count, share.done + share.steps);
    // Places of the slices from `first` on.
    auto look_up = [&](int32_t first) {
      for (int at = threadIdx.x; at < kPlacedSteps * kManySlices; at += kThreads) {
        const int32_t step = first + at / kManySlices;
        const int64_t token = step < to ? (int64_t)walk.token(step) + at % kManySlices * kSlice : q.length;
        int64_t place = -1;
        if (token < q.length) {
          const int32_t page = page_at(a, share.sequence, (int32_t)token);
          if (page >= 0) place = cache_row(a, page, share.key_head, (int32_t)token - divided((int32_t)token, a.page_tokens) * a.page_tokens) * S::kRowBytes;
        }
        lds.places[at] = place;
        if (step >= to) break;
      }
    };
    uint32_t there = 0;  // four bits a step that is asked for: which of its slices are there
    int asked = 0;
    auto issue = [&](int32_t step) {
      const int64_t mine = lds.places[((step - from) % kPlacedSteps) * kManySlices + lane % kManySlices];
      there |= ((uint32_t)__builtin_amdgcn_ballot_w64(mine >= 0) & 15u) << (4 * asked);
      ++asked;
      const int64_t place = max((int64_t)0, (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), slice) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)mine, slice)));
      const uint32_t buffer = (uint32_t)(step % kBuffers) * Lds::kStepBytes;
      if (kWaves == 4 || wave < kManySlices) copy(static_cast<const char*>(a.k) + place, lds_x + buffer);
      if (kWaves == 4 || wave >= kManySlices) copy(static_cast<const char*>(a.v) + place, lds_y + buffer);
    };
    if (from < to) {
      look_up(from);
      __syncthreads();
#pragma unroll
      for (int ahead = 0; ahead < kAhead; ++ahead)
        if (from + ahead < to) issue(from + ahead);
    }
    // The wave's rows, loaded while the first copies are on their way, and what all of them, or any, see, in scalar registers.
    const int32_t first_row = share.tile * kRows + wave * 32, rows = max(0, min(32, q.count * a.group - first_row));
    CacheRow own(a, rule, q, share.key_head, first_row + i);
    const int32_t own_row = own.row >= 0 ? own.row : q.first, own_head = own.row >= 0 ? own.head : share.key_head * a.group;
    const OwnOperand<S, S::kContraction> query(static_cast<const char*>(a.q) + (own_row * a.q_strides.token + own_head * a.q_strides.head) * 2, g, nullptr);
    asm volatile("" : "+v"(own.slope), "+v"(own.drafts));  // (waited for here, not in the loop)
    const int32_t first_token = divided(first_row, a.group), last_token = divided(first_row + max(rows, 1) - 1, a.group);
    const View least = view_at(a, q, max(a.tree ? q.base : q.base + first_token, 0)), most = view_at(a, q, max(a.tree ? q.length - 1 : q.base + last_token, 0));
    const int32_t sure_prompt = prompt_end(a, q), sure_hi = q.base < 0 ? 0 : a.tree ? q.base : least.hi, sure_lo = most.lo;
    const int32_t any_lo = a.tree ? min(least.lo, max(q.base, 0)) : least.lo, any_hi = a.tree ? q.length : most.hi;

    floatx16 sum[S::kDBlocks];
#pragma unroll
    for (auto& t : sum) {
      t = splat(0.f);
      asm volatile("" : "+v"(t));  // (a known zero has the sums copied in every step, 64 moves: three frames over 75K tokens 5.37 / 5.06 ms)
    }
    Softmax soft;
    for (int32_t step = from; step < to; ++step) {
      const int buffer = step % kBuffers;
      const int32_t token = walk.token(step);
      const uint32_t here = there & 15u;
      const bool full = here == 15u && token + kManyStep <= q.length;
      if (kAhead > 1 && step + kAhead <= to) WAIT_VMCNT((kAhead - 1) * kCopies);
      else WAIT_VMCNT(0);
      if (!full && (kWaves == 4 || wave >= kManySlices))
        clear_rows<S>(lds.y[buffer], (here >> slice) & 1u ? max(slice * kSlice, q.length - token) : slice * kSlice, (slice + 1) * kSlice, lane);
      WAIT_LGKMCNT0();
      BARRIER();  // the step is there, and nobody reads the buffer before it any more
      there >>= 4;
      --asked;
      if (step + kAhead < to) {
        if ((step + kAhead - from) % kPlacedSteps == 0) {
          look_up(step + kAhead);
          __syncthreads();
        }
        issue(step + kAhead);
      }
      if (rows > 0 && (token < sure_prompt || (token < any_hi && token + kManyStep > any_lo))) {
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
    }

    const float weight = sum_with_partner(soft.sum);
    if (i < rows) {
      if (share.whole) {
        const int64_t at = (int64_t)own.row * a.heads + own.head;
        const bool real = weight != 0.f;
        store_columns<S::kDBlocks>(static_cast<char*>(a.out) + at * S::kRowBytes, g, 0, sum, 1.f / weight, real);
        if (g == 0) a.lse[at] = real ? (__builtin_fmaf(soft.ref, rule.c2, rule.offset) + __builtin_amdgcn_logf(weight)) * 0.6931471805599453f : kMinusInf;
      } else {
        float* const piece = share.piece(a, D) + (wave * 32 + i) * piece_row(D);
#pragma unroll
        for (int db = 0; db < S::kDBlocks; ++db)
#pragma unroll
          for (int j = 0; j < 4; ++j) *reinterpret_cast<floatx4*>(piece + db * 32 + 8 * j + 4 * g) = floatx4{sum[db][4 * j], sum[db][4 * j + 1], sum[db][4 * j + 2], sum[db][4 * j + 3]};
        if (g == 0) *reinterpret_cast<float2*>(piece + D) = float2{soft.ref, weight};
      }
    }
    if (!kLine || !share.next(a)) break;
    __syncthreads();  // nobody reads the buffers any more
  }
  share.leave(a, true);
}

template <int D, int kRows>
__global__ __launch_bounds__(256) void many_rows_join_kernel(AttendArgs a) {
  join_pieces<D, kRows, 256, 1>(a);
}

template <int D, int kWaves, int kBuffers>
hipError_t launch_many_rows(const AttendArgs& a, hipStream_t stream) {
  constexpr int kRows = kWaves * 32, kRowsAtOnce = 1024 / D;  // of a workgroup that joins
  const int64_t items = a.tiles * a.kv_heads, workgroups = a.way == kShares ? a.workgroups : items * (a.way == kParts ? a.most_parts : 1);
  if (workgroups < 1 || workgroups > 0xffffff || (a.way == kShares && workgroups % 8 != 0)) return hipErrorInvalidValue;  // (2^32 threads)
  if (a.way == kShares) many_rows_kernel<D, true, kWaves, kBuffers><<<(unsigned)workgroups, kWaves * 64, 0, stream>>>(a);
  else many_rows_kernel<D, false, kWaves, kBuffers><<<(unsigned)workgroups, kWaves * 64, 0, stream>>>(a);
  if (a.way != kItems) {
    const int64_t rows = (int64_t)((a.tokens + a.sequences - 1) / a.sequences) * a.group, row_groups = ((rows < kRows ? rows : kRows) + kRowsAtOnce - 1) / kRowsAtOnce;
    many_rows_join_kernel<D, kRows><<<dim3((unsigned)(a.way == kShares ? workgroups : items), (unsigned)row_groups), 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_many(const AttendArgs& a, hipStream_t stream) {
  if (a.tile_rows == 256) return a.D == 64 ? launch_many_rows<64, 8, 4>(a, stream) : launch_many_rows<128, 8, 4>(a, stream);
  if (a.tile_rows == 128) return a.D == 64 ? launch_many_rows<64, 4, 4>(a, stream) : launch_many_rows<128, 4, 2>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace ca
