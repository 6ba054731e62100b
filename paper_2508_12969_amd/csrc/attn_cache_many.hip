// Attention over a paged cache for many rows a sequence: frames, prompts, trees of drafts with grouped heads.  See attn_cache.h.
#include <type_traits>

#include "attn_cache.h"

namespace ca {
namespace {

constexpr int kManyWaves = kManyRows / 32, kManyThreads = kManyWaves * 64, kManySlices = kManyStep / kSlice;
static_assert(kManyWaves == kManySlices, "a wave copies a slice");
constexpr int kManyItemCost = 4;     // steps that a workgroup does in the time that it takes to begin an item; 16 trees with 2 / 3 / 4: 88 / 82 / 78 us
constexpr int kPlacedSteps = 128;    // whose slices are looked up together

// Waves per SIMD that the registers leave room for: a third at head dim 64 (three frames over 75K tokens, 10 heads, two / three 2.74 / 2.50 ms, four prompts of 9K, 32 heads, 1104 / 982 us; with
// shares of a line, whose launches are short, six sequences of 52 rows 35 / 44 us; four spill).
constexpr int many_waves(int D, bool line) { return D == 64 && !line ? 3 : 2; }

template <class S>
struct ManyLds {
  static constexpr int kStepBytes = kManyStep * S::kRowBytes;
  char x[2][kStepBytes], y[2][kStepBytes];
  float frames[kManyWaves][kManyStep];
  int64_t places[kPlacedSteps * kManySlices];  // where slices lie, -1: not there
};

// A workgroup takes a tile of 128 rows, 32 a wave, over steps of 64 tokens that the waves copy together, a slice each, while the step before is computed.  (Tiles of 256 rows, which read their keys
// half as often, with copies three steps ahead: 100 rows a key head 90 / 91 us, 225 rows 160 / 160, 75 rows 81 / 71, a frame of 1560 rows 401 / 391.)
// kCapped: both forms of capped scores are there, as two loops, and a tile takes one of them, by what its rows see (the table's room, known before the launch, says nothing of that; a kernel for each
// form and one with both, all tiles in the fast form: three frames over 75K tokens 4.92 / 5.01 ms, 16 trees over 9K 82 / 84 us).  All waves of a workgroup take the same one, whose barriers they share; with the
// choice in a scalar register the loops' registers spill (41 of them at head dim 128, three frames 5.33 / 7.64 ms).
template <int D, bool kLine, bool kCapped>
__global__ __attribute__((amdgpu_flat_work_group_size(kManyThreads, kManyThreads), amdgpu_waves_per_eu(many_waves(D, kLine), many_waves(D, kLine)))) void many_rows_kernel(AttendArgs a) {
  typedef CacheShape<D> S;
  typedef ManyLds<S> Lds;
  constexpr int kBlocks = kManyStep / 32;
  __shared__ Lds lds;
  __shared__ LineLds found;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, g = lane >> 5;
  // Neighbours on the line, or tiles of one key head, are on one XCD (a frame of 13 tiles a head in chunks of 13 / as the ids come 391 / 418 us, 85 tiles in chunks of 64 / 8 4.90 / 5.09 ms).
  const int64_t total = gridDim.x, workgroup = a.way == kShares ? blockIdx.x % 8 * (total / 8) + blockIdx.x / 8 : xcd_launch_order(blockIdx.x, total, min(a.tiles, kXcdChunk));
  Share<kManyRows, kManyStep, kManyThreads, kManyItemCost> share;
  if (!share.begin(a, found, workgroup)) {
    share.leave(a, false);
    return;
  }
  const SliceCopy<S> copy(lane);
  const Fragments<S> frag(lane);
  const uint32_t lds_x = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.x[0] + wave * S::kSliceBytes;
  const uint32_t lds_y = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.y[0] + wave * S::kSliceBytes;
  while (true) {
    const Sequence& q = share.q;
    const Walk<kManyStep> walk = share.walk;
    const int32_t from = min(walk.count, share.done), to = min(walk.count, share.done + share.steps);
    if constexpr (kCapped) {
      const int32_t first = share.tile * kManyRows, last = min(first + kManyRows, q.count * a.group) - 1;
      share.fine = a.cap > kMostFastCap || Sure(a, q, divided(first, a.group), divided(last, a.group)).tokens() <= kFineTokens;
    }
    const CacheRule rule(a, share.fine);
    // Places of the slices from `first` on.
    auto look_up = [&](int32_t first) {
      for (int at = threadIdx.x; at < kPlacedSteps * kManySlices; at += kManyThreads) {
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
    uint32_t there = 0;  // of the step that was asked for last: which of its slices are there
    auto issue = [&](int32_t step) {
      const int64_t mine = lds.places[((step - from) % kPlacedSteps) * kManySlices + lane % kManySlices];
      there = (uint32_t)__builtin_amdgcn_ballot_w64(mine >= 0) & 15u;
      const int64_t place = max((int64_t)0, (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), wave) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)mine, wave)));
      const uint32_t buffer = (uint32_t)(step & 1) * Lds::kStepBytes;
      copy(static_cast<const char*>(a.k) + place, lds_x + buffer);
      copy(static_cast<const char*>(a.v) + place, lds_y + buffer);
    };
    if (from < to) {
      look_up(from);
      __syncthreads();
      issue(from);
    }
    // The wave's rows, loaded while the first copies are on their way, and what all of them, or any, see, in scalar registers.
    const int32_t first_row = share.tile * kManyRows + wave * 32, rows = max(0, min(32, q.count * a.group - first_row));
    CacheRow own(a, rule, q, share.key_head, first_row + i);
    const int32_t own_row = own.row >= 0 ? own.row : q.first, own_head = own.row >= 0 ? own.head : share.key_head * a.group;
    const OwnOperand<S, S::kContraction> query(static_cast<const char*>(a.q) + (own_row * a.q_strides.token + own_head * a.q_strides.head) * 2, g, nullptr);
    asm volatile("" : "+v"(own.slope), "+v"(own.drafts));  // (waited for here, not in the loop)
    const int32_t first_token = divided(first_row, a.group), last_token = divided(first_row + max(rows, 1) - 1, a.group);
    const View least = view_at(a, q, max(a.tree ? q.base : q.base + first_token, 0)), most = view_at(a, q, max(a.tree ? q.length - 1 : q.base + last_token, 0));
    const Sure sure(a, q, first_token, last_token);
    const int32_t any_lo = a.tree ? min(least.lo, max(q.base, 0)) : least.lo, any_hi = a.tree ? q.length : most.hi;

    floatx16 sum[S::kDBlocks];
#pragma unroll
    for (auto& t : sum) {
      t = splat(0.f);
      asm volatile("" : "+v"(t));  // (a known zero has the sums copied in every step, 64 moves: three frames over 75K tokens 5.37 / 5.06 ms)
    }
    Softmax soft;
    const auto take_steps = [&](auto fine) {
      for (int32_t step = from; step < to; ++step) {
        const int buffer = step & 1;
        const int32_t token = walk.token(step);
        const uint32_t here = there;
        const bool full = here == 15u && token + kManyStep <= q.length;
        WAIT_VMCNT(0);
        if (!full) clear_rows<S>(lds.y[buffer], (here >> wave) & 1u ? max(wave * kSlice, q.length - token) : wave * kSlice, (wave + 1) * kSlice, lane);
        WAIT_LGKMCNT0();
        BARRIER();  // the step is there, and nobody reads the other buffer any more
        if (step + 1 < to) {
          if ((step + 1 - from) % kPlacedSteps == 0) {
            look_up(step + 1);
            __syncthreads();
          }
          issue(step + 1);
        }
        if (rows > 0 && (token < sure.prompt || (token < any_hi && token + kManyStep > any_lo))) {
          const LdsTile x = (LdsTile)lds.x[buffer], y = (LdsTile)lds.y[buffer];
          floatx16 p[kBlocks];
#pragma unroll
          for (int b = 0; b < kBlocks; ++b) p[b] = block_product<S>(frag, x, b, query, splat(0.f));
          if constexpr (kCapped)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
              if constexpr (fine) cap_scores<16>(rule, p[b]);
              else cap_scores_fast(rule, p[b]);
            }
          if (a.slopes) {
            lds.frames[wave][lane] = frame_of_token(a, q, token + lane);
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) bias_scores(own, p[b], lds.frames[wave], b, g);
          }
          if (!full || !sure.sees(token, token + kManyStep))
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
    };
    if (kCapped && share.fine) take_steps(std::true_type());
    else take_steps(std::false_type());

    const float weight = sum_with_partner(soft.sum);
    if (i < rows) {
      if (share.whole) {
        const int64_t at = (int64_t)own.row * a.heads + own.head;
        const bool real = weight != 0.f;
        store_columns<S::kDBlocks>(static_cast<char*>(a.out) + at * S::kRowBytes, g, 0, sum, 1.f / weight, real);
        if (g == 0) a.lse[at] = real ? rule.log_sum_exp(soft.ref, weight) : kMinusInf;
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

template <int D>
__global__ __launch_bounds__(kManyThreads) void many_rows_join_kernel(AttendArgs a) {
  join_pieces<D, __bf16, kManyRows, kManyThreads, 1>(a);
}

template <int D>
hipError_t launch_many_rows(const AttendArgs& a, hipStream_t stream) {
  constexpr int kRowsAtOnce = kManyThreads / (D / 4);  // of a workgroup that joins
  const int64_t items = a.tiles * a.kv_heads, workgroups = a.way == kShares ? a.workgroups : items * (a.way == kParts ? a.most_parts : 1);
  if (workgroups < 1 || workgroups > 0xffffff || (a.way == kShares && workgroups % 8 != 0)) return hipErrorInvalidValue;  // (2^32 threads)
  const auto launch = [&](auto line, auto capped) { many_rows_kernel<D, line, capped><<<(unsigned)workgroups, kManyThreads, 0, stream>>>(a); };
  const bool capped = a.cap > 0.f;
  if (a.way == kShares) capped ? launch(std::true_type(), std::true_type()) : launch(std::true_type(), std::false_type());
  else capped ? launch(std::false_type(), std::true_type()) : launch(std::false_type(), std::false_type());
  if (a.way != kItems) {
    const int64_t rows = (int64_t)((a.tokens + a.sequences - 1) / a.sequences) * a.group, row_groups = ((rows < kManyRows ? rows : kManyRows) + kRowsAtOnce - 1) / kRowsAtOnce;
    many_rows_join_kernel<D><<<dim3((unsigned)(a.way == kShares ? workgroups : items), (unsigned)row_groups), kManyThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_many(const AttendArgs& a, hipStream_t stream) {
  return a.D == 64 ? launch_many_rows<64>(a, stream) : launch_many_rows<128>(a, stream);
}

}  // namespace ca
