// Attention over a paged cache for few rows a sequence: single tokens, drafts.  See attn_cache.h.
#include "attn_cache.h"

namespace ca {
namespace {

constexpr int kFewWaves = 4, kFewThreads = kFewWaves * 64;
constexpr int kFewItemCost = 14;  // steps that a workgroup's four waves do in the time that it takes to begin an item; 32 single tokens with 8 / 14 / 20: 162 / 160 / 161 us

// A wave's own part of LDS: two buffers of a step; at the end its sums, row by row.
template <class S>
struct FewWave {
  static constexpr int kStepBytes = kFewStep * S::kRowBytes, kSumRow = piece_row(S::D);
  union {
    char steps[2][2][kStepBytes];          // [buffer][keys, values]
    float sums[kFewRows][kSumRow];         // D sums, then the reference and the sum of weights
  };
  float frames[kFewStep];
};

// Of an item the waves of a workgroup take a quarter of the steps each; they join their sums at the end.
template <int D>
__global__ __launch_bounds__(kFewThreads) __attribute__((amdgpu_waves_per_eu(D == 128 ? 1 : 2))) void few_rows_kernel(AttendArgs a) {
  typedef CacheShape<D> S;
  __shared__ FewWave<S> lds[kFewWaves];
  __shared__ LineLds found;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, g = lane >> 5;
  Share<kFewRows, kFewStep, kFewThreads, kFewItemCost> share;
  if (!share.begin(a, found, blockIdx.x)) {
    share.leave(a, false);
    return;
  }
  const CacheRule rule(a, true);
  const SliceCopy<S> copy(lane);
  const Fragments<S> frag(lane);
  FewWave<S>& mine = lds[wave];
  const uint32_t lds_steps = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine.steps[0][0];
  while (true) {
    const Sequence& q = share.q;
    const int32_t s = share.sequence, key_head = share.key_head;
    const Walk<kFewStep> walk = share.walk;
    const int32_t first_row = share.tile * kFewRows, rows = min(kFewRows, q.count * a.group - first_row);
    const int32_t first_token = divided(first_row, a.group), last_token = divided(first_row + rows - 1, a.group);
    CacheRow own(a, rule, q, key_head, first_row + i);
    const int32_t own_row = own.row >= 0 ? own.row : q.first + first_token, own_head = own.row >= 0 ? own.head : key_head * a.group;
    const Sure sure(a, q, first_token, last_token);

    floatx16 sum[S::kDBlocks];
#pragma unroll
    for (auto& t : sum) t = splat(0.f);
    Softmax soft;

    const int32_t end = min(share.done + share.steps, walk.count), part = (share.steps + kFewWaves - 1) / kFewWaves;
    const int32_t from = min(end, share.done + wave * part), to = min(end, from + part);
    SlicePlaces<2, kFewStep> places;
    auto issue = [&](int32_t step) {
      places.at_step(a, q, s, key_head, walk, step, from, to, lane, S::kRowBytes);
      WAIT_LGKMCNT0();  // nothing still reads the buffer
      const uint32_t to_lds = lds_steps + (uint32_t)(step & 1) * 2 * FewWave<S>::kStepBytes;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int64_t at = places.at(step, c);
        copy(static_cast<const char*>(a.k) + at, to_lds + c * S::kSliceBytes);
        copy(static_cast<const char*>(a.v) + at, to_lds + FewWave<S>::kStepBytes + c * S::kSliceBytes);
      }
    };
    uint32_t there = 0, next_there = 0;
    if (from < to) {
      issue(from);
      there = places.mask(from);
    }
    // (loaded while the first copies are on their way)
    const OwnOperand<S, S::kContraction> query(static_cast<const char*>(a.q) + (own_row * a.q_strides.token + own_head * a.q_strides.head) * 2, g, nullptr);
    asm volatile("" : "+v"(own.slope), "+v"(own.drafts));  // (waited for here, not in the loop)
    for (int32_t step = from; step < to; ++step) {
      if (step + 1 < to) {
        issue(step + 1);
        next_there = places.mask(step + 1);
        WAIT_VMCNT(4 * S::kSliceLoads);
      } else {
        WAIT_VMCNT(0);
      }
      const LdsTile x = (LdsTile)mine.steps[step & 1][0], y = (LdsTile)mine.steps[step & 1][1];
      const int32_t token = walk.token(step);
      if (there != 3) clear_rows<S>(mine.steps[step & 1][1], there & 1 ? kSlice : 0, there & 2 ? kSlice : kFewStep, lane);
      if (token + kFewStep > q.length) clear_rows<S>(mine.steps[step & 1][1], q.length - token, kFewStep, lane);
      floatx16 p = block_product<S>(frag, x, 0, query, splat(0.f));
      if (rule.capped) cap_scores<16>(rule, p);
      if (a.slopes) {
        if (lane < kFewStep) mine.frames[lane] = frame_of_token(a, q, token + lane);
        __builtin_amdgcn_wave_barrier();
        bias_scores(own, p, mine.frames, 0, g);
      }
      if (there != 3 || !sure.sees(token, token + kFewStep)) hide_tokens(a, q, own, p, token, there, g);
      soften<1, S::kDBlocks>(rule, soft, reinterpret_cast<floatx16(&)[1]>(p), sum);
      bf16x8 weights[2];
      rounded(p, weights);
      block_sums<S>(frag, y, 0, weights, sum);
      there = next_there;
    }

    // the wave's sums, row by row
    const float total = sum_with_partner(soft.sum);
    WAIT_LGKMCNT0();
#pragma unroll
    for (int db = 0; db < S::kDBlocks; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<floatx4*>(&mine.sums[i][db * 32 + 8 * j + 4 * g]) = floatx4{sum[db][4 * j], sum[db][4 * j + 1], sum[db][4 * j + 2], sum[db][4 * j + 3]};
    if (g == 0) mine.sums[i][D] = soft.ref, mine.sums[i][D + 1] = total;
    __syncthreads();
    finish_rows<D, __bf16, kFewWaves>(a, rule, share, lds, first_row, rows);
    if (!share.next(a)) break;
    __syncthreads();  // (the sums lie where the next steps go)
  }
  share.leave(a, true);
}

template <int D>
__global__ __launch_bounds__(kFewThreads) void few_rows_join_kernel(AttendArgs a) {
  join_pieces<D, __bf16, kFewRows, kFewThreads, kFewThreads / (D / 4)>(a);
}

template <int D>
hipError_t launch_few_rows(const AttendArgs& a, hipStream_t stream) {
  const int64_t workgroups = a.way == kShares ? a.workgroups : a.tiles * a.kv_heads;
  if (a.way == kParts || workgroups < 1 || workgroups > 0xffffff) return hipErrorInvalidValue;  // (2^32 threads)
  few_rows_kernel<D><<<(unsigned)workgroups, kFewThreads, 0, stream>>>(a);
  if (a.way == kShares) {
    // a workgroup for every row that a sequence has on average, as far as a tile has them
    const int64_t rows = (int64_t)((a.tokens + a.sequences - 1) / a.sequences) * a.group;
    few_rows_join_kernel<D><<<dim3((unsigned)workgroups, (unsigned)(rows < kFewRows ? rows : kFewRows)), kFewThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_few(const AttendArgs& a, hipStream_t stream) { return a.D == 64 ? launch_few_rows<64>(a, stream) : launch_few_rows<128>(a, stream); }

}  // namespace ca
