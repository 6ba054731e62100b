// Attention over a paged cache for few rows a sequence: single tokens, drafts.  See attn_cache.h.
#include "attn_cache.h"

namespace ca {
namespace {

constexpr int kFewRows = 32, kFewStep = 32, kFewWaves = 4, kFewThreads = kFewWaves * 64;

// A wave's own part of LDS: two buffers of a step; at the end its sums, row by row.
template <class S>
struct FewWave {
  static constexpr int kStepBytes = kFewStep * S::kRowBytes, kSumRow = S::D + 4;  // (rows of sums begin in different banks)
  union {
    char steps[2][2][kStepBytes];          // [buffer][keys, values]
    float sums[kFewRows][kSumRow];         // D sums, then the reference and the sum of weights
  };
  float frames[kFewStep];
};

// A workgroup takes a tile of 32 rows, its waves a quarter of the steps each; they join their sums at the end.
template <int D>
__global__ __launch_bounds__(kFewThreads) __attribute__((amdgpu_waves_per_eu(D == 128 ? 1 : 2))) void few_rows_kernel(AttendArgs a) {
  typedef CacheShape<D> S;
  __shared__ FewWave<S> lds[kFewWaves];
  __shared__ LocateLds found;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, g = lane >> 5;
  const int32_t key_head = (int32_t)(blockIdx.x % (uint32_t)a.kv_heads);
  int32_t s;
  int64_t tile, all;
  if (!locate<kFewThreads>(a, blockIdx.x / (uint32_t)a.kv_heads, found, s, tile, all, [&](const Sequence& q) { return (int64_t)row_tiles(a, q, kFewRows); })) return;
  const Sequence q = sequence_at(a, s);
  const CacheRule rule(a);
  const int64_t first_row = tile * kFewRows;
  const int rows = (int)min((int64_t)kFewRows, (int64_t)q.count * a.group - first_row);
  const int32_t first_token = (int32_t)(first_row / a.group), last_token = (int32_t)((first_row + rows - 1) / a.group);
  const Walk<kFewStep> walk = walk_of<kFewStep>(a, q, first_token, last_token);
  CacheRow own(a, rule, q, key_head, first_row + i);
  const int32_t own_row = own.row >= 0 ? own.row : q.first + first_token, own_head = own.row >= 0 ? own.head : key_head * a.group;
  asm volatile("" : "+v"(own.slope), "+v"(own.drafts));  // (waited for here, not in the loop)
  const OwnOperand<S, S::kContraction> query(static_cast<const char*>(a.q) + (own_row * a.q_strides.token + own_head * a.q_strides.head) * 2, g, nullptr);
  // what all rows of the tile see, in scalar registers
  const int32_t sure_prompt = prompt_end(a, q), sure_hi = q.base < 0 ? 0 : a.tree ? q.base : view_at(a, q, q.base + first_token).hi;
  const int32_t sure_lo = view_at(a, q, a.tree ? max(q.length - 1, 0) : max(q.base + last_token, 0)).lo;

  const SliceCopy<S> copy(lane);
  const Fragments<S> frag(lane);
  FewWave<S>& mine = lds[wave];
  const uint32_t lds_steps = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine.steps[0][0];
  floatx16 sum[S::kDBlocks];
#pragma unroll
  for (auto& t : sum) t = splat(0.f);
  Softmax soft;

  const int32_t part = (walk.count + kFewWaves - 1) / kFewWaves, from = min(walk.count, wave * part), to = min(walk.count, from + part);
  SlicePlaces<2, kFewStep> places;
  auto issue = [&](int32_t step) {
    if (step == from || step - places.first >= places.kSteps) places.fetch(a, q, s, key_head, walk, step, to, lane, S::kRowBytes);
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
    if (rule.capped) {
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(p[r] * rule.bend));
    }
    if (a.slopes) {
      if (lane < kFewStep) mine.frames[lane] = frame_of_token(a, q, token + lane);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const floatx4 f = read4(mine.frames, 0, j, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) p[4 * j + e] = __builtin_fmaf(__builtin_fabsf((float)own.view.frame - f[e]), own.slope, p[4 * j + e]);
      }
    }
    const bool sure = token + kFewStep <= sure_hi && (token >= sure_lo || token + kFewStep <= sure_prompt) && there == 3;
    if (!sure) hide_tokens(a, q, own, p, token, there, g);
    float mx = p[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, p[r]);
    mx = max_with_partner(mx);
    const bool moves = mx > soft.ref + kLazyLog2 / rule.c2;
    if (__builtin_amdgcn_ballot_w64(moves) != 0) {
      const float ref = moves ? mx : soft.ref;
      const float alpha = moves && soft.ref != kMinusInf ? __builtin_amdgcn_exp2f((soft.ref - ref) * rule.c2) : 1.f;
      soft.ref = ref;
      soft.sum *= alpha;
#pragma unroll
      for (int db = 0; db < S::kDBlocks; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[db][r] *= alpha;
    }
    const float shift = soft.ref == kMinusInf ? 0.f : -soft.ref * rule.c2;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], rule.c2, shift));
      soft.sum += p[r];
    }
    bf16x8 weights[2];
    rounded(p, weights);
    block_sums<S>(frag, y, 0, weights, sum);
    there = next_there;
  }

  // the wave's sums, row by row
  const float weight = sum_with_partner(soft.sum);
  WAIT_LGKMCNT0();
#pragma unroll
  for (int db = 0; db < S::kDBlocks; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<floatx4*>(&mine.sums[i][db * 32 + 8 * j + 4 * g]) = floatx4{sum[db][4 * j], sum[db][4 * j + 1], sum[db][4 * j + 2], sum[db][4 * j + 3]};
  if (g == 0) mine.sums[i][D] = soft.ref, mine.sums[i][D + 1] = weight;
  __syncthreads();
  for (int item = threadIdx.x; item < rows * (D / 4); item += kFewThreads) {
    const int r = item / (D / 4), c = item % (D / 4) * 4;
    float ref = kMinusInf, total = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) ref = fmaxf(ref, lds[w].sums[r][D]);
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float there_ref = lds[w].sums[r][D], factor = there_ref == kMinusInf ? 0.f : __builtin_amdgcn_exp2f((there_ref - ref) * rule.c2);
      total += lds[w].sums[r][D + 1] * factor;
      o += *reinterpret_cast<const floatx4*>(&lds[w].sums[r][c]) * factor;
    }
    const int32_t t = (int32_t)((first_row + r) / a.group), head = key_head * a.group + (int32_t)(first_row + r - (int64_t)t * a.group);
    const int64_t at = (int64_t)(q.first + t) * a.heads + head;
    const bool real = total != 0.f;
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (__bf16)(real ? o[e] / total : 0.f);
    *reinterpret_cast<bf16x4*>(static_cast<char*>(a.out) + (at * D + c) * 2) = v;
    if (c == 0) a.lse[at] = real ? (__builtin_fmaf(ref, rule.c2, rule.offset) + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : kMinusInf;
  }
}

}  // namespace

hipError_t launch_attend(const AttendArgs& a, hipStream_t stream) {
  const int64_t workgroups = a.tiles * a.kv_heads;
  if (workgroups < 1 || workgroups > 0xffffff) return hipErrorInvalidValue;  // (2^32 threads)
  if (a.D == 64) few_rows_kernel<64><<<(unsigned)workgroups, kFewThreads, 0, stream>>>(a);
  else few_rows_kernel<128><<<(unsigned)workgroups, kFewThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ca
