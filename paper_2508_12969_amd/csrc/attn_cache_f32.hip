// Attention over a paged cache in fp32.  See attn_cache.h.
//
// The shape is that of few_rows_kernel, on the f32 matrix instructions (16 x 16 x 4): a wave walks over its own steps of 16 tokens, S^T = K Q^T and O^T += V^T P^T, with two tiles of 16 rows as the
// columns.  A lane holds, of row lane % 16 of either, the scores of tokens 4 (lane / 16) + r, which are the second product's operand as they are.  Nothing is rounded but sums.  Bound: HBM as long as
// a sequence has few rows (the matrix instructions do 32 rows of a step in the time that HBM takes for it), the matrix instructions beyond.
#include "attn_cache.h"

namespace ca {
namespace {

constexpr int kF32Waves = 4, kF32Threads = kF32Waves * 64, kF32Step = kSlice, kF32Columns = kFewRows / 16;
constexpr int kF32ItemCost = 14;  // as few_rows_kernel's, whose steps are as many bytes

template <int D_>
struct F32Shape {
  static constexpr int D = D_, kRowBytes = D * 4, kChunksPerRow = D / 4, kRowsPerLoad = 1024 / kRowBytes, kLoads = kSlice / kRowsPerLoad, kStepBytes = kSlice * kRowBytes;
  static constexpr int kBlocks = D / 16;  // of 16 channels
  static_assert(kLoads % 4 == 0, "copies are written for loads by fours");
};

template <class S>
struct F32Wave {
  union {
    char steps[2][2][S::kStepBytes];            // [buffer][keys, values]
    float sums[kFewRows][piece_row(S::D)];      // at the end: D sums, then the reference and the sum of weights
  };
  float frames[kF32Step];
};

// Logical 16-byte chunk c of row r lies at physical chunk c ^ r: read by rows (16 rows, one chunk) or by channels (64 bytes of rows 4 g + r) the places are in different banks.
template <class S>
struct F32Copy {
  uint32_t voff[S::kLoads];
  __device__ __forceinline__ explicit F32Copy(int lane) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int within = lane / S::kChunksPerRow, phys = lane % S::kChunksPerRow;
      voff[i] = (uint32_t)(within * S::kRowBytes + ((phys ^ (i * S::kRowsPerLoad + within)) << 4));
    }
  }
  __device__ __forceinline__ void operator()(const char* slice, uint32_t lds) const {
#pragma unroll
    for (int i = 0; i < S::kLoads; i += 4) {
      const uint32_t m0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds + (uint32_t)i * 1024u));
      asm volatile(
          "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %[v0], %[sb] offset:0\n\t"
          "global_load_lds_dwordx4 %[v1], %[sb] offset:1024\n\t"
          "global_load_lds_dwordx4 %[v2], %[sb] offset:2048\n\t"
          "global_load_lds_dwordx4 %[v3], %[sb] offset:%[o3]\n\t"
          :
          : [o3] "n"(3 * 1024), [m0] "s"(m0), [v0] "v"(voff[i]), [v1] "v"(voff[i + 1]), [v2] "v"(voff[i + 2]), [v3] "v"(voff[i + 3]), [sb] "s"(slice + i * 1024)
          : "memory");
    }
  }
};

// Over the four lanes that hold a row: lane ^ 32, then lane ^ 16.
__device__ __forceinline__ float row_max(float x) {
  float a = max_with_partner(x), b = a;
  asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  return fmaxf(a, b);
}
__device__ __forceinline__ float sum_of_row(float x) {
  float a = sum_with_partner(x), b = a;
  asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  return a + b;
}

template <int D>
__global__ __launch_bounds__(kF32Threads) __attribute__((amdgpu_waves_per_eu(D == 128 ? 1 : 2))) void f32_kernel(AttendArgs a) {
  typedef F32Shape<D> S;
  __shared__ F32Wave<S> lds[kF32Waves];
  __shared__ LineLds found;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  Share<kFewRows, kF32Step, kF32Threads, kF32ItemCost> share;
  if (!share.begin(a, found, blockIdx.x)) {
    share.leave(a, false);
    return;
  }
  const CacheRule rule(a, true);
  const F32Copy<S> copy(lane);
  F32Wave<S>& mine = lds[wave];
  const uint32_t lds_steps = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine.steps[0][0];
  while (true) {
    const Sequence& q = share.q;
    const Walk<kF32Step> walk = share.walk;
    const int32_t first_row = share.tile * kFewRows, rows = min(kFewRows, q.count * a.group - first_row);
    const int32_t first_token = divided(first_row, a.group), last_token = divided(first_row + rows - 1, a.group);
    const Sure sure(a, q, first_token, last_token);
    const int columns = rows > 16 ? 2 : 1;  // tiles of rows in use

    const int32_t end = min(share.done + share.steps, walk.count), part = (share.steps + kF32Waves - 1) / kF32Waves;
    const int32_t from = min(end, share.done + wave * part), to = min(end, from + part);
    SlicePlaces<1, kF32Step> places;
    auto issue = [&](int32_t step) {
      places.at_step(a, q, share.sequence, share.key_head, walk, step, from, to, lane, S::kRowBytes);
      WAIT_LGKMCNT0();  // nothing still reads the buffer
      const uint32_t to_lds = lds_steps + (uint32_t)(step & 1) * 2 * S::kStepBytes;
      const int64_t at = places.at(step, 0);
      copy(static_cast<const char*>(a.k) + at, to_lds);
      copy(static_cast<const char*>(a.v) + at, to_lds + S::kStepBytes);
    };
    uint32_t there = 0, next_there = 0;
    if (from < to) {
      issue(from);
      there = places.mask(from);
    }
    CacheRow own[kF32Columns] = {{a, rule, q, share.key_head, first_row + i}, {a, rule, q, share.key_head, first_row + 16 + i}};
    floatx4 query[kF32Columns][S::kBlocks], sum[kF32Columns][S::kBlocks];
    Softmax soft[kF32Columns];
#pragma unroll
    for (int c = 0; c < kF32Columns; ++c) {
      const int32_t row = own[c].row >= 0 ? own[c].row : q.first + first_token, head = own[c].row >= 0 ? own[c].head : share.key_head * a.group;
      const floatx4* const from_row = reinterpret_cast<const floatx4*>(static_cast<const float*>(a.q) + row * a.q_strides.token + head * a.q_strides.head) + g;
#pragma unroll
      for (int t = 0; t < S::kBlocks; ++t) {
        query[c][t] = from_row[4 * t];
        sum[c][t] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int t = 0; t < S::kBlocks; ++t) asm volatile("" : "+v"(query[c][t]), "+v"(sum[c][t]));  // (waited for here, not in the loop)
      asm volatile("" : "+v"(own[c].slope), "+v"(own[c].drafts));
    }
    for (int32_t step = from; step < to; ++step) {
      if (step + 1 < to) {
        issue(step + 1);
        next_there = places.mask(step + 1);
        WAIT_VMCNT(2 * S::kLoads);
      } else {
        WAIT_VMCNT(0);
      }
      const char *const x = mine.steps[step & 1][0], *const y = mine.steps[step & 1][1];
      const int32_t token = walk.token(step);
      if (there == 0 || token + kF32Step > q.length) clear_rows<S>(mine.steps[step & 1][1], there ? q.length - token : 0, kF32Step, lane);
      floatx4 p[kF32Columns] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      auto scores = [&](auto both) {
#pragma unroll
        for (int t = 0; t < S::kBlocks; ++t) {
          const floatx4 k = *reinterpret_cast<const floatx4*>(x + i * S::kRowBytes + (((4 * t + g) ^ i) << 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], query[0][t][e], p[0], 0, 0, 0);
            if constexpr (both) p[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], query[1][t][e], p[1], 0, 0, 0);
          }
        }
      };
      columns == 2 ? scores(std::true_type()) : scores(std::false_type());
      if (a.slopes) {
        if (lane < kF32Step) mine.frames[lane] = frame_of_token(a, q, token + lane);
        __builtin_amdgcn_wave_barrier();
      }
      const bool all_seen = there != 0 && sure.sees(token, token + kF32Step);
#pragma unroll
      for (int c = 0; c < kF32Columns; ++c) {
        if (c >= columns) break;
        if (rule.capped) cap_scores<4>(rule, p[c]);
        if (a.slopes) {
#pragma unroll
          for (int r = 0; r < 4; ++r) p[c][r] = __builtin_fmaf(__builtin_fabsf((float)own[c].view.frame - mine.frames[4 * g + r]), own[c].slope, p[c][r]);
        }
        if (!all_seen) {
#pragma unroll
          for (int r = 0; r < 4; ++r) p[c][r] = there != 0 && sees_token(a, q, own[c], token + 4 * g + r) ? p[c][r] : kMinusInf;
        }
        const float mx = row_max(fmaxf(fmaxf(p[c][0], p[c][1]), fmaxf(p[c][2], p[c][3])));
        const bool moves = mx > soft[c].ref + kLazyLog2 / rule.c2;
        if (__builtin_amdgcn_ballot_w64(moves) != 0) {
          const float ref = moves ? mx : soft[c].ref;
          const float alpha = moves && soft[c].ref != kMinusInf ? __builtin_amdgcn_exp2f((soft[c].ref - ref) * rule.c2) : 1.f;
          soft[c].ref = ref;
          soft[c].sum *= alpha;
#pragma unroll
          for (int t = 0; t < S::kBlocks; ++t) sum[c][t] *= alpha;
        }
        const float shift = soft[c].ref == kMinusInf ? 0.f : -soft[c].ref * rule.c2;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[c][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[c][r], rule.c2, shift));
          soft[c].sum += p[c][r];
        }
      }
      auto sums = [&](auto both) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 4 * g + r;
#pragma unroll
          for (int t = 0; t < S::kBlocks; ++t) {
            const float v = *reinterpret_cast<const float*>(y + row * S::kRowBytes + (((4 * t + (i >> 2)) ^ row) << 4) + (i & 3) * 4);
            sum[0][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[0][r], sum[0][t], 0, 0, 0);
            if constexpr (both) sum[1][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[1][r], sum[1][t], 0, 0, 0);
          }
        }
      };
      columns == 2 ? sums(std::true_type()) : sums(std::false_type());
      there = next_there;
    }

    // the wave's sums, row by row
    WAIT_LGKMCNT0();
#pragma unroll
    for (int c = 0; c < kF32Columns; ++c) {
      const float total = sum_of_row(soft[c].sum);
#pragma unroll
      for (int t = 0; t < S::kBlocks; ++t) *reinterpret_cast<floatx4*>(&mine.sums[16 * c + i][16 * t + 4 * g]) = sum[c][t];
      if (g == 0) mine.sums[16 * c + i][D] = soft[c].ref, mine.sums[16 * c + i][D + 1] = total;
    }
    __syncthreads();
    finish_rows<D, float, kF32Waves>(a, rule, share, lds, first_row, rows);
    if (!share.next(a)) break;
    __syncthreads();  // (the sums lie where the next steps go)
  }
  share.leave(a, true);
}

template <int D>
__global__ __launch_bounds__(kF32Threads) void f32_join_kernel(AttendArgs a) {
  join_pieces<D, float, kFewRows, kF32Threads, kF32Threads / (D / 4)>(a);
}

template <int D>
hipError_t launch_f32(const AttendArgs& a, hipStream_t stream) {
  const int64_t workgroups = a.way == kShares ? a.workgroups : a.tiles * a.kv_heads;
  if (a.many || a.way == kParts || workgroups < 1 || workgroups > 0xffffff) return hipErrorInvalidValue;  // (2^32 threads)
  f32_kernel<D><<<(unsigned)workgroups, kF32Threads, 0, stream>>>(a);
  if (a.way == kShares) {
    const int64_t rows = (int64_t)((a.tokens + a.sequences - 1) / a.sequences) * a.group;
    f32_join_kernel<D><<<dim3((unsigned)workgroups, (unsigned)(rows < kFewRows ? rows : kFewRows)), kF32Threads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_f32(const AttendArgs& a, hipStream_t stream) { return a.D == 64 ? launch_f32<64>(a, stream) : launch_f32<128>(a, stream); }

}  // namespace ca
