// Scored attention on the bf16 matrix instructions: scores that are capped, biased and masked, forwards and backwards.
//
//   s = scale q.k;  s = cap tanh(s / cap);  s -= slope |p_q - p_k|;  visible where documents agree and p_k <= limit_q
//   O = softmax(s) V,  L = log sum exp s
//   P = exp(s - L),  dV = P^T dO,  dP = dO V^T,  dS = P (dP - rowsum(dO O)) (1 - tanh^2),  dQ = scale dS K,  dK = scale dS^T Q
//
// One shape of kernel serves all of them.  A workgroup owns a tile of queries (forward, dQ) or of keys (dK, dV), a wave 32 of its
// tokens, one a lane: they are the columns of every product, and stay in registers.  The tokens of the other side stream through LDS in steps of two
// tensors X and Y: keys and values, or queries and gradients dO.  With S^T = X own^T, a lane holds the scores of its token, so that the
// weights, rounded to bf16, are register for register the second operand of the products that follow, which read X or Y transposed from LDS:
//             own         X, Y     S        dP       sums
//   forward   q           k, v     X q^T    -        O^T  += Y^T P
//   dQ        q, dO       k, v     X q^T    Y dO^T   dQ^T += X^T dS
//   dK, dV    k, v        q, dO    X k^T    Y v^T    dK^T += X^T dS,  dV^T += Y^T P
// Sums over tokens are fp32 in the matrix accumulators; weights and dS are rounded to bf16 as their products' operands, as in the other bf16 kernels.
//
// A step of X and Y is copied straight into LDS while the one before is computed (two buffers, one barrier a step).  Both are read by rows and
// transposed, so one swizzle of the 16-byte chunks serves both patterns (see swizzle).  What the scores need of the streamed tokens (position, document, limit;
// log-sum-exp and delta backwards) is copied the same way.  The list of a row is cut into steps up front, 512 tiles at a time, by all threads: steps without a
// token and, by the tiles' ranges of documents, positions and limits, tiles without a visible pair are left out, and tiles with nothing but visible pairs are marked, so
// that the others alone compare anything.
#pragma once

#include "attn_bf16_common.h"
#include "scored.h"

namespace ca {
namespace {

enum ScoredKernel { kScoredForward, kScoredDQ, kScoredDKV, kScoredDK, kScoredDV };
constexpr bool owns_keys(ScoredKernel k) { return k == kScoredDKV || k == kScoredDK || k == kScoredDV; }

template <int B_, int D_>
struct ScoredShape {
  static constexpr int B = B_, D = D_;
  static constexpr int kWaves = B / 32, kThreads = kWaves * 64;
  // Tokens of a step: two buffers of X and Y take 64 KiB (B = 128, D = 128) or 32 KiB of LDS.
  static constexpr int kStep = D == 64 ? 64 : B / 2;
  static constexpr int kHalves = B / kStep;          // steps of a tile
  static constexpr int kBlocks = kStep / 32;
  static constexpr int kRowBytes = D * 2, kChunksPerRow = D / 8, kRowsPerLoad = 1024 / kRowBytes;
  static constexpr int kStepBytes = kStep * kRowBytes;
  static constexpr int kLoads = kStepBytes / 1024 / kWaves;  // wave-wide copies of X (and of Y) per wave
  static constexpr int kContraction = D / 16, kDBlocks = D / 32;
  static constexpr int kInfoRows = 6;                // position, document, limit, -, log-sum-exp, delta
  static constexpr int kListTiles = 512;             // tiles of a list cut into steps at a time
  static_assert(kLoads == 2 || kLoads == 4, "copies are written for two or four loads");
};

template <class S>
struct ScoredLds {
  char x[2][S::kStepBytes], y[2][S::kStepBytes];
  float info[2][S::kInfoRows][S::kStep];
  uint32_t steps[S::kListTiles * S::kHalves + 2];
  int counts[S::kWaves];
};

// Logical 16-byte chunk c of row r lies at physical chunk c ^ swizzle(r).  Read by rows (16 consecutive rows, one logical chunk) the 16 places are
// distinct; read transposed (four rows of 64 consecutive bytes) every row lies in another 64-byte group.
template <int D>
__device__ __forceinline__ int swizzle(int row) {
  return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

// A word of the step list: tile id, which part of the tile, and bits 25-31: its padding class (without arrays), or 1: compare (with).
__device__ __forceinline__ int step_tile(uint32_t w) { return (int)(w & 0xffffffu); }
__device__ __forceinline__ int step_half(uint32_t w) { return (int)(w >> 24) & 1; }
__device__ __forceinline__ int step_kind(uint32_t w) { return (int)(w >> 25); }

// Copies of a step's X and Y, asynchronous.
template <class S>
struct StepCopy {
  uint32_t voff[S::kLoads];
  int wave, lane;
  __device__ __forceinline__ StepCopy(int wave_, int lane_) : wave(wave_), lane(lane_) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int row = i * S::kRowsPerLoad + lane / S::kChunksPerRow, phys = lane % S::kChunksPerRow;  // (the wave's first row is a multiple of 16)
      voff[i] = (uint32_t)((lane / S::kChunksPerRow) * S::kRowBytes + ((phys ^ swizzle<S::D>(row)) << 4));
    }
  }
  __device__ __forceinline__ void tensor(const char* step, uint32_t lds) const {
    const uint32_t slice = (uint32_t)(wave * S::kLoads) * 1024u;
    const char* sb = step + slice;
    const uint32_t m0 = lds + slice;
    if constexpr (S::kLoads == 4) {
      asm volatile(
          "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %[v0], %[sb] offset:0\n\t"
          "global_load_lds_dwordx4 %[v1], %[sb] offset:1024\n\t"
          "global_load_lds_dwordx4 %[v2], %[sb] offset:2048\n\t"
          "global_load_lds_dwordx4 %[v3], %[sb] offset:3072\n\t"
          :
          : [m0] "s"(m0), [v0] "v"(voff[0]), [v1] "v"(voff[1]), [v2] "v"(voff[2]), [v3] "v"(voff[3]), [sb] "s"(sb)
          : "memory");
    } else {
      asm volatile(
          "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %[v0], %[sb] offset:0\n\t"
          "global_load_lds_dwordx4 %[v1], %[sb] offset:1024\n\t"
          :
          : [m0] "s"(m0), [v0] "v"(voff[0]), [v1] "v"(voff[1]), [sb] "s"(sb)
          : "memory");
    }
  }
  // `rows` rows of kStep words, B words apart in memory, one after the other in LDS; a wave-wide load moves 64 words, and `wave_of` says whose turn it is.
  // rows * kStep is a multiple of 64.
  __device__ __forceinline__ void words(const float* from, uint32_t lds, int rows, int wave_of) const {
    constexpr int kRowsAtOnce = 64 / S::kStep;
    for (int r = 0; r < rows; r += kRowsAtOnce, ++wave_of) {
      if (wave_of % S::kWaves != wave) continue;
      const uint32_t off = (uint32_t)((lane / S::kStep) * S::B + lane % S::kStep) * 4u;
      const float* sb = from + r * S::B;
      const uint32_t m0 = lds + (uint32_t)(r * S::kStep) * 4u;
      asm volatile(
          "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
          "global_load_lds_dword %[v], %[sb] offset:0\n\t"
          :
          : [m0] "s"(m0), [v] "v"(off), [sb] "s"(sb)
          : "memory");
    }
  }
};

// May any query of q see a key of k?  Does every query that is there see every slot of k?
__device__ __forceinline__ bool any_visible(const TileLine& q, const TileLine& k) {
  return q.doc_min <= k.doc_max && k.doc_min <= q.doc_max && k.pos_min <= q.limit_max;
}
__device__ __forceinline__ bool all_visible(const TileLine& q, const TileLine& k) {
  return q.doc_min == q.doc_max && k.doc_min == q.doc_min && k.doc_max == q.doc_min && k.pos_max <= q.limit_min;
}

// Cuts `count` tiles of a list into steps; the number of these.  All threads take part.
template <class S, bool kLine, ScoredKernel K>
__device__ __forceinline__ int cut_steps(const ScoredArgs& a, const int32_t* meta, int count, const TileLine& own, const TileLine* tiles, ScoredLds<S>& lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const auto mask = reinterpret_cast<const uint32_t*>(a.class_mask);
  int total = 0;
  for (int first = 0; first < count; first += S::kThreads) {
    bool keep[2] = {false, false};
    uint32_t word = 0;
    if (first + tid < count) {
      const uint32_t w = (uint32_t)meta[first + tid];
      const int tile = (int)(w & 0xffffffu), cls = (int)(w >> 24) & 0x7f;
#pragma unroll
      for (int h = 0; h < S::kHalves; ++h) {
        uint32_t valid = 0;
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b) valid |= mask[cls * 4 + h * S::kBlocks + b];
        keep[h] = valid != 0;
      }
      word = (uint32_t)tile | (uint32_t)cls << 25;
      if constexpr (kLine) {
        const TileLine other = tiles[tile];
        const bool compare = owns_keys(K) ? !all_visible(other, own) : !(other.whole && all_visible(own, other));
        word = (uint32_t)tile | (compare ? 1u << 25 : 0u);
        if (!(owns_keys(K) ? any_visible(other, own) : any_visible(own, other))) keep[0] = keep[1] = false;
      }
    }
    const uint64_t b0 = __builtin_amdgcn_ballot_w64(keep[0]), b1 = __builtin_amdgcn_ballot_w64(keep[1]);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    int at = total + __popcll(b0 & below) + __popcll(b1 & below);
    if (lane == 0) lds.counts[wave] = __popcll(b0) + __popcll(b1);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < S::kWaves; ++w) {
      const int c = lds.counts[w];
      if (w < wave) at += c;
      total += c;
    }
    if (keep[0]) lds.steps[at++] = word;
    if (keep[1]) lds.steps[at] = word | 1u << 24;
    __syncthreads();
  }
  return __builtin_amdgcn_readfirstlane(total);
}

// LDS offsets of a lane's operand fragments.
template <class S>
struct Fragments {
  uint32_t row, row_swizzle, g, column[S::kDBlocks];
  __device__ __forceinline__ explicit Fragments(int lane) {
    const int i = lane & 31;
    g = (uint32_t)(lane >> 5);
    row = (uint32_t)(i * S::kRowBytes);
    row_swizzle = (uint32_t)swizzle<S::D>(i);
    // a transposing read covers rows 4 g + (lane % 16) / 4 (and those 8 further on) and the 8 bytes of channels 32 db + 16 ((lane / 16) % 2) + 4 (lane % 4)
    const int r = 4 * (int)g + ((lane & 15) >> 2), chunk = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
    for (int db = 0; db < S::kDBlocks; ++db)
      column[db] = (uint32_t)(r * S::kRowBytes + (((db * 4 + chunk) ^ swizzle<S::D>(r)) << 4) + (lane & 1) * 8);
  }
  // rows 32 block .. + 31, channels 16 s .. + 15
  __device__ __forceinline__ bf16x8 by_rows(LdsTile lds, int block, int s) const {
    const uint32_t off = (uint32_t)(block * 32 * S::kRowBytes) + row + ((((uint32_t)(2 * s) + g) ^ row_swizzle) << 4);
    return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>(lds + off);
  }
  // transposed: channels 32 db .. + 31, rows 32 block + 16 t .. + 15 in the order of a lane's accumulator registers
  __device__ __forceinline__ bf16x8 transposed(LdsTile lds, int block, int t, int db) const {
    const uint32_t at = (uint32_t)((block * 32 + t * 16) * S::kRowBytes);
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shortx4 __attribute__((address_space(3)))*)(lds + (at + column[db])));
    // eight rows further on the swizzle differs in the second bit
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shortx4 __attribute__((address_space(3)))*)(lds + (at + 8 * S::kRowBytes + (column[db] ^ 32u))));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// The scalars that turn products into scores, in raw units (before the scale): s' = s / scale.
struct ScoreRule {
  bool capped, biased;
  float bend, cap_raw;   // tanh(s / cap) = 1 - 2 / (2^(bend s') + 1)
  float slope_raw;       // minus the slope, per position
  float c2;              // scale log2(e)
  __device__ __forceinline__ ScoreRule(const ScoredArgs& a, int64_t head) {
    c2 = a.scale * kLog2e;
    capped = a.cap > 0.f;
    bend = capped ? 2.f * c2 / a.cap : 0.f;
    cap_raw = a.cap / a.scale;
    biased = a.slopes != nullptr;
    slope_raw = biased ? -a.slopes[head] / a.scale : 0.f;
  }
};

// Caps 16 scores; `steep` receives 1 - tanh^2 = 4 r (1 - r), r = 1 / (2^(bend s') + 1), where the caller wants it.
template <bool kSteep>
__device__ __forceinline__ void cap_scores(const ScoreRule& rule, floatx16& s, floatx16& steep) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float w = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[r] * rule.bend) + 1.f);
    s[r] = __builtin_fmaf(-2.f * rule.cap_raw, w, rule.cap_raw);
    if constexpr (kSteep) steep[r] = 4.f * (w - w * w);
  }
}

// Masks the padding slots of a block of 32 streamed keys (no arrays given), as QueryWave::mask_padding_keys does.
__device__ __forceinline__ void mask_slots(floatx16& s, uint32_t bits) {
  if (bits == 0xffffffffu) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int bit = 8 * (r / 4) + (r % 4);
    const uint32_t lo = 0u - ((bits >> bit) & 1u), hi = 0u - ((bits >> (bit + 4)) & 1u);
    const uint64_t keep = (uint64_t)lo | ((uint64_t)hi << 32);
    asm("v_cndmask_b32 %0, %1, %0, %2" : "+v"(s[r]) : "v"(kMinusInf), "s"(keep));
  }
}

typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(4))) int intx4;
__device__ __forceinline__ floatx4 read4(const float* row, int block, int i, int g) {
  return *reinterpret_cast<const floatx4*>(row + block * 32 + 8 * i + 4 * g);
}

// Bias and comparison of a block's scores.  own_*: of the lane's token; info: rows of the step's tokens.  own_limit is the lane's where it is a query, the
// streamed tokens' limits are read where they are.
template <class S, ScoredKernel K>
__device__ __forceinline__ void bias_and_compare(const ScoreRule& rule, floatx16& s, const float (&info)[S::kInfoRows][S::kStep], int block, int g, bool compare, float own_pos,
                                                 int own_doc, float own_limit) {
  if (!rule.biased && !compare) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const floatx4 pos = read4(info[kLinePosition], block, i, g);
    if (rule.biased)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[4 * i + e] = __builtin_fmaf(__builtin_fabsf(own_pos - pos[e]), rule.slope_raw, s[4 * i + e]);
    if (compare) {
      const intx4 doc = __builtin_bit_cast(intx4, read4(info[kLineDocument], block, i, g));
      floatx4 limit;
      if constexpr (owns_keys(K)) limit = read4(info[kLineLimit], block, i, g);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool reached = owns_keys(K) ? own_pos <= limit[e] : pos[e] <= own_limit;
        s[4 * i + e] = reached && doc[e] == own_doc ? s[4 * i + e] : kMinusInf;
      }
    }
  }
}

__device__ __forceinline__ void rounded(const floatx16& p, bf16x8 (&out)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) out[t][e] = (__bf16)p[8 * t + e];
}

template <class S>
__device__ __forceinline__ void load_own(const char* row, int g, bf16x8 (&own)[S::kContraction]) {
#pragma unroll
  for (int s = 0; s < S::kContraction; ++s) own[s] = *reinterpret_cast<const bf16x8*>(row + s * 32 + g * 16);
  // waited for here: in the loop the vector-memory counter belongs to the copies alone
#pragma unroll
  for (int s = 0; s < S::kContraction; ++s) asm volatile("" : "+v"(own[s]));
}

template <class S>
__device__ __forceinline__ void store_columns(char* row, int g, const floatx16 (&acc)[S::kDBlocks], float factor, bool real) {
#pragma unroll
  for (int db = 0; db < S::kDBlocks; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)(real ? acc[db][4 * r4 + e] * factor : 0.f);
      *reinterpret_cast<bf16x4*>(row + (db * 32 + 8 * r4 + 4 * g) * 2) = v;
    }
}

// S^T of a block: 32 streamed tokens x the lane's token
template <class S>
__device__ __forceinline__ floatx16 block_product(const Fragments<S>& f, LdsTile lds, int block, const bf16x8 (&own)[S::kContraction]) {
  floatx16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
#pragma unroll
  for (int s = 0; s < S::kContraction; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.by_rows(lds, block, s), own[s], acc, 0, 0, 0);
  return acc;
}

// sums^T += (block of the streamed tensor)^T weights
template <class S>
__device__ __forceinline__ void block_sums(const Fragments<S>& f, LdsTile lds, int block, const bf16x8 (&w)[2], floatx16 (&acc)[S::kDBlocks]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int db = 0; db < S::kDBlocks; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.transposed(lds, block, t, db), w[t], acc[db], 0, 0, 0);
}

// The softmax state of the lane's query and one step of it: see QueryWave::softmax for the lagging reference.  The row sum adds up the weights before they
// are rounded, because the log-sum-exp is an output of its own (a sum of rounded weights is off by up to 2^-8 where a row has few keys).
struct Softmax {
  float ref = kMinusInf, sum = 0.f;  // reference in raw units; this lane's share of the sum
};

template <class S, bool kLine, ScoredKernel K>
__global__ __attribute__((amdgpu_flat_work_group_size(S::kThreads, S::kThreads), amdgpu_waves_per_eu(2, 2))) void scored_kernel(ScoredArgs a) {
  constexpr bool kForward = K == kScoredForward, kKeys = owns_keys(K);
  constexpr bool kSum1 = K == kScoredDQ || K == kScoredDKV || K == kScoredDK, kSum2 = kForward || K == kScoredDKV || K == kScoredDV;
  __shared__ __attribute__((aligned(1024))) ScoredLds<S> lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, g = lane >> 5;
  const int64_t rows = (int64_t)a.num_heads * a.n;
  const int64_t linear = xcd_launch_order(blockIdx.x, gridDim.x, xcd_chunk(gridDim.x));
  const int64_t batch = linear / rows, row = a.order[linear - batch * rows], head = row / a.n, tile = row - head * a.n;
  const int64_t plane = batch * a.num_heads + head, plane_bytes = a.n * (int64_t)S::B * S::kRowBytes;
  const char* const X = static_cast<const char*>(kKeys ? a.q : a.k) + plane * plane_bytes;
  const char* const Y = static_cast<const char*>(kKeys ? a.dout : a.v) + plane * plane_bytes;
  const float* const line = kLine ? a.line + batch * a.n * kLineRows * S::B : nullptr;
  const float* const stats = kForward ? nullptr : a.rows + plane * a.n * 2 * S::B;
  const ScoreRule rule(a, head);

  // the lane's token
  const QuerySlot slot = query_slot<S::B>(a, tile, wave * 32, i);
  const bool active = slot.wave_active;
  const int64_t own_row = tile * S::B + slot.slot;
  bool there = slot.real;
  float own_pos = 0.f, own_limit = __builtin_inff(), own_lse = 0.f, own_delta = 0.f;
  int own_doc = 0;
  if constexpr (kLine) {
    const float* t = line + tile * kLineRows * S::B + slot.slot;
    own_pos = t[kLinePosition * S::B];
    own_limit = t[kLineLimit * S::B];
    own_doc = __builtin_bit_cast(int, t[kLineDocument * S::B]);
    there = there && own_doc >= 0;
    if (own_doc < 0) own_doc = -2;  // sees nothing, not even tokens without a document
  }
  bf16x8 own1[S::kContraction], own2[kSum1 ? S::kContraction : 1];
  load_own<S>(static_cast<const char*>(kKeys ? a.k : a.q) + plane * plane_bytes + own_row * S::kRowBytes, g, own1);
  if constexpr (kSum1) load_own<S>(static_cast<const char*>(kKeys ? a.v : a.dout) + plane * plane_bytes + own_row * S::kRowBytes, g, own2);
  if constexpr (K == kScoredDQ) {
    own_lse = stats[tile * 2 * S::B + slot.slot];
    own_delta = stats[tile * 2 * S::B + S::B + slot.slot];
    asm volatile("" : "+v"(own_lse), "+v"(own_delta));
  }
  asm volatile("" : "+v"(own_pos), "+v"(own_limit), "+v"(own_doc));

  floatx16 sum1[kSum1 ? S::kDBlocks : 1], sum2[kSum2 ? S::kDBlocks : 1];
#pragma unroll
  for (auto& t : sum1)
#pragma unroll
    for (int r = 0; r < 16; ++r) t[r] = 0.f;
#pragma unroll
  for (auto& t : sum2)
#pragma unroll
    for (int r = 0; r < 16; ++r) t[r] = 0.f;
  Softmax soft;

  const StepCopy<S> copy(wave, lane);
  const Fragments<S> frag(lane);
  const uint32_t lds_x = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.x[0], lds_y = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.y[0];
  const uint32_t lds_info = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.info[0][0];
  constexpr uint32_t kInfoBytes = S::kInfoRows * S::kStep * 4;
  auto issue = [&](uint32_t w, int buffer) {
    const int64_t first = (int64_t)step_tile(w) * S::B + step_half(w) * S::kStep;
    copy.tensor(X + first * S::kRowBytes, lds_x + buffer * S::kStepBytes);
    copy.tensor(Y + first * S::kRowBytes, lds_y + buffer * S::kStepBytes);
    if constexpr (kLine)
      copy.words(line + (int64_t)step_tile(w) * kLineRows * S::B + step_half(w) * S::kStep, lds_info + buffer * kInfoBytes, kKeys ? 4 : 2, 0);
    if constexpr (kKeys)
      copy.words(stats + (int64_t)step_tile(w) * 2 * S::B + step_half(w) * S::kStep, lds_info + buffer * kInfoBytes + 4 * S::kStep * 4, 2, 2);
  };

  const TileLine* const tiles = kLine ? a.tiles + batch * a.n : nullptr;
  TileLine own_tile{};
  if constexpr (kLine) own_tile = tiles[tile];
  const int64_t begin = a.row_ptr[row];
  const int count = (int)(a.row_ptr[row + 1] - begin);
  for (int first = 0; first < count; first += S::kListTiles) {
    const int steps = cut_steps<S, kLine, K>(a, a.col_meta + begin + first, min(S::kListTiles, count - first), own_tile, tiles, lds);
    if (steps == 0) continue;
    uint32_t word = __builtin_amdgcn_readfirstlane(lds.steps[0]), next = 0;
    if (steps > 1) next = __builtin_amdgcn_readfirstlane(lds.steps[1]);
    issue(word, 0);
    for (int step = 0; step < steps; ++step) {
      const int buffer = step & 1;
      uint32_t after = 0;
      if (step + 2 < steps) after = lds.steps[step + 2];
      WAIT_VMCNT(0);
      WAIT_LGKMCNT0();
      BARRIER();  // the step's X and Y are there, and nobody reads the other buffer any more
      if (step + 1 < steps) issue(next, buffer ^ 1);
      if (active) {
        const LdsTile x = (LdsTile)lds.x[buffer], y = (LdsTile)lds.y[buffer];
        const float(&info)[S::kInfoRows][S::kStep] = lds.info[buffer];
        const bool compare = kLine && step_kind(word) != 0;
        const auto valid = CONST_PTR(uint32_t, a.class_mask) + (kLine ? 0 : step_kind(word) * 4 + step_half(word) * S::kBlocks);
        if constexpr (kForward) {
          floatx16 s[S::kBlocks], unused;
#pragma unroll
          for (int b = 0; b < S::kBlocks; ++b) s[b] = block_product<S>(frag, x, b, own1);
          if (rule.capped)
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) cap_scores<false>(rule, s[b], unused);
          if constexpr (kLine) {
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) bias_and_compare<S, K>(rule, s[b], info, b, g, compare, own_pos, own_doc, own_limit);
          } else if (step_kind(word) != 0) {
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) mask_slots(s[b], __builtin_amdgcn_readfirstlane(valid[b]));
          }
          float mx = s[0][0];
#pragma unroll
          for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
          mx = max_with_partner(mx);
          const bool moves = mx > soft.ref + kLazyLog2 / rule.c2;
          if (__builtin_amdgcn_ballot_w64(moves) != 0) {
            const float to = moves ? mx : soft.ref;
            const float alpha = moves && soft.ref != kMinusInf ? __builtin_amdgcn_exp2f((soft.ref - to) * rule.c2) : 1.f;
            soft.ref = to;
            soft.sum *= alpha;
#pragma unroll
            for (int db = 0; db < S::kDBlocks; ++db)
#pragma unroll
              for (int r = 0; r < 16; ++r) sum2[db][r] *= alpha;
          }
          const float shift = soft.ref == kMinusInf ? 0.f : -soft.ref * rule.c2;
#pragma unroll
          for (int b = 0; b < S::kBlocks; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], rule.c2, shift));
              soft.sum += s[b][r];
            }
            bf16x8 p[2];
            rounded(s[b], p);
            block_sums<S>(frag, y, b, p, sum2);
          }
        } else {
#pragma unroll
          for (int b = 0; b < S::kBlocks; ++b) {
            floatx16 steep;
            floatx16 s = block_product<S>(frag, x, b, own1);
            if (rule.capped) cap_scores<kSum1>(rule, s, steep);
            if constexpr (kLine) {
              bias_and_compare<S, K>(rule, s, info, b, g, compare, own_pos, own_doc, own_limit);
            } else if (K == kScoredDQ && step_kind(word) != 0) {
              mask_slots(s, __builtin_amdgcn_readfirstlane(valid[b]));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              floatx4 lse;
              if constexpr (kKeys) lse = read4(info[4], b, j, g);
#pragma unroll
              for (int e = 0; e < 4; ++e) s[4 * j + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * j + e], rule.c2, -(kKeys ? lse[e] : own_lse)));
            }
            if constexpr (kSum2) {
              bf16x8 p[2];
              rounded(s, p);
              block_sums<S>(frag, y, b, p, sum2);
            }
            if constexpr (kSum1) {
            const floatx16 dp = block_product<S>(frag, y, b, own2);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              floatx4 delta;
              if constexpr (kKeys) delta = read4(info[5], b, j, g);
#pragma unroll
              for (int e = 0; e < 4; ++e) s[4 * j + e] *= dp[4 * j + e] - (kKeys ? delta[e] : own_delta);
            }
            if (rule.capped)
#pragma unroll
              for (int r = 0; r < 16; ++r) s[r] *= steep[r];
            bf16x8 ds[2];
            rounded(s, ds);
            block_sums<S>(frag, x, b, ds, sum1);
            }
          }
        }
      }
      word = next;
      next = __builtin_amdgcn_readfirstlane(after);
    }
    WAIT_LGKMCNT0();
    BARRIER();  // before the list and the buffers are filled again
  }

  const int64_t at = plane * plane_bytes + own_row * S::kRowBytes;
  if constexpr (kForward) {
    const float sum = sum_with_partner(soft.sum);
    const bool empty = !there || sum == 0.f;
    store_columns<S>(static_cast<char*>(a.out) + at, g, sum2, 1.f / sum, !empty);
    if (g == 0) a.lse[plane * a.n * S::B + own_row] = empty ? kMinusInf : (soft.ref * rule.c2 + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
  }
  if constexpr (K == kScoredDQ) store_columns<S>(static_cast<char*>(a.dq) + at, g, sum1, a.scale, there);
  if constexpr (kKeys) {
    if constexpr (kSum1) store_columns<S>(static_cast<char*>(a.dk) + at, g, sum1, a.scale, there);
    if constexpr (kSum2) store_columns<S>(static_cast<char*>(a.dv) + at, g, sum2, 1.f, there);
  }
}

template <ScoredKernel K, int B, int D>
hipError_t launch_shape(const ScoredArgs& a, hipStream_t stream) {
  using S = ScoredShape<B, D>;
  const int64_t workgroups = (int64_t)a.batch * a.num_heads * a.n;
  if (workgroups < 1 || workgroups > 0x7fffffff) return hipErrorInvalidValue;
  if (a.line) scored_kernel<S, true, K><<<(unsigned)workgroups, S::kThreads, 0, stream>>>(a);
  else scored_kernel<S, false, K><<<(unsigned)workgroups, S::kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <ScoredKernel K, int D>
hipError_t launch_scored(const ScoredArgs& a, hipStream_t stream) {
  if (a.D != D || (a.B != 64 && a.B != 128)) return hipErrorInvalidValue;
  return a.B == 64 ? launch_shape<K, 64, D>(a, stream) : launch_shape<K, 128, D>(a, stream);
}

}  // namespace
}  // namespace ca
