// Scored attention on the bf16 matrix instructions: scores that are capped, biased and masked, forwards and backwards.
//
//   s = scale q.k;  s = cap tanh(s / cap);  s -= slope |p_q - p_k|;  visible where documents agree and p_k <= limit_q
//   O = softmax(s) V,  L = log sum exp s
//   P = exp(s - L),  dV = P^T dO,  dP = dO V^T,  dS = P (dP - rowsum(dO O)) (1 - tanh^2),  dQ = scale dS K,  dK = scale dS^T Q
//
// One shape of kernel serves all of them.  A workgroup owns 128 queries (forward, dQ) or keys (dK, dV), a tile or two neighbours (ScoredWalk), a wave 32 of
// them, one a lane: they are the columns of every product, and stay in registers.  The tokens of the other side stream through LDS in steps of two
// tensors X and Y: keys and values, or queries and gradients dO.  With S^T = X own^T, a lane holds the scores of its token, so that the
// weights, rounded to bf16, are register for register the second operand of the products that follow, which read X or Y transposed from LDS:
//             own         X, Y     S        dP       sums
//   forward   q           k, v     X q^T    -        O^T  += Y^T P
//   dQ        q, dO       k, v     X q^T    Y dO^T   dQ^T += X^T dS,  and X^T P (RowSums)
//   dK, dV    k, v        q, dO    X k^T    Y v^T    dK^T += X^T dS,  dV^T += Y^T P
// Sums over tokens are fp32 in the matrix accumulators; weights and dS are rounded to bf16 as their products' operands, as in the other bf16 kernels.
//
// A step of X and Y is copied straight into LDS while the one before is computed (two buffers, one barrier a step).  Both are read by rows and
// transposed, so one swizzle of the 16-byte chunks serves both patterns (see swizzle).  What the scores need of the streamed tokens (position, document, limit;
// log-sum-exp and delta backwards) is copied the same way.  Which steps there are is settled before (ScoredWalk): with token arrays, by the tiles' ranges of documents, positions and
// limits, tiles without a visible pair are left out, and those with nothing but visible pairs are marked, so that the others alone compare anything.
#pragma once

#include "attn_bf16_common.h"
#include "scored.h"

namespace ca {
namespace {

enum ScoredKernel { kScoredForward, kScoredDQ, kScoredDKV };

// Waves per SIMD that a kernel's registers leave room for.  Head dim 64, measured at 8K and 20K tokens, 12 heads: forward with two / four 311 / 294 and 745 / 664 us;
// gradients with two and 64-token buffers / three, with half of those and the own operands in LDS 905 / 884 and 2054 / 1986 us.  Head dim 128 has registers for
// two; the forward kernel with three and 32-token buffers takes the same time (20K tokens in all: the products' power is the limit).
constexpr int scored_waves(ScoredKernel k, int D) { return D == 128 ? 2 : k == kScoredForward ? 4 : 3; }

template <int B_, int D_, int kStep_ = 64>
struct ScoredShape {
  static constexpr int B = B_, D = D_;               // B: tokens of a tile
  static constexpr int kWaves = kGroupTokens / 32, kThreads = kWaves * 64;
  static constexpr int kTiles = kGroupTokens / B;    // tiles of a group
  static constexpr int kStep = kStep_;               // streamed tokens in a buffer: a step, or half of one
  static constexpr int kSubs = 64 / kStep;
  static constexpr int kBlocks = kStep / 32;
  static constexpr int kRowBytes = D * 2, kChunksPerRow = D / 8, kRowsPerLoad = 1024 / kRowBytes;
  static constexpr int kStepBytes = kStep * kRowBytes;
  static constexpr int kLoads = kStepBytes / 1024 / kWaves;  // wave-wide copies of X (and of Y) per wave
  static constexpr int kContraction = D / 16, kDBlocks = D / 32;
  static constexpr int kInfoRows = 6;                // position, document, limit, -, log-sum-exp, delta
  static_assert(kLoads == 1 || kLoads == 2 || kLoads == 4, "copies are written for one, two or four loads");
};

template <class S, int kOwnSteps>
struct ScoredLds {
  char x[2][S::kStepBytes], y[2][S::kStepBytes];
  float info[2][S::kInfoRows][64];
  bf16x8 own[kOwnSteps > 0 ? S::kWaves * kOwnSteps * 64 : 1];  // of the waves' own operands, see OwnOperand
};

// Logical 16-byte chunk c of row r lies at physical chunk c ^ swizzle(r).  Read by rows (16 consecutive rows, one logical chunk) the 16 places are
// distinct; read transposed (four rows of 64 consecutive bytes) every row lies in another 64-byte group.
template <int D>
__device__ __forceinline__ int swizzle(int row) {
  return D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

__device__ __forceinline__ int step_tile(uint32_t w) { return (int)(w & 0xffffffu); }
__device__ __forceinline__ int step_half(uint32_t w) { return (int)(w >> 24) & 1; }
__device__ __forceinline__ int step_class(uint32_t w) { return (int)(w >> 25) & 15; }
constexpr uint32_t kStepCompares = 1u << 29;

// Copies of a step's X and Y, asynchronous.
template <class S>
struct StepCopy {
  uint32_t voff[S::kLoads];
  int wave, lane;
  __device__ __forceinline__ StepCopy(int wave_, int lane_) : wave(wave_), lane(lane_) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int row = (wave * S::kLoads + i) * S::kRowsPerLoad + lane / S::kChunksPerRow, phys = lane % S::kChunksPerRow;
      voff[i] = (uint32_t)((lane / S::kChunksPerRow) * S::kRowBytes + ((phys ^ swizzle<S::D>(row)) << 4));
    }
  }
  __device__ __forceinline__ void tensor(const char* step, uint32_t lds) const {
    const uint32_t slice = (uint32_t)(wave * S::kLoads) * 1024u;
    const char* sb = step + slice;
    const uint32_t m0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds + slice));
    if constexpr (S::kLoads == 4) {
      asm volatile(
          "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %[v0], %[sb] offset:0\n\t"
          "global_load_lds_dwordx4 %[v1], %[sb] offset:1024\n\t"
          "global_load_lds_dwordx4 %[v2], %[sb] offset:2048\n\t"
          "global_load_lds_dwordx4 %[v3], %[sb] offset:%[o3]\n\t"
          :
          : [o3] "n"(3 * 1024), [m0] "s"(m0), [v0] "v"(voff[0]), [v1] "v"(voff[1]), [v2] "v"(voff[2]), [v3] "v"(voff[3]), [sb] "s"(sb)
          : "memory");
    } else if constexpr (S::kLoads == 2) {
      asm volatile(
          "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %[v0], %[sb] offset:0\n\t"
          "global_load_lds_dwordx4 %[v1], %[sb] offset:1024\n\t"
          :
          : [m0] "s"(m0), [v0] "v"(voff[0]), [v1] "v"(voff[1]), [sb] "s"(sb)
          : "memory");
    } else {
      copy_rows(m0, sb, voff[0]);
    }
  }
  // `rows` rows of a step's 64 words, B words apart in memory, one after the other in LDS: row r by wave first_wave + r.
  __device__ __forceinline__ void words(const float* from, uint32_t lds, int rows, int first_wave) const {
    const int r = (wave - first_wave) & (S::kWaves - 1);
    if (r >= rows) return;
    const float* sb = from + r * S::B;
    const uint32_t off = (uint32_t)lane * 4u, m0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds + (uint32_t)(r * 64) * 4u));
    asm volatile(
        "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
        "global_load_lds_dword %[v], %[sb] offset:0\n\t"
        :
        : [m0] "s"(m0), [v] "v"(off), [sb] "s"(sb)
        : "memory");
  }
};

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

// The scalars that turn products q.k into scores.  Scores are held in a unit of their own, x, with log2(e) s = c2 x + offset: without a cap x is the
// product itself, with one x = -1 / (2^(bend q.k) + 1), which is (tanh(s / cap) - 1) / 2: the last steps of the tanh are part of the factor and of an offset
// that the softmax does not see.
struct ScoreRule {
  bool capped, biased;
  float bend, c2, offset;
  float slope;           // minus the slope, in units of x per position
  float slope2;          // the same in powers of two
  __device__ __forceinline__ ScoreRule(const ScoredArgs& a, int64_t head) {
    capped = a.cap > 0.f;
    bend = capped ? 2.f * a.scale * kLog2e / a.cap : 0.f;
    c2 = (capped ? 2.f * a.cap : a.scale) * kLog2e;
    offset = capped ? a.cap * kLog2e : 0.f;
    biased = a.slopes != nullptr;
    slope = biased ? -a.slopes[head] / (capped ? 2.f * a.cap : a.scale) : 0.f;
    slope2 = biased ? -a.slopes[head] * kLog2e : 0.f;
  }
};

// Caps 16 scores.
__device__ __forceinline__ void cap_scores(const ScoreRule& rule, floatx16& s) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(s[r] * rule.bend));
}

// Masks the padding slots of a block of 32 streamed tokens where pairs are not compared, as QueryWave::mask_padding_keys does.
__device__ __forceinline__ void mask_slots(floatx16& s, uint32_t bits, float hidden) {
  if (bits == 0xffffffffu) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int bit = 8 * (r / 4) + (r % 4);
    const uint32_t lo = 0u - ((bits >> bit) & 1u), hi = 0u - ((bits >> (bit + 4)) & 1u);
    const uint64_t keep = (uint64_t)lo | ((uint64_t)hi << 32);
    asm("v_cndmask_b32 %0, %1, %0, %2" : "+v"(s[r]) : "v"(hidden), "s"(keep));
  }
}

typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(4))) int intx4;
__device__ __forceinline__ floatx4 read4(const float* row, int block, int i, int g) {
  return *reinterpret_cast<const floatx4*>(row + block * 32 + 8 * i + 4 * g);
}

// Bias of a block's scores.  own_pos: of the lane's token; info: rows of the step's tokens.
template <class S>
__device__ __forceinline__ void bias_scores(const ScoreRule& rule, floatx16& s, const float (&info)[S::kInfoRows][64], int block, int g, float own_pos) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const floatx4 pos = read4(info[kLinePosition], block, i, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[4 * i + e] = __builtin_fmaf(__builtin_fabsf(own_pos - pos[e]), rule.slope, s[4 * i + e]);
  }
}

// Documents and limits of a block: hidden pairs get the score `hidden`.  own_limit is the lane's where it is a query; else the streamed tokens' limits are read.
template <class S, ScoredKernel K>
__device__ __forceinline__ void hide_scores(floatx16& s, const float (&info)[S::kInfoRows][64], int block, int g, float own_pos, int own_doc, float own_limit, float hidden) {
  constexpr bool kKeys = K == kScoredDKV;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const floatx4 reach = read4(info[kKeys ? kLineLimit : kLinePosition], block, i, g);
    const intx4 doc = __builtin_bit_cast(intx4, read4(info[kLineDocument], block, i, g));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool seen = (int)(kKeys ? own_pos <= reach[e] : reach[e] <= own_limit) & (int)(doc[e] == own_doc);
      s[4 * i + e] = seen ? s[4 * i + e] : hidden;
    }
  }
}

__device__ __forceinline__ void rounded(const floatx16& p, bf16x8 (&out)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) out[t][e] = (__bf16)p[8 * t + e];
}

// A token's own operand: the fragments of its first kInRegisters contraction steps are held in registers, those of the others in LDS, lane by lane (read by the
// wave that wrote them).
template <class S, int kInRegisters>
struct OwnOperand {
  bf16x8 held[kInRegisters > 0 ? kInRegisters : 1];
  const bf16x8* rest;
  __device__ __forceinline__ OwnOperand(const char* row, int g, bf16x8* lds) : rest(lds) {
    const bf16x8* from = reinterpret_cast<const bf16x8*>(row + g * 16);
#pragma unroll
    for (int s = 0; s < kInRegisters; ++s) held[s] = from[2 * s];
#pragma unroll
    for (int s = kInRegisters; s < S::kContraction; ++s) lds[(s - kInRegisters) * 64] = from[2 * s];
    // waited for here: in the loop the vector-memory counter belongs to the copies alone
#pragma unroll
    for (int s = 0; s < kInRegisters; ++s) asm volatile("" : "+v"(held[s]));
  }
  __device__ __forceinline__ bf16x8 at(int s) const { return s < kInRegisters ? held[s < kInRegisters ? s : 0] : rest[(s - kInRegisters) * 64]; }
};

__device__ __forceinline__ floatx16 splat(float x) {
  floatx16 v;
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = x;
  return v;
}

// S^T of a block, 32 streamed tokens x the lane's token, added to acc
template <class S, class Own>
__device__ __forceinline__ floatx16 block_product(const Fragments<S>& f, LdsTile lds, int block, const Own& own, floatx16 acc) {
#pragma unroll
  for (int s = 0; s < S::kContraction; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.by_rows(lds, block, s), own.at(s), acc, 0, 0, 0);
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

// The same for two sums of the same tensor.
template <class S>
__device__ __forceinline__ void block_sums(const Fragments<S>& f, LdsTile lds, int block, const bf16x8 (&w)[2], floatx16 (&acc)[S::kDBlocks], const bf16x8 (&w2)[2],
                                           floatx16 (&acc2)[S::kDBlocks]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int db = 0; db < S::kDBlocks; ++db) {
      const bf16x8 v = f.transposed(lds, block, t, db);
      acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[t], acc[db], 0, 0, 0);
      acc2[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w2[t], acc2[db], 0, 0, 0);
    }
}

__device__ __forceinline__ float sum_of_rounded(const bf16x8 (&w)[2], float sum) {
  bf16x2 ones;
  ones[0] = ones[1] = (__bf16)1.0f;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(w[t], w[t], 0, 1), ones, sum, false);
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(w[t], w[t], 2, 3), ones, sum, false);
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(w[t], w[t], 4, 5), ones, sum, false);
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(w[t], w[t], 6, 7), ones, sum, false);
  }
  return sum;
}

// The softmax state of the lane's query: see QueryWave::softmax for the lagging reference.  The row sum adds up the weights before they
// are rounded, because the log-sum-exp is an output of its own (a sum of rounded weights is off by up to 2^-8 where a row has few keys).
struct Softmax {
  float ref = kMinusInf, sum = 0.f;  // reference in units of x; this lane's share of the sum
};

// What the lane's query of dQ adds up besides, over its share of the keys.  delta comes from the rounded result, and dS is rounded as an operand; both shift all of
// a row's dS the same way, and such a shift meets the weighted mean of the keys, which is not small.  In exact arithmetic P (dP - delta) sums to zero over a row, and so the
// row's sums say what the shift is: `lean` is by how much delta is off, `excess` what rounding added.  dQ is put right at the end by as much of
// sum2 = sum of (P steep) K, and delta by lean, for dK.  Without a cap excess is the sum of the rounded dS, both in one, and delta is put right by that: what rounding adds to
// it is small beside the roundings of dK's own dS.  (Relative error of dQ / dK at scores of a spread of 3: 3.6e-3 / 2.7e-3 without, 2.2e-3 / 2.2e-3 with, of which
// 1.7e-3 is the rounding of the result.  It is one product more, of seven: 36K tokens, dense, forwards not counted, 17.0 / 17.8 ms at head dim 128 and 9.1 / 9.3 at 64, the latter as it is now.)
struct RowSums {
  float lean = 0.f, excess = 0.f, weight = 0.f;  // sums of P (dP - delta), of dS rounded less dS, of P steep; without a cap of dS rounded alone
};

// The lane's token, and what becomes of its sums.
template <class S, bool kLine>
struct OwnToken {
  int32_t tile, row;    // row: in the plane
  bool active, there;   // the wave has tokens at all; the token is in the grid and has a document that is not negative
  bool writes;          // it has a row
  float pos = 0.f, limit = __builtin_inff();
  int doc = 0;
  __device__ __forceinline__ OwnToken(const ScoredArgs& a, int64_t batch, int64_t first_tile, int wave, int i) {
    constexpr int kWavesPerTile = S::B / 32;
    tile = (int32_t)first_tile + wave / kWavesPerTile;
    writes = tile < a.n;
    if (!writes) tile = (int32_t)a.n - 1;
    const QuerySlot slot = query_slot<S::B>(a, tile, wave % kWavesPerTile * 32, i);
    active = slot.wave_active && writes;
    row = tile * S::B + slot.slot;
    there = slot.real && writes;
    if constexpr (kLine) {
      const float* t = a.line + ((batch * a.n + tile) * kLineRows * S::B + slot.slot);
      pos = t[kLinePosition * S::B];
      limit = t[kLineLimit * S::B];
      doc = __builtin_bit_cast(int, t[kLineDocument * S::B]);
      there = there && doc >= 0;
      if (doc < 0) doc = -2;  // sees nothing, not even tokens without a document
    }
  }
};

// What the tokens of a wave that are there have in common, in scalar registers: a streamed token outside of it has no pair with the wave.  Where pairs are compared, a
// wave leaves out what it has no pair with (two lanes' worth of reads and a ballot a step; 9K tokens, three clips in a causal order, forward and backward: 1420 / 1360 us
// without / with, 8K tokens causal at head dim 64, few steps compared: 139 / 141).
template <bool kKeys>
struct WaveLine {
  int doc_min = 0x7fffffff, doc_max = -1;
  float reach = kKeys ? __builtin_inff() : kMinusInf;  // lowest position of the keys, highest limit of the queries
  template <class Token>
  __device__ __forceinline__ explicit WaveLine(const Token& own) {
    if (own.there) doc_min = doc_max = own.doc, reach = kKeys ? own.pos : own.limit;
#pragma unroll
    for (int step = 1; step < 32; step *= 2) {  // (both halves of a wave hold the same tokens)
      doc_min = min(doc_min, __shfl_xor(doc_min, step));
      doc_max = max(doc_max, __shfl_xor(doc_max, step));
      reach = kKeys ? fminf(reach, __shfl_xor(reach, step)) : fmaxf(reach, __shfl_xor(reach, step));
    }
    doc_min = __builtin_amdgcn_readfirstlane(doc_min);
    doc_max = __builtin_amdgcn_readfirstlane(doc_max);
    reach = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, reach)));
  }
  // With which of the lanes' streamed tokens may the wave have a pair?
  __device__ __forceinline__ uint64_t meets(int doc, float x) const {
    return __builtin_amdgcn_ballot_w64((int)(doc >= doc_min) & (int)(doc <= doc_max) & (int)(kKeys ? reach <= x : x <= reach));
  }
};

template <class S, ScoredKernel K>
constexpr int sums_of() {
  return K == kScoredForward ? 1 : 2;
}

__device__ __forceinline__ float log_sum_exp(const ScoreRule& rule, const Softmax& soft, float sum) {
  return (__builtin_fmaf(soft.ref, rule.c2, rule.offset) + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}
template <int kBlocks>
__device__ __forceinline__ void store_columns(char* row, int g, int first_block, const floatx16* acc, float factor, bool real) {
#pragma unroll
  for (int db = 0; db < kBlocks; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)(real ? acc[db][4 * r4 + e] * factor : 0.f);
      *reinterpret_cast<bf16x4*>(row + ((first_block + db) * 32 + 8 * r4 + 4 * g) * 2) = v;
    }
}
// Of sums of dS: with a cap they are made without the -4 of 1 - tanh^2 = -4 x (1 + x).
__device__ __forceinline__ float gradient_factor(const ScoredArgs& a, const ScoreRule& rule) { return rule.capped ? -4.f * a.scale : a.scale; }
// Writes channel blocks first_block .. + kBlocks - 1 of a token's results.  state: Softmax (forward) or RowSums (dQ).
template <class S, ScoredKernel K, int kBlocks, class Token, class State>
__device__ __forceinline__ void store_results(const ScoredArgs& a, const ScoreRule& rule, int64_t plane, const Token& own, int g, const State& state, int first_block,
                                              const floatx16* sum1, const floatx16* sum2) {
  if (!own.writes) return;
  const int64_t at = (plane * a.n * S::B + own.row) * S::kRowBytes;
  if constexpr (K == kScoredForward) {
    const float sum = sum_with_partner(state.sum);
    const bool real = own.there && sum != 0.f;
    if (g == 0 && first_block == 0) a.lse[plane * a.n * S::B + own.row] = real ? log_sum_exp(rule, state, sum) : kMinusInf;
    store_columns<kBlocks>(static_cast<char*>(a.out) + at, g, first_block, sum2, 1.f / sum, real);
  } else if constexpr (K == kScoredDQ) {
    const float excess = sum_with_partner(state.excess);
    float lean = excess, shift = excess;
    if (rule.capped) {
      const float weight = sum_with_partner(state.weight);
      lean = sum_with_partner(state.lean);
      shift = lean + (weight != 0.f ? excess / weight : 0.f);
    }
    floatx16 sum[kBlocks];  // (changed in place, sum1 would be copied in every step: 20K tokens, forward and backward, 4120 / 3975 us)
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[db][r] = __builtin_fmaf(-shift, sum2[db][r], sum1[db][r]);
    store_columns<kBlocks>(static_cast<char*>(a.dq) + at, g, first_block, sum, gradient_factor(a, rule), own.there);
    if (g == 0 && first_block == 0) a.rows[(plane * a.n * 2 + own.tile + 1) * S::B + own.row] -= lean;  // (tile * 2 * B + B + slot)
  } else {
    store_columns<kBlocks>(static_cast<char*>(a.dk) + at, g, first_block, sum1, gradient_factor(a, rule), own.there);
    store_columns<kBlocks>(static_cast<char*>(a.dv) + at, g, first_block, sum2, 1.f, own.there);
  }
}

// An item, in scalar registers.
__device__ __forceinline__ ScoredItem item_at(const ScoredItem* p) {
  const auto w = CONST_PTR(uint32_t, p);
  uint32_t v[6];
#pragma unroll
  for (int i = 0; i < 6; ++i) v[i] = __builtin_amdgcn_readfirstlane(w[i]);
  return ScoredItem{(int64_t)((uint64_t)v[1] << 32 | v[0]), (int32_t)v[2], (int32_t)v[3], (int32_t)v[4], (int32_t)v[5]};
}

// A wave's part of a share: floatx4 per lane, lane by lane, so that every store is whole lines.
template <class S, ScoredKernel K>
__device__ __forceinline__ float* share_at(const ScoredArgs& a, int64_t share, int wave) {
  constexpr int64_t kWaveFloats = share_floats(S::D, sums_of<S, K>()) / S::kWaves;
  return a.share_sums + (share * S::kWaves + wave) * kWaveFloats;
}

// kCapped: of gradients, whose registers a branch more costs (it spills 25 of them at head dim 64, and takes 1.7 times as long); the forward kernel asks the rule
// (compiled in 0.98 to 1.02 of the time).  With a cap all scores lie in x = -1 .. 0 (ScoreRule), and 0 could be the reference of their softmax, without a
// maximum: 33K tokens took 0.96 to 0.99 of the time, but the largest weight of a row, 1 as it is, would be rounded as well (relative error at 256 tokens 2.0e-3 / 2.2e-3).
template <class S, bool kLine, ScoredKernel K, bool kCapped>
__global__ __attribute__((amdgpu_flat_work_group_size(S::kThreads, S::kThreads), amdgpu_waves_per_eu(scored_waves(K, S::D), scored_waves(K, S::D)))) void scored_kernel(ScoredArgs a) {
  constexpr bool kForward = K == kScoredForward, kKeys = (K == kScoredDKV);
  // Gradients: two sums and both own operands would be 192 registers at head dim 128, of 256; the second operand and a part of the first are kept in LDS, as much as two
  // workgroups of a compute unit have room for (head dim 64: both, for three).  With the second alone there the kernel of dK and dV spills, and takes 1.2 times as long.
  constexpr int kHeld1 = kForward ? S::kContraction : S::D == 128 ? 5 : 0;
  constexpr int kOwnSteps1 = S::kContraction - kHeld1, kOwnSteps2 = kForward ? 0 : S::kContraction;
  __shared__ __attribute__((aligned(1024))) ScoredLds<S, kOwnSteps1 + kOwnSteps2> lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, g = lane >> 5;
  const int64_t total = a.header ? CONST_PTR(int32_t, &a.header->items)[0] : gridDim.x;
  if (blockIdx.x >= total) return;  // (all of its threads)
  const int64_t linear = xcd_launch_order(blockIdx.x, total, xcd_chunk(total)), entry = a.header ? 0 : linear / a.num_items;
  const ScoredItem item = item_at(a.items + (linear - entry * a.num_items));
  const int64_t batch = a.header ? item.batch : entry;
  const int64_t groups = (a.n + S::kTiles - 1) / S::kTiles, head = item.group / groups, first_tile = (item.group - head * groups) * S::kTiles;
  const int64_t plane = batch * a.num_heads + head, plane_bytes = a.n * (int64_t)S::B * S::kRowBytes;
  const char* const X = static_cast<const char*>(kKeys ? a.q : a.k) + plane * plane_bytes;
  const char* const Y = static_cast<const char*>(kKeys ? a.dout : a.v) + plane * plane_bytes;
  const float* const line = kLine ? a.line + batch * a.n * kLineRows * S::B : nullptr;
  const float* const stats = kForward ? nullptr : a.rows + plane * a.n * 2 * S::B;
  const ScoreRule rule(a, head);

  OwnToken<S, kLine> own(a, batch, first_tile, wave, i);
  float own_lse = 0.f, own_delta = 0.f;
  bf16x8* const own_lds = lds.own + wave * (kOwnSteps1 + kOwnSteps2) * 64 + lane;
  const int64_t own_at = plane * plane_bytes + (int64_t)own.row * S::kRowBytes;
  const OwnOperand<S, kHeld1> own1(static_cast<const char*>(kKeys ? a.k : a.q) + own_at, g, own_lds);
  const std::conditional_t<kForward, int, OwnOperand<S, 0>> own2 = [&] {
    if constexpr (kForward) return 0;
    else return OwnOperand<S, 0>(static_cast<const char*>(kKeys ? a.v : a.dout) + own_at, g, own_lds + kOwnSteps1 * 64);
  }();
  if constexpr (K == kScoredDQ) {
    const float* const t = stats + ((int64_t)own.tile * S::B + own.row);  // (tile * 2 * B + slot)
    own_lse = t[0];
    own_delta = t[S::B];
    asm volatile("" : "+v"(own_lse), "+v"(own_delta));
  }
  asm volatile("" : "+v"(own.pos), "+v"(own.limit), "+v"(own.doc));
  const WaveLine<kKeys> wave_line(own);
  const uint32_t member = 1u << (30 + wave / (S::B / 32));  // the wave's tile in a step's word

  floatx16 sum1[kForward ? 1 : S::kDBlocks], sum2[S::kDBlocks];
#pragma unroll
  for (auto& t : sum1)
#pragma unroll
    for (int r = 0; r < 16; ++r) t[r] = 0.f;
#pragma unroll
  for (auto& t : sum2)
#pragma unroll
    for (int r = 0; r < 16; ++r) t[r] = 0.f;
  Softmax soft;
  RowSums row;
  // dP - delta: the product of dP begins at minus delta, which saves a subtraction a value.  For queries it takes 16 registers more: head dim 128 has none left, and 64 with
  // token arrays would spill 25
  constexpr bool kDeltaFirst = kKeys || (S::D == 64 && !kLine);
  floatx16 minus_delta = splat(!kKeys && kDeltaFirst ? own_delta : 0.f);
  if constexpr (!kForward && !kKeys && kDeltaFirst) asm volatile("" : "+v"(minus_delta));

  // Gradients: a wave that has its weights ready goes before one that still makes them, so that matrix pipe and vector ALU are in use together (without / with: 8K tokens at head
  // dim 64 1241 / 1183 us, 9K tokens with arrays 1273 / 1243, 20K 3944 / 3878).  Plain calls at head dim 128 are bound by power, and lose 3 % by it; around the products of scores
  // it gave 0.98 to 1.01, in the forward kernel 0.96 to 1.01.
  constexpr bool kSumsFirst = S::D == 64 || kLine;
  const StepCopy<S> copy(wave, lane);
  const Fragments<S> frag(lane);
  const uint32_t lds_x = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.x[0], lds_y = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.y[0];
  const uint32_t lds_info = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds.info[0][0];
  constexpr uint32_t kInfoBytes = S::kInfoRows * 64 * 4;
  auto issue = [&](uint32_t w, int sub, int buffer) {
    const int64_t first = (int64_t)step_tile(w) * S::B + step_half(w) * 64 + sub * S::kStep;
    copy.tensor(X + first * S::kRowBytes, lds_x + buffer * S::kStepBytes);
    copy.tensor(Y + first * S::kRowBytes, lds_y + buffer * S::kStepBytes);
    if (kLine && (rule.biased || (w & kStepCompares) != 0)) copy.words(line + (int64_t)step_tile(w) * kLineRows * S::B + step_half(w) * 64, lds_info + buffer * kInfoBytes, kKeys ? 3 : 2, 0);
    if constexpr (kKeys) copy.words(stats + (int64_t)step_tile(w) * 2 * S::B + step_half(w) * 64, lds_info + buffer * kInfoBytes + 4 * 64 * 4, 2, 2);
  };

  // words are fetched two steps ahead of their use (the runs are readable two words past their end)
  const auto words = CONST_PTR(uint32_t, a.steps + item.first);
  const int steps = item.count * S::kSubs;
  uint32_t word = words[0], next = words[1 / S::kSubs];
  if (steps > 0) issue(word, 0, 0);
  {
    for (int step = 0; step < steps; ++step) {
      const int buffer = step & 1, sub = S::kSubs == 1 ? 0 : step & 1, first_block = sub * S::kBlocks;
      const uint32_t after = words[(step + 2) / S::kSubs];
      WAIT_VMCNT(0);
      WAIT_LGKMCNT0();
      BARRIER();  // the step's X and Y are there, and nobody reads the other buffer any more
      if (step + 1 < steps) issue(next, S::kSubs == 1 ? 0 : sub ^ 1, buffer ^ 1);
      const float(&info)[S::kInfoRows][64] = lds.info[buffer];
      const bool compare = kLine && (word & kStepCompares) != 0;
      bool visit = own.active && (word & member) != 0;
      if constexpr (kLine) {
        if (visit && compare) {
          const uint64_t met = wave_line.meets(__builtin_bit_cast(int, info[kLineDocument][lane]), info[kKeys ? kLineLimit : kLinePosition][lane]);
          visit = S::kStep == 64 ? met != 0 : (uint32_t)(met >> (first_block * 32)) != 0;
        }
      }
      if (visit) {
        const LdsTile x = (LdsTile)lds.x[buffer], y = (LdsTile)lds.y[buffer];
        const int cls = compare ? 0 : step_class(word);  // (padding slots have a document of their own)
        const auto valid = CONST_PTR(uint32_t, a.class_mask) + (cls * 4 + step_half(word) * 2 + first_block);
        if constexpr (kForward) {
          floatx16 s[S::kBlocks];
#pragma unroll
          for (int b = 0; b < S::kBlocks; ++b) s[b] = block_product<S>(frag, x, b, own1, splat(0.f));
          if (rule.capped)
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) cap_scores(rule, s[b]);
          if (kLine && rule.biased)
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) bias_scores<S>(rule, s[b], info, first_block + b, g, own.pos);
          if (kLine && compare)
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) hide_scores<S, K>(s[b], info, first_block + b, g, own.pos, own.doc, own.limit, kMinusInf);
          if (cls != 0) {
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) mask_slots(s[b], __builtin_amdgcn_readfirstlane(valid[b]), kMinusInf);
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
            floatx16 less = minus_delta;
            if constexpr (kKeys)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const floatx4 d = read4(info[5], first_block + b, j, g);
                less[4 * j] = d[0], less[4 * j + 1] = d[1], less[4 * j + 2] = d[2], less[4 * j + 3] = d[3];
              }
            floatx16 s = block_product<S>(frag, x, b, own1, splat(0.f)), dp = block_product<S>(frag, y, b, own2, less);
            // Both products end here.  Without it the compiler begins the weights while registers still hold the products' operands, and up to 36 values go to memory
            // at head dim 128 (forward and backward at 20K tokens, 6 heads: 4176 / 3998 us; at head dim 64, 8K tokens: 1315 / 1301).
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kCapped) cap_scores(rule, s);
            constexpr float kHidden = kCapped ? -1e18f : kMinusInf;  // (no weight either way; its square is finite, for steep)
            if (kLine && compare) hide_scores<S, K>(s, info, first_block + b, g, own.pos, own.doc, own.limit, kHidden);
            // (padding queries too, whose weights are zero with any score but NaN: their zeros times an infinite key)
            if (cls != 0) mask_slots(s, __builtin_amdgcn_readfirstlane(valid[b]), kHidden);
            // s -> P (dQ: P steep), dp -> dS.  One value at a time, so that nothing else is held: steep = 1 - tanh^2 = -4 x (1 + x) is made from x when it is used, its -4 is left to the
            // results (gradient_factor), the bias goes into the exponent.
            auto weigh = [&](auto biased) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                floatx4 lse, pos;
                if constexpr (kKeys) lse = read4(info[4], first_block + b, j, g);
                if constexpr (biased) pos = read4(info[kLinePosition], first_block + b, j, g);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float v = s[4 * j + e];
                  float shift = kKeys ? -lse[e] : -own_lse;
                  if constexpr (biased) shift = __builtin_fmaf(__builtin_fabsf(own.pos - pos[e]), rule.slope2, shift);
                  float p = __builtin_amdgcn_exp2f(__builtin_fmaf(v, rule.c2, shift)), t = p * (kDeltaFirst ? dp[4 * j + e] : dp[4 * j + e] + own_delta);
                  if constexpr (!kKeys && kCapped) row.lean += t;
                  if constexpr (kCapped) {
                    const float steep = __builtin_fmaf(v, v, v);
                    t *= steep;
                    if constexpr (!kKeys) row.excess -= t, p *= steep;
                  }
                  s[4 * j + e] = p;
                  dp[4 * j + e] = t;
                }
              }
            };
            if (kLine && rule.biased) weigh(std::bool_constant<kLine>());
            else weigh(std::false_type());
            bf16x8 p[2], ds[2];
            rounded(s, p);
            rounded(dp, ds);
            if constexpr (kSumsFirst) __builtin_amdgcn_s_setprio(1);
            if constexpr (kKeys) {
              block_sums<S>(frag, y, b, p, sum2);
              block_sums<S>(frag, x, b, ds, sum1);
            } else {
              row.excess = sum_of_rounded(ds, row.excess);
              if constexpr (kCapped) row.weight = sum_of_rounded(p, row.weight);
              block_sums<S>(frag, x, b, ds, sum1, p, sum2);
            }
            if constexpr (kSumsFirst) __builtin_amdgcn_s_setprio(0);
          }
        }
      }
      word = next;
      next = after;
    }
  }

  const auto state = [&] {
    if constexpr (kForward) return soft;
    else return row;
  }();
  if (item.share < 0) {
    store_results<S, K, S::kDBlocks>(a, rule, plane, own, g, state, 0, sum1, sum2);
    return;
  }
  floatx4* out = reinterpret_cast<floatx4*>(share_at<S, K>(a, entry * a.shares + item.share, wave)) + lane;
  *out = kForward ? floatx4{soft.ref, soft.sum, 0.f, 0.f} : floatx4{row.lean, row.excess, row.weight, 0.f};
  out += 64;
  auto leave = [&](const floatx16* sums) {
#pragma unroll
    for (int j = 0; j < 4 * S::kDBlocks; ++j, out += 64) *out = floatx4{sums[j / 4][j % 4 * 4], sums[j / 4][j % 4 * 4 + 1], sums[j / 4][j % 4 * 4 + 2], sums[j / 4][j % 4 * 4 + 3]};
  };
  if constexpr (!kForward) leave(sum1);
  leave(sum2);
}

// Adds up the shares of a group, in their order, and writes its results: a workgroup takes 32 tokens, a wave 32 channels of them.  Bound: latency, and the shares
// once.
template <class S, bool kLine, ScoredKernel K>
__global__ __launch_bounds__(S::kDBlocks * 64) void scored_merge_kernel(ScoredArgs a) {
  constexpr bool kForward = K == kScoredForward;
  constexpr int kAhead = 4;  // shares that are loaded before the first is added
  const int lane = threadIdx.x & 63, block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 31, g = lane >> 5;
  const int wave = blockIdx.x % S::kWaves;
  const int64_t linear = blockIdx.x / S::kWaves, entry = a.header ? 0 : linear / a.num_merges;
  if (a.header && linear >= CONST_PTR(int32_t, &a.header->merges)[0]) return;
  const ScoredMerge merge = a.merges[linear - entry * a.num_merges];
  const int64_t batch = a.header ? merge.batch : entry;
  const int64_t groups = (a.n + S::kTiles - 1) / S::kTiles, head = merge.group / groups, first_tile = (merge.group - head * groups) * S::kTiles;
  const int64_t plane = batch * a.num_heads + head;
  const ScoreRule rule(a, head);
  const OwnToken<S, kLine> own(a, batch, first_tile, wave, i);
  floatx16 sum1, sum2;
#pragma unroll
  for (int r = 0; r < 16; ++r) sum1[r] = sum2[r] = 0.f;
  Softmax soft;
  RowSums row;
  for (int first = 0; first < merge.shares; first += kAhead) {
    floatx4 stats[kAhead], part1[kAhead][4], part2[kAhead][4];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (first + k >= merge.shares) break;
      const floatx4* in = reinterpret_cast<const floatx4*>(share_at<S, K>(a, entry * a.shares + merge.first_share + first + k, wave)) + lane;
      stats[k] = *in;
      in += 64 + block * 256;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (!kForward) part1[k][j] = in[j * 64];
        part2[k][j] = in[(kForward ? 0 : S::kDBlocks * 256) + j * 64];
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (first + k >= merge.shares) break;
      float weight = 1.f, old = 1.f;
      if constexpr (kForward) {
        const float ref = fmaxf(soft.ref, stats[k][0]);
        old = soft.ref == kMinusInf ? 0.f : __builtin_amdgcn_exp2f((soft.ref - ref) * rule.c2);
        weight = stats[k][0] == kMinusInf ? 0.f : __builtin_amdgcn_exp2f((stats[k][0] - ref) * rule.c2);
        soft.sum = soft.sum * old + stats[k][1] * weight;  // (a share without a finite score has no weight, but NaN stays)
        soft.ref = ref;
      } else {
        row.lean += stats[k][0];
        row.excess += stats[k][1];
        row.weight += stats[k][2];
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (!kForward) sum1[r] += part1[k][r / 4][r % 4];
        sum2[r] = __builtin_fmaf(weight, part2[k][r / 4][r % 4], sum2[r] * old);
      }
    }
  }
  if constexpr (kForward) store_results<S, K, 1>(a, rule, plane, own, g, soft, block, &sum1, &sum2);
  else store_results<S, K, 1>(a, rule, plane, own, g, row, block, &sum1, &sum2);
}

template <class S, bool kLine, ScoredKernel K>
hipError_t launch_items(const ScoredArgs& a, hipStream_t stream) {
  const int64_t entries = a.header ? 1 : a.batch, items = entries * a.num_items, merges = entries * a.num_merges;
  if (items < 1 || items > 0xffffff || merges * S::kWaves > 0xffffff) return hipErrorInvalidValue;  // (2^32 threads)
  if (K != kScoredForward && a.cap > 0.f) scored_kernel<S, kLine, K, K != kScoredForward><<<(unsigned)items, S::kThreads, 0, stream>>>(a);
  else scored_kernel<S, kLine, K, false><<<(unsigned)items, S::kThreads, 0, stream>>>(a);
  if (merges > 0) scored_merge_kernel<S, kLine, K><<<(unsigned)(merges * S::kWaves), S::kDBlocks * 64, 0, stream>>>(a);
  return hipGetLastError();
}

template <ScoredKernel K, int D, int kStep = 64>
hipError_t launch_scored(const ScoredArgs& a, hipStream_t stream) {
  if (a.D != D || (a.B != 64 && a.B != 128)) return hipErrorInvalidValue;
  if (a.line) return a.B == 64 ? launch_items<ScoredShape<64, D, kStep>, true, K>(a, stream) : launch_items<ScoredShape<128, D, kStep>, true, K>(a, stream);
  return a.B == 64 ? launch_items<ScoredShape<64, D, kStep>, false, K>(a, stream) : launch_items<ScoredShape<128, D, kStep>, false, K>(a, stream);
}

}  // namespace
}  // namespace ca
