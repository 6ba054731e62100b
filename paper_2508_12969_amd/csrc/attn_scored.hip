// Scored attention, forward: the kernel is in attn_scored.h.  Here too: what the tokens' arrays are turned into first, and the row statistics of the backward
// pass.
#include "attn_scored.h"

namespace ca {
namespace {

// One workgroup a tile: the arrays in tile order, and what the tile's tokens have in common.  Tokens that are not there have document -1.
__global__ void line_kernel(ScoredArgs a) {
  __shared__ TileLine shared[2];
  const int64_t tile = blockIdx.x, batch = blockIdx.y;
  const int slot = threadIdx.x;
  const Token k = token_of_place(a, (uint32_t)(tile * a.B + slot));
  float pos = 0.f, limit = __builtin_inff();
  int doc = -1;
  if (k.natural >= 0) {
    const int64_t at = batch * a.N_real + k.natural;
    doc = a.documents ? a.documents[at] : 0;
    if (doc < 0) doc = -1;
    if (a.positions) pos = (float)a.positions[at];
    if (a.limits) limit = (float)a.limits[at];
  }
  float* const out = a.line + (batch * a.n + tile) * kLineRows * a.B + slot;
  out[kLinePosition * a.B] = pos;
  out[kLineDocument * a.B] = __builtin_bit_cast(float, doc);
  out[kLineLimit * a.B] = limit;
  out[3 * a.B] = 0.f;
  const float inf = __builtin_inff();
  TileLine t{doc >= 0 ? doc : 0x7fffffff, doc >= 0 ? doc : -1, doc >= 0 ? pos : inf, doc >= 0 ? pos : -inf, doc >= 0 ? limit : inf, doc >= 0 ? limit : -inf, doc >= 0, 0};
  for (int step = 1; step < 64; step *= 2) {
    t.doc_min = min(t.doc_min, __shfl_xor(t.doc_min, step));
    t.doc_max = max(t.doc_max, __shfl_xor(t.doc_max, step));
    t.pos_min = fminf(t.pos_min, __shfl_xor(t.pos_min, step));
    t.pos_max = fmaxf(t.pos_max, __shfl_xor(t.pos_max, step));
    t.limit_min = fminf(t.limit_min, __shfl_xor(t.limit_min, step));
    t.limit_max = fmaxf(t.limit_max, __shfl_xor(t.limit_max, step));
    t.whole = t.whole & __shfl_xor(t.whole, step);
  }
  if ((slot & 63) == 0) shared[slot >> 6] = t;
  __syncthreads();
  if (slot != 0) return;
  if (a.B > 64) {
    const TileLine o = shared[1];
    t.doc_min = min(t.doc_min, o.doc_min);
    t.doc_max = max(t.doc_max, o.doc_max);
    t.pos_min = fminf(t.pos_min, o.pos_min);
    t.pos_max = fmaxf(t.pos_max, o.pos_max);
    t.limit_min = fminf(t.limit_min, o.limit_min);
    t.limit_max = fmaxf(t.limit_max, o.limit_max);
    t.whole = t.whole & o.whole;
  }
  a.tiles[batch * a.n + tile] = t;
}

// Per query: the log-sum-exp in powers of two, less the offset of a cap (ScoreRule) (plus infinity where it has none, so that all weights are zero backwards), and
// delta = sum of dO O, which is what dP of every key is reduced by.  Bound: HBM, dO and O once.
template <int D>
__global__ __launch_bounds__(256) void row_stats_kernel(ScoredArgs a, int64_t rows) {
  constexpr int kLanes = D / 8, kRows = 256 / kLanes;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;  // of all planes
  const int lane = threadIdx.x % kLanes;
  if (row >= rows) return;
  const bf16x8 x = reinterpret_cast<const bf16x8*>(static_cast<const char*>(a.o) + row * (D * 2))[lane];
  const bf16x8 y = reinterpret_cast<const bf16x8*>(static_cast<const char*>(a.dout) + row * (D * 2))[lane];
  float delta = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) delta += (float)x[e] * (float)y[e];
#pragma unroll
  for (int step = 1; step < kLanes; step *= 2) delta += __shfl_xor(delta, step);
  if (lane != 0) return;
  const float lse = a.lse_in[row];
  const bool empty = lse == kMinusInf;
  const int64_t tile = row / a.B, slot = row - tile * a.B;
  float* const out = a.rows + tile * 2 * a.B + slot;
  out[0] = empty ? __builtin_inff() : (a.cap > 0.f ? lse - a.cap : lse) * kLog2e;
  out[a.B] = empty ? 0.f : delta;
}

}  // namespace

hipError_t launch_line(const ScoredArgs& a, hipStream_t stream) {
  line_kernel<<<dim3((unsigned)a.n, (unsigned)a.batch), (unsigned)a.B, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_row_stats(const ScoredArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.batch * a.num_heads * a.N_pad, per = 256 / (a.D / 8), workgroups = (rows + per - 1) / per;
  if (workgroups > 0x7fffffff) return hipErrorInvalidValue;
  if (a.D == 64) row_stats_kernel<64><<<(unsigned)workgroups, 256, 0, stream>>>(a, rows);
  else row_stats_kernel<128><<<(unsigned)workgroups, 256, 0, stream>>>(a, rows);
  return hipGetLastError();
}

hipError_t launch_scored_forward(const ScoredArgs& a, hipStream_t stream) {
  return a.D == 64 ? launch_scored<kScoredForward, 64>(a, stream) : launch_scored<kScoredForward, 128>(a, stream);
}

}  // namespace ca
