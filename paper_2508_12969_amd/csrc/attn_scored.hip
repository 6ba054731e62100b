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
  TileLine t{doc >= 0 ? doc : 0x7fffffff, doc >= 0 ? doc : -1, doc >= 0 ? pos : inf, doc >= 0 ? pos : -inf, doc >= 0 ? limit : inf, doc >= 0 ? limit : -inf, k.natural < 0 || doc >= 0, 0};
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
// minus delta, delta = sum of dO O, which is what dP of every key is reduced by.  Bound: HBM, dO and O once.
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
  out[a.B] = empty ? 0.f : -delta;
}

// May any query of q see a key of k?  Does every query that is there see every slot of k?
__device__ __forceinline__ bool any_visible(const TileLine& q, const TileLine& k) {
  return q.doc_min <= k.doc_max && k.doc_min <= q.doc_max && k.pos_min <= q.limit_max;
}
__device__ __forceinline__ bool all_visible(const TileLine& q, const TileLine& k) {
  return q.doc_min == q.doc_max && k.doc_min == q.doc_min && k.doc_max == q.doc_min && k.pos_max <= q.limit_min;
}

constexpr int kVisitThreads = 256, kItemThreads = 1024;
struct VisitPair {
  Visits walk[2];
};

// Inclusive sum over the workgroup's threads; `waves`: a word of LDS for each wave.  *total receives the sum of all.
template <int kThreads>
__device__ __forceinline__ int sum_up_to(int x, int* waves, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int step = 1; step < 64; step *= 2) {
    const int y = __shfl_up(x, step);
    if (lane >= step) x += y;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) x += waves[w];
    all += waves[w];
  }
  *total = all;
  return x;
}

// The runs of a call whose arrays hide something: a workgroup takes a group's run and keeps the steps with visible pairs, in their order.  Bound: latency.
template <int B>
__global__ __launch_bounds__(kVisitThreads) void visit_kernel(ScoredArgs a, VisitPair pair) {
  constexpr int kTiles = kGroupTokens / B;
  __shared__ int waves[kVisitThreads / 64];
  const Visits v = blockIdx.z ? pair.walk[1] : pair.walk[0];
  const int tid = threadIdx.x;
  const int64_t group = blockIdx.x, batch = blockIdx.y;
  const TileLine* const tiles = a.tiles + batch * a.n;
  const int64_t per_head = (a.n + kTiles - 1) / kTiles, first_tile = group % per_head * kTiles;
  TileLine own[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) own[t] = tiles[min(first_tile + t, a.n - 1)];  // (no step names a tile that is not there)
  const int64_t begin = v.first[group], count = v.first[group + 1] - begin;
  uint32_t* const out = v.steps + batch * v.total + begin;
  int kept = 0;
  for (int64_t first = 0; first < count; first += kVisitThreads) {
    uint32_t word = 0, members = 0;
    if (first + tid < count) {
      word = v.from[begin + first + tid];
      members = word >> 30;
      const TileLine other = tiles[word & 0xffffffu];
      bool compare = false;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        if (!(v.keys ? any_visible(other, own[t]) : any_visible(own[t], other))) members &= ~(1u << t);
        // (streamed tokens that are not there are compared, so that an infinite token of the group's meets none of their values; the group's own write zeros)
        const bool all = other.whole && (v.keys ? all_visible(other, own[t]) : all_visible(own[t], other));
        compare = compare || ((members >> t & 1) != 0 && !all);
      }
      word = (word & 0x1fffffffu) | (compare ? 1u << 29 : 0u) | members << 30;
    }
    int all;
    const int at = kept + sum_up_to<kVisitThreads>(members != 0, waves, &all) - 1;
    if (members) out[at] = word;
    kept += all;
  }
  if (tid == 0) v.counts[batch * v.groups + group] = kept;
}

// Items of a launch from the runs' lengths, by one workgroup a walk: long runs are cut into equal parts, and items put into the order of their lengths, in 256
// classes (their order within a class changes nothing but who begins first).  Bound: latency; it reads the lengths three times.
__global__ __launch_bounds__(kItemThreads) void items_kernel(VisitPair pair, int64_t batch, int places) {
  __shared__ int waves[kItemThreads / 64], longest_shared, bucket[256];
  __shared__ unsigned long long total_shared;
  const Visits v = blockIdx.x ? pair.walk[1] : pair.walk[0];
  const int tid = threadIdx.x;
  const int64_t n = batch * v.groups;
  if (tid == 0) longest_shared = 0, total_shared = 0;
  if (tid < 256) bucket[tid] = 0;
  __syncthreads();
  int longest = 0;
  unsigned long long total = 0;
  for (int64_t i = tid; i < n; i += kItemThreads) {
    const int c = v.counts[i];
    longest = max(longest, c);
    total += (unsigned)c;
  }
#pragma unroll
  for (int step = 1; step < 64; step *= 2) {
    longest = max(longest, __shfl_xor(longest, step));
    total += __shfl_xor(total, step);
  }
  if ((tid & 63) == 0) {
    atomicMax(&longest_shared, longest);
    atomicAdd(&total_shared, total);
  }
  __syncthreads();
  longest = longest_shared;
  const int64_t ideal = (int64_t)((total_shared + places - 1) / places);
  // a run may be a tenth longer than an even share of the work before it is worth cutting
  const int target = (int)(10 * (int64_t)longest <= 11 * ideal ? max(longest, 1) : max(kLeastSteps, ideal));
  const int per_class = max(1, (min(longest, target) + 255) / 256);
  auto parts_of = [&](int c) { return max(1, (c + target - 1) / target); };
  auto class_of = [&](int c, int parts) { return 255 - min(255, (c + parts - 1) / parts / per_class); };
  for (int64_t i = tid; i < n; i += kItemThreads) {
    const int c = v.counts[i], parts = parts_of(c);
    atomicAdd(&bucket[class_of(c, parts)], parts);
  }
  __syncthreads();
  int all;
  const int mine = tid < 256 ? bucket[tid] : 0, upto = sum_up_to<kItemThreads>(mine, waves, &all);
  if (tid < 256) bucket[tid] = upto - mine;
  if (tid == 0) v.header->items = all;
  // Shares and merges are numbered in the order of the groups (below 2^16 and 2^15: both fit one sum).
  int before = 0;
  for (int64_t first = 0; first < n; first += kItemThreads) {
    const int64_t i = first + tid;
    const int c = i < n ? v.counts[i] : 0, parts = parts_of(c), shares = parts > 1 ? parts : 0, both = shares | (shares ? 1 << 16 : 0);
    const int at = before + sum_up_to<kItemThreads>(both, waves, &all) - both, share = at & 0xffff;
    before += all;
    if (i < n) {
      const int b = (int)(i / v.groups), g = (int)(i - b * v.groups), size = (c + parts - 1) / parts;
      if (shares) v.merges[at >> 16] = ScoredMerge{g, share, shares, b};
      const int64_t run = b * v.total + v.first[g];
      const int slot = atomicAdd(&bucket[class_of(c, parts)], parts);
      for (int k = 0; k < parts; ++k) {
        const int from = min(c, k * size);
        v.items[slot + k] = ScoredItem{run + from, min(c - from, size), g, shares ? share + k : -1, b};
      }
    }
  }
  if (tid == 0) v.header->merges = before >> 16;
}

}  // namespace

hipError_t launch_line(const ScoredArgs& a, hipStream_t stream) {
  line_kernel<<<dim3((unsigned)a.n, (unsigned)a.batch), (unsigned)a.B, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_visits(const ScoredArgs& a, const Visits* visits, int count, hipStream_t stream) {
  const dim3 grid((unsigned)visits[0].groups, (unsigned)a.batch, (unsigned)count);
  const VisitPair pair{visits[0], visits[count - 1]};
  if (a.B == 64) visit_kernel<64><<<grid, kVisitThreads, 0, stream>>>(a, pair);
  else visit_kernel<128><<<grid, kVisitThreads, 0, stream>>>(a, pair);
  items_kernel<<<(unsigned)count, kItemThreads, 0, stream>>>(pair, a.batch, (int)scored_places(a.D));
  return hipGetLastError();
}

hipError_t launch_row_stats(const ScoredArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.batch * a.num_heads * a.N_pad, per = 256 / (a.D / 8), workgroups = (rows + per - 1) / per;
  if (workgroups > 0xffffff) return hipErrorInvalidValue;  // (2^32 threads)
  if (a.D == 64) row_stats_kernel<64><<<(unsigned)workgroups, 256, 0, stream>>>(a, rows);
  else row_stats_kernel<128><<<(unsigned)workgroups, 256, 0, stream>>>(a, rows);
  return hipGetLastError();
}

hipError_t launch_scored_forward(const ScoredArgs& a, hipStream_t stream) {
  return a.D == 64 ? launch_scored<kScoredForward, 64>(a, stream) : launch_scored<kScoredForward, 128>(a, stream);
}

}  // namespace ca
