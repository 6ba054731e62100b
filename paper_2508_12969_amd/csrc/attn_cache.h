// Attention of new tokens over a paged cache, on the bf16 matrix instructions.
//
//   s = scale q.k;  s = cap tanh(s / cap);  s -= slope |frame_q - frame_k|;  O = softmax(s) V,  L = log sum exp s
//
// The rows of a sequence and a key head are its new tokens times the query heads that share the key head, token by token.  A wave owns 32 of them, one a lane: they are the columns of
// S^T = K Q^T and O^T += V^T P^T (as in attn_scored.h, whose fragments and products these are), so that a row's maximum and sum stay in its lane and the rounded weights are, register for
// register, the second product's operand.  Keys and values stream through LDS in steps of 32 tokens a wave or 64 a workgroup, copied straight from the pages: 16 rows of a page, a
// "slice", are one contiguous piece whatever the page length.  The weights are rounded to bf16 because the matrix instructions take both operands in one type, and V is bf16 (results are off by 2.3e-3 in
// norm, by 1.7e-3 of their own rounding alone); they are summed up as they were before, in fp32.
//
// What a row sees of its sequence is the prompt and a range lo <= token < hi that follows from its frame, and among drafts the bits of its word.  So the steps that a tile of rows walks are two runs in closed form
// (Walk), without a list, and only steps at the ends of a range compare anything.
#pragma once

#include "attn_scored.h"
#include "cache_tokens.h"

namespace ca {
namespace {

constexpr int kSlice = 16;  // tokens

template <int D_>
struct CacheShape {
  static constexpr int D = D_;
  static constexpr int kRowBytes = D * 2, kChunksPerRow = D / 8, kRowsPerLoad = 1024 / kRowBytes;
  static constexpr int kSliceLoads = kSlice / kRowsPerLoad;  // wave-wide copies of a slice
  static constexpr int kSliceBytes = kSlice * kRowBytes;
  static constexpr int kContraction = D / 16, kDBlocks = D / 32;
};

// Bits of a draft, of the new tokens that there are; and where it stands.
__device__ __forceinline__ uint64_t draft_bits(const AttendArgs& a, const Sequence& q, int32_t row) {
  const uint64_t bits = a.tree[row];
  return q.count < kMostDrafts ? bits & (((uint64_t)1 << q.count) - 1) : bits;
}
__device__ __forceinline__ int32_t draft_place(const Sequence& q, uint64_t bits) { return max(q.base + max((int)__popcll(bits), 1) - 1, 0); }

// What rows at a place of their sequence see.
struct View {
  int32_t lo, hi;  // behind the prompt
  int32_t frame;
};
__device__ __forceinline__ int32_t frame_at(const CacheArgs& a, const Sequence& q, int32_t place) { return place < q.origin ? -1 : divided(place - q.origin, a.span); }
__device__ __forceinline__ View view_at(const AttendArgs& a, const Sequence& q, int32_t place) {
  View v;
  v.frame = frame_at(a, q, place);
  const int64_t end = a.causal ? q.origin + (v.frame + (int64_t)1) * a.span : q.length;
  const int64_t begin = a.window && v.frame >= a.window ? q.origin + ((int64_t)v.frame - a.window + 1) * a.span : q.origin;
  v.hi = (int32_t)min(end, (int64_t)q.length);
  v.lo = (int32_t)min(begin, (int64_t)q.length);
  return v;
}

// Tokens of a prompt that are seen as such (a draft is not, wherever it lies).
__device__ __forceinline__ int32_t prompt_end(const AttendArgs& a, const Sequence& q) { return a.tree ? max(0, min(q.origin, q.base)) : q.origin; }

// Steps of kStep tokens that a tile of rows walks over: those of the prompt, then those of all its rows' ranges.
template <int kStep>
struct Walk {
  int32_t prompt, jump, count;  // steps of the prompt; what is added to the number of a later one; all
  __device__ __forceinline__ int32_t token(int32_t step) const { return (step + (step < prompt ? 0 : jump)) * kStep; }
};
template <int kStep>
__device__ __forceinline__ Walk<kStep> walk_of(const AttendArgs& a, const Sequence& q, int32_t first_token, int32_t last_token) {
  const int32_t least = max(q.base + (a.tree ? 0 : first_token), 0), most = a.tree ? q.length - 1 : q.base + last_token;
  const View low = view_at(a, q, least), high = view_at(a, q, most);
  const int32_t hi = a.tree ? q.length : high.hi;
  Walk<kStep> w;
  w.prompt = (prompt_end(a, q) + kStep - 1) / kStep;
  const int32_t from = max(w.prompt, min(low.lo, a.tree ? max(q.base, 0) : low.lo) / kStep), to = (hi + kStep - 1) / kStep;
  w.jump = from - w.prompt;
  w.count = most < 0 ? 0 : w.prompt + max(0, to - from);
  return w;
}

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// The sequences on a line on which each takes up weight(sequence) places, one after the other.  All threads of a workgroup make it and ask it together.
struct LineLds {
  int64_t waves[8], rest, weight;
  int32_t sequence;
  Sequence q;
};
template <int kThreads>
struct SequenceLine {
  int32_t from, to;   // the thread's sequences
  int64_t at, own;    // where they begin, what they take up
  Sequence last;      // of them
  int64_t all;        // places, in scalar registers
  template <class Weight>
  __device__ __forceinline__ SequenceLine(const CacheArgs& a, LineLds& lds, Weight&& weight) {
    if (a.sequences == 1) {  // nothing to look for
      last = sequence_at(a, 0);
      all = own = weight(last);
      return;
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t per = (a.sequences + kThreads - 1) / kThreads;
    from = min(tid * per, a.sequences), to = min(from + per, a.sequences);
    own = 0;
    for (int32_t s = from; s < to; ++s) last = sequence_at(a, s), own += weight(last);
    int64_t up = own;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
      const int64_t other = __shfl_up(up, step);
      if (lane >= step) up += other;
    }
    if (lane == 63) lds.waves[wave] = up;
    if (tid == 0) lds.sequence = -1;
    __syncthreads();
    at = up - own;
    int64_t total = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < wave) at += lds.waves[w];
      total += lds.waves[w];
    }
    all = uniform64(total);
  }
  // The sequence that holds a place, what it takes up and how far behind its first the place is; false: there is no such place.
  template <class Weight>
  __device__ __forceinline__ bool find(const CacheArgs& a, LineLds& lds, int64_t place, int32_t& sequence, Sequence& q, int64_t& takes, int64_t& rest, Weight&& weight) const {
    if (a.sequences == 1) {
      sequence = 0, q = last, takes = all, rest = place;
      return place >= 0 && place < all;
    }
    if (place >= at && place < at + own) {
      int64_t here = at, w = own;
      int32_t s = from;
      Sequence mine = last;
      if (to - from > 1)
        for (;; ++s) {
          mine = sequence_at(a, s);
          w = weight(mine);
          if (place < here + w) break;
          here += w;
        }
      lds.sequence = s;
      lds.q = mine;
      lds.weight = w;
      lds.rest = place - here;
    }
    __syncthreads();
    sequence = __builtin_amdgcn_readfirstlane(lds.sequence);
    if (sequence < 0) return false;
    q.first = __builtin_amdgcn_readfirstlane(lds.q.first), q.count = __builtin_amdgcn_readfirstlane(lds.q.count);
    q.length = __builtin_amdgcn_readfirstlane(lds.q.length), q.origin = __builtin_amdgcn_readfirstlane(lds.q.origin), q.base = __builtin_amdgcn_readfirstlane(lds.q.base);
    takes = uniform64(lds.weight);
    rest = uniform64(lds.rest);
    return true;
  }
};

__device__ __forceinline__ int32_t row_tiles(const AttendArgs& a, const Sequence& q, int rows) { return (q.count * a.group + rows - 1) / rows; }  // (rows of a call: at most 2^30)

// Steps of a tile of rows.
template <int kRows, int kStep>
__device__ __forceinline__ Walk<kStep> tile_walk(const AttendArgs& a, const Sequence& q, int32_t tile) {
  const int32_t first = tile * kRows, last = min(first + kRows, q.count * a.group) - 1;
  return walk_of<kStep>(a, q, divided(first, a.group), divided(last, a.group));
}

// A workgroup's share of a launch of items (tiles of rows and key heads), in one of three ways.
//   kItems   an item a workgroup.
//   kShares  The steps of all items lie on one line: sequences, their key heads, their tiles.  A workgroup takes an even share of the line, whatever items that cuts: a batch of sequences of
//            very different lengths is as even as one of equal ones.  An item takes up kItemCost places before its steps, for the time it takes to begin one.
//   kParts   Items are cut into equal parts.  Tiles of one key head and part begin together, on one XCD, and walk over their keys side by side: its L2 serves all of them.
// Sums of an item that is cut are left as pieces, which a second kernel joins.  An item without steps has one, with nothing to read: its results are written.
template <int kRows, int kStep, int kThreads, int kItemCost>
struct Share {
  int32_t sequence, key_head, tile, tiles;
  Sequence q;
  Walk<kStep> walk;
  int32_t count, done, steps;  // of the item: its steps, those before this workgroup's, this workgroup's
  bool whole;                  // they are all
  int64_t size, left, place;   // kShares: places of a share, those not taken yet, its number; kParts: place of the item
  int32_t part, parts;         // kParts
  int32_t begun = 0;           // pieces of an item that begins here
  bool fine = true;            // how the item's capped scores are held, see CacheRule

  __device__ __forceinline__ static int64_t places_of(const AttendArgs& a, const Sequence& q) {
    int64_t all = 0;
    for (int32_t t = 0, n = row_tiles(a, q, kRows); t < n; ++t) all += kItemCost + max(1, tile_walk<kRows, kStep>(a, q, t).count);
    return all * a.kv_heads;
  }
  // false: there is nothing to do
  __device__ __forceinline__ bool begin(const AttendArgs& a, LineLds& lds, int64_t workgroup) {
    place = workgroup;
    const auto tiles_of = [&](const Sequence& s) { return (int64_t)row_tiles(a, s, kRows); };
    const auto all_places = [&](const Sequence& s) { return places_of(a, s); };
    int64_t rest, takes;
    tile = done = 0;
    if (a.way == kShares) {
      const SequenceLine<kThreads> line(a, lds, all_places);
      size = max((int64_t)a.least_steps, divided64(line.all + a.workgroups - 1, a.workgroups));
      left = min(size, line.all - workgroup * size);
      if (left < 1 || !line.find(a, lds, workgroup * size, sequence, q, takes, rest, all_places)) return false;
      tiles = row_tiles(a, q, kRows);
      const int64_t per_head = a.kv_heads == 1 ? takes : divided64(takes, a.kv_heads);
      key_head = a.kv_heads == 1 ? 0 : (int32_t)divided64(rest, per_head);
      rest -= key_head * per_head;
      for (int32_t c; (c = kItemCost + max(1, tile_walk<kRows, kStep>(a, q, tile).count)) <= rest; ++tile) rest -= c;
      return take_share(a, (int32_t)rest);
    }
    const int64_t items = a.tiles * a.kv_heads;
    part = (int32_t)((uint32_t)workgroup / (uint32_t)items);  // (launches have fewer than 2^24 workgroups)
    place = workgroup - part * items;
    key_head = (int32_t)((uint32_t)place / (uint32_t)a.tiles);
    const SequenceLine<kThreads> line(a, lds, tiles_of);
    // the last tiles come first: in a causal order they see most
    if (!line.find(a, lds, a.tiles - 1 - (place - key_head * a.tiles), sequence, q, takes, rest, tiles_of)) return false;
    tiles = (int32_t)takes;
    tile = (int32_t)rest;
    walk = tile_walk<kRows, kStep>(a, q, tile);
    count = max(1, walk.count);
    parts = a.way == kParts ? max(1, min((count + a.part_steps - 1) / a.part_steps, a.most_parts)) : 1;
    const int32_t each = (count + parts - 1) / parts;
    done = min(count, part * each);
    steps = min(count - done, each);
    whole = parts == 1;
    if (part == 0 && parts > 1) begun = parts;
    return part < parts;
  }
  // What is left of the share begins `from` places behind the first of the item.  false: it ends before the item's steps.
  __device__ __forceinline__ bool take_share(const AttendArgs& a, int32_t from) {
    walk = tile_walk<kRows, kStep>(a, q, tile);
    count = max(1, walk.count);
    const int32_t all = kItemCost + count, to = (int32_t)min((int64_t)all, from + left), rest = all - to;
    left -= to - from;
    done = max(0, from - kItemCost);
    steps = max(0, to - kItemCost) - done;
    whole = steps == count;
    if (steps > 0 && done == 0 && rest > 0) begun = size >= rest ? 2 : 1 + (int32_t)((uint32_t)(rest + (int32_t)size - 1) / (uint32_t)size);
    return steps > 0;
  }
  // Rows of sums of this piece.
  __device__ __forceinline__ float* piece(const AttendArgs& a, int D) const {
    return a.pieces + (a.way == kShares ? place * 2 + (done > 0) : place * a.most_parts + part) * kRows * piece_row(D);
  }
  // The next item; false: there is none.
  __device__ __forceinline__ bool next(const AttendArgs& a) {
    if (a.way != kShares || left < 1) return false;
    if (++tile == tiles) {
      tile = 0;
      if (++key_head == a.kv_heads) {
        key_head = 0;
        do q = sequence_at(a, ++sequence);
        while (q.count == 0);
        tiles = row_tiles(a, q, kRows);
      }
    }
    return take_share(a, 0);
  }
  // What the second kernel has to know: of an item that begins here, in how many pieces it lies.
  __device__ __forceinline__ void leave(const AttendArgs& a, bool any) const {
    if (a.way == kItems || (a.way == kParts && part > 0)) return;
    if (threadIdx.x != 0) return;
    const int32_t first_row = tile * kRows;
    a.splits[place] = any && begun > 1 ? CacheSplit{q.first, key_head, first_row, min(kRows, q.count * a.group - first_row), begun, fine} : CacheSplit{0, 0, 0, 0, 0, 0};
  }
};

// Scores are held in a unit of their own, x, with s = unit x + offset.  Without a cap that is the product q.k itself.  With one, z = scale / cap q.k, it is one of two:
// fine, tanh(z): where the |z| of a wave's block are at most 0.35, z + z u (c0 + u (c1 + u c2)), u = z^2 (least largest relative error, 2^-24.5, by weighted least squares on Chebyshev nodes), else
//   1 - 2 / (2^(2 log2(e) z) + 1), off by 2^-24 of one.  Its constants are literals or in scalar registers (coefficients with powers of scale / cap in them, an operation less: 16 capped trees 94 / 85 us).
// fast, (tanh(z) - 1) / 2 (as ScoreRule has it), off by 2^-23 at most however small z is, which puts a score off by cap 2^-22 at most: the log-sum-exp of a few tokens shows that, of more it averages out.
//   For tiles of many rows that all see more than kFineTokens tokens, with caps up to kMostFastCap (2^-16 then): two forms and a branch between them take registers that those kernels do not have
//   (fast / fine: 16 trees over 9K tokens 80 / 85 us, three frames over 75K 4.83 / 4.95 ms and 3.29 / 3.80 at head dim 64; kernels of few rows are the same, and have the fine form alone).
constexpr float kSmall = 0.35f, kMostFastCap = 64.f;
constexpr int32_t kFineTokens = 4096;
__device__ __forceinline__ float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }
struct CacheRule {
  float unit, offset, c2;  // log2(e) (s - offset) = c2 x
  float inner, bend;       // z = inner q.k, 2 log2(e) z = bend q.k
  bool capped;
  __device__ __forceinline__ CacheRule(const AttendArgs& a, bool fine) : capped(a.cap > 0.f) {
    unit = !capped ? a.scale : fine ? a.cap : 2.f * a.cap;
    offset = capped && !fine ? a.cap : 0.f;
    c2 = uniform(unit * kLog2e);
    inner = uniform(capped ? a.scale / a.cap : 1.f);
    bend = uniform(2.f * kLog2e * inner);
  }
  // (the reference's own score first: beside the offset alone a logarithm loses places)
  __device__ __forceinline__ float log_sum_exp(float ref, float total) const { return __builtin_fmaf(__builtin_amdgcn_logf(total), 0.6931471805599453f, __builtin_fmaf(ref, unit, offset)); }
};

// A lane's row.
struct CacheRow {
  int32_t row;        // of the packed tensors; -1: there is none
  int32_t head;       // of the query
  View view;          // nothing where it has no place
  int32_t prompt;     // what it sees of it
  uint64_t drafts;
  float slope;        // in units of the scores, negative
  __device__ __forceinline__ CacheRow(const AttendArgs& a, const CacheRule& rule, const Sequence& q, int32_t key_head, int32_t index) {
    const int32_t i = divided(index, a.group);
    head = key_head * a.group + (index - i * a.group);
    row = i < q.count ? q.first + i : -1;
    const bool there = row >= 0 && q.base + i >= 0;
    drafts = there && a.tree ? draft_bits(a, q, row) : 0;
    view = view_at(a, q, !there ? 0 : a.tree ? draft_place(q, drafts) : q.base + i);
    prompt = prompt_end(a, q);
    if (a.tree) view.hi = min(view.hi, max(q.base, 0));
    if (!there) view.lo = view.hi = prompt = 0;
    slope = a.slopes ? -a.slopes[head] / rule.unit : 0.f;
  }
};

// q.k -> x
template <int kScores, class Scores>
__device__ __forceinline__ void cap_scores(const CacheRule& rule, Scores& s) {
  float most = 0.f;
#pragma unroll
  for (int r = 0; r < kScores; ++r) most = fmaxf(most, __builtin_fabsf(s[r]));
  if (__builtin_amdgcn_ballot_w64(!(most * rule.inner <= kSmall)) == 0) {
#pragma unroll
    for (int r = 0; r < kScores; ++r) {
      const float z = s[r] * rule.inner, u = z * z;
      s[r] = __builtin_fmaf(z, u * __builtin_fmaf(u, __builtin_fmaf(u, -0.0491593f, 0.1330001f), -0.3333267f), z);
    }
  } else {
#pragma unroll
    for (int r = 0; r < kScores; ++r) s[r] = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s[r] * rule.bend)), 1.f);
  }
}

__device__ __forceinline__ void cap_scores_fast(const CacheRule& rule, floatx16& s) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(s[r] * rule.bend));
}

// frames: of the step's tokens
__device__ __forceinline__ void bias_scores(const CacheRow& own, floatx16& s, const float* frames, int block, int g) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const floatx4 f = read4(frames, block, j, g);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[4 * j + e] = __builtin_fmaf(__builtin_fabsf((float)own.view.frame - f[e]), own.slope, s[4 * j + e]);
  }
}

// Scores -> weights.  The reference lags behind the maximum (see QueryWave::softmax); sums are put in relation to a new one when it moves.
template <int kBlocks, int kDBlocks>
__device__ __forceinline__ void soften(const CacheRule& rule, Softmax& soft, floatx16 (&s)[kBlocks], floatx16 (&sum)[kDBlocks]) {
  float mx = s[0][0];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
  mx = max_with_partner(mx);
  const bool moves = mx > soft.ref + kLazyLog2 / rule.c2;
  if (__builtin_amdgcn_ballot_w64(moves) != 0) {
    const float ref = moves ? mx : soft.ref;
    const float alpha = moves && soft.ref != kMinusInf ? __builtin_amdgcn_exp2f((soft.ref - ref) * rule.c2) : 1.f;
    soft.ref = ref;
    soft.sum *= alpha;
#pragma unroll
    for (int db = 0; db < kDBlocks; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[db][r] *= alpha;
  }
  const float shift = soft.ref == kMinusInf ? 0.f : -soft.ref * rule.c2;
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], rule.c2, shift));
      soft.sum += s[b][r];
    }
}

// What rows first_token to last_token of a sequence see in any case: of the prompt, and from lo to hi.
struct Sure {
  int32_t prompt, lo, hi;
  __device__ __forceinline__ Sure(const AttendArgs& a, const Sequence& q, int32_t first_token, int32_t last_token) {
    prompt = prompt_end(a, q);
    hi = q.base < 0 ? 0 : a.tree ? q.base : view_at(a, q, q.base + first_token).hi;
    lo = view_at(a, q, a.tree ? max(q.length - 1, 0) : max(q.base + last_token, 0)).lo;
  }
  __device__ __forceinline__ bool sees(int32_t token, int32_t end) const { return end <= hi && (token >= lo || end <= prompt); }
  __device__ __forceinline__ int32_t tokens() const { return prompt + max(0, hi - max(lo, prompt)); }
};

// Copies a slice (16 rows of a page) into LDS, asynchronously; logical chunks lie where swizzle() puts them.
template <class S>
struct SliceCopy {
  uint32_t voff[S::kSliceLoads];
  __device__ __forceinline__ explicit SliceCopy(int lane) {
#pragma unroll
    for (int i = 0; i < S::kSliceLoads; ++i) {
      const int within = lane / S::kChunksPerRow, phys = lane % S::kChunksPerRow;
      voff[i] = (uint32_t)(within * S::kRowBytes + ((phys ^ swizzle<S::D>(i * S::kRowsPerLoad + within)) << 4));
    }
  }
  __device__ __forceinline__ void operator()(const char* slice, uint32_t lds) const {
    const uint32_t m0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
    if constexpr (S::kSliceLoads == 4) {
      asm volatile(
          "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %[v0], %[sb] offset:0\n\t"
          "global_load_lds_dwordx4 %[v1], %[sb] offset:1024\n\t"
          "global_load_lds_dwordx4 %[v2], %[sb] offset:2048\n\t"
          "global_load_lds_dwordx4 %[v3], %[sb] offset:%[o3]\n\t"
          :
          : [o3] "n"(3 * 1024), [m0] "s"(m0), [v0] "v"(voff[0]), [v1] "v"(voff[1]), [v2] "v"(voff[2]), [v3] "v"(voff[3]), [sb] "s"(slice)
          : "memory");
    } else {
      static_assert(S::kSliceLoads == 2, "copies are written for two or four loads");
      asm volatile(
          "s_mov_b32 m0, %[m0]\n\ts_nop 0\n\t"
          "global_load_lds_dwordx4 %[v0], %[sb] offset:0\n\t"
          "global_load_lds_dwordx4 %[v1], %[sb] offset:1024\n\t"
          :
          : [m0] "s"(m0), [v0] "v"(voff[0]), [v1] "v"(voff[1]), [sb] "s"(slice)
          : "memory");
    }
  }
};

// Where the slices of 64 / kSlices steps lie, one a lane, fetched by all lanes at once; the table is read some steps before the places are needed.
template <int kSlices, int kStep>
struct SlicePlaces {
  static constexpr int kSteps = 64 / kSlices;
  int32_t first = 0;      // step of lane 0
  int64_t offset = 0;     // bytes; of a slice that is not there: 0, a place that can be read
  uint64_t there = 0;     // a bit a lane
  int32_t page = -1;      // of the steps asked for
  __device__ __forceinline__ int64_t token_of(const Sequence& q, const Walk<kStep>& w, int32_t step, int32_t end, int lane) const {
    const int32_t mine = step + lane / kSlices;
    return mine < end ? (int64_t)w.token(mine) + lane % kSlices * kSlice : q.length;
  }
  __device__ __forceinline__ void ask(const AttendArgs& a, const Sequence& q, int32_t s, const Walk<kStep>& w, int32_t step, int32_t end, int lane) {
    const int64_t token = token_of(q, w, step, end, lane);
    page = token < q.length ? a.table[(int64_t)s * a.table_width + divided((int32_t)token, a.page_tokens)] : -1;
  }
  __device__ __forceinline__ void take(const AttendArgs& a, const Sequence& q, int32_t head, const Walk<kStep>& w, int32_t step, int32_t end, int lane, int row_bytes) {
    first = step;
    const int64_t token = token_of(q, w, step, end, lane);
    const bool here = page >= 0 && page < a.num_pages;
    const int32_t slot = (int32_t)token - divided((int32_t)token, a.page_tokens) * a.page_tokens;
    offset = here ? cache_row(a, page, head, slot) * row_bytes : 0;
    there = __builtin_amdgcn_ballot_w64(here);
  }
  // Called for every step in turn, from `begin` on.
  __device__ __forceinline__ void at_step(const AttendArgs& a, const Sequence& q, int32_t s, int32_t head, const Walk<kStep>& w, int32_t step, int32_t begin, int32_t end, int lane,
                                          int row_bytes) {
    if (step == begin) ask(a, q, s, w, step, end, lane);
    if (step == begin || step - first == kSteps) take(a, q, head, w, step, end, lane, row_bytes);
    if (step - first == kSteps / 2 && first + kSteps < end) ask(a, q, s, w, first + kSteps, end, lane);
  }
  __device__ __forceinline__ int64_t at(int32_t step, int slice) const {
    const int from = (step - first) * kSlices + slice;
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(offset >> 32), from) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)offset, from));
  }
  __device__ __forceinline__ uint32_t mask(int32_t step) const { return (uint32_t)(there >> ((step - first) * kSlices)) & ((1u << kSlices) - 1); }
};

// Rows of a step that hold no token become zero: what lies there is multiplied by a weight of zero, and may be anything.
template <class S>
__device__ __forceinline__ void clear_rows(char* y, int first_row, int rows, int lane) {
  for (int r = first_row; r < rows; ++r)
    if (lane < S::kChunksPerRow) *reinterpret_cast<intx4*>(y + r * S::kRowBytes + lane * 16) = intx4{0, 0, 0, 0};
}

// Does a row see a token that is there?
__device__ __forceinline__ bool sees_token(const AttendArgs& a, const Sequence& q, const CacheRow& own, int32_t token) {
  const int32_t draft = token - q.base;
  const bool drafted = a.tree && draft >= 0 && draft < kMostDrafts && (own.drafts >> draft) & 1u;
  return (int)(token < own.prompt) | ((int)(token >= own.view.lo) & (int)(token < own.view.hi)) | (int)drafted;
}

// Hides what a row does not see in a block of 32 tokens from `token` on; slices: which of its two are there.
__device__ __forceinline__ void hide_tokens(const AttendArgs& a, const Sequence& q, const CacheRow& own, floatx16& s, int32_t token, uint32_t slices, int g) {
  const int32_t at = token + 4 * g, lo = own.view.lo - at, hi = own.view.hi - at, prompt = own.prompt - at;
  uint32_t drafts = 0;
  if (a.tree) {
    const int32_t shift = at - q.base;  // bit of the lane's first token
    if (shift > -32 && shift < kMostDrafts) drafts = (uint32_t)(shift >= 0 ? own.drafts >> shift : own.drafts << -shift);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int c = 8 * (r / 4) + (r % 4);
    const bool seen = (int)(c < prompt) | ((int)(c >= lo) & (int)(c < hi)) | (int)((drafts >> c) & 1u);
    s[r] = seen && ((slices >> (r / 8)) & 1u) ? s[r] : kMinusInf;
  }
}

// Frame of a token of the cache, for the bias: drafts stand where their words say.
__device__ __forceinline__ float frame_of_token(const AttendArgs& a, const Sequence& q, int32_t token) {
  const bool draft = a.tree && token >= q.base && token < q.length;
  return (float)frame_at(a, q, draft ? draft_place(q, draft_bits(a, q, q.first + (token - q.base))) : token);
}

// Writes a row's four channels from the joined sums.  T: of the results.
template <int D, class T>
__device__ __forceinline__ void store_row(const AttendArgs& a, const CacheRule& rule, int32_t first, int32_t key_head, int32_t row, int channel, const floatx4& o, float ref, float total) {
  typedef T Four __attribute__((ext_vector_type(4)));
  const int32_t t = divided(row, a.group), head = key_head * a.group + (row - t * a.group);
  const int64_t at = (int64_t)(first + t) * a.heads + head;
  const bool real = total != 0.f;
  Four v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (T)(real ? o[e] / total : 0.f);
  *reinterpret_cast<Four*>(static_cast<T*>(a.out) + at * D + channel) = v;
  if (channel == 0) a.lse[at] = real ? rule.log_sum_exp(ref, total) : kMinusInf;
}

// Sums of a row of which parts were made with references of their own.
struct Joined {
  float ref = kMinusInf, total = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(const CacheRule& rule, float part_ref, float part_total, const floatx4& part) {
    const float to = fmaxf(ref, part_ref), old = ref == kMinusInf ? 0.f : __builtin_amdgcn_exp2f((ref - to) * rule.c2);
    const float fresh = part_ref == kMinusInf ? 0.f : __builtin_amdgcn_exp2f((part_ref - to) * rule.c2);
    ref = to;
    total = total * old + part_total * fresh;  // (NaN stays, whatever its weight)
    o = o * old + part * fresh;
  }
};

// Joins what the waves of a workgroup have summed up for a tile of `rows` rows, each row by row in its own part of LDS (lds[wave].sums), and writes the results, or a piece of them.
template <int D, class T, int kWaves, class Wave, class Shared>
__device__ __forceinline__ void finish_rows(const AttendArgs& a, const CacheRule& rule, const Shared& share, const Wave* lds, int32_t first_row, int rows) {
  float* const piece = share.whole ? nullptr : share.piece(a, D);
  for (int item = threadIdx.x; item < rows * (D / 4); item += kWaves * 64) {
    const int r = item / (D / 4), c = item % (D / 4) * 4;
    Joined j;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) j.add(rule, lds[w].sums[r][D], lds[w].sums[r][D + 1], *reinterpret_cast<const floatx4*>(&lds[w].sums[r][c]));
    if (share.whole) {
      store_row<D, T>(a, rule, share.q.first, share.key_head, first_row + r, c, j.o, j.ref, j.total);
    } else {
      *reinterpret_cast<floatx4*>(piece + r * piece_row(D) + c) = j.o;
      if (c == 0) *reinterpret_cast<float2*>(piece + r * piece_row(D) + D) = float2{j.ref, j.total};
    }
  }
}

// Joins the pieces of the item that begins at place blockIdx.x, in their order.  Threads take four channels of a row each, and kParts of them together a part of the
// pieces.  Bound: latency, and the pieces once.
template <int D, class T, int kRows, int kThreads, int kParts>
__device__ __forceinline__ void join_pieces(const AttendArgs& a) {
  constexpr int kColumns = D / 4, kRowsAtOnce = kThreads / kColumns / kParts;
  __shared__ floatx4 sums[kParts > 1 ? kRowsAtOnce : 1][kParts][kColumns];
  __shared__ float2 stats[kParts > 1 ? kRowsAtOnce : 1][kParts];
  const CacheSplit split = a.splits[blockIdx.x];
  if (split.pieces == 0) return;
  const CacheRule rule(a, split.fine != 0);
  const int column = threadIdx.x % kColumns, part = threadIdx.x / kColumns % kParts, within = threadIdx.x / kColumns / kParts;
  for (int r0 = blockIdx.y * kRowsAtOnce; r0 < split.rows; r0 += gridDim.y * kRowsAtOnce) {
    const int r = r0 + within;
    Joined j;
    if (r < split.rows) {
#pragma unroll 4
      for (int k = part; k < split.pieces; k += kParts) {
        const int64_t piece = a.way == kShares ? ((int64_t)blockIdx.x + k) * 2 + (k > 0) : (int64_t)blockIdx.x * a.most_parts + k;
        const float* from = a.pieces + (piece * kRows + r) * piece_row(D);
        const float2 stat = *reinterpret_cast<const float2*>(from + D);
        j.add(rule, stat.x, stat.y, *reinterpret_cast<const floatx4*>(from + column * 4));
      }
    }
    if constexpr (kParts > 1) {
      sums[within][part][column] = j.o;
      if (column == 0) stats[within][part] = float2{j.ref, j.total};
      __syncthreads();
      if (part == 0)
        for (int k = 1; k < kParts && k < split.pieces; ++k) j.add(rule, stats[within][k].x, stats[within][k].y, sums[within][k][column]);
    }
    if (r < split.rows && part == 0) store_row<D, T>(a, rule, split.first, split.key_head, split.first_row + r, column * 4, j.o, j.ref, j.total);
    if constexpr (kParts > 1) __syncthreads();
  }
}

}  // namespace
}  // namespace ca
