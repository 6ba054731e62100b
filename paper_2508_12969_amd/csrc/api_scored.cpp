// C-ABI entry points of scored attention: lists and items of its launches, argument checks, launches (attn_scored.hip, attn_scored_back.hip).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <functional>
#include <new>
#include <queue>
#include <vector>

#include "api_common.h"
#include "scored.h"

using ca::aligned16;
using ca::fail;
using ca::hip_fail;
using ca::ranges_overlap;
using ca::set_error;

namespace {

int64_t padded256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int check_scores(const ca_layout* L, const ca_scores* s) {
  if (!L || !s) return fail(CA_ERR_INVALID_ARG, "null argument");
  const ca_problem& p = L->prob;
  if (p.dtype != CA_BF16 || (L->B != 64 && L->B != 128) || (p.head_dim != 64 && p.head_dim != 128)) {
    set_error("scored attention supports bf16 with tile sizes 64/128 and head_dim 64/128; got dtype=%d B=%lld D=%d", p.dtype, (long long)L->B, p.head_dim);
    return CA_ERR_UNSUPPORTED;
  }
  if (p.batch > 65535 || (int64_t)p.batch * p.num_heads * L->n > 0x7fffffff) return fail(CA_ERR_UNSUPPORTED, "more than 65535 batch entries or 2^31 - 1 rows");
  if (L->n > 0xffffff) return fail(CA_ERR_UNSUPPORTED, "more than 2^24 - 1 tiles");  // (a step's word has 24 bits for one)
  // capped scores are held as (tanh - 1) / 2 and off by a few 2^-24 of the cap
  if (s->cap != 0.f && !(s->cap >= ca::kLeastCap && s->cap <= ca::kMostCap)) return fail(CA_ERR_INVALID_ARG, "cap must be 0 or between 2^-16 and 4096");
  if (s->slopes && !s->positions) return fail(CA_ERR_INVALID_ARG, "slopes need positions");
  if (s->limits && !s->positions) return fail(CA_ERR_INVALID_ARG, "limits need positions");
  if (!aligned4(s->slopes) || !aligned4(s->positions) || !aligned4(s->limits) || !aligned4(s->documents))
    return fail(CA_ERR_INVALID_ARG, "slopes, positions, limits and documents must be 4-byte aligned");
  return CA_OK;
}

// Do the tokens need a line of their own in the workspace?  Positions alone change nothing.
bool has_line(const ca_scores* s) { return s->slopes || s->limits || s->documents; }

struct Range {
  const void* at;
  int64_t bytes;
};

// Results may not overlap each other or anything that is read.
int check_apart(std::vector<Range> results, const std::vector<Range>& inputs) {
  for (size_t i = 0; i < results.size(); ++i) {
    if (!results[i].bytes) continue;
    for (const Range& in : inputs)
      if (in.at && ranges_overlap(results[i].at, results[i].bytes, in.at, in.bytes)) return fail(CA_ERR_INVALID_ARG, "results and workspace must not overlap the inputs");
    for (size_t j = i + 1; j < results.size(); ++j)
      if (results[j].bytes && ranges_overlap(results[i].at, results[i].bytes, results[j].at, results[j].bytes))
        return fail(CA_ERR_INVALID_ARG, "results and workspace must not overlap each other");
  }
  return CA_OK;
}

int check_workspace(const void* workspace, int64_t bytes, int64_t need) {
  if (need > 0 && (!workspace || !aligned16(workspace) || bytes < need)) {
    set_error("the call needs a 16-byte aligned workspace of %lld bytes; got %lld", (long long)need, (long long)(workspace ? bytes : 0));
    return CA_ERR_INVALID_ARG;
  }
  return CA_OK;
}

std::vector<Range> token_arrays(const ca_layout* L, const ca_scores* s) {
  const int64_t bytes = (int64_t)L->prob.batch * L->N_real * 4;
  return {{s->positions, bytes}, {s->limits, bytes}, {s->documents, bytes}, {s->slopes, (int64_t)L->prob.num_heads * 4}};
}

constexpr int64_t kMaxScoredShareBytes = (int64_t)128 << 20;

// When the last workgroup ends, in steps, if runs longer than `target` are cut into equal parts of at most that.
int64_t end_of_launch(const std::vector<int64_t>& costs, int64_t batch, int64_t places_count, int64_t target) {
  std::vector<int64_t> pieces;
  bool shares = false;
  for (int64_t c : costs) {
    const int64_t parts = std::max<int64_t>(1, (c + target - 1) / target);
    shares = shares || parts > 1;
    for (int64_t i = 0; i < parts; ++i) pieces.push_back((c + parts - 1) / parts + ca::kItemSteps + (parts > 1 ? ca::kShareSteps : 0));
  }
  std::sort(pieces.begin(), pieces.end(), std::greater<int64_t>());
  std::priority_queue<int64_t, std::vector<int64_t>, std::greater<int64_t>> places;
  for (int64_t i = 0; i < places_count; ++i) places.push(0);
  int64_t end = 0;
  for (int64_t b = 0; b < batch; ++b)
    for (int64_t c : pieces) {
      const int64_t at = places.top() + c;
      places.pop();
      places.push(at);
      end = std::max(end, at);
    }
  return end + (shares ? ca::kMergeSteps : 0);
}

// Longest part of a run, in steps: runs are cut where the launch would end with a few long ones, or leave compute units without work.
int64_t part_steps(const std::vector<int64_t>& costs, int64_t batch, int64_t places, int64_t share_bytes) {
  const int64_t whole = (int64_t)1 << 40;
  int64_t total = 0;
  for (int64_t c : costs) total += c;
  if ((int64_t)costs.size() * batch > 16 * places) return whole;  // (no run is long beside so many)
  int64_t best = whole, best_end = end_of_launch(costs, batch, places, whole);
  const int64_t ideal = std::max<int64_t>(1, total * batch / places);
  for (int64_t divisor = 1; divisor <= 4; ++divisor) {
    const int64_t target = std::max(ca::kLeastSteps, (ideal + divisor - 1) / divisor);
    int64_t shares = 0;
    for (int64_t c : costs) shares += c > target ? (c + target - 1) / target : 0;
    if (shares * batch * share_bytes > kMaxScoredShareBytes) break;
    const int64_t end = end_of_launch(costs, batch, places, target);
    if (20 * end < 19 * best_end) best = target, best_end = end;  // (not for a few per cent)
  }
  return best;
}

// The lists of the layout's rows (or columns), as runs of groups, and the items of a launch.
int make_walk(const ca_layout* L, bool columns, ca::ScoredWalk& walk) {
  if (L->class_mask.size() > 16) return fail(CA_ERR_UNSUPPORTED, "too many padding classes for scored attention");
  const int64_t n = L->n, heads = L->prob.num_heads, rows = heads * n, tiles = ca::kGroupTokens / L->B, per_head = (n + tiles - 1) / tiles, groups = heads * per_head;
  std::vector<int64_t> ptr_t;
  std::vector<int32_t> idx_t;
  if (columns) {
    ptr_t.assign(rows + 1, 0);
    idx_t.resize(L->col_idx.size());
    for (int64_t head = 0; head < heads; ++head)
      for (int64_t i = L->row_ptr[head * n]; i < L->row_ptr[(head + 1) * n]; ++i) ++ptr_t[head * n + L->col_idx[i] + 1];
    for (int64_t r = 0; r < rows; ++r) ptr_t[r + 1] += ptr_t[r];
    std::vector<int64_t> at(ptr_t.begin(), ptr_t.end() - 1);
    for (int64_t row = 0; row < rows; ++row)
      for (int64_t i = L->row_ptr[row]; i < L->row_ptr[row + 1]; ++i) idx_t[at[row / n * n + L->col_idx[i]]++] = (int32_t)(row % n);
  }
  const int64_t* const ptr = columns ? ptr_t.data() : L->row_ptr.data();
  const int32_t* const idx = columns ? idx_t.data() : L->col_idx.data();
  bool has[16][2] = {};  // does half h of a tile of class c hold a token?
  for (size_t c = 0; c < L->class_mask.size(); ++c)
    for (int64_t h = 0; h < L->B / 64; ++h) has[c][h] = (L->class_mask[c].w[2 * h] | L->class_mask[c].w[2 * h + 1]) != 0;
  std::vector<int64_t> costs(groups);
  walk.first.assign(groups + 1, 0);
  walk.steps.reserve(L->col_idx.size() * (L->B / 64) / tiles + 2);
  for (int64_t g = 0; g < groups; ++g) {
    const int64_t row = g / per_head * n + g % per_head * tiles;
    const bool second = tiles == 2 && g % per_head * tiles + 1 < n;
    int64_t i = ptr[row], j = second ? ptr[row + 1] : 0;
    const int64_t i_end = ptr[row + 1], j_end = second ? ptr[row + 2] : 0;
    while (i < i_end || j < j_end) {
      const int32_t a = i < i_end ? idx[i] : INT32_MAX, b = j < j_end ? idx[j] : INT32_MAX, t = std::min(a, b), cls = L->tile_class[t];
      for (uint32_t h = 0; h < (uint32_t)(L->B / 64); ++h)
        if (has[cls][h]) walk.steps.push_back((uint32_t)t | h << 24 | (uint32_t)cls << 25 | (a == t ? 1u << 30 : 0u) | (b == t ? 1u << 31 : 0u));
      i += a == t;
      j += b == t;
    }
    walk.first[g + 1] = (int64_t)walk.steps.size();
    costs[g] = walk.first[g + 1] - walk.first[g];
    if (costs[g] > INT_MAX / 2) return fail(CA_ERR_UNSUPPORTED, "a list is too long for scored attention");
  }
  walk.steps.push_back(0);  // the kernels fetch two words ahead
  walk.steps.push_back(0);
  const int64_t D = L->prob.head_dim, most = part_steps(costs, L->prob.batch, ca::scored_places(D), ca::share_floats(D, 2) * 4);
  for (int64_t g = 0; g < groups; ++g) {
    const int64_t count = costs[g], parts = std::max<int64_t>(1, (count + most - 1) / most), size = (count + parts - 1) / parts;
    if (parts > 1) walk.merges.push_back({(int32_t)g, (int32_t)walk.shares, (int32_t)parts, 0});
    for (int64_t i = 0; i < parts; ++i) {
      const int64_t from = std::min(count, i * size), to = std::min(count, from + size);
      walk.items.push_back({walk.first[g] + from, (int32_t)(to - from), (int32_t)g, parts > 1 ? (int32_t)(walk.shares + i) : -1, 0});
    }
    walk.shares += parts > 1 ? parts : 0;
  }
  std::stable_sort(walk.items.begin(), walk.items.end(), [](const ca::ScoredItem& a, const ca::ScoredItem& b) { return a.count > b.count; });
  if (((int64_t)walk.items.size() + ca::most_shares(D)) * L->prob.batch > INT_MAX) return fail(CA_ERR_UNSUPPORTED, "more than 2^31 - 1 workgroups");
  walk.made = true;
  return CA_OK;
}

// The layout's walk, made on the host if it is not there yet.
int walk_of(ca_layout* L, bool columns, ca::ScoredWalk** walk) {
  try {
    std::shared_ptr<ca::ScoredState> state;
    {
      std::lock_guard<std::mutex> lock(L->upload_mutex);
      if (!L->scored) L->scored = std::make_shared<ca::ScoredState>();
      state = L->scored;
    }
    std::lock_guard<std::mutex> lock(state->mutex);
    ca::ScoredWalk& w = columns ? state->columns : state->rows;
    if (!w.made) {
      ca::ScoredWalk fresh;
      const int st = make_walk(L, columns, fresh);
      if (st != CA_OK) return st;
      w = std::move(fresh);
    }
    *walk = &w;
    return CA_OK;
  } catch (const std::bad_alloc&) {
    return fail(CA_ERR_ALLOC, "out of host memory while making the lists of scored attention");
  }
}

// The same on the device, with the layout's own tables.
int upload_walk(ca_layout* L, bool columns, hipStream_t stream, ca::ScoredWalk** walk) {
  int st = ca::ensure_uploaded(L, stream);
  if (st == CA_OK) st = walk_of(L, columns, walk);
  if (st != CA_OK) return st;
  ca::ScoredWalk& w = **walk;
  std::lock_guard<std::mutex> lock(L->scored->mutex);
  if (w.block) return CA_OK;
  if (stream) {
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    const hipError_t e = hipStreamIsCapturing(stream, &cap);
    if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
    if (cap != hipStreamCaptureStatusNone)
      return fail(CA_ERR_INVALID_ARG, "the lists of scored attention are not on the device yet and the stream is being captured: call compact_attn_layout_upload_scored "
                                      "before the capture");
  }
  struct Part {
    const void* from;
    size_t bytes;
    void** to;
  };
  const Part parts[] = {{w.steps.data(), w.steps.size() * sizeof(uint32_t), reinterpret_cast<void**>(&w.dev_steps)},
                        {w.first.data(), w.first.size() * sizeof(int64_t), reinterpret_cast<void**>(&w.dev_first)},
                        {w.items.data(), w.items.size() * sizeof(ca::ScoredItem), reinterpret_cast<void**>(&w.dev_items)},
                        {w.merges.data(), w.merges.size() * sizeof(ca::ScoredMerge), reinterpret_cast<void**>(&w.dev_merges)}};
  size_t bytes = 0;
  for (const Part& p : parts) bytes += (size_t)padded256((int64_t)p.bytes);
  void* block = nullptr;
  hipError_t e = hipMalloc(&block, bytes);
  if (e != hipSuccess) {
    set_error("hipMalloc of %zu bytes for the lists of scored attention failed: %s", bytes, hipGetErrorString(e));
    (void)hipGetLastError();
    return CA_ERR_ALLOC;
  }
  unsigned char* at = static_cast<unsigned char*>(block);
  for (const Part& p : parts) {
    *p.to = at;
    if (e == hipSuccess && p.bytes) e = hipMemcpy(at, p.from, p.bytes, hipMemcpyHostToDevice);
    at += padded256((int64_t)p.bytes);
  }
  if (e != hipSuccess) {
    (void)hipFree(block);
    return hip_fail(e, "hipMemcpy of the lists of scored attention");
  }
  w.block = static_cast<unsigned char*>(block);
  return CA_OK;
}

// Do the arrays hide something, so that runs are made on the device?  (Slopes alone do not.)
bool is_masked(const ca_scores* s) { return s->limits || s->documents; }

// Parts of a call's workspace, in their order.
struct Workspace {
  int64_t line = 0, tiles = 0, rows = 0, steps[2] = {0, 0}, counts[2] = {0, 0}, items[2] = {0, 0}, merges[2] = {0, 0}, headers = 0, shares = 0;
  int64_t bytes() const {
    int64_t all = line + tiles + rows + headers + shares;
    for (int i = 0; i < 2; ++i) all += steps[i] + counts[i] + items[i] + merges[i];
    return all;
  }
};

int64_t groups_of(const ca::ScoredWalk& w) { return (int64_t)w.first.size() - 1; }

// Most shares that runs made on the device can have.
int64_t shares_made(const ca::ScoredWalk& w, int64_t batch, int64_t D) {
  int64_t all = 0;
  for (int64_t g = 0; g < groups_of(w) && all < ca::most_shares(D); ++g) {
    const int64_t count = w.first[g + 1] - w.first[g];
    if (count > ca::kLeastSteps) all += batch * ((count + ca::kLeastSteps - 1) / ca::kLeastSteps);
  }
  return std::min(all, ca::most_shares(D));
}

int workspace_of(ca_layout* L, const ca_scores* s, bool backward, Workspace& w) {
  const ca_problem& p = L->prob;
  ca::ScoredWalk* walks[2] = {nullptr, nullptr};
  int st = walk_of(L, false, &walks[0]);
  if (st == CA_OK && backward) st = walk_of(L, true, &walks[1]);
  if (st != CA_OK) return st;
  if (has_line(s)) {
    w.line = ca::line_bytes(p.batch, L->n, L->B);
    w.tiles = ca::tile_line_bytes(p.batch, L->n);
  }
  if (backward) w.rows = padded256(ca::row_stat_bytes((int64_t)p.batch * p.num_heads, L->n, L->B));
  for (int i = 0; i < (backward ? 2 : 1); ++i) {
    const ca::ScoredWalk& walk = *walks[i];
    const int64_t groups = groups_of(walk), share_bytes = ca::share_floats(p.head_dim, backward ? 2 : 1) * 4;
    if (is_masked(s)) {
      w.steps[i] = padded256((p.batch * walk.first[groups] + 2) * 4);
      w.counts[i] = padded256(p.batch * groups * 4);
      w.items[i] = padded256((p.batch * groups + ca::most_shares(p.head_dim)) * (int64_t)sizeof(ca::ScoredItem));
      w.merges[i] = padded256(ca::most_merges(p.head_dim) * (int64_t)sizeof(ca::ScoredMerge));
      w.headers = 256;
      w.shares = std::max(w.shares, padded256(shares_made(walk, p.batch, p.head_dim) * share_bytes));
    } else {
      w.shares = std::max(w.shares, padded256(p.batch * walk.shares * share_bytes));
    }
  }
  return CA_OK;
}

// Where a walk's launches find their items.
void set_walk(ca::ScoredArgs& a, const ca::ScoredWalk& w) {
  a.steps = w.dev_steps;
  a.items = w.dev_items;
  a.merges = w.dev_merges;
  a.header = nullptr;
  a.num_items = (int64_t)w.items.size();
  a.num_merges = (int64_t)w.merges.size();
  a.shares = w.shares;
}
void set_walk(ca::ScoredArgs& a, const ca::Visits& v) {
  a.steps = v.steps;
  a.items = v.items;
  a.merges = v.merges;
  a.header = v.header;
  a.num_items = a.batch * v.groups + ca::most_shares(a.D);
  a.num_merges = std::min(ca::most_merges(a.D), a.batch * v.groups);
  a.shares = 0;
}

// Arguments of a call's launches; visits: the walks that are made on the device, one or two (0 where none is).
ca::ScoredArgs scored_args(const ca_layout* L, const ca_scores* s, const Workspace& w, void* workspace, ca::ScoredWalk* const (&walks)[2], ca::Visits (&visits)[2],
                           int& num_visits) {
  const ca_problem& p = L->prob;
  ca::ScoredArgs a{};
  ca::fill_grid(a, L);
  a.tile_class = L->dev.tile_class;
  a.class_mask = L->dev.class_mask;
  a.class_perm = L->dev.class_perm;
  a.batch = p.batch;
  a.num_heads = p.num_heads;
  a.D = p.head_dim;
  a.n = L->n;
  a.scale = L->scale;
  a.cap = s->cap;
  a.slopes = s->slopes;
  a.positions = s->positions;
  a.limits = s->limits;
  a.documents = s->documents;
  unsigned char* at = static_cast<unsigned char*>(workspace);
  auto take = [&](int64_t bytes) {
    unsigned char* const here = bytes ? at : nullptr;
    at += bytes;
    return here;
  };
  a.line = reinterpret_cast<float*>(take(w.line));
  a.tiles = reinterpret_cast<ca::TileLine*>(take(w.tiles));
  a.rows = reinterpret_cast<float*>(take(w.rows));
  ca::VisitCounts* const headers = reinterpret_cast<ca::VisitCounts*>(take(w.headers));
  num_visits = 0;
  for (int i = 0; i < 2 && walks[i] && headers; ++i) {
    ca::Visits& v = visits[num_visits++];
    v.from = walks[i]->dev_steps;
    v.first = walks[i]->dev_first;
    v.groups = groups_of(*walks[i]);
    v.total = walks[i]->first[v.groups];
    v.keys = i;
    v.steps = reinterpret_cast<uint32_t*>(take(w.steps[i]));
    v.counts = reinterpret_cast<int32_t*>(take(w.counts[i]));
    v.items = reinterpret_cast<ca::ScoredItem*>(take(w.items[i]));
    v.merges = reinterpret_cast<ca::ScoredMerge*>(take(w.merges[i]));
    v.header = headers + i;
  }
  a.share_sums = reinterpret_cast<float*>(take(w.shares));
  return a;
}

// The token arrays in tile order, and the walks that depend on them.
hipError_t launch_tokens(const ca::ScoredArgs& a, const ca::Visits (&visits)[2], int num_visits, hipStream_t stream) {
  hipError_t e = a.line ? ca::launch_line(a, stream) : hipSuccess;
  if (e == hipSuccess && num_visits > 0) e = ca::launch_visits(a, visits, num_visits, stream);
  return e;
}

}  // namespace

ca::ScoredState::~ScoredState() {
  if (rows.block) (void)hipFree(rows.block);
  if (columns.block) (void)hipFree(columns.block);
}

extern "C" {

int compact_attn_scored_workspace(ca_layout* L, const ca_scores* scores, int32_t backward, int64_t* workspace_bytes) {
  ca::clear_error();
  if (!workspace_bytes) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (backward != 0 && backward != 1) return fail(CA_ERR_INVALID_ARG, "backward must be 0 or 1");
  int st = check_scores(L, scores);
  if (st != CA_OK) return st;
  Workspace w;
  st = workspace_of(L, scores, backward != 0, w);
  *workspace_bytes = st == CA_OK ? w.bytes() : 0;
  return st;
}

int compact_attn_layout_upload_scored(ca_layout* L, int32_t backward) {
  ca::clear_error();
  if (backward != 0 && backward != 1) return fail(CA_ERR_INVALID_ARG, "backward must be 0 or 1");
  const ca_scores plain{};
  int st = check_scores(L, &plain);
  ca::ScoredWalk* walk = nullptr;
  if (st == CA_OK) st = upload_walk(L, false, nullptr, &walk);
  if (st == CA_OK && backward) st = upload_walk(L, true, nullptr, &walk);
  return st;
}

int compact_attn_forward_scored(const void* q, const void* k, const void* v, ca_layout* L, const ca_scores* scores, void* out, float* lse, void* workspace,
                                int64_t workspace_bytes, void* stream) {
  ca::clear_error();
  if (!q || !k || !v || !out || !lse) return fail(CA_ERR_INVALID_ARG, "null argument");
  int st = check_scores(L, scores);
  if (st != CA_OK) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned4(lse)) return fail(CA_ERR_INVALID_ARG, "tensors must be 16-byte aligned, lse 4-byte");
  Workspace w;
  st = workspace_of(L, scores, false, w);
  const int64_t need = w.bytes(), bytes = ca::tensor_bytes(*L), lse_bytes = bytes / L->prob.head_dim * 2;
  if (st == CA_OK) st = check_workspace(workspace, workspace_bytes, need);
  if (st != CA_OK) return st;
  try {
    std::vector<Range> inputs = token_arrays(L, scores);
    for (const void* t : {q, k, v}) inputs.push_back({t, bytes});
    st = check_apart({{out, bytes}, {lse, lse_bytes}, {workspace, need}}, inputs);
  } catch (const std::bad_alloc&) {
    return fail(CA_ERR_ALLOC, "out of host memory");
  }
  ca::ScoredWalk* walks[2] = {nullptr, nullptr};
  if (st == CA_OK) st = upload_walk(L, false, (hipStream_t)stream, &walks[0]);
  if (st != CA_OK) return st;
  ca::Visits visits[2]{};
  int num_visits = 0;
  ca::ScoredArgs a = scored_args(L, scores, w, workspace, walks, visits, num_visits);
  num_visits ? set_walk(a, visits[0]) : set_walk(a, *walks[0]);
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.lse = lse;
  hipError_t e = launch_tokens(a, visits, num_visits, (hipStream_t)stream);
  if (e == hipSuccess) e = ca::launch_scored_forward(a, (hipStream_t)stream);
  return e == hipSuccess ? CA_OK : hip_fail(e, "scored attention launch");
}

int compact_attn_backward_scored(const void* dout, const void* q, const void* k, const void* v, const void* out, const float* lse, ca_layout* L, const ca_scores* scores,
                                 void* dq, void* dk, void* dv, void* workspace, int64_t workspace_bytes, void* stream) {
  ca::clear_error();
  if (!dout || !q || !k || !v || !out || !lse || !dq || !dk || !dv) return fail(CA_ERR_INVALID_ARG, "null argument");
  int st = check_scores(L, scores);
  if (st != CA_OK) return st;
  for (const void* t : {dout, q, k, v, out, (const void*)dq, (const void*)dk, (const void*)dv})
    if (!aligned16(t)) return fail(CA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  if (!aligned4(lse)) return fail(CA_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  Workspace w;
  st = workspace_of(L, scores, true, w);
  const int64_t need = w.bytes(), bytes = ca::tensor_bytes(*L), lse_bytes = bytes / L->prob.head_dim * 2;
  if (st == CA_OK) st = check_workspace(workspace, workspace_bytes, need);
  if (st != CA_OK) return st;
  try {
    std::vector<Range> inputs = token_arrays(L, scores);
    for (const void* t : {dout, q, k, v, out}) inputs.push_back({t, bytes});
    inputs.push_back({lse, lse_bytes});
    st = check_apart({{dq, bytes}, {dk, bytes}, {dv, bytes}, {workspace, need}}, inputs);
  } catch (const std::bad_alloc&) {
    return fail(CA_ERR_ALLOC, "out of host memory");
  }
  ca::ScoredWalk* walks[2] = {nullptr, nullptr};
  if (st == CA_OK) st = upload_walk(L, false, (hipStream_t)stream, &walks[0]);
  if (st == CA_OK) st = upload_walk(L, true, (hipStream_t)stream, &walks[1]);
  if (st != CA_OK) return st;
  ca::Visits visits[2]{};
  int num_visits = 0;
  ca::ScoredArgs a = scored_args(L, scores, w, workspace, walks, visits, num_visits);
  num_visits ? set_walk(a, visits[0]) : set_walk(a, *walks[0]);
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = out;
  a.dout = dout;
  a.lse_in = lse;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  hipError_t e = launch_tokens(a, visits, num_visits, (hipStream_t)stream);
  if (e == hipSuccess) e = ca::launch_row_stats(a, (hipStream_t)stream);
  if (e == hipSuccess) e = ca::launch_scored_dq(a, (hipStream_t)stream);
  if (e == hipSuccess) {
    num_visits ? set_walk(a, visits[1]) : set_walk(a, *walks[1]);
    e = ca::launch_scored_dkv(a, (hipStream_t)stream);
  }
  return e == hipSuccess ? CA_OK : hip_fail(e, "scored attention gradient launch");
}

}  // extern "C"
