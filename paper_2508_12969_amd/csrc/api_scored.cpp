// C-ABI entry points of scored attention: lists and items of its launches, argument checks, launches (attn_scored.hip, attn_scored_back.hip).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
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

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int check_scores(const ca_layout* L, const ca_scores* s) {
  if (!L || !s) return fail(CA_ERR_INVALID_ARG, "null argument");
  const ca_problem& p = L->prob;
  if (p.dtype != CA_BF16 || (L->B != 64 && L->B != 128) || (p.head_dim != 64 && p.head_dim != 128)) {
    set_error("scored attention supports bf16 with tile sizes 64/128 and head_dim 64/128; got dtype=%d B=%lld D=%d", p.dtype, (long long)L->B, p.head_dim);
    return CA_ERR_UNSUPPORTED;
  }
  if (p.batch > 65535 || (int64_t)p.batch * p.num_heads * L->n > 0x7fffffff) return fail(CA_ERR_UNSUPPORTED, "more than 65535 batch entries or 2^31 - 1 rows");
  if (!(s->cap >= 0.f) || std::isinf(s->cap)) return fail(CA_ERR_INVALID_ARG, "cap must be finite and not negative");
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

// Steps of 64 tokens that a workgroup's other work is worth (start, own tokens, results), and what a share adds; a workgroup's
// places: two per compute unit.  From launches of one tile length: a row of no steps takes 9 to 11 us, a step 1.3 to 1.7.
constexpr int64_t kItemSteps = 6, kShareSteps = 4, kMergeSteps = 5, kPlaces = 512;
constexpr int64_t kMaxScoredShareBytes = (int64_t)128 << 20;

// When the last workgroup ends, in steps, if runs longer than `target` are cut into equal parts of at most that.
int64_t end_of_launch(const std::vector<int64_t>& costs, int64_t batch, int64_t target) {
  std::vector<int64_t> pieces;
  bool shares = false;
  for (int64_t c : costs) {
    const int64_t parts = std::max<int64_t>(1, (c + target - 1) / target);
    shares = shares || parts > 1;
    for (int64_t i = 0; i < parts; ++i) pieces.push_back((c + parts - 1) / parts + kItemSteps + (parts > 1 ? kShareSteps : 0));
  }
  std::sort(pieces.begin(), pieces.end(), std::greater<int64_t>());
  std::priority_queue<int64_t, std::vector<int64_t>, std::greater<int64_t>> places;
  for (int64_t i = 0; i < kPlaces; ++i) places.push(0);
  int64_t end = 0;
  for (int64_t b = 0; b < batch; ++b)
    for (int64_t c : pieces) {
      const int64_t at = places.top() + c;
      places.pop();
      places.push(at);
      end = std::max(end, at);
    }
  return end + (shares ? kMergeSteps : 0);
}

// Longest part of a run, in steps: runs are cut where the launch would end with a few long ones, or leave compute units without work.  masked: documents and
// limits will leave out parts of the runs, which ones is not known here; the longest may stay whole while the others shrink, so runs are cut as if the launch
// were half as much work.
int64_t part_steps(const std::vector<int64_t>& costs, int64_t batch, int64_t share_bytes, bool masked) {
  const int64_t whole = (int64_t)1 << 40;
  int64_t total = 0;
  for (int64_t c : costs) total += c;
  if ((int64_t)costs.size() * batch > 16 * kPlaces) return whole;  // (no run is long beside so many)
  int64_t best = whole, best_end = end_of_launch(costs, batch, whole);
  const int64_t ideal = std::max<int64_t>(1, total * batch / kPlaces);
  for (int64_t divisor = masked ? 2 : 1; divisor <= 4; ++divisor) {
    const int64_t target = std::max<int64_t>(8, (ideal + divisor - 1) / divisor);
    int64_t shares = 0;
    for (int64_t c : costs) shares += c > target ? (c + target - 1) / target : 0;
    if (shares == 0) break;
    if (shares * batch * share_bytes > kMaxScoredShareBytes) break;
    if (masked) return target;
    const int64_t end = end_of_launch(costs, batch, target);
    if (20 * end < 19 * best_end) best = target, best_end = end;  // (not for a few per cent)
  }
  return best;
}

// The lists of the layout's rows (or columns), as groups, and the items of a launch.
int make_walk(const ca_layout* L, bool columns, ca::ScoredWalk& walk) {
  if (L->class_mask.size() > 32) return fail(CA_ERR_UNSUPPORTED, "too many padding classes for scored attention");
  const int64_t n = L->n, heads = L->prob.num_heads, rows = heads * n, tiles = ca::kGroupTokens / L->B, groups = (n + tiles - 1) / tiles;
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
  std::vector<int64_t> first(heads * groups + 1, 0), costs(heads * groups);
  walk.words.reserve(L->col_idx.size());
  for (int64_t g = 0; g < heads * groups; ++g) {
    const int64_t row = g / groups * n + g % groups * tiles;
    const bool second = tiles == 2 && g % groups * tiles + 1 < n;
    int64_t i = ptr[row], j = second ? ptr[row + 1] : 0;
    const int64_t i_end = ptr[row + 1], j_end = second ? ptr[row + 2] : 0;
    while (i < i_end || j < j_end) {
      const int32_t a = i < i_end ? idx[i] : INT32_MAX, b = j < j_end ? idx[j] : INT32_MAX, t = std::min(a, b);
      walk.words.push_back((uint32_t)t | (uint32_t)L->tile_class[t] << 24 | (a == t ? 1u << 30 : 0u) | (b == t ? 1u << 31 : 0u));
      i += a == t;
      j += b == t;
    }
    first[g + 1] = (int64_t)walk.words.size();
    if (first[g + 1] - first[g] > INT32_MAX / 2) return fail(CA_ERR_UNSUPPORTED, "a list is too long for scored attention");
    costs[g] = (first[g + 1] - first[g]) * (L->B / 64);
  }
  const int sums = columns ? ca::kv_sums(L->prob.head_dim) : 1;
  for (int masked = 0; masked < 2; ++masked) {
    ca::ScoredPlan& plan = walk.plans[masked];
    const int64_t words_at_once = std::max<int64_t>(1, part_steps(costs, L->prob.batch, ca::share_floats(L->prob.head_dim, sums) * 4, masked) / (L->B / 64));
    for (int64_t g = 0; g < heads * groups; ++g) {
      const int64_t count = first[g + 1] - first[g], parts = std::max<int64_t>(1, (count + words_at_once - 1) / words_at_once), size = (count + parts - 1) / parts;
      if (parts > 1) plan.merges.push_back({(int32_t)g, (int32_t)plan.shares, (int32_t)parts, 0});
      for (int64_t i = 0; i < parts; ++i) {
        const int64_t from = std::min(count, i * size), to = std::min(count, from + size);
        plan.items.push_back({first[g] + from, (int32_t)(to - from), (int32_t)g, parts > 1 ? (int32_t)(plan.shares + i) : -1, 0});
      }
      plan.shares += parts > 1 ? parts : 0;
    }
    std::stable_sort(plan.items.begin(), plan.items.end(), [](const ca::ScoredItem& a, const ca::ScoredItem& b) { return a.count > b.count; });
    if ((int64_t)plan.items.size() * L->prob.batch > 0x7fffffff) return fail(CA_ERR_UNSUPPORTED, "more than 2^31 - 1 workgroups");
  }
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
  auto padded = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
  size_t bytes = padded(w.words.size() * sizeof(uint32_t)), at[2][2];
  for (int i = 0; i < 2; ++i) {
    at[i][0] = bytes;
    bytes += padded(w.plans[i].items.size() * sizeof(ca::ScoredItem));
    at[i][1] = bytes;
    bytes += padded(w.plans[i].merges.size() * sizeof(ca::ScoredMerge));
  }
  void* p = nullptr;
  hipError_t e = hipMalloc(&p, bytes);
  if (e != hipSuccess) {
    set_error("hipMalloc of %zu bytes for the lists of scored attention failed: %s", bytes, hipGetErrorString(e));
    (void)hipGetLastError();
    return CA_ERR_ALLOC;
  }
  unsigned char* const d = static_cast<unsigned char*>(p);
  auto put = [&](size_t to, const void* from, size_t size) {
    if (e == hipSuccess && size) e = hipMemcpy(d + to, from, size, hipMemcpyHostToDevice);
  };
  put(0, w.words.data(), w.words.size() * sizeof(uint32_t));
  for (int i = 0; i < 2; ++i) {
    put(at[i][0], w.plans[i].items.data(), w.plans[i].items.size() * sizeof(ca::ScoredItem));
    put(at[i][1], w.plans[i].merges.data(), w.plans[i].merges.size() * sizeof(ca::ScoredMerge));
  }
  if (e != hipSuccess) {
    (void)hipFree(p);
    return hip_fail(e, "hipMemcpy of the lists of scored attention");
  }
  w.dev_words = reinterpret_cast<uint32_t*>(d);
  for (int i = 0; i < 2; ++i) {
    w.plans[i].dev_items = reinterpret_cast<ca::ScoredItem*>(d + at[i][0]);
    w.plans[i].dev_merges = reinterpret_cast<ca::ScoredMerge*>(d + at[i][1]);
  }
  w.block = d;
  return CA_OK;
}

bool is_masked(const ca_scores* s) { return s->limits || s->documents; }

void set_walk(ca::ScoredArgs& a, const ca::ScoredWalk& w, const ca_scores* s) {
  const ca::ScoredPlan& plan = w.plans[is_masked(s)];
  a.words = w.dev_words;
  a.items = plan.dev_items;
  a.merges = plan.dev_merges;
  a.num_items = (int64_t)plan.items.size();
  a.num_merges = (int64_t)plan.merges.size();
  a.shares = plan.shares;
}

int64_t padded256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Bytes of a call's workspace: the tokens' line, the row statistics, the shares.
int workspace_bytes_of(ca_layout* L, const ca_scores* s, bool backward, int64_t* bytes) {
  const ca_problem& p = L->prob;
  ca::ScoredWalk *rows = nullptr, *columns = nullptr;
  int st = walk_of(L, false, &rows);
  if (st == CA_OK && backward) st = walk_of(L, true, &columns);
  if (st != CA_OK) return st;
  int64_t shares = p.batch * rows->plans[is_masked(s)].shares * ca::share_floats(p.head_dim, 1) * 4;
  if (backward) shares = std::max(shares, p.batch * columns->plans[is_masked(s)].shares * ca::share_floats(p.head_dim, ca::kv_sums(p.head_dim)) * 4);
  *bytes = (has_line(s) ? ca::line_bytes(p.batch, L->n, L->B) + ca::tile_line_bytes(p.batch, L->n) : 0) +
           (backward ? padded256(ca::row_stat_bytes((int64_t)p.batch * p.num_heads, L->n, L->B)) : 0) + shares;
  return CA_OK;
}

ca::ScoredArgs scored_args(const ca_layout* L, const ca_scores* s, bool backward, void* workspace) {
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
  unsigned char* w = static_cast<unsigned char*>(workspace);
  if (has_line(s)) {
    a.line = reinterpret_cast<float*>(w);
    w += ca::line_bytes(p.batch, L->n, L->B);
    a.tiles = reinterpret_cast<ca::TileLine*>(w);
    w += ca::tile_line_bytes(p.batch, L->n);
  }
  if (backward) {
    a.rows = reinterpret_cast<float*>(w);
    w += padded256(ca::row_stat_bytes((int64_t)p.batch * p.num_heads, L->n, L->B));
  }
  a.share_sums = reinterpret_cast<float*>(w);
  return a;
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
  const int st = check_scores(L, scores);
  if (st != CA_OK) return st;
  return workspace_bytes_of(L, scores, backward != 0, workspace_bytes);
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
  int64_t need = 0;
  const int64_t bytes = ca::tensor_bytes(*L), lse_bytes = bytes / L->prob.head_dim * 2;
  st = workspace_bytes_of(L, scores, false, &need);
  if (st == CA_OK) st = check_workspace(workspace, workspace_bytes, need);
  if (st != CA_OK) return st;
  try {
    std::vector<Range> inputs = token_arrays(L, scores);
    for (const void* t : {q, k, v}) inputs.push_back({t, bytes});
    st = check_apart({{out, bytes}, {lse, lse_bytes}, {workspace, need}}, inputs);
  } catch (const std::bad_alloc&) {
    return fail(CA_ERR_ALLOC, "out of host memory");
  }
  ca::ScoredWalk* rows = nullptr;
  if (st == CA_OK) st = upload_walk(L, false, (hipStream_t)stream, &rows);
  if (st != CA_OK) return st;
  ca::ScoredArgs a = scored_args(L, scores, false, workspace);
  set_walk(a, *rows, scores);
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.lse = lse;
  hipError_t e = a.line ? ca::launch_line(a, (hipStream_t)stream) : hipSuccess;
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
  int64_t need = 0;
  const int64_t bytes = ca::tensor_bytes(*L), lse_bytes = bytes / L->prob.head_dim * 2;
  st = workspace_bytes_of(L, scores, true, &need);
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
  ca::ScoredWalk *rows = nullptr, *columns = nullptr;
  if (st == CA_OK) st = upload_walk(L, false, (hipStream_t)stream, &rows);
  if (st == CA_OK) st = upload_walk(L, true, (hipStream_t)stream, &columns);
  if (st != CA_OK) return st;
  ca::ScoredArgs a = scored_args(L, scores, true, workspace);
  set_walk(a, *rows, scores);
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = out;
  a.dout = dout;
  a.lse_in = lse;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  hipError_t e = a.line ? ca::launch_line(a, (hipStream_t)stream) : hipSuccess;
  if (e == hipSuccess) e = ca::launch_row_stats(a, (hipStream_t)stream);
  if (e == hipSuccess) e = ca::launch_scored_dq(a, (hipStream_t)stream);
  if (e == hipSuccess) {
    set_walk(a, *columns, scores);
    e = ca::launch_scored_dkv(a, (hipStream_t)stream);
  }
  return e == hipSuccess ? CA_OK : hip_fail(e, "scored attention gradient launch");
}

}  // extern "C"
