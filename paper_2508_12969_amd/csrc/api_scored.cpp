// C-ABI entry points of scored attention: transposed lists, argument checks, launches (attn_scored.hip, attn_scored_back.hip).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <numeric>
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

int64_t workspace_bytes_of(const ca_layout* L, const ca_scores* s, bool backward) {
  const ca_problem& p = L->prob;
  return (has_line(s) ? ca::line_bytes(p.batch, L->n, L->B) + ca::tile_line_bytes(p.batch, L->n) : 0) +
         (backward ? ca::row_stat_bytes((int64_t)p.batch * p.num_heads, L->n, L->B) : 0);
}

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

// For every (head, key tile) the query tiles that keep it, on the device.
int ensure_transposed(ca_layout* L, hipStream_t stream) {
  std::lock_guard<std::mutex> lock(L->upload_mutex);
  if (L->dev.transposed_block) return CA_OK;
  if (stream) {
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    const hipError_t e = hipStreamIsCapturing(stream, &cap);
    if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
    if (cap != hipStreamCaptureStatusNone)
      return fail(CA_ERR_INVALID_ARG, "the layout's transposed lists are not on the device yet and the stream is being captured: call compact_attn_layout_upload_backward "
                                      "before the capture");
  }
  const int64_t n = L->n, rows = (int64_t)L->prob.num_heads * n, nnz = (int64_t)L->col_idx.size();
  auto padded = [](int64_t bytes) { return (bytes + 255) / 256 * 256; };
  const int64_t ptr_bytes = padded((rows + 1) * 8), meta_bytes = padded(nnz * 4), order_bytes = padded(rows * 4);
  std::vector<unsigned char> image((size_t)(ptr_bytes + meta_bytes + order_bytes), 0);
  int64_t* const ptr = reinterpret_cast<int64_t*>(image.data());
  int32_t* const meta = reinterpret_cast<int32_t*>(image.data() + ptr_bytes);
  int32_t* const order = reinterpret_cast<int32_t*>(image.data() + ptr_bytes + meta_bytes);
  for (int64_t head = 0; head < L->prob.num_heads; ++head)
    for (int64_t i = L->row_ptr[head * n]; i < L->row_ptr[(head + 1) * n]; ++i) ++ptr[head * n + L->col_idx[i] + 1];
  for (int64_t r = 0; r < rows; ++r) ptr[r + 1] += ptr[r];
  std::vector<int64_t> at(ptr, ptr + rows);
  for (int64_t row = 0; row < rows; ++row) {
    const int64_t head = row / n, tile = row - head * n;
    const int32_t word = (int32_t)((uint32_t)tile | (uint32_t)L->tile_class[tile] << 24);
    for (int64_t i = L->row_ptr[row]; i < L->row_ptr[row + 1]; ++i) meta[at[head * n + L->col_idx[i]]++] = word;
  }
  std::iota(order, order + rows, 0);
  std::stable_sort(order, order + rows, [&](int32_t x, int32_t y) { return ptr[x + 1] - ptr[x] > ptr[y + 1] - ptr[y]; });

  void* block = nullptr;
  hipError_t e = hipMalloc(&block, image.size());
  if (e != hipSuccess) {
    set_error("hipMalloc of %zu bytes for the transposed lists failed: %s", image.size(), hipGetErrorString(e));
    (void)hipGetLastError();
    return CA_ERR_ALLOC;
  }
  e = hipMemcpy(block, image.data(), image.size(), hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    (void)hipFree(block);
    return hip_fail(e, "hipMemcpy of the transposed lists");
  }
  unsigned char* const d = static_cast<unsigned char*>(block);
  L->dev.transposed_row_ptr = reinterpret_cast<int64_t*>(d);
  L->dev.transposed_meta = reinterpret_cast<int32_t*>(d + ptr_bytes);
  L->dev.transposed_order = reinterpret_cast<int32_t*>(d + ptr_bytes + meta_bytes);
  L->dev.transposed_block = d;
  return CA_OK;
}

int ensure_backward(ca_layout* L, hipStream_t stream) {
  const int st = ca::ensure_uploaded(L, stream);
  if (st != CA_OK) return st;
  try {
    return ensure_transposed(L, stream);
  } catch (const std::bad_alloc&) {
    return fail(CA_ERR_ALLOC, "out of host memory while making the transposed lists");
  }
}

ca::ScoredArgs scored_args(const ca_layout* L, const ca_scores* s, void* workspace) {
  const ca_problem& p = L->prob;
  ca::ScoredArgs a{};
  ca::fill_grid(a, L);
  a.row_ptr = L->dev.row_ptr;
  a.col_meta = L->dev.col_meta;
  a.order = L->dev.order;
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
  a.rows = reinterpret_cast<float*>(w);
  return a;
}

}  // namespace

extern "C" {

int compact_attn_scored_workspace(const ca_layout* L, const ca_scores* scores, int32_t backward, int64_t* workspace_bytes) {
  ca::clear_error();
  if (!workspace_bytes) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (backward != 0 && backward != 1) return fail(CA_ERR_INVALID_ARG, "backward must be 0 or 1");
  const int st = check_scores(L, scores);
  if (st != CA_OK) return st;
  *workspace_bytes = workspace_bytes_of(L, scores, backward != 0);
  return CA_OK;
}

int compact_attn_layout_upload_backward(ca_layout* L) {
  ca::clear_error();
  if (!L) return fail(CA_ERR_INVALID_ARG, "null layout");
  return ensure_backward(L, nullptr);
}

int compact_attn_forward_scored(const void* q, const void* k, const void* v, ca_layout* L, const ca_scores* scores, void* out, float* lse, void* workspace,
                                int64_t workspace_bytes, void* stream) {
  ca::clear_error();
  if (!q || !k || !v || !out || !lse) return fail(CA_ERR_INVALID_ARG, "null argument");
  int st = check_scores(L, scores);
  if (st != CA_OK) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned4(lse)) return fail(CA_ERR_INVALID_ARG, "tensors must be 16-byte aligned, lse 4-byte");
  const int64_t need = workspace_bytes_of(L, scores, false), bytes = ca::tensor_bytes(*L), lse_bytes = bytes / L->prob.head_dim * 2;
  st = check_workspace(workspace, workspace_bytes, need);
  if (st != CA_OK) return st;
  try {
    std::vector<Range> inputs = token_arrays(L, scores);
    for (const void* t : {q, k, v}) inputs.push_back({t, bytes});
    st = check_apart({{out, bytes}, {lse, lse_bytes}, {workspace, need}}, inputs);
  } catch (const std::bad_alloc&) {
    return fail(CA_ERR_ALLOC, "out of host memory");
  }
  if (st == CA_OK) st = ca::ensure_uploaded(L, (hipStream_t)stream);
  if (st != CA_OK) return st;
  ca::ScoredArgs a = scored_args(L, scores, workspace);
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
  const int64_t need = workspace_bytes_of(L, scores, true), bytes = ca::tensor_bytes(*L), lse_bytes = bytes / L->prob.head_dim * 2;
  st = check_workspace(workspace, workspace_bytes, need);
  if (st != CA_OK) return st;
  try {
    std::vector<Range> inputs = token_arrays(L, scores);
    for (const void* t : {dout, q, k, v, out}) inputs.push_back({t, bytes});
    inputs.push_back({lse, lse_bytes});
    st = check_apart({{dq, bytes}, {dk, bytes}, {dv, bytes}, {workspace, need}}, inputs);
  } catch (const std::bad_alloc&) {
    return fail(CA_ERR_ALLOC, "out of host memory");
  }
  if (st == CA_OK) st = ensure_backward(L, (hipStream_t)stream);
  if (st != CA_OK) return st;
  ca::ScoredArgs a = scored_args(L, scores, workspace);
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
    a.row_ptr = L->dev.transposed_row_ptr;
    a.col_meta = L->dev.transposed_meta;
    a.order = L->dev.transposed_order;
    e = ca::launch_scored_dkv(a, (hipStream_t)stream);
  }
  return e == hipSuccess ? CA_OK : hip_fail(e, "scored attention gradient launch");
}

}  // extern "C"
