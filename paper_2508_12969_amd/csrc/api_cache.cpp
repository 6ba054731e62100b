// C-ABI entry points of the paged cache: argument checks, launches (cache.hip, attn_cache.hip).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "api_common.h"
#include "cache.h"
#include "scored.h"

using ca::aligned16;
using ca::elem_size;
using ca::fail;
using ca::hip_fail;
using ca::ranges_overlap;
using ca::set_error;

namespace {

constexpr int64_t kMostTokens = (int64_t)1 << 30, kMostBytes = (int64_t)1 << 46;
constexpr int32_t kMostSequences = 1 << 20;
constexpr int64_t kWholeTokens = 1024;  // sequences of at most so many are not cut: 16 of up to 600 / 900 / 2000 tokens, cut / whole, 17.6 / 12.8, 18.5 / 16.9, 19.4 / 27.0 us
constexpr int64_t kLeastFewSteps = 8, kLeastManySteps = 8;  // of a workgroup's share: 256 and 512 tokens
constexpr int32_t kItemSequences = 512;  // every workgroup looks through all sequences for its own: of more, only as many workgroups as the device holds do
constexpr int64_t kMostItems = 0xffffff / 64;  // 64 parts of each are a launch
constexpr int64_t kSideBySide = 512;   // rows of a sequence from which on tiles walk side by side

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int check_cache(const ca_cache* c) {
  if (!c) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (!c->k || !c->v || !c->table || !c->lengths || !c->starts) return fail(CA_ERR_INVALID_ARG, "pages, table, lengths and starts of a cache must not be null");
  if (c->dtype != CA_F32 && c->dtype != CA_BF16) return fail(CA_ERR_INVALID_ARG, "dtype must be a ca_dtype value");
  if (c->num_pages < 1 || c->num_pages > 0x7fffffff || c->kv_heads < 1 || c->head_dim < 1 || c->sequences < 1 || c->table_width < 1 || c->tokens < 0)
    return fail(CA_ERR_INVALID_ARG, "sizes of a cache must be positive, with fewer than 2^31 pages");
  if (c->page_tokens < 16 || c->page_tokens > 65536 || c->page_tokens % 16 != 0) return fail(CA_ERR_INVALID_ARG, "page_tokens must be a multiple of 16 up to 65536");
  if ((int64_t)c->table_width * c->page_tokens > kMostTokens) return fail(CA_ERR_INVALID_ARG, "a sequence of the table must have fewer than 2^30 tokens");
  if (c->frame_height < 1 || c->frame_width < 1 || (int64_t)c->frame_height * c->frame_width > kMostTokens)
    return fail(CA_ERR_INVALID_ARG, "frame_height and frame_width must be positive, their product at most 2^30");
  if ((int64_t)c->head_dim * elem_size(c->dtype) % 16 != 0) return fail(CA_ERR_INVALID_ARG, "rows must be a multiple of 16 bytes");
  const int most = c->dtype == CA_BF16 ? 512 : 256;
  if (c->head_dim > most || c->kv_heads > 65535 || c->sequences > kMostSequences) {
    set_error("a cache takes head_dim up to %d in this type, 65535 heads and 2^20 sequences; got D=%d, %d heads, %d sequences", most, c->head_dim, c->kv_heads, c->sequences);
    return CA_ERR_UNSUPPORTED;
  }
  const int64_t head_bytes = (int64_t)c->page_tokens * c->head_dim * elem_size(c->dtype);  // at most 2^26, times 2^16 heads
  if (c->num_pages > kMostBytes / (head_bytes * c->kv_heads)) return fail(CA_ERR_INVALID_ARG, "pages of more than 2^46 bytes");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(CA_ERR_INVALID_ARG, "pages must be 16-byte aligned");
  if (!aligned4(c->table) || !aligned4(c->lengths) || !aligned4(c->starts) || !aligned4(c->origins))
    return fail(CA_ERR_INVALID_ARG, "table, lengths, starts and origins must be 4-byte aligned");
  return CA_OK;
}

int64_t page_bytes(const ca_cache* c) { return c->num_pages * c->kv_heads * c->page_tokens * c->head_dim * elem_size(c->dtype); }

void fill_cache(ca::CacheArgs& a, const ca_cache* c) {
  a.k = c->k;
  a.v = c->v;
  a.num_pages = c->num_pages;
  a.page_tokens = c->page_tokens;
  a.kv_heads = c->kv_heads;
  a.sequences = c->sequences;
  a.table_width = c->table_width;
  a.tokens = c->tokens;
  a.frame_h = c->frame_height;
  a.frame_w = c->frame_width;
  a.span = c->frame_height * c->frame_width;
  a.table = c->table;
  a.lengths = c->lengths;
  a.starts = c->starts;
  a.origins = c->origins;
}

// Strides of a packed tensor of `heads` heads, and the bytes from its first to the end of its last element.
int packed_strides(const ca_cache* c, const ca_strides* s, int32_t heads, const char* name, ca::TokenStrides& out, int64_t& bytes) {
  out = {(int64_t)heads * c->head_dim, c->head_dim};
  if (s) {
    const int64_t unit = 16 / elem_size(c->dtype);
    const std::pair<int64_t, int64_t> steps[] = {{s->head, heads}, {s->token, c->tokens}};
    for (const auto& [stride, count] : steps)
      if (stride < 0 || stride > ((int64_t)1 << 40) / std::max<int64_t>(1, count - 1) || stride % unit != 0) {
        set_error("strides of %s must be multiples of 16 bytes, not negative, and lead over fewer than 2^40 elements", name);
        return CA_ERR_INVALID_ARG;
      }
    out = {s->token, s->head};
  }
  bytes = c->tokens < 1 ? 0 : ((c->tokens - 1) * out.token + (heads - 1) * out.head + c->head_dim) * elem_size(c->dtype);
  return CA_OK;
}

struct Range {
  const void* at;
  int64_t bytes;
};

// Results may not overlap each other or anything that is read; a cache's arrays are read by every call.
int check_apart(const ca_cache* c, std::initializer_list<Range> results, std::initializer_list<Range> inputs) {
  const Range arrays[] = {{c->table, (int64_t)c->sequences * c->table_width * 4}, {c->lengths, (int64_t)c->sequences * 4}, {c->starts, ((int64_t)c->sequences + 1) * 4},
                          {c->origins, (int64_t)c->sequences * 4}};
  auto meets = [](const Range& a, const Range& b) { return a.at && b.at && a.bytes > 0 && b.bytes > 0 && ranges_overlap(a.at, a.bytes, b.at, b.bytes); };
  for (const Range* r = results.begin(); r != results.end(); ++r) {
    for (const Range& in : inputs)
      if (meets(*r, in)) return fail(CA_ERR_INVALID_ARG, "results and workspace must not overlap the inputs");
    for (const Range& in : arrays)
      if (meets(*r, in)) return fail(CA_ERR_INVALID_ARG, "results and workspace must not overlap the cache's arrays");
    for (const Range* other = r + 1; other != results.end(); ++other)
      if (meets(*r, *other)) return fail(CA_ERR_INVALID_ARG, "results and workspace must not overlap each other");
  }
  return CA_OK;
}

int check_append(const ca_append* p, const ca_cache* c) {
  if (!p) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (!p->q != !p->q_out) return fail(CA_ERR_INVALID_ARG, "both q and q_out or none");
  if (c->tokens > 0 && (!p->k || !p->v)) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (2 * (int64_t)c->kv_heads > 65535) return fail(CA_ERR_UNSUPPORTED, "more than 65535 heads of keys and values");
  if (p->q && (p->heads < 1 || p->heads > 65535 - 2 * (int64_t)c->kv_heads)) return fail(CA_ERR_INVALID_ARG, "heads must be positive, and with those of keys and values at most 65535");
  for (const void* t : {p->q, p->k, p->v, (const void*)p->q_out, p->q_weight, p->k_weight})
    if (!aligned16(t)) return fail(CA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  if (p->normed != 0 && p->normed != 1) return fail(CA_ERR_INVALID_ARG, "normed must be 0 or 1");
  if (!p->normed && (p->q_weight || p->k_weight)) return fail(CA_ERR_INVALID_ARG, "weights belong to a norm");
  if (!p->q && p->q_weight) return fail(CA_ERR_INVALID_ARG, "q_weight without q");
  if (p->normed && (!(p->eps >= 0.f) || std::isinf(p->eps))) return fail(CA_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (!p->rotary) return CA_OK;
  if (p->rotary->channels > c->head_dim) return fail(CA_ERR_INVALID_ARG, "more rotated channels than the head has");
  if (p->where && p->where->positions) {
    if (!aligned4(p->where->positions)) return fail(CA_ERR_INVALID_ARG, "positions must be 4-byte aligned");
  } else if (p->where) {
    for (int i = 0; i < 3; ++i)
      if (p->rotary->axes[i].channels && p->where->origin[i] < 0) return fail(CA_ERR_INVALID_ARG, "origins must not be negative");
  }
  return CA_OK;
}

int check_attend(const ca_cache* c, const ca_reach* r, int32_t heads) {
  if (c->head_dim != 64 && c->head_dim != 128) {
    set_error("attention over a cache supports head_dim 64 and 128; got D=%d", c->head_dim);
    return CA_ERR_UNSUPPORTED;
  }
  if (heads < 1 || heads > 65535 || heads % c->kv_heads != 0) return fail(CA_ERR_INVALID_ARG, "heads must be a multiple of kv_heads, at most 65535");
  if (!r) return CA_OK;
  if (std::isnan(r->scale) || std::isinf(r->scale) || (r->scale > 0.f && (r->scale < 0x1p-100f || r->scale > 0x1p100f)))  // (what is made of it, and of it and the cap, stays a number)
    return fail(CA_ERR_INVALID_ARG, "scale must be finite, and between 2^-100 and 2^100 where it is positive");
  if (r->cap != 0.f && !(r->cap >= ca::kLeastCap && r->cap <= ca::kMostCap)) return fail(CA_ERR_INVALID_ARG, "cap must be 0 or between 2^-16 and 4096");
  if (r->causal != 0 && r->causal != 1) return fail(CA_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (r->window < 0) return fail(CA_ERR_INVALID_ARG, "window must not be negative");
  if (!aligned4(r->slopes) || (reinterpret_cast<uintptr_t>(r->tree) & 7u) != 0) return fail(CA_ERR_INVALID_ARG, "slopes must be 4-byte aligned, tree 8-byte");
  return CA_OK;
}

// Parts of a call's workspace, in their order.
struct Workspace {
  int64_t splits = 0, pieces = 0;
  int64_t bytes() const { return splits + pieces; }
};

int64_t padded256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Equal parts of items of up to `steps` steps: launches of few items would leave compute units without work, or end with a round that is not full.  A workgroup takes as long as
// kItemSteps steps besides its own, and kPieceSteps more where its sums are joined.
void cut_items(ca::AttendArgs& a, int64_t steps) {
  constexpr int64_t kItemSteps = 6, kPieceSteps = 4, kMostParts = 63, kMostPieceBytes = (int64_t)256 << 20;
  const int64_t items = a.tiles * a.kv_heads, piece_bytes = (int64_t)ca::kManyRows * ca::piece_row(a.D) * 4, places = ca::many_places(a.D);
  int64_t best = 1, best_end = 0;
  for (int64_t parts = 1; parts <= kMostParts; ++parts) {
    const int64_t size = (steps + parts - 1) / parts;
    if (parts > 1 && (size < kLeastManySteps || items * parts * piece_bytes > kMostPieceBytes)) break;
    const int64_t rounds = (items * parts + places - 1) / places, end = rounds * (size + kItemSteps + (parts > 1 ? kPieceSteps : 0));
    if (parts == 1 || 50 * end < 49 * best_end) best = parts, best_end = end;  // (not for a per cent)
  }
  a.way = best > 1 ? ca::kParts : ca::kItems;
  a.most_parts = (int32_t)best;
  a.part_steps = (int32_t)((steps + best - 1) / best);
}

// How a call's launch is shared out (Share).  Tiles that walk side by side cost their keys one reading, an even line cuts anything evenly: three frames over 75K tokens 4.9 / 6.0 ms, but 8 sequences
// of very different lengths with 680 rows each 211 / 120 us.  So the former where all tiles are alike (one sequence, all of it seen), or so many that they are even without being cut.  What no
// window takes up in the workspace, and what one does, is asked for alike.  Few rows or many goes by the average: how many each sequence has is known on the device alone (a prompt of 2000 tokens beside 200
// single ones 652 us, in two calls 623; a prompt of 1000 beside 255, which go as few, 832 and 812).
int fill_attend(ca::AttendArgs& a, Workspace& w, const ca_cache* c, int32_t heads, bool window) {
  fill_cache(a, c);
  a.heads = heads;
  a.group = heads / c->kv_heads;
  a.D = c->head_dim;
  const int64_t most_tokens = (int64_t)c->table_width * c->page_tokens, rows = (int64_t)((c->tokens + (int64_t)c->sequences - 1) / c->sequences) * a.group;
  a.many = rows > ca::kFewRows && c->dtype == CA_BF16;
  const int64_t tile = a.many ? ca::kManyRows : ca::kFewRows, piece_bytes = tile * ca::piece_row(a.D) * 4;
  a.tiles = (int64_t)c->tokens * a.group / tile + std::min(c->tokens, c->sequences);
  if ((int64_t)c->tokens * a.group > kMostTokens) return fail(CA_ERR_UNSUPPORTED, "more rows than a launch takes");
  const int64_t items = a.tiles * c->kv_heads;
  a.way = ca::kItems;  // (items of a few steps are not worth a second launch)
  const bool itemized = c->sequences <= kItemSequences && items <= kMostItems, side_by_side = itemized && a.many && rows >= kSideBySide && ((c->sequences == 1 && !window) || items >= 2 * ca::many_places(a.D));
  if (side_by_side) {
    cut_items(a, (most_tokens + ca::kManyStep - 1) / ca::kManyStep);
    if (a.way == ca::kParts) {
      w.splits = padded256(items * (int64_t)sizeof(ca::CacheSplit));
      w.pieces = items * a.most_parts * piece_bytes;
    }
  } else if (most_tokens > kWholeTokens || !itemized) {
    a.way = ca::kShares;
    a.workgroups = a.many ? ca::kManyWorkgroups : ca::few_workgroups(a.D);
    a.least_steps = a.many ? kLeastManySteps : kLeastFewSteps;
    w.splits = padded256(a.workgroups * (int64_t)sizeof(ca::CacheSplit));
    w.pieces = (int64_t)a.workgroups * 2 * piece_bytes;
  }
  return CA_OK;
}

}  // namespace

extern "C" {

int compact_attn_cache_append(const ca_append* p, const ca_cache* c, void* stream) {
  ca::clear_error();
  int st = check_cache(c);
  if (st == CA_OK) st = check_append(p, c);
  if (st != CA_OK) return st;
  ca::AppendArgs a{};
  const int32_t heads = p->q ? p->heads : 0;
  int64_t q_bytes = 0, k_bytes = 0, v_bytes = 0;
  if (p->q) st = packed_strides(c, p->q_strides, heads, "q", a.q_strides, q_bytes);
  if (st == CA_OK) st = packed_strides(c, p->k_strides, c->kv_heads, "k", a.k_strides, k_bytes);
  if (st == CA_OK) st = packed_strides(c, p->v_strides, c->kv_heads, "v", a.v_strides, v_bytes);
  if (st != CA_OK) return st;
  const int64_t row = (int64_t)c->head_dim * elem_size(c->dtype);
  if (c->tokens >= (1 << 26) - (row > 512 ? 3 : 0))  // (a launch has fewer than 2^32 threads; rows of more than 512 bytes are a wave's)
    return fail(CA_ERR_UNSUPPORTED, "2^26 new tokens and more, or 2^26 - 3 of rows of more than 512 bytes");
  const int64_t out_bytes = (int64_t)c->tokens * heads * row, pages = page_bytes(c);
  const void* const positions = p->rotary && p->where ? p->where->positions : nullptr;
  st = check_apart(c, {{p->q_out, out_bytes}, {c->k, pages}, {c->v, pages}},
                   {{p->q, q_bytes}, {p->k, k_bytes}, {p->v, v_bytes}, {p->q_weight, row}, {p->k_weight, row}, {positions, (int64_t)c->tokens * 12}});
  if (st != CA_OK || c->tokens == 0) return st;
  fill_cache(a, c);
  a.D = c->head_dim;
  a.eps = p->eps;
  a.sign = 1.f;
  a.q = p->q;
  a.k_new = p->k;
  a.v_new = p->v;
  a.q_out = p->q_out;
  a.heads = heads;
  a.q_weight = p->q_weight;
  a.k_weight = p->k_weight;
  if (p->rotary) {
    st = ca::fill_rotation(a, p->rotary, (hipStream_t)stream);
    if (st != CA_OK) return st;
    a.where = static_cast<const int32_t*>(positions);
    for (int i = 0; i < 3; ++i) a.origin[i] = p->where && p->rotary->axes[i].channels ? p->where->origin[i] : 0;
  }
  const hipError_t e = ca::launch_append(a, c->dtype == CA_BF16, p->normed != 0, (hipStream_t)stream);
  return e == hipSuccess ? CA_OK : hip_fail(e, "cache append launch");
}

int compact_attn_cache_workspace(const ca_cache* c, int32_t heads, int64_t* workspace_bytes) {
  ca::clear_error();
  if (!workspace_bytes) return fail(CA_ERR_INVALID_ARG, "null argument");
  *workspace_bytes = 0;
  int st = check_cache(c);
  if (st == CA_OK) st = check_attend(c, nullptr, heads);
  ca::AttendArgs a{};
  Workspace w, windowed;
  if (st == CA_OK) st = fill_attend(a, w, c, heads, false);
  if (st == CA_OK) st = fill_attend(a, windowed, c, heads, true);
  if (st == CA_OK) *workspace_bytes = std::max(w.bytes(), windowed.bytes());
  return st;
}

int compact_attn_cache_attend(const void* q, const ca_strides* q_strides, int32_t heads, const ca_cache* c, const ca_reach* r, void* out, float* lse, void* workspace,
                              int64_t workspace_bytes, void* stream) {
  ca::clear_error();
  if (!r) return fail(CA_ERR_INVALID_ARG, "null argument");
  int st = check_cache(c);
  if (st == CA_OK) st = check_attend(c, r, heads);
  if (st != CA_OK) return st;
  if (c->tokens > 0 && (!q || !out || !lse)) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (!aligned16(q) || !aligned16(out) || !aligned4(lse)) return fail(CA_ERR_INVALID_ARG, "tensors must be 16-byte aligned, lse 4-byte");
  ca::AttendArgs a{};
  int64_t q_bytes = 0;
  st = packed_strides(c, q_strides, heads, "q", a.q_strides, q_bytes);
  Workspace w;
  if (st == CA_OK) st = fill_attend(a, w, c, heads, r->window > 0);
  if (st != CA_OK) return st;
  const int64_t need = c->tokens > 0 ? w.bytes() : 0, rows = (int64_t)c->tokens * heads, pages = page_bytes(c);
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) {
    set_error("the call needs a 16-byte aligned workspace of %lld bytes; got %lld", (long long)need, (long long)(workspace ? workspace_bytes : 0));
    return CA_ERR_INVALID_ARG;
  }
  st = check_apart(c, {{out, rows * c->head_dim * elem_size(c->dtype)}, {lse, rows * 4}, {workspace, need}},
                   {{q, q_bytes}, {c->k, pages}, {c->v, pages}, {r->slopes, (int64_t)heads * 4}, {r->tree, (int64_t)c->tokens * 8}});
  if (st != CA_OK || c->tokens == 0) return st;
  a.splits = static_cast<ca::CacheSplit*>(workspace);
  a.pieces = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + w.splits);
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.scale = r->scale > 0.f ? r->scale : 1.f / std::sqrt((float)c->head_dim);
  a.cap = r->cap;
  a.slopes = r->slopes;
  a.causal = r->causal;
  a.window = r->window;
  a.tree = r->tree;
  const auto launch = c->dtype == CA_F32 ? ca::launch_attend_f32 : a.many ? ca::launch_attend_many : ca::launch_attend_few;
  const hipError_t e = launch(a, (hipStream_t)stream);
  return e == hipSuccess ? CA_OK : hip_fail(e, "cache attention launch");
}

int compact_attn_cache_keep(const ca_cache* c, const int32_t* kept, int32_t width, const int32_t* counts, void* stream) {
  ca::clear_error();
  int st = check_cache(c);
  if (st != CA_OK) return st;
  if (width < 0 || width > ca::kMostDrafts) return fail(CA_ERR_INVALID_ARG, "width must be 0 to 64");
  if (!counts || (width > 0 && !kept)) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (!aligned4(kept) || !aligned4(counts)) return fail(CA_ERR_INVALID_ARG, "kept and counts must be 4-byte aligned");
  const int64_t pages = page_bytes(c);
  st = check_apart(c, {{c->k, pages}, {c->v, pages}}, {{kept, (int64_t)c->sequences * width * 4}, {counts, (int64_t)c->sequences * 4}});
  if (st != CA_OK || c->tokens == 0 || width == 0) return st;
  ca::KeepArgs a{};
  fill_cache(a, c);
  a.kept = kept;
  a.counts = counts;
  a.width = width;
  a.row_bytes = c->head_dim * elem_size(c->dtype);
  const hipError_t e = ca::launch_keep(a, (hipStream_t)stream);
  return e == hipSuccess ? CA_OK : hip_fail(e, "cache keep launch");
}

}  // extern "C"
