// C-ABI entry points of rotary positions and of norms with the rotation: tables, argument checks, launches (rotary.hip).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "api_common.h"
#include "rotary.h"

using ca::aligned16;
using ca::elem_size;
using ca::fail;
using ca::hip_fail;
using ca::ranges_overlap;
using ca::set_error;

namespace {

constexpr int64_t kMaxAngles = (int64_t)1 << 28;

int check_axes(const ca_rotary_axis* axes, int32_t pairing, int32_t method, double magnitude) {
  if (pairing != CA_PAIRS_INTERLEAVED && pairing != CA_PAIRS_HALF) return fail(CA_ERR_INVALID_ARG, "pairing must be a ca_pairing value");
  if (method < CA_STRETCH_LINEAR || method > CA_STRETCH_BANDS) return fail(CA_ERR_INVALID_ARG, "method must be a ca_stretch value");
  if (!std::isfinite(magnitude)) return fail(CA_ERR_INVALID_ARG, "magnitude is not finite");
  int64_t channels = 0, angles = 0;
  for (int i = 0; i < 3; ++i) {
    const ca_rotary_axis& x = axes[i];
    if (x.channels < 0 || x.channels % 2 != 0) return fail(CA_ERR_INVALID_ARG, "channels of an axis must be even and not negative");
    if (x.channels == 0) continue;
    if (x.positions < 1) return fail(CA_ERR_INVALID_ARG, "an axis with channels needs at least one position");
    if (!(x.base > 0) || !std::isfinite(x.base) || !(x.stretch > 0) || !std::isfinite(x.stretch))
      return fail(CA_ERR_INVALID_ARG, "base and stretch must be positive");
    if (method == CA_STRETCH_BANDS &&
        (!(x.trained > 0) || !std::isfinite(x.trained) || !(x.turns_low < x.turns_high) || !std::isfinite(x.turns_low) || !std::isfinite(x.turns_high)))
      return fail(CA_ERR_INVALID_ARG, "bands need trained > 0 and turns_low < turns_high");
    channels += x.channels;
    angles += (int64_t)x.positions * (x.channels / 2);
  }
  if (channels == 0) return fail(CA_ERR_INVALID_ARG, "no axis has channels");
  if (channels > 65536 || angles > kMaxAngles) return fail(CA_ERR_INVALID_ARG, "more than 65536 channels or 2^28 angles");
  return CA_OK;
}

double frequency(const ca_rotary_axis& x, int32_t method, int pair) {
  const double c = x.channels;
  double base = x.base;
  if (method == CA_STRETCH_BASE && x.channels > 2) base *= std::pow(x.stretch, c / (c - 2));
  const double f = std::pow(base, -2.0 * pair / c);
  if (method == CA_STRETCH_LINEAR) return f / x.stretch;
  if (method == CA_STRETCH_BASE) return f;
  const double turns = x.trained * f / (2 * 3.14159265358979323846);
  const double keep = std::min(1.0, std::max(0.0, (turns - x.turns_low) / (x.turns_high - x.turns_low)));
  return keep * f + (1 - keep) * f / x.stretch;
}

// Puts the table on the current device at its first use, as ensure_uploaded does with a layout's tables.
int ensure_rotary_uploaded(ca_rotary* r, hipStream_t stream) {
  std::lock_guard<std::mutex> lock(r->upload_mutex);
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (r->dev) {
    if (dev == r->device) return CA_OK;
    set_error("the rotary table lives on device %d but the current device is %d", r->device, dev);
    return CA_ERR_INVALID_ARG;
  }
  if (stream) {
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    e = hipStreamIsCapturing(stream, &cap);
    if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
    if (cap != hipStreamCaptureStatusNone)
      return fail(CA_ERR_INVALID_ARG, "the rotary table is not on the device yet and the stream is being captured: call compact_attn_rotary_upload before the capture");
  }
  void* p = nullptr;
  const size_t bytes = r->angles.size() * sizeof(float);
  e = hipMalloc(&p, bytes);
  if (e != hipSuccess) {
    set_error("hipMalloc of %zu bytes for the rotary table failed: %s", bytes, hipGetErrorString(e));
    (void)hipGetLastError();
    return CA_ERR_ALLOC;
  }
  e = hipMemcpy(p, r->angles.data(), bytes, hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    (void)hipFree(p);
    return hip_fail(e, "hipMemcpy of the rotary table");
  }
  r->dev = static_cast<float*>(p);
  r->device = dev;
  return CA_OK;
}

// Strides of a tensor; those of a contiguous one of `tokens` tokens where s is null.
ca::RowStrides strides_of(const ca_layout* L, const ca_strides* s, int64_t tokens) {
  if (s) return {s->batch, s->head, s->token};
  const int64_t D = L->prob.head_dim;
  return {L->prob.num_heads * tokens * D, tokens * D, D};
}

// Bytes from the first to the end of the last element.
int64_t extent(const ca_layout* L, const ca::RowStrides& s, int64_t tokens) {
  const ca_problem& p = L->prob;
  return ((p.batch - 1) * s.batch + (p.num_heads - 1) * s.head + (tokens - 1) * s.token + p.head_dim) * elem_size(p.dtype);
}

int check_strides(const ca_layout* L, const ca_strides* s, const char* name) {
  if (!s) return CA_OK;
  const ca_problem& p = L->prob;
  const int64_t unit = 16 / elem_size(p.dtype);
  const std::pair<int64_t, int64_t> steps[] = {{s->batch, p.batch}, {s->head, p.num_heads}, {s->token, L->N_real}};
  for (const auto& [stride, count] : steps)
    if (stride < 0 || stride > ((int64_t)1 << 40) / std::max<int64_t>(1, count - 1) || stride % unit != 0) {
      set_error("strides of %s must be multiples of 16 bytes, not negative, and lead over fewer than 2^40 elements", name);
      return CA_ERR_INVALID_ARG;
    }
  return CA_OK;
}

// Rows of a tensor that is written: sorted by stride, each step over all that the smaller ones span.
int check_apart(const ca_layout* L, const ca_strides* s, const char* name) {
  if (!s) return CA_OK;
  const ca_problem& p = L->prob;
  std::pair<int64_t, int64_t> steps[3] = {{s->batch, p.batch}, {s->head, p.num_heads}, {s->token, L->N_real}};
  std::sort(steps, steps + 3);
  int64_t span = p.head_dim;
  for (const auto& [stride, count] : steps) {
    if (count <= 1) continue;
    if (stride < span) {
      set_error("rows of %s share memory", name);
      return CA_ERR_INVALID_ARG;
    }
    span += stride * (count - 1);
  }
  return CA_OK;
}

// Do rows of two natural-order tensors that are written share memory?  Both are sums of steps, so the distance of a row of b from one of a is
// b - a + sum of m * stride over the terms, and a term's m lies in a known range (steps that both have are one term: their difference).  Each term narrows down
// what the later, shorter ones can still bring to less than a row; where one tensor's rows are nested as the other's, that leaves a few m a term, whatever their number.
struct Term {
  int64_t stride, least, most;  // of m
};
bool reaches_row(const Term* term, const Term* end, int64_t distance, int64_t row) {
  if (term == end) return distance > -row && distance < row;
  int64_t below = 0, above = 0;  // what the terms after this one add
  for (const Term* t = term + 1; t != end; ++t) below += t->least * t->stride, above += t->most * t->stride;
  // -row < distance + m stride + above  and  distance + m stride + below < row
  auto floor_div = [](int64_t x, int64_t by) { return x / by - (x % by < 0); };
  const int64_t first = std::max(term->least, floor_div(-row - distance - above, term->stride) + 1);
  const int64_t last = std::min(term->most, floor_div(row - distance - below - 1, term->stride));
  for (int64_t m = first; m <= last; ++m)
    if (reaches_row(term + 1, end, distance + m * term->stride, row)) return true;
  return false;
}
bool rows_share_memory(const ca_layout* L, const void* a, const ca::RowStrides& sa, const void* b, const ca::RowStrides& sb) {
  const ca_problem& p = L->prob;
  if (!ranges_overlap(a, extent(L, sa, L->N_real), b, extent(L, sb, L->N_real))) return false;
  const struct {
    int64_t a, b, count;
  } steps[] = {{sa.batch, sb.batch, p.batch}, {sa.head, sb.head, p.num_heads}, {sa.token, sb.token, L->N_real}};
  Term terms[6];
  int n = 0;
  for (const auto& s : steps) {
    if (s.count <= 1) continue;
    if (s.a == s.b) {
      terms[n++] = {s.a, 1 - s.count, s.count - 1};
    } else {
      terms[n++] = {s.a, 1 - s.count, 0};
      terms[n++] = {s.b, 0, s.count - 1};
    }
  }
  std::sort(terms, terms + n, [](const Term& x, const Term& y) { return x.stride > y.stride; });
  const int64_t bytes = static_cast<const char*>(b) - static_cast<const char*>(a);  // (both are 16-byte aligned)
  return reaches_row(terms, terms + n, bytes / elem_size(p.dtype), p.head_dim);
}

int check_rows_support(const ca_layout* L) {
  const ca_problem& p = L->prob;
  const int most = p.dtype == CA_BF16 ? 512 : 256;
  if (p.head_dim > most || p.batch > 65535 || p.num_heads > 65535) {
    set_error("rotation and norms take head_dim up to %d in this type, and 65535 heads and batch entries; got D=%d, %d heads, batch %d", most, p.head_dim,
              p.num_heads, p.batch);
    return CA_ERR_UNSUPPORTED;
  }
  return CA_OK;
}

// Geometry, rotation and positions of a launch, with their checks; uploads the table.
int fill_rows(ca::RowArgs& a, const ca_layout* L, ca_rotary* r, const ca_where* where, int32_t tiled, hipStream_t stream) {
  const ca_problem& p = L->prob;
  if (tiled != 0 && tiled != 1) return fail(CA_ERR_INVALID_ARG, "tiled must be 0 or 1");
  a.batch = p.batch;
  a.heads = p.num_heads;
  a.D = p.head_dim;
  fill_grid(a, L);
  a.tiled = tiled;
  a.sign = 1.f;
  if (!r) return CA_OK;
  if (r->channels > p.head_dim) return fail(CA_ERR_INVALID_ARG, "more rotated channels than the head has");
  const int32_t grid[3] = {p.T, p.H, p.W};
  if (where && where->positions) {
    if ((reinterpret_cast<uintptr_t>(where->positions) & 3u) != 0) return fail(CA_ERR_INVALID_ARG, "positions must be 4-byte aligned");
  } else {
    for (int i = 0; i < 3; ++i) {
      const int32_t origin = where ? where->origin[i] : 0;
      if (r->axes[i].channels == 0) continue;
      if (origin < 0 || (int64_t)origin + grid[i] > r->axes[i].positions) {
        set_error("axis %d: positions %d to %lld lie outside of the table's %d", i, origin, (long long)origin + grid[i] - 1, r->axes[i].positions);
        return CA_ERR_INVALID_ARG;
      }
    }
  }
  const int st = ca::fill_rotation(a, r, stream);
  if (st != CA_OK) return st;
  a.where = where ? where->positions : nullptr;
  for (int i = 0; i < 3; ++i) a.origin[i] = where && r->axes[i].channels ? where->origin[i] : 0;
  return CA_OK;
}

// Checks shared by the norm calls; fills everything but the results.
int check_norm(const ca_norm* m, const ca_layout* L) {
  if (!m || !L || !m->q || !m->k) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (!aligned16(m->q) || !aligned16(m->k) || !aligned16(m->q_weight) || !aligned16(m->k_weight))
    return fail(CA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  if (!(m->eps >= 0.f) || std::isinf(m->eps)) return fail(CA_ERR_INVALID_ARG, "eps must be finite and not negative");
  int st = check_rows_support(L);
  if (st == CA_OK) st = check_strides(L, m->q_strides, "q");
  if (st == CA_OK) st = check_strides(L, m->k_strides, "k");
  return st;
}

// What is read besides the tensors: weights and positions.  (Positions are not, without a rotation.)
bool overlaps_small_inputs(const ca_layout* L, const void* at, int64_t bytes, const ca_norm* m, const ca_rotary* rotary, const ca_where* where) {
  const ca_problem& p = L->prob;
  const int64_t weight_bytes = (int64_t)p.head_dim * elem_size(p.dtype);
  if (m && ((m->q_weight && ranges_overlap(at, bytes, m->q_weight, weight_bytes)) || (m->k_weight && ranges_overlap(at, bytes, m->k_weight, weight_bytes)))) return true;
  return rotary && where && where->positions && ranges_overlap(at, bytes, where->positions, (int64_t)p.batch * L->N_real * 3 * (int64_t)sizeof(int32_t));
}

int64_t plane_elements(const ca_layout* L) { return (int64_t)L->prob.batch * L->prob.num_heads * L->prob.head_dim; }

}  // namespace

int ca::fill_rotation(RowRule& a, ca_rotary* r, hipStream_t stream) {
  const int st = ensure_rotary_uploaded(r, stream);
  if (st != CA_OK) return st;
  a.angles = r->dev;
  a.half = r->pairing == CA_PAIRS_HALF;
  a.rotated = r->channels;
  for (int i = 0; i < 3; ++i) {
    a.first[i] = r->first[i];
    a.pairs[i] = r->axes[i].channels / 2;
    a.positions[i] = r->axes[i].positions;
  }
  return CA_OK;
}

extern "C" {

int compact_attn_build_rotary(const ca_rotary_axis* axes, int32_t pairing, int32_t method, double magnitude, ca_rotary** out) {
  ca::clear_error();
  if (out) *out = nullptr;
  if (!axes || !out) return fail(CA_ERR_INVALID_ARG, "null argument");
  const int st = check_axes(axes, pairing, method, magnitude);
  if (st != CA_OK) return st;
  ca_rotary* r = new (std::nothrow) ca_rotary();
  if (!r) return fail(CA_ERR_ALLOC, "out of host memory");
  try {
    r->pairing = pairing;
    for (int i = 0; i < 3; ++i) {
      r->axes[i] = axes[i];
      if (axes[i].channels == 0) r->axes[i].positions = 0;
      const ca_rotary_axis& x = r->axes[i];
      const int pairs = x.channels / 2;
      r->first[i] = (int64_t)r->angles.size() / 2;
      r->channels += x.channels;
      r->angles.resize(r->angles.size() + (size_t)x.positions * pairs * 2);
      for (int k = 0; k < pairs; ++k) {
        const double f = frequency(x, method, k);
        float* at = r->angles.data() + 2 * (r->first[i] + k);
        for (int64_t p = 0; p < x.positions; ++p, at += 2 * pairs) {
          at[0] = (float)(magnitude * std::cos(p * f));
          at[1] = (float)(magnitude * std::sin(p * f));
        }
      }
    }
  } catch (const std::bad_alloc&) {
    delete r;
    return fail(CA_ERR_ALLOC, "out of host memory for the rotary table");
  }
  *out = r;
  return CA_OK;
}

int compact_attn_rotary_angles(const ca_rotary* r, int32_t axis, const float** cos_sin) {
  ca::clear_error();
  if (!r || !cos_sin) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (axis < 0 || axis > 2) return fail(CA_ERR_INVALID_ARG, "axis must be 0, 1 or 2");
  *cos_sin = r->axes[axis].channels ? r->angles.data() + 2 * r->first[axis] : nullptr;
  return CA_OK;
}

int compact_attn_rotary_upload(ca_rotary* r) {
  ca::clear_error();
  if (!r) return fail(CA_ERR_INVALID_ARG, "null table");
  return ensure_rotary_uploaded(r, nullptr);
}

void compact_attn_free_rotary(ca_rotary* r) {
  if (!r) return;
  if (r->dev) (void)hipFree(r->dev);
  delete r;
}

int compact_attn_rotate(const void* src, const ca_strides* src_strides, void* dst, const ca_strides* dst_strides, const ca_layout* L, ca_rotary* rotary,
                        const ca_where* where, int32_t tiled, int32_t transpose, void* stream) {
  ca::clear_error();
  if (!src || !dst || !L || !rotary) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (!aligned16(src) || !aligned16(dst)) return fail(CA_ERR_INVALID_ARG, "src and dst must be 16-byte aligned");
  if (transpose != 0 && transpose != 1) return fail(CA_ERR_INVALID_ARG, "transpose must be 0 or 1");
  if (tiled == 1 && (transpose ? src_strides : dst_strides)) return fail(CA_ERR_INVALID_ARG, "a tensor in tile order is contiguous: its strides must be NULL");
  int st = check_rows_support(L);
  if (st == CA_OK) st = check_strides(L, src_strides, "src");
  if (st == CA_OK) st = check_strides(L, dst_strides, "dst");
  if (st == CA_OK) st = check_apart(L, dst_strides, "dst");
  if (st != CA_OK) return st;
  const int64_t src_tokens = tiled && transpose ? L->N_pad : L->N_real, dst_tokens = tiled && !transpose ? L->N_pad : L->N_real;
  ca::RowArgs a{};
  a.src_strides = strides_of(L, src_strides, src_tokens);
  a.dst_strides = strides_of(L, dst_strides, dst_tokens);
  if (ranges_overlap(src, extent(L, a.src_strides, src_tokens), dst, extent(L, a.dst_strides, dst_tokens)))
    return fail(CA_ERR_INVALID_ARG, "src and dst must not overlap");
  if (overlaps_small_inputs(L, dst, extent(L, a.dst_strides, dst_tokens), nullptr, rotary, where)) return fail(CA_ERR_INVALID_ARG, "dst must not overlap the positions");
  st = fill_rows(a, L, rotary, where, tiled, (hipStream_t)stream);
  if (st != CA_OK) return st;
  a.src[0] = src;
  a.dst[0] = dst;
  a.tensors = 1;
  a.sign = transpose ? -1.f : 1.f;
  const hipError_t e = ca::launch_rotate(a, L->prob.dtype == CA_BF16, transpose != 0, (hipStream_t)stream);
  return e == hipSuccess ? CA_OK : hip_fail(e, "rotation launch");
}

int compact_attn_norm_rotate(const ca_norm* m, void* q_out, void* k_out, const ca_layout* L, void* stream) {
  ca::clear_error();
  if (!q_out || !k_out) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (!aligned16(q_out) || !aligned16(k_out)) return fail(CA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  int st = check_norm(m, L);
  if (st != CA_OK) return st;
  const int64_t tokens = m->tiled ? L->N_pad : L->N_real, out_bytes = plane_elements(L) * tokens * elem_size(L->prob.dtype);
  ca::RowArgs a{};
  a.src_strides = strides_of(L, m->q_strides, L->N_real);
  a.src_strides1 = strides_of(L, m->k_strides, L->N_real);
  a.dst_strides = a.dst_strides1 = strides_of(L, nullptr, tokens);
  const int64_t q_bytes = extent(L, a.src_strides, L->N_real), k_bytes = extent(L, a.src_strides1, L->N_real);
  for (const void* out : {q_out, k_out})
    if (ranges_overlap(out, out_bytes, m->q, q_bytes) || ranges_overlap(out, out_bytes, m->k, k_bytes) || overlaps_small_inputs(L, out, out_bytes, m, m->rotary, m->where))
      return fail(CA_ERR_INVALID_ARG, "results must not overlap the inputs");
  if (ranges_overlap(q_out, out_bytes, k_out, out_bytes)) return fail(CA_ERR_INVALID_ARG, "results must not overlap each other");
  st = fill_rows(a, L, m->rotary, m->where, m->tiled, (hipStream_t)stream);
  if (st != CA_OK) return st;
  a.src[0] = m->q; a.src[1] = m->k;
  a.dst[0] = q_out; a.dst[1] = k_out;
  a.weight[0] = m->q_weight; a.weight[1] = m->k_weight;
  a.eps = m->eps;
  a.tensors = 2;
  const hipError_t e = ca::launch_norm_rotate(a, L->prob.dtype == CA_BF16, (hipStream_t)stream);
  return e == hipSuccess ? CA_OK : hip_fail(e, "norm launch");
}

int compact_attn_norm_workspace(const ca_layout* L, int64_t* workspace_bytes) {
  ca::clear_error();
  if (!L || !workspace_bytes) return fail(CA_ERR_INVALID_ARG, "null argument");
  const int st = check_rows_support(L);
  if (st != CA_OK) return st;
  *workspace_bytes = (int64_t)ca::kMaxGradientBlocks * 2 * L->prob.head_dim * (int64_t)sizeof(float);
  return CA_OK;
}

int compact_attn_norm_rotate_backward(const ca_norm* m, const void* dq_out, const void* dk_out, void* dq, const ca_strides* dq_strides, void* dk,
                                      const ca_strides* dk_strides, float* dq_weight, float* dk_weight, const ca_layout* L, void* workspace,
                                      int64_t workspace_bytes, void* stream) {
  ca::clear_error();
  if (!dq_out || !dk_out || !dq || !dk) return fail(CA_ERR_INVALID_ARG, "null argument");
  if (!aligned16(dq_out) || !aligned16(dk_out) || !aligned16(dq) || !aligned16(dk)) return fail(CA_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  if (!dq_weight != !dk_weight) return fail(CA_ERR_INVALID_ARG, "both weight gradients or none");
  int st = check_norm(m, L);
  if (st == CA_OK) st = check_strides(L, dq_strides, "dq");
  if (st == CA_OK) st = check_strides(L, dk_strides, "dk");
  if (st == CA_OK) st = check_apart(L, dq_strides, "dq");
  if (st == CA_OK) st = check_apart(L, dk_strides, "dk");
  if (st != CA_OK) return st;
  int64_t need = 0;
  const int64_t weight_bytes = L->prob.head_dim * (int64_t)sizeof(float);
  if (dq_weight) {
    need = (int64_t)ca::kMaxGradientBlocks * 2 * weight_bytes;
    if (!workspace || !aligned16(workspace) || workspace_bytes < need) return fail(CA_ERR_INVALID_ARG, "weight gradients need a 16-byte aligned workspace of compact_attn_norm_workspace bytes");
    if ((reinterpret_cast<uintptr_t>(dq_weight) & 3u) != 0 || (reinterpret_cast<uintptr_t>(dk_weight) & 3u) != 0)
      return fail(CA_ERR_INVALID_ARG, "weight gradients must be 4-byte aligned");
  }
  const int64_t tokens = m->tiled ? L->N_pad : L->N_real, dy_bytes = plane_elements(L) * tokens * elem_size(L->prob.dtype);
  ca::RowArgs a{};
  a.src_strides = a.src_strides1 = strides_of(L, nullptr, tokens);
  a.x_strides = strides_of(L, m->q_strides, L->N_real);
  a.x_strides1 = strides_of(L, m->k_strides, L->N_real);
  a.dst_strides = strides_of(L, dq_strides, L->N_real);
  a.dst_strides1 = strides_of(L, dk_strides, L->N_real);
  struct Range {
    const void* at;
    int64_t bytes;
  };
  const Range inputs[] = {{dq_out, dy_bytes}, {dk_out, dy_bytes}, {m->q, extent(L, a.x_strides, L->N_real)}, {m->k, extent(L, a.x_strides1, L->N_real)}};
  const Range results[] = {{dq, extent(L, a.dst_strides, L->N_real)}, {dk, extent(L, a.dst_strides1, L->N_real)},
                           {dq_weight, need ? weight_bytes : 0}, {dk_weight, need ? weight_bytes : 0}, {need ? workspace : nullptr, need}};
  for (const Range& out : results) {
    if (!out.bytes) continue;
    bool apart = !overlaps_small_inputs(L, out.at, out.bytes, m, m->rotary, m->where);
    for (const Range& in : inputs) apart = apart && !ranges_overlap(out.at, out.bytes, in.at, in.bytes);
    if (!apart) return fail(CA_ERR_INVALID_ARG, "results and workspace must not overlap the inputs");
  }
  // dq and dk may be interleaved in one tensor (strides): their rows count, not what lies between them
  if (rows_share_memory(L, dq, a.dst_strides, dk, a.dst_strides1)) return fail(CA_ERR_INVALID_ARG, "rows of dq and dk share memory");
  for (int i = 0; i < 5; ++i)
    for (int j = std::max(2, i + 1); j < 5; ++j)
      if (results[i].bytes && results[j].bytes && ranges_overlap(results[i].at, results[i].bytes, results[j].at, results[j].bytes))
        return fail(CA_ERR_INVALID_ARG, "results and workspace must not overlap each other");
  st = fill_rows(a, L, m->rotary, m->where, m->tiled, (hipStream_t)stream);
  if (st != CA_OK) return st;
  a.src[0] = dq_out; a.src[1] = dk_out;
  a.x[0] = m->q; a.x[1] = m->k;
  a.dst[0] = dq; a.dst[1] = dk;
  a.weight[0] = m->q_weight; a.weight[1] = m->k_weight;
  a.eps = m->eps;
  a.tensors = 2;
  a.sign = -1.f;
  if (need) {
    a.partial = static_cast<float*>(workspace);
    a.dweight[0] = dq_weight;
    a.dweight[1] = dk_weight;
  }
  const hipError_t e = ca::launch_norm_rotate_backward(a, L->prob.dtype == CA_BF16, (hipStream_t)stream);
  return e == hipSuccess ? CA_OK : hip_fail(e, "norm gradient launch");
}

}  // extern "C"
