// Host-side exercise of the paged cache's entry points for a build with AddressSanitizer and UndefinedBehaviorSanitizer (host code only; no kernel is launched and no GPU
// is needed).  Random calls: what reaches a launch is compared with what was asked for, every part of a workspace is written from end to end, and launches stay within
// their limits.  Any sanitizer report aborts the run; a wrong result prints a message and exits with status 1.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "cache.h"
#include "compact_attn.h"
#include "layout.h"

extern "C" {
hipError_t hipGetDevice(int* device) {
  *device = 0;
  return hipSuccess;
}
const char* hipGetErrorString(hipError_t) { return ""; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* status) {
  *status = hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipMalloc(void** p, size_t bytes) {
  *p = std::malloc(bytes);
  return hipSuccess;
}
hipError_t hipFree(void* p) {
  std::free(p);
  return hipSuccess;
}
hipError_t hipMemcpy(void* dst, const void* src, size_t bytes, hipMemcpyKind) {
  std::memcpy(dst, src, bytes);
  return hipSuccess;
}
}

namespace {

int failures = 0;
#define CHECK(cond)                                                 \
  do {                                                              \
    if (!(cond)) {                                                  \
      std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); \
      ++failures;                                                   \
    }                                                               \
  } while (0)

std::vector<char> g_workspace;
const ca_cache* g_cache = nullptr;
int g_ways[3][2], g_appends = 0, g_keeps = 0;

void same_cache(const ca::CacheArgs& a) {
  const ca_cache& c = *g_cache;
  CHECK(a.k == c.k && a.v == c.v && a.num_pages == c.num_pages && a.page_tokens == c.page_tokens && a.kv_heads == c.kv_heads && a.sequences == c.sequences);
  CHECK(a.table == c.table && a.lengths == c.lengths && a.starts == c.starts && a.origins == c.origins && a.table_width == c.table_width && a.tokens == c.tokens);
  CHECK(a.frame_h == c.frame_height && a.frame_w == c.frame_width && a.span == c.frame_height * c.frame_width);
}

hipError_t attend(const ca::AttendArgs& a, bool many) {
  same_cache(a);
  const ca_cache& c = *g_cache;
  CHECK(a.many == many && a.group * a.kv_heads == a.heads && a.D == c.head_dim && a.scale > 0);
  const int64_t tile = many ? ca::kManyRows : ca::kFewRows, items = a.tiles * a.kv_heads;
  // however the rows are dealt out to the sequences, there is room for their tiles
  CHECK(a.tiles >= std::min<int64_t>(c.tokens, c.sequences) && a.tiles >= ((int64_t)c.tokens * a.group + tile - 1) / tile);
  ++g_ways[a.way][many];
  int64_t splits = 0, pieces = 0;
  if (a.way == ca::kShares) {
    CHECK(a.workgroups > 0 && a.workgroups % 8 == 0 && a.workgroups <= 512 && a.least_steps > 0);
    splits = a.workgroups, pieces = 2 * (int64_t)a.workgroups;
  } else {
    CHECK(items * (a.way == ca::kParts ? a.most_parts : 1) <= 0xffffff);
    CHECK(c.sequences <= 512);
    if (a.way == ca::kParts) {
      CHECK(many && a.most_parts > 1 && a.part_steps > 0);
      CHECK((int64_t)a.part_steps * a.most_parts * ca::kManyStep >= (int64_t)c.table_width * c.page_tokens);
      splits = items, pieces = items * a.most_parts;
    }
  }
  char* const first = reinterpret_cast<char*>(a.splits);
  char* const second = reinterpret_cast<char*>(a.pieces);
  if (splits) {
    const int64_t split_bytes = splits * (int64_t)sizeof(ca::CacheSplit), piece_bytes = pieces * tile * ca::piece_row(a.D) * 4;
    CHECK(first >= g_workspace.data() && first + split_bytes <= second && second + piece_bytes <= g_workspace.data() + g_workspace.size());
    CHECK(reinterpret_cast<uintptr_t>(second) % 16 == 0);
    std::memset(first, 0x5a, (size_t)split_bytes);
    std::memset(second, 0x5a, (size_t)piece_bytes);
  }
  return hipSuccess;
}

}  // namespace

namespace ca {
static char g_error[512];
void set_error(const char* format, ...) {
  va_list args;
  va_start(args, format);
  std::vsnprintf(g_error, sizeof(g_error), format, args);
  va_end(args);
}
void clear_error() { g_error[0] = 0; }
hipError_t launch_append(const AppendArgs& a, bool bf16, bool, hipStream_t) {
  same_cache(a);
  CHECK(bf16 == (g_cache->dtype == CA_BF16) && a.D == g_cache->head_dim && a.sign == 1.f);
  CHECK((a.heads > 0) == (a.q != nullptr) && (a.heads > 0) == (a.q_out != nullptr));
  ++g_appends;
  return hipSuccess;
}
hipError_t launch_keep(const KeepArgs& a, hipStream_t) {
  same_cache(a);
  CHECK(a.row_bytes == g_cache->head_dim * (g_cache->dtype == CA_BF16 ? 2 : 4) && a.width <= kMostDrafts && a.row_bytes <= 1024);
  ++g_keeps;
  return hipSuccess;
}
hipError_t launch_attend_few(const AttendArgs& a, hipStream_t) { return attend(a, false); }
hipError_t launch_attend_many(const AttendArgs& a, hipStream_t) { return attend(a, true); }
hipError_t launch_attend_f32(const AttendArgs& a, hipStream_t) {
  CHECK(g_cache->dtype == CA_F32 && a.way != kParts);
  return attend(a, false);
}
int fill_rotation(RowRule& a, ca_rotary* r, hipStream_t) {
  a.angles = reinterpret_cast<const float*>(r);
  return CA_OK;
}
}  // namespace ca

int main() {
  std::mt19937_64 rng(7);
  auto pick = [&](int64_t lo, int64_t hi) { return (int64_t)(lo + rng() % (uint64_t)(hi - lo + 1)); };
  auto any_of = [&](std::initializer_list<int64_t> values) { return values.begin()[rng() % values.size()]; };
  // addresses far apart, that nothing reads
  auto at = [](int i) { return reinterpret_cast<void*>((uintptr_t)(i + 1) << 48); };
  for (int turn = 0; turn < 4000; ++turn) {
    ca_cache c{};
    c.k = at(0), c.v = at(1);
    c.page_tokens = (int32_t)(16 * any_of({1, 2, 3, 4, 8, 16, 225, 4096}));
    c.kv_heads = (int32_t)any_of({1, 2, 3, 8, 40, 128});
    c.head_dim = (int32_t)any_of({64, 128, 128, 8, 256, 512});
    c.dtype = (int32_t)any_of({CA_BF16, CA_BF16, CA_BF16, CA_F32});
    c.num_pages = any_of({1, 7, 100000});
    c.sequences = (int32_t)any_of({1, 1, 2, 16, 500, 513, 3000, 1 << 20});
    c.table_width = (int32_t)std::max<int64_t>(1, std::min<int64_t>(any_of({1, 5, 100, 4000, 1 << 26}), ((int64_t)1 << 30) / c.page_tokens));
    c.tokens = (int32_t)any_of({0, 1, 16, 500, 3600, 75600, 2000000, (1 << 26) - 1, 0x7fffffff});
    c.frame_height = (int32_t)any_of({1, 1, 30, 32768}), c.frame_width = (int32_t)any_of({1, 1, 52, 32768});
    c.table = static_cast<int32_t*>(at(2)), c.lengths = static_cast<int32_t*>(at(3)), c.starts = static_cast<int32_t*>(at(4));
    c.origins = pick(0, 1) ? static_cast<int32_t*>(at(5)) : nullptr;
    g_cache = &c;
    const int32_t group = (int32_t)any_of({1, 1, 4, 5, 40}), heads = c.kv_heads * group;
    ca_reach r{};
    r.cap = (float)any_of({0, 0, 20});
    r.causal = (int32_t)pick(0, 1);
    r.window = (int32_t)any_of({0, 0, 4, 0x7fffffff});
    int64_t need = -1;
    const int st = compact_attn_cache_workspace(&c, heads, &need);
    CHECK(st == CA_OK || st == CA_ERR_UNSUPPORTED || st == CA_ERR_INVALID_ARG);
    if (st == CA_OK) {
      CHECK(need >= 0 && need <= ((int64_t)1 << 29));
      g_workspace.assign((size_t)need + 16, 0);
      char* const aligned = g_workspace.data() + (16 - reinterpret_cast<uintptr_t>(g_workspace.data()) % 16) % 16;
      const int call = compact_attn_cache_attend(at(6), nullptr, heads, &c, &r, at(7), static_cast<float*>(at(8)), need ? aligned : nullptr, need, nullptr);
      CHECK(call == CA_OK);
      if (need > 256 && c.tokens > 0 && r.window == 0) {
        const int small = compact_attn_cache_attend(at(6), nullptr, heads, &c, &r, at(7), static_cast<float*>(at(8)), aligned, 1, nullptr);
        CHECK(small == CA_OK || small == CA_ERR_INVALID_ARG);
      }
    }
    ca_append p{};
    const bool queries = pick(0, 1);
    p.k = at(6), p.v = at(9);
    if (queries) p.q = at(10), p.q_out = at(11), p.heads = heads;
    p.normed = (int32_t)pick(0, 1);
    p.eps = 1e-6f;
    const ca_strides strides{0, any_of({128, 64, 4, 512, -64}), any_of({4096, 8192, 12, (int64_t)1 << 41})};
    if (pick(0, 3) == 0) p.k_strides = &strides;
    const int appended = compact_attn_cache_append(&p, &c, nullptr);
    CHECK(appended == CA_OK || appended == CA_ERR_INVALID_ARG || appended == CA_ERR_UNSUPPORTED);
    const int kept = compact_attn_cache_keep(&c, static_cast<int32_t*>(at(12)), (int32_t)pick(0, 64), static_cast<int32_t*>(at(13)), nullptr);
    CHECK(kept == CA_OK || kept == CA_ERR_INVALID_ARG || kept == CA_ERR_UNSUPPORTED);
  }
  CHECK(g_ways[ca::kItems][0] > 0 && g_ways[ca::kItems][1] > 0 && g_ways[ca::kShares][0] > 0 && g_ways[ca::kShares][1] > 0 && g_ways[ca::kParts][1] > 0 && g_ways[ca::kParts][0] == 0);
  CHECK(g_appends > 0 && g_keeps > 0);
  if (failures) return 1;
  std::printf("cache host checks passed: items %d + %d, shares %d + %d, parts %d, %d appended, %d kept\n", g_ways[0][0], g_ways[0][1], g_ways[1][0], g_ways[1][1], g_ways[2][1], g_appends, g_keeps);
  return 0;
}
