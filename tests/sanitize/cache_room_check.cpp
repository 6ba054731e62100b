// Host-side check of how much room a launch over the paged cache is given, for a build with AddressSanitizer and UndefinedBehaviorSanitizer (host code only; no kernel is launched and no GPU is
// needed).  Where new tokens lie is known on the device alone, so a launch has to have tiles for the worst way in which they can be dealt out to the sequences: that is found here by trying
// all of them (a table over sequences and rows).  A wrong result prints a message and exits with status 1.
#include <algorithm>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "cache.h"
#include "compact_attn.h"

extern "C" {
hipError_t hipGetDevice(int* device) {
  *device = 0;
  return hipSuccess;
}
const char* hipGetErrorString(hipError_t) { return ""; }
}

namespace {

int failures = 0, seen[3][2];

// Most tiles that `tokens` new tokens of `group` rows each can have in `sequences` sequences.
int64_t most_tiles(int tokens, int sequences, int group, int64_t tile) {
  std::vector<int64_t> best((size_t)tokens + 1, -1);
  best[0] = 0;
  for (int s = 0; s < sequences; ++s)
    for (int all = tokens; all >= 0; --all)
      for (int here = 1; here <= all; ++here)
        if (best[all - here] >= 0) best[all] = std::max(best[all], best[all - here] + ((int64_t)here * group + tile - 1) / tile);
  return *std::max_element(best.begin(), best.end());
}

hipError_t attend(const ca::AttendArgs& a, bool many) {
  const int64_t tile = many ? ca::kManyRows : ca::kFewRows, most = most_tiles(a.tokens, a.sequences, a.group, tile);
  if (a.tiles < most) {
    std::printf("FAILED: %d tokens in %d sequences, %d rows each, can have %lld tiles of %lld, room for %lld\n", a.tokens, a.sequences, a.group, (long long)most, (long long)tile, (long long)a.tiles);
    ++failures;
  }
  ++seen[a.way][many];
  return hipSuccess;
}

}  // namespace

namespace ca {
void set_error(const char*, ...) {}
void clear_error() {}
hipError_t launch_append(const AppendArgs&, bool, bool, hipStream_t) { return hipSuccess; }
hipError_t launch_keep(const KeepArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_attend_few(const AttendArgs& a, hipStream_t) { return attend(a, false); }
hipError_t launch_attend_many(const AttendArgs& a, hipStream_t) { return attend(a, true); }
hipError_t launch_attend_f32(const AttendArgs& a, hipStream_t) { return attend(a, false); }
int fill_rotation(RowRule&, ca_rotary*, hipStream_t) { return CA_OK; }
}  // namespace ca

int main() {
  std::mt19937_64 rng(11);
  auto pick = [&](int64_t lo, int64_t hi) { return (int64_t)(lo + rng() % (uint64_t)(hi - lo + 1)); };
  auto at = [](int i) { return reinterpret_cast<void*>((uintptr_t)(i + 1) << 48); };  // addresses far apart, that nothing reads
  if (most_tiles(64, 2, 1, 32) != 3 || most_tiles(5, 9, 1, 32) != 5 || most_tiles(33, 1, 4, 128) != 2) ++failures;  // 33 + 31 rows; a row each; 132 rows
  for (int turn = 0; turn < 3000; ++turn) {
    ca_cache c{};
    c.k = at(0), c.v = at(1);
    c.page_tokens = 64, c.kv_heads = (int32_t)pick(1, 8), c.head_dim = 64, c.dtype = pick(0, 3) ? CA_BF16 : CA_F32, c.num_pages = 1000;
    c.sequences = (int32_t)pick(1, 12), c.table_width = pick(0, 1) ? 10 : 500;
    c.tokens = (int32_t)(pick(0, 3) ? pick(1, 70) : pick(70, 300));
    c.frame_height = c.frame_width = 1;
    c.table = static_cast<int32_t*>(at(2)), c.lengths = static_cast<int32_t*>(at(3)), c.starts = static_cast<int32_t*>(at(4));
    const int32_t group = (int32_t)(pick(0, 1) ? pick(1, 8) : pick(1, 60)), heads = c.kv_heads * group;
    ca_reach r{};
    r.window = (int32_t)pick(0, 1);
    int64_t need = 0;
    if (compact_attn_cache_workspace(&c, heads, &need) != CA_OK ||
        compact_attn_cache_attend(at(5), nullptr, heads, &c, &r, at(6), static_cast<float*>(at(7)), need ? at(8) : nullptr, need, nullptr) != CA_OK)
      ++failures;
  }
  if (!(seen[ca::kItems][0] && seen[ca::kItems][1] && seen[ca::kShares][0] && seen[ca::kShares][1] && seen[ca::kParts][1])) ++failures;
  if (failures) return 1;
  std::printf("cache room checks passed\n");
  return 0;
}
