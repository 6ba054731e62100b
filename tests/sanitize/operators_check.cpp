// Host-side exercise of rotation, norms and scored attention for a build with AddressSanitizer and UndefinedBehaviorSanitizer (host code only; no kernel is launched
// and no GPU is needed).  The lists that scored attention walks over are compared with the layout's tile lists, for rows and for columns, as the launches find them;
// every part of a workspace is written from end to end, and parts may not overlap; rotary tables are built and read, and calls made with strides of all kinds.  Any sanitizer
// report aborts the run; a wrong result prints a message and exits with status 1.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <vector>

#include "compact_attn.h"
#include "kernels.h"
#include "layout.h"
#include "rotary.h"
#include "scored.h"

// The few runtime calls, on host memory.
extern "C" {
hipError_t hipGetDevice(int* device) {
  *device = 0;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* value, hipDeviceAttribute_t, int) {
  *value = 256;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
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
hipError_t hipMemset(void* dst, int value, size_t bytes) {
  std::memset(dst, value, bytes);
  return hipSuccess;
}
}

namespace {

int failures = 0;
#define CHECK(cond)                                                        \
  do {                                                                     \
    if (!(cond)) {                                                         \
      std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond);        \
      ++failures;                                                          \
    }                                                                      \
  } while (0)

const ca_layout* g_layout = nullptr;  // of the call being made
std::vector<char> g_workspace;
std::vector<std::pair<const char*, const char*>> g_claimed;  // parts of it
int g_launches = 0, g_cut = 0;
volatile uint32_t g_ahead = 0;

void claim(void* at, int64_t bytes) {
  if (bytes == 0) return;
  char* const p = static_cast<char*>(at);
  CHECK(p >= g_workspace.data() && p + bytes <= g_workspace.data() + g_workspace.size());
  for (const auto& [from, to] : g_claimed) CHECK(p + bytes <= from || p >= to);
  g_claimed.push_back({p, p + bytes});
  std::memset(p, 0x5a, (size_t)bytes);  // (ends exactly where it may)
}

// Does half h of a tile hold a token?
bool half_has_token(const ca_layout* L, int64_t tile, int half) {
  if (tile >= L->n_vid) return true;
  const ca_problem& p = L->prob;
  const int64_t kt = tile / (L->nH * L->nW), kh = tile / L->nW % L->nH, kw = tile % L->nW;
  for (int slot = 64 * half; slot < std::min<int64_t>(64 * half + 64, L->B); ++slot)
    if (kt * p.tt + slot / (p.th * p.tw) < p.T && kh * p.th + slot / p.tw % p.th < p.H && kw * p.tw + slot % p.tw < p.W) return true;
  return false;
}

// The items of a launch that walks over the layout's rows or columns, against its tile lists.
void check_items(const ca::ScoredArgs& a, bool columns) {
  const ca_layout* L = g_layout;
  const int64_t n = L->n, tiles = ca::kGroupTokens / L->B, per_head = (n + tiles - 1) / tiles, heads = L->prob.num_heads;
  std::map<int32_t, std::vector<const ca::ScoredItem*>> of;
  for (int64_t i = 0; i < a.num_items; ++i) {
    of[a.items[i].group].push_back(&a.items[i]);
    if (i > 0) CHECK(a.items[i].count <= a.items[i - 1].count);  // longest first
  }
  CHECK((int64_t)of.size() == heads * per_head);
  std::map<int32_t, const ca::ScoredMerge*> merged;
  for (int64_t i = 0; i < a.num_merges; ++i) CHECK(merged.emplace(a.merges[i].group, &a.merges[i]).second);
  std::vector<char> taken((size_t)a.shares, 0);
  for (int64_t head = 0; head < heads; ++head) {
    std::vector<char> keep((size_t)(n * n), 0);
    for (int64_t row = 0; row < n; ++row)
      for (int64_t i = L->row_ptr[head * n + row]; i < L->row_ptr[head * n + row + 1]; ++i) keep[(size_t)(columns ? L->col_idx[i] * n + row : row * n + L->col_idx[i])] = 1;
    for (int64_t g = 0; g < per_head; ++g) {
      std::vector<uint32_t> want;
      for (int64_t t = 0; t < n; ++t) {
        uint32_t members = 0;
        for (int64_t k = 0; k < tiles; ++k)
          if (g * tiles + k < n && keep[(size_t)((g * tiles + k) * n + t)]) members |= 1u << k;
        for (int half = 0; members && half < L->B / 64; ++half)
          if (half_has_token(L, t, half)) want.push_back((uint32_t)t | (uint32_t)half << 24 | (uint32_t)L->tile_class[t] << 25 | members << 30);
      }
      auto& mine = of[(int32_t)(head * per_head + g)];
      std::sort(mine.begin(), mine.end(), [](const ca::ScoredItem* x, const ca::ScoredItem* y) { return x->first < y->first; });
      std::vector<uint32_t> got;
      for (const ca::ScoredItem* it : mine) {
        CHECK(it->first == mine[0]->first + (int64_t)got.size());
        got.insert(got.end(), a.steps + it->first, a.steps + it->first + it->count);
        g_ahead = a.steps[it->first + it->count] ^ a.steps[it->first + it->count + 1];  // the kernels fetch two words ahead
      }
      CHECK(got == want);
      const auto m = merged.find((int32_t)(head * per_head + g));
      CHECK((m != merged.end()) == (mine.size() > 1));
      if (mine.size() == 1) CHECK(mine[0]->share == -1);
      if (m == merged.end()) continue;
      ++g_cut;
      CHECK(m->second->shares == (int32_t)mine.size());
      for (size_t k = 0; k < mine.size(); ++k) {
        const int64_t share = m->second->first_share + (int64_t)k;
        CHECK(mine[k]->share == share && share >= 0 && share < a.shares && !taken[(size_t)share]);
        if (share >= 0 && share < a.shares) taken[(size_t)share] = 1;
      }
    }
  }
  for (char t : taken) CHECK(t);
}

hipError_t scored_launch(const ca::ScoredArgs& a, bool columns, int sums) {
  ++g_launches;
  const int64_t share_bytes = ca::share_floats(a.D, sums) * 4;
  if (!a.header) {
    check_items(a, columns);
    const auto before = g_claimed;
    if (a.shares) claim(a.share_sums, a.batch * a.shares * share_bytes);
    g_claimed = before;  // dQ and dK/dV use the same shares one after the other
  } else {
    CHECK(a.num_merges <= ca::most_merges(a.D) && a.shares == 0);
  }
  return hipSuccess;
}

}  // namespace

namespace ca {
hipError_t launch_permute(const PermuteArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_attn_f32(const AttnArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_attn_f32_planes(const PlaneArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_attn_bf16(const SplitArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_attn_bf16_ways(const SplitArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_attn_bf16_pair(const SplitArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_attn_bf16_merge(const SplitArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_tile_mass(const MassArgs&, hipStream_t) { return hipErrorInvalidValue; }

hipError_t launch_line(const ScoredArgs& a, hipStream_t) {
  claim(a.line, (int64_t)a.batch * a.n * kLineRows * a.B * 4);
  claim(a.tiles, (int64_t)a.batch * a.n * (int64_t)sizeof(TileLine));
  return hipSuccess;
}
hipError_t launch_visits(const ScoredArgs& a, const Visits* visits, int count, hipStream_t) {
  for (int i = 0; i < count; ++i) {
    const Visits& v = visits[i];
    CHECK(v.first[v.groups] == v.total && v.keys == i);
    claim(v.steps, (a.batch * v.total + 2) * 4);
    claim(v.counts, a.batch * v.groups * 4);
    claim(v.items, (a.batch * v.groups + most_shares(a.D)) * (int64_t)sizeof(ScoredItem));
    claim(v.merges, most_merges(a.D) * (int64_t)sizeof(ScoredMerge));
    claim(v.header, sizeof(VisitCounts));
    // the most shares that the device can make of these runs: it cuts into parts of at least kLeastSteps
    int64_t shares = 0;
    for (int64_t g = 0; g < v.groups; ++g) {
      const int64_t c = v.first[g + 1] - v.first[g];
      if (c > kLeastSteps) shares += a.batch * ((c + kLeastSteps - 1) / kLeastSteps);
    }
    const auto before = g_claimed;
    claim(a.share_sums, std::min(shares, most_shares(a.D)) * share_floats(a.D, a.rows ? 2 : 1) * 4);
    g_claimed = before;
  }
  return hipSuccess;
}
hipError_t launch_row_stats(const ScoredArgs& a, hipStream_t) {
  claim(a.rows, (int64_t)a.batch * a.num_heads * a.n * 2 * a.B * 4);
  return hipSuccess;
}
hipError_t launch_scored_forward(const ScoredArgs& a, hipStream_t) { return scored_launch(a, false, 1); }
hipError_t launch_scored_dq(const ScoredArgs& a, hipStream_t) { return scored_launch(a, false, 2); }
hipError_t launch_scored_dkv(const ScoredArgs& a, hipStream_t) { return scored_launch(a, true, 2); }

hipError_t launch_rotate(const RowArgs& a, bool, bool, hipStream_t) {
  ++g_launches;
  float sum = 0.f;  // the table's ends
  for (int i = 0; i < 3; ++i)
    if (a.pairs[i]) sum += a.angles[2 * a.first[i]] + a.angles[2 * (a.first[i] + (int64_t)a.positions[i] * a.pairs[i]) - 1];
  CHECK(std::isfinite(sum));
  return hipSuccess;
}
hipError_t launch_norm_rotate(const RowArgs& a, bool bf16, hipStream_t s) { return a.angles ? launch_rotate(a, bf16, false, s) : (++g_launches, hipSuccess); }
hipError_t launch_norm_rotate_backward(const RowArgs& a, bool bf16, hipStream_t s) {
  if (a.partial) claim(a.partial, (int64_t)kMaxGradientBlocks * 2 * a.D * 4);
  return launch_norm_rotate(a, bf16, s);
}
}  // namespace ca

namespace {

char* fake(int i) { return reinterpret_cast<char*>((uintptr_t)0x10000000000 * (i + 1)); }  // addresses that are never read

void scored_calls(std::mt19937& rng, ca_layout* L) {
  g_layout = L;
  const bool upload_first = rng() % 2;
  if (upload_first) CHECK(compact_attn_layout_upload_scored(L, (int)(rng() % 2)) == CA_OK);
  for (int kind = 0; kind < 5; ++kind) {
    ca_scores s{};
    if (kind == 1) s.cap = 20.f;
    if (kind >= 2) s.positions = reinterpret_cast<int32_t*>(fake(10));
    if (kind == 2 || kind == 4) s.slopes = reinterpret_cast<float*>(fake(11));
    if (kind >= 3) s.documents = reinterpret_cast<int32_t*>(fake(12));
    if (kind == 4) s.limits = reinterpret_cast<int32_t*>(fake(13));
    for (int backward = 0; backward < 2; ++backward) {
      int64_t need = -1;
      CHECK(compact_attn_scored_workspace(L, &s, backward, &need) == CA_OK && need >= 0);
      g_workspace.assign((size_t)need, 0);
      g_claimed.clear();
      void* const ws = need ? g_workspace.data() : nullptr;
      const int before = g_launches;
      float* const lse = reinterpret_cast<float*>(fake(5));
      if (need && !backward) CHECK(compact_attn_forward_scored(fake(0), fake(1), fake(2), L, &s, fake(3), lse, ws, need - 1, nullptr) == CA_ERR_INVALID_ARG);
      if (backward)
        CHECK(compact_attn_backward_scored(fake(4), fake(0), fake(1), fake(2), fake(3), lse, L, &s, fake(6), fake(7), fake(8), ws, need, nullptr) == CA_OK);
      else
        CHECK(compact_attn_forward_scored(fake(0), fake(1), fake(2), L, &s, fake(3), lse, ws, need, nullptr) == CA_OK);
      CHECK(g_launches >= before + (backward ? 2 : 1));
    }
  }
}

void random_scored(std::mt19937& rng, int rep) {
  const int tiles[6][3] = {{1, 8, 8}, {2, 8, 8}, {4, 4, 4}, {1, 8, 16}, {2, 4, 16}, {4, 4, 8}};
  const int* tile = tiles[rng() % 6];
  const int B = tile[0] * tile[1] * tile[2];
  ca_problem p{};
  p.T = 1 + (int)(rng() % 7), p.H = 1 + (int)(rng() % 30), p.W = 1 + (int)(rng() % 40);
  p.tt = tile[0], p.th = tile[1], p.tw = tile[2];
  p.n_text = B * (int)(rng() % 3);
  p.batch = 1 + (int)(rng() % 3), p.num_heads = 1 + (int)(rng() % 4), p.head_dim = rng() % 2 ? 64 : 128;
  p.dtype = CA_BF16;
  const int64_t n = (int64_t)((p.T + p.tt - 1) / p.tt) * ((p.H + p.th - 1) / p.th) * ((p.W + p.tw - 1) / p.tw) + p.n_text / B;
  const int share = rep % 5 == 0 ? 0 : rep % 5 == 1 ? 100 : (int)(rng() % 100);  // of the tiles, in per cent; rows without any among them
  std::vector<std::vector<int64_t>> ptr(p.num_heads);
  std::vector<std::vector<int32_t>> idx(p.num_heads);
  std::vector<const int64_t*> ptrs;
  std::vector<const int32_t*> idxs;
  for (int h = 0; h < p.num_heads; ++h) {
    ptr[h].push_back(0);
    for (int64_t r = 0; r < n; ++r) {
      if (share == 100 || rng() % 6)
        for (int64_t t = 0; t < n; ++t)
          if ((int)(rng() % 100) < share) idx[h].push_back((int32_t)t);
      ptr[h].push_back((int64_t)idx[h].size());
    }
    ptrs.push_back(ptr[h].data());
    idxs.push_back(idx[h].data());
  }
  ca_layout* L = nullptr;
  CHECK(compact_attn_layout_from_csr(&p, ptrs.data(), idxs.data(), &L) == CA_OK);
  if (!L) return;
  scored_calls(rng, L);
  compact_attn_free_layout(L);
}

// One head that keeps everything: long runs, which are cut into shares (288 runs on 768 places; at head dim 128 two parts each would be two rounds on 512, and
// four take more memory than shares may).
void long_scored(std::mt19937& rng, int tt, int head_dim) {
  ca_problem p{};
  p.T = 9, p.H = 61, p.W = 64, p.tt = tt, p.th = 8, p.tw = 8, p.batch = 1, p.num_heads = 1, p.head_dim = head_dim, p.dtype = CA_BF16;
  const ca_group group{8, {7, 7}, {-1, -1}};
  const ca_head head{1, 0, &group};
  ca_layout* L = nullptr;
  CHECK(compact_attn_build_layout(&p, &head, &L) == CA_OK);
  const int before = g_cut;
  scored_calls(rng, L);
  CHECK(g_cut > before || head_dim == 128);
  compact_attn_free_layout(L);
}

void rotary(std::mt19937& rng) {
  std::uniform_real_distribution<double> unit(0.1, 1.0);
  ca_problem p{};
  p.T = 1 + (int)(rng() % 5), p.H = 1 + (int)(rng() % 9), p.W = 1 + (int)(rng() % 9);
  p.tt = 1 + (int)(rng() % 3), p.th = 1 + (int)(rng() % 4), p.tw = 1 + (int)(rng() % 4);
  p.n_text = p.tt * p.th * p.tw * (int)(rng() % 2);
  p.batch = 1 + (int)(rng() % 2), p.num_heads = 1 + (int)(rng() % 3), p.dtype = rng() % 2 ? CA_BF16 : CA_F32;
  p.head_dim = 8 * (1 + (int)(rng() % 16));
  std::vector<ca_head> heads((size_t)p.num_heads, ca_head{0, 0, nullptr});
  ca_layout* L = nullptr;
  CHECK(compact_attn_build_layout(&p, heads.data(), &L) == CA_OK);
  g_layout = L;
  ca_rotary_axis axes[3];
  const int32_t grid[3] = {p.T, p.H, p.W};
  for (int i = 0; i < 3; ++i) axes[i] = {(int32_t)(2 * (rng() % 12)), grid[i] + (int32_t)(rng() % 3), 1e4 * unit(rng), 8 * unit(rng), 100 * unit(rng), 1.0, 4.0};
  const int32_t method = (int32_t)(rng() % 3);
  ca_rotary* table = nullptr;
  const int st = compact_attn_build_rotary(axes, (int32_t)(rng() % 2), method, 1.0, &table);
  CHECK((st == CA_OK) == (axes[0].channels + axes[1].channels + axes[2].channels > 0) && (st == CA_OK) == (table != nullptr));
  for (int i = 0; table && i < 3; ++i) {
    const float* at = nullptr;
    CHECK(compact_attn_rotary_angles(table, i, &at) == CA_OK && (at != nullptr) == (axes[i].channels > 0));
    for (int64_t k = 0; at && k < (int64_t)axes[i].positions * axes[i].channels / 2; ++k)
      CHECK(std::fabs((double)at[2 * k] * at[2 * k] + (double)at[2 * k + 1] * at[2 * k + 1] - 1) < 1e-6);
  }
  int64_t need = -1;
  CHECK(compact_attn_norm_workspace(L, &need) == CA_OK);
  g_workspace.assign((size_t)need, 0);
  auto strides = [&]() -> ca_strides {
    const int64_t D = p.head_dim, N = L->N_real, wild[] = {INT64_MIN, INT64_MAX, -8, 4, (int64_t)1 << 40, ((int64_t)1 << 40) + 8, 0};
    ca_strides s = rng() % 2 ? ca_strides{p.num_heads * N * D, D, p.num_heads * D} : ca_strides{3 * p.num_heads * N * D, D, 3 * p.num_heads * D};
    if (rng() % 3 == 0) (rng() % 3 == 0 ? s.batch : rng() % 2 ? s.head : s.token) = wild[rng() % 7];
    return s;
  };
  for (int rep = 0; rep < 40; ++rep) {
    const ca_strides s[4] = {strides(), strides(), strides(), strides()};
    auto maybe = [&](int i) { return rng() % 3 ? &s[i] : nullptr; };
    const ca_where where{{(int32_t)(rng() % 3) - (int32_t)(rng() % 2), rng() % 9 ? 0 : INT32_MAX, 0}, rng() % 2 ? reinterpret_cast<int32_t*>(fake(9)) : nullptr};
    const int32_t tiled = (int32_t)(rng() % 2), transpose = (int32_t)(rng() % 2);
    if (table) (void)compact_attn_rotate(fake(0), maybe(0), fake(1), maybe(1), L, table, rng() % 2 ? &where : nullptr, tiled, transpose, nullptr);
    const ca_norm norm{fake(0), fake(1), maybe(0), maybe(1), rng() % 2 ? fake(2) : nullptr, nullptr, rng() % 2 ? table : nullptr, rng() % 2 ? &where : nullptr, 1e-6f, tiled};
    (void)compact_attn_norm_rotate(&norm, fake(3), fake(4), L, nullptr);
    g_claimed.clear();
    const bool weights = rng() % 2;
    char* const dk = rng() % 2 ? fake(6) : fake(5) + 16 * (int64_t)(rng() % 4096) - 16 * (int64_t)(rng() % 4096);
    (void)compact_attn_norm_rotate_backward(&norm, fake(3), fake(4), fake(5), maybe(2), dk, maybe(3), weights ? reinterpret_cast<float*>(fake(7)) : nullptr,
                                            weights ? reinterpret_cast<float*>(fake(8)) : nullptr, L, weights ? g_workspace.data() : nullptr, weights ? need : 0, nullptr);
  }
  compact_attn_free_rotary(table);
  compact_attn_free_layout(L);
}

}  // namespace

int main() {
  std::mt19937 rng(11);
  for (int rep = 0; rep < 40; ++rep) random_scored(rng, rep);
  for (int head_dim : {64, 128})
    for (int tt : {1, 2}) long_scored(rng, tt, head_dim);
  const int before = g_launches;
  for (int rep = 0; rep < 60; ++rep) rotary(rng);
  CHECK(g_launches > before + 600);  // (a good part of the calls is made, the others are refused)
  std::printf("%d launches, %d runs in shares\n", g_launches, g_cut);
  if (failures) {
    std::printf("%d checks failed\n", failures);
    return 1;
  }
  std::printf("operator host checks passed\n");
  return 0;
}
