// Rows of channels, and what a lane does with its part of one: norms, the rotation and its pairings.  Shared by the kernels that walk over rows (rotary.hip, cache.hip).
#pragma once

#include <type_traits>

#include "rotary.h"

namespace ca {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float floatx4;

template <class T>
struct Row;
template <>
struct Row<__bf16> {
  static constexpr int kVec = 8;
  typedef bf16x8 Chunk;
};
template <>
struct Row<float> {
  static constexpr int kVec = 4;
  typedef floatx4 Chunk;
};

// A lane's part of a row: channels first .. first + kVec - 1 (live: there are such channels).
struct Part {
  int lanes_log2;  // lanes of a row
  int first;
  int row;         // of the wave's rows
  bool live;
};
template <class T>
__device__ __forceinline__ Part part_of(const RowRule& a, int lane) {
  Part p;
  const int chunks = a.D / Row<T>::kVec;
  p.lanes_log2 = chunks > 1 ? 32 - __builtin_clz((unsigned)(chunks - 1)) : 0;
  const int c = lane & ((1 << p.lanes_log2) - 1);
  p.live = c < chunks;
  p.first = (p.live ? c : 0) * Row<T>::kVec;
  p.row = lane >> p.lanes_log2;
  return p;
}

// Sum over the lanes of a row: within 16 lanes by lane exchanges on the vector ALU.
__device__ __forceinline__ float row_sum(float x, int lanes_log2) {
  auto dpp = [](float v, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  if (lanes_log2 > 0) x += dpp(x, std::integral_constant<int, 0xB1>());   // quad_perm 1 0 3 2
  if (lanes_log2 > 1) x += dpp(x, std::integral_constant<int, 0x4E>());   // quad_perm 2 3 0 1
  if (lanes_log2 > 2) x += dpp(x, std::integral_constant<int, 0x141>());  // the other quad of eight lanes
  if (lanes_log2 > 3) x += dpp(x, std::integral_constant<int, 0x140>());  // the other eight of sixteen
  if (lanes_log2 > 4) x += __shfl_xor(x, 16);
  if (lanes_log2 > 5) x += __shfl_xor(x, 32);
  return x;
}

// The rotation as the lane sees it: y[e] = c[e] x[e] + s[e] partner[e], where the partner of a channel is the other one of its pair.
template <int kVec>
struct Turn {
  float c[kVec], s[kVec];
};

// What the partner adds.  Nothing where its factor is zero, as it is for channels that nothing turns (in no pair, or of an axis without a position): zero times an
// infinity would be NaN there, and a zero that is added would lose the sign of another; minus zero does not.
__device__ __forceinline__ float from_partner(float factor, float partner) { return factor == 0.f ? -0.f : factor * partner; }

template <int kVec>
__device__ __forceinline__ void no_turn(Turn<kVec>& turn) {
#pragma unroll
  for (int e = 0; e < kVec; ++e) turn.c[e] = 1.f, turn.s[e] = 0.f;
}

// at0, at1, at2: the row's positions on the three axes.  What is chosen by axis is taken out of the arguments first: chosen within them, they are copied to private memory (rotation of 20K
// tokens, 80 channels 36 / 46 us without / with).  Angles asked for one by one as their positions are compared took 37 / 31 us (now) there, 16 tokens appended to a cache 17 / 11 us.
template <class T, bool kHalf>
__device__ __forceinline__ void make_turn(const RowRule& a, const Part& p, int at0, int at1, int at2, Turn<Row<T>::kVec>& turn) {
  constexpr int kVec = Row<T>::kVec;
  constexpr int kStep = kHalf ? 1 : 2;
  const int half = a.rotated / 2;
  const int pairs0 = a.pairs[0], pairs1 = a.pairs[1], pairs2 = a.pairs[2], limit0 = a.positions[0], limit1 = a.positions[1], limit2 = a.positions[2];
  const uint32_t first0 = (uint32_t)a.first[0], first1 = (uint32_t)a.first[1], first2 = (uint32_t)a.first[2];  // (tables have at most 2^28 angles)
  float2 angles[kVec];  // all are asked for before the first is looked at: where nothing turns, or past the table, one that is there
  int pos[kVec], limit[kVec];
#pragma unroll
  for (int e = 0; e < kVec; e += kStep) {
    const int ch = min(p.first + e, a.rotated - kStep);
    const int pair = kHalf ? (ch < half ? ch : ch - half) : ch >> 1;
    const int axis = pair < pairs0 ? 0 : pair < pairs0 + pairs1 ? 1 : 2;
    const int within = pair - (axis == 0 ? 0 : axis == 1 ? pairs0 : pairs0 + pairs1);
    const int pairs = axis == 0 ? pairs0 : axis == 1 ? pairs1 : pairs2;
    const uint32_t first = axis == 0 ? first0 : axis == 1 ? first1 : first2;
    pos[e] = axis == 0 ? at0 : axis == 1 ? at1 : at2;
    limit[e] = axis == 0 ? limit0 : axis == 1 ? limit1 : limit2;
    const uint32_t index = first + (uint32_t)max(min(pos[e], limit[e] - 1), 0) * (uint32_t)pairs + (uint32_t)within;
    angles[e] = reinterpret_cast<const float2*>(a.angles)[index];
  }
#pragma unroll
  for (int e = 0; e < kVec; e += kStep) {
    const int ch = p.first + e;
    const bool turns = ch < a.rotated && pos[e] >= 0, past = turns && pos[e] >= limit[e];
    const float c = past ? __builtin_nanf("") : turns ? angles[e].x : 1.f, s = past ? __builtin_nanf("") : turns ? angles[e].y * a.sign : 0.f;
    turn.c[e] = c;
    if constexpr (kHalf) {
      turn.s[e] = !turns ? 0.f : ch < half ? -s : s;
    } else {
      turn.c[e + 1] = c;
      turn.s[e] = turns ? -s : 0.f;
      turn.s[e + 1] = s;
    }
  }
}

// Pairings: neighbouring channels are in one lane.  Channels half the rotated ones apart are exchanged between the lanes of a row, word by word; where half of
// them is an odd number of bf16 channels (kApart) they straddle words and are read from memory a second time, one by one.
enum Pairing { kNeighbours, kHalves, kApart };

typedef __attribute__((ext_vector_type(4))) int intx4;

// Where the partners of a lane's four words are: in word (i + turn) % 4, or where that is odd and the partner lies below, (i - turn) % 4, of lane[i].
template <class T>
struct Exchange {
  int turn;           // wave-uniform
  int lane[4];        // byte address of the lane for ds_bpermute
  bool below[4], has[4];
  __device__ __forceinline__ Exchange(const RowRule& a, const Part& p, int wave_lane) {
    constexpr int kPerWord = 4 / sizeof(T);
    const int half = a.rotated / 2 / kPerWord;
    turn = half & 3;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int word = p.first / kPerWord + i;
      has[i] = a.angles && word < 2 * half;
      below[i] = word >= half;
      const int partner = has[i] ? (below[i] ? word - half : word + half) : word;
      lane[i] = (((wave_lane >> p.lanes_log2) << p.lanes_log2) + (partner >> 2)) * 4;
    }
  }
  __device__ __forceinline__ typename Row<T>::Chunk operator()(const typename Row<T>::Chunk& own) const {
    intx4 v = __builtin_bit_cast(intx4, own);
    if (turn & 1) v = __builtin_shufflevector(v, v, 1, 2, 3, 0);
    if (turn & 2) v = __builtin_shufflevector(v, v, 2, 3, 0, 1);
    intx4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      out[i] = __builtin_amdgcn_ds_bpermute(lane[i], v[i]);
      if (turn & 1) {  // (i - turn) % 4 = (i + turn + 2) % 4
        const int low = __builtin_amdgcn_ds_bpermute(lane[i], v[(i + 2) & 3]);
        out[i] = below[i] ? low : out[i];
      }
      out[i] = has[i] ? out[i] : 0;
    }
    return __builtin_bit_cast(typename Row<T>::Chunk, out);
  }
};

// The same from memory, zero where there is no partner.
template <class T>
__device__ __forceinline__ typename Row<T>::Chunk load_partner(const RowRule& a, const Part& p, const T* row) {
  constexpr int kVec = Row<T>::kVec;
  const int half = a.rotated / 2;
  typename Row<T>::Chunk v;
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    const int ch = p.first + e;
    v[e] = a.angles && ch < a.rotated ? row[ch < half ? ch + half : ch - half] : (T)0.f;
  }
  return v;
}

template <class T, Pairing kPairing>
__device__ __forceinline__ void load_weights(const RowRule& a, const Part& p, const void* weight, float (&w)[Row<T>::kVec], float (&wp)[Row<T>::kVec]) {
  constexpr int kVec = Row<T>::kVec;
#pragma unroll
  for (int e = 0; e < kVec; ++e) w[e] = wp[e] = 1.f;
  if (!weight) return;
  const T* row = static_cast<const T*>(weight);
  const auto own = *reinterpret_cast<const typename Row<T>::Chunk*>(row + p.first);
  typename Row<T>::Chunk other = own;
  if constexpr (kPairing != kNeighbours) other = load_partner<T>(a, p, row);
#pragma unroll
  for (int e = 0; e < kVec; ++e) w[e] = (float)own[e], wp[e] = kPairing == kNeighbours ? (float)own[e ^ 1] : (float)other[e];
}

int lanes_log2(const RowRule& a, bool bf16) {
  const int chunks = a.D / (bf16 ? 8 : 4);
  int log2 = 0;
  while ((1 << log2) < chunks) ++log2;
  return log2;
}

// launch(element type, pairing) of the kernel that takes a's rows
template <class Launch>
void with_pairing(const RowRule& a, bool bf16, Launch&& launch) {
  using std::integral_constant;
  if (!bf16) {
    if (a.half) launch(float(), integral_constant<Pairing, kHalves>());
    else launch(float(), integral_constant<Pairing, kNeighbours>());
  } else if (!a.half) {
    launch(__bf16(), integral_constant<Pairing, kNeighbours>());
  } else if (a.rotated / 2 % 2 == 0) {
    launch(__bf16(), integral_constant<Pairing, kHalves>());
  } else {
    launch(__bf16(), integral_constant<Pairing, kApart>());
  }
}

}  // namespace
}  // namespace ca
