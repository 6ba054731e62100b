// Rotary positions, and norms of queries and keys with the rotation in the same pass, forwards and backwards.
//
//   y = R (w n),  n = x r,  r = (mean(x^2) + eps)^-1/2;   R turns pairs of channels by position * frequency.
//   Backwards: u = R^T dy,  dx = r (w u - n mean(w u n)),  dw = sum of u n;  R^T is R with the sines negated.
//
// Bound: HBM, every row (token, head) is read once and written once.  A row is held by D / 8 lanes (bf16; D / 4 for fp32), 16 bytes each, so
// its sums are a few lane exchanges and its rounding is one.  A wave takes 64 / lanes tokens and walks over the heads and
// over q and k with them: the angles (gathered from the small per-axis tables, which stay in L2) and their products with the weights are made
// once per token and tensor, and several heads are loaded before the first is computed, so that enough bytes are in flight.  Tile order costs nothing
// here: a token's place in it is a few integer operations per token, and no pass of its own.
#include <algorithm>

#include "rotary.h"
#include "tokens.h"

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
__device__ __forceinline__ Part part_of(const RowArgs& a, int lane) {
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

template <class T, bool kHalf>
__device__ __forceinline__ void make_turn(const RowArgs& a, const Part& p, const Token& k, int64_t batch, Turn<Row<T>::kVec>& turn) {
  constexpr int kVec = Row<T>::kVec;
#pragma unroll
  for (int e = 0; e < kVec; ++e) turn.c[e] = 1.f, turn.s[e] = 0.f;
  if (!a.angles || k.natural < 0) return;
  int at[3] = {k.at[0], k.at[1], k.at[2]};
  if (a.where) {
    const int32_t* w = a.where + (batch * a.N_real + k.natural) * 3;
#pragma unroll
    for (int i = 0; i < 3; ++i) at[i] = w[i];
  } else if (at[0] >= 0) {
#pragma unroll
    for (int i = 0; i < 3; ++i) at[i] += a.origin[i];
  }
  const int half = a.rotated / 2;
#pragma unroll
  for (int e = 0; e < kVec; e += kHalf ? 1 : 2) {
    const int ch = p.first + e;
    if (ch >= a.rotated) continue;
    const int pair = kHalf ? (ch < half ? ch : ch - half) : ch >> 1;
    const int axis = pair < a.pairs[0] ? 0 : pair < a.pairs[0] + a.pairs[1] ? 1 : 2;
    const int within = pair - (axis == 0 ? 0 : axis == 1 ? a.pairs[0] : a.pairs[0] + a.pairs[1]);
    const int pos = axis == 0 ? at[0] : axis == 1 ? at[1] : at[2];
    const int pairs = axis == 0 ? a.pairs[0] : axis == 1 ? a.pairs[1] : a.pairs[2];
    const int limit = axis == 0 ? a.positions[0] : axis == 1 ? a.positions[1] : a.positions[2];
    const int64_t first = axis == 0 ? a.first[0] : axis == 1 ? a.first[1] : a.first[2];
    float c = 1.f, s = 0.f;
    if (pos >= limit) {
      c = s = __builtin_nanf("");
    } else if (pos >= 0) {
      const float2 cs = reinterpret_cast<const float2*>(a.angles)[first + (int64_t)pos * pairs + within];
      c = cs.x, s = cs.y * a.sign;
    }
    turn.c[e] = c;
    if constexpr (kHalf) {
      turn.s[e] = ch < half ? -s : s;
    } else {
      turn.c[e + 1] = c;
      turn.s[e] = -s;
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
  __device__ __forceinline__ Exchange(const RowArgs& a, const Part& p, int wave_lane) {
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
__device__ __forceinline__ typename Row<T>::Chunk load_partner(const RowArgs& a, const Part& p, const T* row) {
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
__device__ __forceinline__ void load_weights(const RowArgs& a, const Part& p, const void* weight, float (&w)[Row<T>::kVec], float (&wp)[Row<T>::kVec]) {
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

// Forward calls and the transposed rotation.  Rows are walked in the order of dst; heads are split over blockIdx.y where there are few tokens.
// kHeads: rows that are loaded before the first of them is computed (2 / 4 / 8: 20K tokens x 24 rows of 64 channels, forward and gradients 157 / 151 / 149 us; fp32, 7K
// tokens x 16 rows 30 / 28 / 30 us).  Results are stored past the caches, inputs loaded through them; inputs that lie in no cache, stores through / past / both past the caches:
// 33K tokens x 16 heads of 128 64.6 / 61.3 / 59.7 us, 2 x 20K x 12 of 80 42.1 / 36.9 / 44.0, fp32 7K x 16 of 128 33.7 / 27.7 / 34.8 (4.9, 4.6 and 4.7 TB/s as they are); q and k of 75.6K
// tokens x 40 heads, tokens first, 640 us = 5.0 TB/s (a plain copy of 1 GiB: 4.8 to 5.1 TB/s; permute_kernel on such a tensor 6.0 TB/s).  All of these are times of the operator alone: what
// attention, which reads the results next, has of them in the caches either way was not measured.
template <class T, Pairing kPairing, bool kNorm, bool kBack>
__global__ __launch_bounds__(kRowThreads) void rows_kernel(RowArgs a, int heads_per_block) {
  constexpr int kVec = Row<T>::kVec, kHeads = 4;
  typedef typename Row<T>::Chunk Chunk;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Part p = part_of<T>(a, lane);
  const int64_t count = !kBack && a.tiled ? a.N_pad : a.N_real, batch = blockIdx.z;
  const int64_t row = (((int64_t)blockIdx.x * kRowWaves + wave) << (6 - p.lanes_log2)) + p.row;
  const bool live = p.live && row < count;
  const uint32_t at = (uint32_t)(row < count ? row : count - 1);
  const Token k = !kBack && a.tiled ? token_of_place(a, at) : token_of_natural(a, at);
  const bool real = k.natural >= 0;
  const int h0 = blockIdx.y * heads_per_block, h1 = min(a.heads, h0 + heads_per_block);

  Turn<kVec> turn;
  make_turn<T, kPairing != kNeighbours>(a, p, k, batch, turn);
  const Exchange<T> exchange(a, p, lane);
  const int64_t src_row = kBack && a.tiled ? k.place : k.natural, dst_row = !kBack && a.tiled ? k.place : k.natural;

  for (int tensor = 0; tensor < a.tensors; ++tensor) {
    const RowStrides ss = tensor ? a.src_strides1 : a.src_strides, ds = tensor ? a.dst_strides1 : a.dst_strides;
    const T* __restrict__ src = static_cast<const T*>(tensor ? a.src[1] : a.src[0]) + batch * ss.batch + (real ? src_row : 0) * ss.token;
    T* __restrict__ dst = static_cast<T*>(tensor ? a.dst[1] : a.dst[0]) + batch * ds.batch + dst_row * ds.token + p.first;
    float own_c[kVec], other_c[kVec];  // y = own_c x + other_c partner (times r)
#pragma unroll
    for (int e = 0; e < kVec; ++e) own_c[e] = turn.c[e], other_c[e] = turn.s[e];
    if constexpr (kNorm) {
      float w[kVec], wp[kVec];
      load_weights<T, kPairing>(a, p, tensor ? a.weight[1] : a.weight[0], w, wp);
#pragma unroll
      for (int e = 0; e < kVec; ++e) own_c[e] *= w[e], other_c[e] = from_partner(other_c[e], wp[e]);
    }
    for (int h = h0; h < h1; h += kHeads) {
      Chunk own[kHeads], other[kHeads];
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        if (h + i < h1 && live && real) {
          const T* r = src + (h + i) * ss.head;
          own[i] = *reinterpret_cast<const Chunk*>(r + p.first);
          if constexpr (kPairing == kApart) other[i] = load_partner<T>(a, p, r);
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) own[i][e] = other[i][e] = (T)0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < kHeads; ++i) {
        if (h + i >= h1) break;
        if constexpr (kPairing == kHalves) other[i] = exchange(own[i]);
        float r = 1.f;
        if constexpr (kNorm) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < kVec; ++e) sum += live ? (float)own[i][e] * (float)own[i][e] : 0.f;
          r = rsqrtf(row_sum(sum, p.lanes_log2) / a.D + a.eps);
        }
        Chunk y;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float x = (float)own[i][e], xp = kPairing == kNeighbours ? (float)own[i][e ^ 1] : (float)other[i][e];
          y[e] = (T)(r * (own_c[e] * x + from_partner(other_c[e], xp)));
        }
        if (!real)
#pragma unroll
          for (int e = 0; e < kVec; ++e) y[e] = (T)0.f;  // (0 * r is NaN where eps is 0)
        if (live) __builtin_nontemporal_store(y, reinterpret_cast<Chunk*>(dst + (h + i) * ds.head));
      }
    }
  }
}

// Gradients of the norm.  Rows are walked in natural order; a workgroup takes blocks of tokens in turn and adds up its share of the weight
// gradients in registers, then over its waves in LDS, and leaves it in `partial`.
template <class T, Pairing kPairing>
__global__ __launch_bounds__(kRowThreads) void norm_backward_kernel(RowArgs a, int heads_per_block) {
  constexpr int kVec = Row<T>::kVec, kHeads = 2;
  typedef typename Row<T>::Chunk Chunk;
  __shared__ float sums[2][kRowThreads * Row<T>::kVec];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Part p = part_of<T>(a, lane);
  const int rows_log2 = 6 - p.lanes_log2;
  const int64_t blocks_per_batch = (a.N_real + (kRowWaves << rows_log2) - 1) / (kRowWaves << rows_log2), blocks = blocks_per_batch * a.batch;
  const int h0 = blockIdx.y * heads_per_block, h1 = min(a.heads, h0 + heads_per_block);
  const Exchange<T> exchange(a, p, lane);
  float dw[2][kVec];
#pragma unroll
  for (int e = 0; e < kVec; ++e) dw[0][e] = dw[1][e] = 0.f;

  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const int64_t batch = block / blocks_per_batch, row = ((((block - batch * blocks_per_batch) * kRowWaves) + wave) << rows_log2) + p.row;
    const bool live = p.live && row < a.N_real;
    const Token k = token_of_natural(a, (uint32_t)(row < a.N_real ? row : a.N_real - 1));
    Turn<kVec> turn;
    make_turn<T, kPairing != kNeighbours>(a, p, k, batch, turn);
    const int64_t src_row = a.tiled ? k.place : k.natural;
#pragma unroll
    for (int tensor = 0; tensor < 2; ++tensor) {
      const RowStrides ss = tensor ? a.src_strides1 : a.src_strides, ds = tensor ? a.dst_strides1 : a.dst_strides, xs = tensor ? a.x_strides1 : a.x_strides;
      const T* __restrict__ src = static_cast<const T*>(a.src[tensor]) + batch * ss.batch + src_row * ss.token;
      const T* __restrict__ xin = static_cast<const T*>(a.x[tensor]) + batch * xs.batch + k.natural * xs.token + p.first;
      T* __restrict__ dst = static_cast<T*>(a.dst[tensor]) + batch * ds.batch + k.natural * ds.token + p.first;
      float w[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) w[e] = 1.f;
      if (a.weight[tensor]) {
        const Chunk own = *reinterpret_cast<const Chunk*>(static_cast<const T*>(a.weight[tensor]) + p.first);
#pragma unroll
        for (int e = 0; e < kVec; ++e) w[e] = (float)own[e];
      }
      for (int h = h0; h < h1; h += kHeads) {
        Chunk own[kHeads], other[kHeads], x[kHeads];
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
          if (h + i < h1 && live) {
            const T* r = src + (h + i) * ss.head;
            own[i] = *reinterpret_cast<const Chunk*>(r + p.first);
            if constexpr (kPairing == kApart) other[i] = load_partner<T>(a, p, r);
            x[i] = *reinterpret_cast<const Chunk*>(xin + (h + i) * xs.head);
          } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) own[i][e] = other[i][e] = x[i][e] = (T)0.f;
          }
        }
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
          if (h + i >= h1) break;
          if constexpr (kPairing == kHalves) other[i] = exchange(own[i]);
          float u[kVec], squares = 0.f, dot = 0.f;
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const float xe = live ? (float)x[i][e] : 0.f, dyp = kPairing == kNeighbours ? (float)own[i][e ^ 1] : (float)other[i][e];
            u[e] = turn.c[e] * (float)own[i][e] + from_partner(turn.s[e], dyp);
            squares += xe * xe;
            dot += live ? w[e] * u[e] * xe : 0.f;
          }
          const float r = rsqrtf(row_sum(squares, p.lanes_log2) / a.D + a.eps);
          const float lean = row_sum(dot, p.lanes_log2) / a.D * r * r;  // mean(w u n) / r * r: n mean(w u n) = x r * lean / r
          Chunk dx;
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const float xe = (float)x[i][e];
            dx[e] = (T)(r * (w[e] * u[e] - xe * lean));
            dw[tensor][e] += live ? u[e] * xe * r : 0.f;
          }
          if (live) __builtin_nontemporal_store(dx, reinterpret_cast<Chunk*>(dst + (h + i) * ds.head));
        }
      }
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int tensor = 0; tensor < 2; ++tensor)
#pragma unroll
    for (int e = 0; e < kVec; ++e) sums[tensor][(threadIdx.x >> p.lanes_log2 << p.lanes_log2) * kVec + (threadIdx.x & ((1 << p.lanes_log2) - 1)) * kVec + e] = dw[tensor][e];
  __syncthreads();
  // rows of the workgroup lie (lanes of a row) * kVec apart
  const int stride = kVec << p.lanes_log2, rows = kRowThreads >> p.lanes_log2;
  float* out = a.partial + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.D;
  for (int c = threadIdx.x; c < 2 * a.D; c += kRowThreads) {
    const int tensor = c >= a.D, ch = c - tensor * a.D;
    float sum = 0.f;
    for (int r = 0; r < rows; ++r) sum += sums[tensor][r * stride + ch];
    out[c] = sum;
  }
}

// Adds up the workgroups' shares of the weight gradients: 16 channels a workgroup, 64 threads a channel, always in the same order.
__global__ __launch_bounds__(1024) void weight_gradient_kernel(const float* partial, int blocks, int D, float* dq, float* dk) {
  __shared__ float sums[64][17];
  const int channel = threadIdx.x & 15, part = threadIdx.x >> 4, c = blockIdx.x * 16 + channel;
  float sum = 0.f;
  if (c < 2 * D) {
#pragma unroll 8
    for (int b = part; b < blocks; b += 64) sum += partial[(int64_t)b * 2 * D + c];
  }
  sums[part][channel] = sum;
  __syncthreads();
  for (int half = 32; half > 0; half /= 2) {
    if (part < half) sums[part][channel] += sums[part + half][channel];
    __syncthreads();
  }
  if (part == 0 && c < 2 * D) (c < D ? dq[c] : dk[c - D]) = sums[0][channel];
}

int lanes_log2(const RowArgs& a, bool bf16) {
  const int chunks = a.D / (bf16 ? 8 : 4);
  int log2 = 0;
  while ((1 << log2) < chunks) ++log2;
  return log2;
}

// launch(element type, pairing) of the kernel that takes a's rows
template <class Launch>
void with_pairing(const RowArgs& a, bool bf16, Launch&& launch) {
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

// Heads are split over workgroups until there are enough of these to fill the card (2048: eight of four waves on each CU).
int head_blocks(int64_t workgroups, int heads) {
  int blocks = 1;
  while (blocks < heads && workgroups * blocks < 2048) blocks *= 2;
  return std::min(blocks, heads);
}

template <bool kNorm, bool kBack>
hipError_t launch_rows(const RowArgs& a, bool bf16, hipStream_t stream) {
  const int rows = kRowWaves << (6 - lanes_log2(a, bf16));
  const int64_t count = !kBack && a.tiled ? a.N_pad : a.N_real, blocks = (count + rows - 1) / rows;
  int per = (a.heads + head_blocks(blocks * a.batch, a.heads) - 1) / head_blocks(blocks * a.batch, a.heads);
  const dim3 grid((unsigned)blocks, (unsigned)((a.heads + per - 1) / per), (unsigned)a.batch);
  if (blocks > 0xffffff || grid.y > 65535 || grid.z > 65535) return hipErrorInvalidValue;  // (2^32 threads in x)
  with_pairing(a, bf16, [&](auto type, auto pairing) {
    rows_kernel<decltype(type), decltype(pairing)::value, kNorm, kBack><<<grid, kRowThreads, 0, stream>>>(a, per);
  });
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RowArgs& a, bool bf16, bool backward, hipStream_t stream) {
  return backward ? launch_rows<false, true>(a, bf16, stream) : launch_rows<false, false>(a, bf16, stream);
}

hipError_t launch_norm_rotate(const RowArgs& a, bool bf16, hipStream_t stream) { return launch_rows<true, false>(a, bf16, stream); }

hipError_t launch_norm_rotate_backward(const RowArgs& a, bool bf16, hipStream_t stream) {
  const int rows = kRowWaves << (6 - lanes_log2(a, bf16));
  const int64_t blocks = (a.N_real + rows - 1) / rows * a.batch;
  const int split = (int)std::min<int64_t>(head_blocks(blocks, a.heads), std::max<int64_t>(1, kMaxGradientBlocks / std::min<int64_t>(blocks, kMaxGradientBlocks)));
  const int per = (a.heads + split - 1) / split, head_groups = (a.heads + per - 1) / per;
  const dim3 grid((unsigned)std::min<int64_t>(blocks, kMaxGradientBlocks / head_groups), (unsigned)head_groups);
  with_pairing(a, bf16, [&](auto type, auto pairing) {
    norm_backward_kernel<decltype(type), decltype(pairing)::value><<<grid, kRowThreads, 0, stream>>>(a, per);
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.partial) return e;
  weight_gradient_kernel<<<(unsigned)((2 * a.D + 15) / 16), 1024, 0, stream>>>(a.partial, (int)(grid.x * grid.y), a.D, a.dweight[0], a.dweight[1]);
  return hipGetLastError();
}

}  // namespace ca
