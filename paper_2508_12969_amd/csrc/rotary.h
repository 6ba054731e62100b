// Rotary tables and the launch interface of the kernels that read them (rotary.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <mutex>
#include <vector>

#include "compact_attn.h"
#include "tokens.h"

struct ca_rotary {
  ca_rotary_axis axes[3]{};
  int32_t pairing = CA_PAIRS_INTERLEAVED;
  int32_t channels = 0;        // rotated channels of a head
  int64_t first[3] = {0, 0, 0};  // of the axis' angles in `angles`, in (cos, sin) pairs
  std::vector<float> angles;   // per axis [positions][channels / 2] (cos, sin), times the magnitude

  std::mutex upload_mutex;
  int device = -1;
  float* dev = nullptr;
};

namespace ca {

constexpr int kRowThreads = 256, kRowWaves = kRowThreads / 64;
constexpr int kMaxGradientBlocks = 1024;  // workgroups of the norm's backward kernel: each leaves a partial sum of the weight gradients

struct RowStrides {
  int64_t batch, head, token;  // elements
};

// What is done with a row of D channels.
struct RowRule {
  int32_t D;
  float eps;
  // rotation
  const float* angles;         // (cos, sin) pairs; null: no rotation
  int64_t first[3];
  int32_t pairs[3], positions[3];
  int32_t half;                // pairing: channels i and i + rotated/2
  int32_t rotated;
  float sign;                  // of the sine: -1 turns back
};

// One launch over the rows (token, head) of one or two tensors.
struct RowArgs : GridArgs, RowRule {  // rows are walked in the order of dst, which is in tile order (tiled forward) or in natural order
  const void* src[2];
  void* dst[2];
  const void* x[2];            // norm, backward: the forward call's inputs
  RowStrides src_strides, dst_strides, x_strides, src_strides1, dst_strides1, x_strides1;  // of tensor 0 and of tensor 1
  const void* weight[2];       // null: ones
  float* partial;              // norm, backward: [workgroups][tensors][D], or null
  float* dweight[2];
  int32_t tensors, batch, heads;
  int32_t tiled;               // the tensor that is not the model's own is in tile order: dst of forward, src of backward calls
  int32_t origin[3];
  const int32_t* where;        // [batch][N_real][3] or null
};

// The rotation part of a rule; puts the table on the current device at its first use (api_rotary.cpp).
int fill_rotation(RowRule& a, ca_rotary* r, hipStream_t stream);

hipError_t launch_rotate(const RowArgs& a, bool bf16, bool backward, hipStream_t stream);
hipError_t launch_norm_rotate(const RowArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_norm_rotate_backward(const RowArgs& a, bool bf16, hipStream_t stream);

}  // namespace ca
