// Natural order and tile order of the tokens, for kernels that walk over them one by one.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "layout.h"

namespace ca {

struct GridArgs {
  int32_t T, H, W, tt, th, tw, nH, nW, B;
  int64_t n_vid, N_real, N_pad, N_video;
};
inline void fill_grid(GridArgs& a, const ca_layout* L) {
  const ca_problem& p = L->prob;
  a.T = p.T; a.H = p.H; a.W = p.W;
  a.tt = p.tt; a.th = p.th; a.tw = p.tw;
  a.nH = L->nH; a.nW = L->nW;
  a.B = (int32_t)L->B;
  a.n_vid = L->n_vid;
  a.N_real = L->N_real;
  a.N_pad = L->N_pad;
  a.N_video = (int64_t)p.T * p.H * p.W;
}

namespace {

// Token of a row in natural order, -1 for a padding slot, and its coordinates (-1 for text).
struct Token {
  int64_t natural, place;  // place: in tile order
  int at[3];
};

__device__ __forceinline__ Token token_of_natural(const GridArgs& a, uint32_t natural) {
  Token k;
  k.natural = natural;
  k.at[0] = k.at[1] = k.at[2] = -1;
  if (natural >= (uint64_t)a.N_video) {
    k.place = a.n_vid * a.B + (natural - a.N_video);
    return k;
  }
  const uint32_t row = natural / (uint32_t)a.W, x = natural - row * a.W, t = row / (uint32_t)a.H, y = row - t * a.H;
  const uint32_t kt = t / (uint32_t)a.tt, kh = y / (uint32_t)a.th, kw = x / (uint32_t)a.tw;
  k.at[0] = (int)t, k.at[1] = (int)y, k.at[2] = (int)x;
  const uint32_t slot = ((t - kt * a.tt) * a.th + (y - kh * a.th)) * a.tw + (x - kw * a.tw);
  k.place = (int64_t)((kt * a.nH + kh) * a.nW + kw) * a.B + slot;
  return k;
}

__device__ __forceinline__ Token token_of_place(const GridArgs& a, uint32_t place) {
  Token k;
  k.place = place;
  k.at[0] = k.at[1] = k.at[2] = -1;
  const uint32_t tile = place / (uint32_t)a.B, slot = place - tile * a.B;
  if (tile >= (uint64_t)a.n_vid) {
    k.natural = a.N_video + (place - a.n_vid * a.B);
    return k;
  }
  const uint32_t tr = tile / (uint32_t)a.nW, kw = tile - tr * a.nW, kt = tr / (uint32_t)a.nH, kh = tr - kt * a.nH;
  const uint32_t sr = slot / (uint32_t)a.tw, dx = slot - sr * a.tw, dt = sr / (uint32_t)a.th, dy = sr - dt * a.th;
  const int t = (int)(kt * a.tt + dt), y = (int)(kh * a.th + dy), x = (int)(kw * a.tw + dx);
  const bool real = t < a.T && y < a.H && x < a.W;
  k.natural = real ? ((int64_t)t * a.H + y) * a.W + x : -1;
  if (real) k.at[0] = t, k.at[1] = y, k.at[2] = x;
  return k;
}

}  // namespace
}  // namespace ca
