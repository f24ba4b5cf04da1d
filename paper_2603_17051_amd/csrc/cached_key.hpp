// Rotation of the keys that a bf16 cache keeps: in 64 bits, rounded to 32 and then to bf16, whichever kernel stores them (an
// append with or without block means, sinks that move on).  A cached key is then a function of the key and its position alone.  In 32
// bits, with tables rounded to 32, one element in 50000 to 100000 came out as the other neighbour, which the gradients of
// queries over selected blocks (fp32, 16 bits kept) show: 1.2e-5 off, 6e-6 now.  A vector instruction of 64 bits takes as long as one of
// 32 here, and the appends stay bound by their bytes.  (Turning in 32 bits, and in 64 only where an element lies too near a tie to know, one lane
// in 500, was slower: the tables of those come late.)
#pragma once

#include <hip/hip_runtime.h>

#include "kernels.hpp"

namespace astro {

// A frame's temporal pairs, by the first n_t threads of a workgroup
__device__ __forceinline__ void exact_temporal(const DevGeom& g, double2* tab_t, int frame) {
  if ((int)threadIdx.x >= g.n_t) return;
  double s, c;
  sincos((double)frame * g.inv_freq_t[threadIdx.x], &s, &c);
  tab_t[threadIdx.x] = make_double2(c, s);
}

// The (cos, sin) of four consecutive pairs, the first of them number `pair`, for a token in row `row` and column `col`.
struct ExactAngles {
  double2 v[4];
  __device__ __forceinline__ void load_temporal(const DevGeom& g, const double2* tab_t, int pair) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (pair + i < g.n_t) v[i] = tab_t[pair + i];
  }
  // the others: a token's (one load from a selected address)
  __device__ __forceinline__ void load_spatial(const DevGeom& g, int row, int col, int pair) {
    const int nb = g.n_t + g.n_h;
    const double2 *h = g.tab_h64 + (row * g.n_h - g.n_t), *w = g.tab_w64 + (col * g.n_w - nb);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (pair + i >= g.n_t) v[i] = (pair + i < nb ? h : w)[pair + i];
  }
};

// Eight consecutive components (four adjacent pairs) turned.  (Without the empty statement the compiler rounds from 64 bits to bf16 at once, in five
// more instructions an element, and to the other neighbour where the 32-bit value is a tie.)
template <typename X8>
__device__ __forceinline__ X8 cached_key8(const X8& x, const ExactAngles& at) {
  X8 y;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const double a = (double)(float)x[2 * v], b = (double)(float)x[2 * v + 1];
    float lo = (float)fma(at.v[v].x, a, -(at.v[v].y * b)), hi = (float)fma(at.v[v].x, b, at.v[v].y * a);
    asm("" : "+v"(lo), "+v"(hi));
    y[2 * v] = (__bf16)lo;
    y[2 * v + 1] = (__bf16)hi;
  }
  return y;
}

}  // namespace astro
