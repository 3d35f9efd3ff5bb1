// What the kernels of rotary positions share: a pair's turn, and rotating with it.
#ifndef LT_ROTARY_H_
#define LT_ROTARY_H_

#include <hip/hip_runtime.h>

#include "lt_kernels.h"

namespace ltk {

struct Turn {
  float c, s;   // amplitude * cos, amplitude * sin
};

// The turn of pair i at a position.  Quarter turns in 64 bits: the whole ones go, their last two bits are the quadrant,
// and the rest, half a quarter at most, is exact in 32 bits to 2^-25 of itself.  On |x| <= pi / 4 the
// Taylor polynomials to x^9 and x^10 err by 2e-9 and 1e-10, below half a unit of the last place.
__device__ __forceinline__ Turn turn_of(const Rotary& r, int32_t position, uint32_t i) {
  const double q = (double)position * r.turns[i];
  const double whole = rint(q);
  const int quadrant = (int)whole;
  const float x = (float)(q - whole) * 1.57079632679489662f, xx = x * x;
  const float s = x * fmaf(xx, fmaf(xx, fmaf(xx, fmaf(xx, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f), 1.0f);
  const float c = fmaf(xx, fmaf(xx, fmaf(xx, fmaf(xx, fmaf(xx, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.0f);
  const float sn = (quadrant & 1) ? c : s, cs = (quadrant & 1) ? s : c;
  const bool flip_s = (quadrant & 2) != 0, flip_c = ((quadrant + 1) & 2) != 0;
  Turn t;
  t.c = r.amplitude * (flip_c ? -cs : cs);
  t.s = r.amplitude * ((flip_s != (r.back != 0u)) ? -sn : sn);
  return t;
}

__device__ __forceinline__ void rotate(const Turn& t, float x, float y, float* a, float* b) {
  *a = fmaf(x, t.c, -(y * t.s));
  *b = fmaf(y, t.c, x * t.s);
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__bf16 v) { return (float)v; }

}  // namespace ltk
#endif
