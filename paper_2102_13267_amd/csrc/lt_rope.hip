// Rotary positions: out[t][h] = x[t][h] with its first n elements rotated, pair by pair, by an angle that the token's
// position and the pair's frequency give, and the rest as it is; the gradient turns back.
//
// Bound by memory: every element is read and written once.  16 bytes a lane where rows allow, up to four rows of a thread on
// their way while the workgroup computes its tokens' turns (lt_rotary.h).  65536 tokens of 32 x 128 bf16: 174 us, 6.2 TB/s (one thread
// a pair, each with a turn of its own, 550).
//
// Past the last-level cache (256 MB) goes what does not fit it: reads where operand and result together are larger, two rows a
// thread (134 MB + 134 MB alone 51.0 -> 46.0 us, with scores behind it 1414 -> 1405), results where they alone are.  Smaller ones are plain: 33 MB + 33 MB
// among other data that fills the cache take 16.8 us a launch, 12.1 with results stored past it, but whoever reads the result next loses more
// (an elementwise pass behind it 26.6 / 29.1, scores, softmax and product 308 / 320).
#include <hip/hip_runtime.h>

#include "lt_launch.h"
#include "lt_rotary.h"

namespace ltk {
namespace {

template <typename T, int V, bool IL, Past PAST>
__global__ __launch_bounds__(kRowBlock) void lt_rope_kernel(const RopeArgs a) {
  __shared__ Turn turns[kMaxTurns];
  rope_rows<T, V, IL, PAST>(a, blockIdx.x, turns);
}

// Rows that the above does not take: interleaved pairs at odd places, rows of very many slots.  One thread per pair (or element of the rest).
template <typename T>
__global__ __launch_bounds__(kRowBlock) void lt_rope_any_kernel(const RopeArgs a) {
  const uint32_t half = a.rotary.dims / 2u, unit = a.dim - half;   // pairs, then the rest
  const uint64_t n = a.tokens * a.heads.d * unit, stride = (uint64_t)gridDim.x * kRowBlock;
  for (uint64_t i = (uint64_t)blockIdx.x * kRowBlock + threadIdx.x; i < n; i += stride) {
    const uint32_t u = (uint32_t)(i % unit);
    const uint64_t row = i / unit, t = row / a.heads.d;
    const uint32_t h = (uint32_t)(row % a.heads.d);
    const T* x = (const T*)a.x + (int64_t)(t / a.inner.d) * a.s_outer + (int64_t)(t % a.inner.d) * a.s_inner + (int64_t)h * a.s_head;
    T* y = (T*)a.out + row * a.dim;
    if (u >= half) {
      y[half + u] = x[half + u];
      continue;
    }
    const uint32_t p = a.rotary.interleaved ? 2u * u : u, q = a.rotary.interleaved ? 2u * u + 1u : u + half;
    float v, w;
    rotate(turn_of(a.rotary, a.positions[t % a.n_pos.d], u), to_float(x[p]), to_float(x[q]), &v, &w);
    y[p] = (T)v;
    y[q] = (T)w;
  }
}

template <typename T, int V, bool IL>
void launch_rows(const RopeArgs& a, const RopeLayout& l, hipStream_t s) {
  if (l.past == kAllPast) LT_LAUNCH((lt_rope_kernel<T, V, IL, kAllPast>), dim3(l.grid), dim3(kRowBlock), s, a);
  else if (l.past == kReadsPast) LT_LAUNCH((lt_rope_kernel<T, V, IL, kReadsPast>), dim3(l.grid), dim3(kRowBlock), s, a);
  else LT_LAUNCH((lt_rope_kernel<T, V, IL, kNothingPast>), dim3(l.grid), dim3(kRowBlock), s, a);
}

template <typename T>
hipError_t launch_rope_of(RopeArgs a, hipStream_t s) {
  constexpr int kMost = 16 / sizeof(T);
  RopeLayout l;
  if (lay_out(&a, sizeof(T), &l)) {
    if (a.rotary.interleaved) {
      if (l.v == kMost) launch_rows<T, kMost, true>(a, l, s);
      else if (l.v == 4u) launch_rows<T, 4, true>(a, l, s);
      else launch_rows<T, 2, true>(a, l, s);
    } else {
      if (l.v == kMost) launch_rows<T, kMost, false>(a, l, s);
      else if (l.v == 4u) launch_rows<T, 4, false>(a, l, s);
      else if (l.v == 2u) launch_rows<T, 2, false>(a, l, s);
      else launch_rows<T, 1, false>(a, l, s);
    }
    return hipGetLastError();
  }
  const uint64_t n = (a.tokens * a.heads.d * (a.dim - a.rotary.dims / 2u) + kRowBlock - 1) / kRowBlock;
  LT_LAUNCH(lt_rope_any_kernel<T>, dim3((uint32_t)(n < 65536u ? n : 65536u)), dim3(kRowBlock), s, a);
  return hipGetLastError();
}

hipError_t launch_rope(const void* args, hipStream_t s) {
  const RopeArgs& a = *(const RopeArgs*)args;
  if (a.tokens * a.heads.d * a.dim == 0) return hipSuccess;
  if (!fit_to_run(a)) return hipErrorInvalidValue;
  return a.dtype == kF32 ? launch_rope_of<float>(a, s) : a.dtype == kBF16 ? launch_rope_of<__bf16>(a, s) : hipErrorInvalidValue;
}

const bool registered = set_operator(kOpRope, launch_rope);

}  // namespace
}  // namespace ltk
