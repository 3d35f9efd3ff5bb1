// Rotary positions: out[t][h] = x[t][h] with its first n elements rotated, pair by pair, by an angle that the token's
// position and the pair's frequency give, and the rest as it is; the gradient turns back.
//
// One thread per pair (or element of the rest) of every head.
#include <hip/hip_runtime.h>

#include "lt_launch.h"
#include "lt_rotary.h"

namespace ltk {
namespace {

constexpr uint32_t kRopeBlock = 256;

template <typename T>
__global__ __launch_bounds__(kRopeBlock) void lt_rope_kernel(const RopeArgs a) {
  const uint32_t half = a.rotary.dims / 2u, unit = a.dim - half;   // pairs, then the rest
  const uint64_t n = a.tokens * a.heads * unit, stride = (uint64_t)gridDim.x * kRopeBlock;
  for (uint64_t i = (uint64_t)blockIdx.x * kRopeBlock + threadIdx.x; i < n; i += stride) {
    const uint32_t u = (uint32_t)(i % unit);
    const uint64_t row = i / unit, t = row / a.heads;
    const uint32_t h = (uint32_t)(row % a.heads);
    const T* x = (const T*)a.x + (int64_t)(t / a.inner) * a.s_outer + (int64_t)(t % a.inner) * a.s_inner + (int64_t)h * a.s_head;
    T* y = (T*)a.out + row * a.dim;
    if (u >= half) {
      y[half + u] = x[half + u];
      continue;
    }
    const uint32_t p = a.rotary.interleaved ? 2u * u : u, q = a.rotary.interleaved ? 2u * u + 1u : u + half;
    float v, w;
    rotate(turn_of(a.rotary, a.positions[t % a.n_pos], u), to_float(x[p]), to_float(x[q]), &v, &w);
    y[p] = (T)v;
    y[q] = (T)w;
  }
}

hipError_t launch_rope(const void* args, hipStream_t s) {
  const RopeArgs& a = *(const RopeArgs*)args;
  const uint64_t n = a.tokens * a.heads * (a.dim - a.rotary.dims / 2u);
  if (n == 0) return hipSuccess;
  if (!a.x || !a.positions || !a.out || a.inner == 0 || a.n_pos == 0 || a.rotary.dims > a.dim || a.rotary.dims > 2u * kMaxPairs) return hipErrorInvalidValue;
  const uint32_t grid = (uint32_t)((n + kRopeBlock - 1) / kRopeBlock < 65536u ? (n + kRopeBlock - 1) / kRopeBlock : 65536u);
  if (a.dtype == kF32) LT_LAUNCH(lt_rope_kernel<float>, dim3(grid), dim3(kRopeBlock), s, a);
  else if (a.dtype == kBF16) LT_LAUNCH(lt_rope_kernel<__bf16>, dim3(grid), dim3(kRopeBlock), s, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

const bool registered = set_operator(kOpRope, launch_rope);

}  // namespace
}  // namespace ltk
