// Dropout whose mask is never stored: out = (bits >= level ? x * scale : 0) + residual, where an element's 16 bits come from its
// place alone: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011), counter (i / 8, site, step), key
// seed.  Ten rounds of two 32 x 32 -> 64 bit products give 128 bits, eight elements' worth.
#include <hip/hip_runtime.h>

#include "lt_launch.h"

namespace ltk {
namespace {

constexpr uint32_t kBlock = 256;

struct Words {
  uint32_t w[4];
};

__device__ __forceinline__ Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)q;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Words{{c0, c1, c2, c3}};
}

// One thread, eight elements.  A dropped element is 0 whatever it was (selected, not multiplied).
template <typename T>
__global__ __launch_bounds__(kBlock) void lt_dropout_kernel(const DropoutArgs a) {
  const uint64_t block = (uint64_t)blockIdx.x * kBlock + threadIdx.x, at = block * 8u;
  if (at >= a.n) return;
  const uint64_t seed = (uint64_t)a.state[0], step = (uint64_t)a.state[1];
  const Words r = philox((uint32_t)block, a.site, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)seed, (uint32_t)(seed >> 32));
  const T* x = (const T*)a.x + at;
  const T* more = a.residual ? (const T*)a.residual + at : nullptr;
  T* out = (T*)a.out + at;
  const uint32_t left = a.n - at < 8u ? (uint32_t)(a.n - at) : 8u;
#pragma unroll
  for (uint32_t j = 0; j < 8u; ++j) {
    if (j >= left) break;
    const uint32_t bits = (r.w[j >> 1] >> (16u * (j & 1u))) & 0xffffu;
    float v = bits >= a.level ? (float)x[j] * a.scale : 0.0f;
    if (more) v += (float)more[j];
    out[j] = (T)v;
  }
}

hipError_t launch_dropout(const void* args, hipStream_t s) {
  const DropoutArgs& a = *(const DropoutArgs*)args;
  if (a.n == 0) return hipSuccess;
  if (a.n >= (uint64_t)1 << 35 || a.level > 65535u) return hipErrorInvalidValue;
  // (below 2^35 elements: below 2^32 threads)
  const dim3 grid((uint32_t)((a.n + 8u * kBlock - 1) / (8u * kBlock)));
  if (a.dtype == kF32) LT_LAUNCH(lt_dropout_kernel<float>, grid, dim3(kBlock), s, a);
  else if (a.dtype == kBF16) LT_LAUNCH(lt_dropout_kernel<__bf16>, grid, dim3(kBlock), s, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

const bool registered = set_operator(kOpDropout, launch_dropout);

}  // namespace
}  // namespace ltk
