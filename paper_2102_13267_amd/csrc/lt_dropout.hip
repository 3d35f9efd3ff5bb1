// Dropout whose mask is never stored: out = (bits >= level ? x * scale : 0) + residual, where an element's 16 bits come from its
// place alone: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011), counter (i / 8, site, step), key
// seed.  Ten rounds of two 32 x 32 -> 64 bit products give 128 bits, eight elements' worth: sixteen bits each, because 32 would take as long to compute as
// the elements take to travel.
//
// Bound by memory: every element is read and written once, 16 bytes a load.  16384 x 4096 bf16: 42 us, 6.4 TB/s, with a residual
// 61 us, 6.6 TB/s (element by element 113 and 220).
// Past the last-level cache (256 MB) goes what does not fit it: without that 51 and 72 us; 16384 x 1024 takes 11.0 us through it and 12.6 past it.
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

// Eight elements as they are moved: 16 bytes at a time.
typedef uint32_t Quad __attribute__((ext_vector_type(4)));
template <typename T>
struct Eight {
  static constexpr int kQuads = sizeof(T) / 2;
  Quad q[kQuads];
  template <bool PAST>
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kQuads; ++i) q[i] = PAST ? __builtin_nontemporal_load((const Quad*)p + i) : ((const Quad*)p)[i];
  }
  template <bool PAST>
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
      if (PAST) __builtin_nontemporal_store(q[i], (Quad*)p + i);
      else ((Quad*)p)[i] = q[i];
    }
  }
  __device__ __forceinline__ float get(int j) const {
    const uint32_t word = sizeof(T) == 4 ? q[j / 4][j % 4] : q[0][j / 2];   // (a bit cast of a vector's element itself takes the first)
    return __builtin_bit_cast(float, sizeof(T) == 4 ? word : j & 1 ? word & 0xffff0000u : word << 16);
  }
  __device__ __forceinline__ void set_pair(int j, float a, float b) {   // elements 2 j and 2 j + 1
    if (sizeof(T) == 4) {
      q[j / 2][j % 2 * 2] = __builtin_bit_cast(uint32_t, a);
      q[j / 2][j % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, b);
    } else {
      typedef __bf16 V2 __attribute__((ext_vector_type(2)));
      q[0][j] = __builtin_bit_cast(uint32_t, V2{(__bf16)a, (__bf16)b});
    }
  }
};

__device__ __forceinline__ bool kept(const Words& r, uint32_t j, uint32_t level) { return ((r.w[j >> 1] >> (16u * (j & 1u))) & 0xffffu) >= level; }

// One thread, eight elements, on their way while the words are computed.  A dropped element is 0 whatever it was (selected,
// not multiplied).  (Sixteen elements a thread: 12.1 us where eight take 11.0 at 16384 x 1024 bf16, 169 where they take 162 at 262144 x 1024.)
template <typename T, bool MORE, bool PAST>
__global__ __launch_bounds__(kBlock) void lt_dropout_kernel(const DropoutArgs a) {
  const uint64_t block = (uint64_t)blockIdx.x * kBlock + threadIdx.x, whole = a.n / 8u;
  if (block * 8u >= a.n) return;
  const T* const x = (const T*)a.x;
  const T* const more = (const T*)a.residual;
  T* const out = (T*)a.out;
  Eight<T> v, w;
  if (block < whole) {
    v.template load<PAST>(x + block * 8u);
    if (MORE) w.template load<PAST>(more + block * 8u);
  }
  const uint64_t seed = (uint64_t)a.state[0], step = (uint64_t)a.state[1];
  const Words r = philox((uint32_t)block, a.site, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)seed, (uint32_t)(seed >> 32));
  if (block < whole) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo = kept(r, 2 * j, a.level) ? v.get(2 * j) * a.scale : 0.0f, hi = kept(r, 2 * j + 1, a.level) ? v.get(2 * j + 1) * a.scale : 0.0f;
      if (MORE) {
        lo += w.get(2 * j);
        hi += w.get(2 * j + 1);
      }
      v.set_pair(j, lo, hi);
    }
    v.template store<PAST>(out + block * 8u);
  } else {   // the last few
#pragma unroll
    for (uint32_t j = 0; j < 7u; ++j) {
      const uint64_t at = block * 8u + j;
      if (at >= a.n) break;
      float e = kept(r, j, a.level) ? (float)x[at] * a.scale : 0.0f;
      if (MORE) e += (float)more[at];
      out[at] = (T)e;
    }
  }
}

// Operands that do not start at 16 bytes (a window's): element by element.
template <typename T>
__global__ __launch_bounds__(kBlock) void lt_dropout_any_kernel(const DropoutArgs a) {
  const uint64_t block = (uint64_t)blockIdx.x * kBlock + threadIdx.x, at = block * 8u;
  if (at >= a.n) return;
  const uint64_t seed = (uint64_t)a.state[0], step = (uint64_t)a.state[1];
  const Words r = philox((uint32_t)block, a.site, (uint32_t)step, (uint32_t)(step >> 32), (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
  for (uint32_t j = 0; j < 8u; ++j) {
    if (at + j >= a.n) break;
    float v = kept(r, j, a.level) ? (float)((const T*)a.x)[at + j] * a.scale : 0.0f;
    if (a.residual) v += (float)((const T*)a.residual)[at + j];
    ((T*)a.out)[at + j] = (T)v;
  }
}

template <typename T, bool MORE>
void launch_of(const DropoutArgs& a, hipStream_t s) {
  const dim3 grid((uint32_t)((a.n + 8u * kBlock - 1) / (8u * kBlock)));
  if (a.n * sizeof(T) * (MORE ? 3u : 2u) >= ((uint64_t)256 << 20)) LT_LAUNCH((lt_dropout_kernel<T, MORE, true>), grid, dim3(kBlock), s, a);
  else LT_LAUNCH((lt_dropout_kernel<T, MORE, false>), grid, dim3(kBlock), s, a);
}

template <typename T>
hipError_t launch_typed(const DropoutArgs& a, hipStream_t s) {
  if ((((uintptr_t)a.x | (uintptr_t)a.residual | (uintptr_t)a.out) & 15u) != 0) LT_LAUNCH(lt_dropout_any_kernel<T>, dim3((uint32_t)((a.n + 8u * kBlock - 1) / (8u * kBlock))), dim3(kBlock), s, a);
  else if (a.residual) launch_of<T, true>(a, s);
  else launch_of<T, false>(a, s);
  return hipGetLastError();
}

hipError_t launch_dropout(const void* args, hipStream_t s) {
  const DropoutArgs& a = *(const DropoutArgs*)args;
  if (a.n == 0) return hipSuccess;
  // (below 2^35 elements: at most 2^32 - 256 threads)
  if (a.n > ((uint64_t)1 << 35) - 2048u || a.level > 65535u) return hipErrorInvalidValue;
  return a.dtype == kF32 ? launch_typed<float>(a, s) : a.dtype == kBF16 ? launch_typed<__bf16>(a, s) : hipErrorInvalidValue;
}

const bool registered = set_operator(kOpDropout, launch_dropout);

}  // namespace
}  // namespace ltk
