// A paged cache of keys and values: new rows written into it (the keys rotated by their positions on the way), and
// the attention of one new token a sequence over what the sequence has in it.
//
// The cache is [pages][2][key heads][rows][dim]; sequence s holds position p in row p % rows of page table[s][p / rows].
// What lengths and tables say is checked here, key by key: nothing outside the cache is read or written.
#include <hip/hip_runtime.h>

#include "lt_launch.h"
#include "lt_rotary.h"

namespace ltk {
namespace {

constexpr uint32_t kBlock = 256;
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ uint32_t divide(const Divider& d, uint32_t n) { return (uint32_t)(((uint64_t)n * d.magic) >> (31u + d.shift)); }

// ---- new rows ------------------------------------------------------------------------------------
__global__ __launch_bounds__(kBlock) void lt_cache_copy_kernel(const AppendArgs a) {
  const uint64_t n = a.cache_elems * (a.cache_dtype == kF32 ? 4u : 2u), stride = (uint64_t)gridDim.x * kBlock * 16u;
  for (uint64_t i = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) * 16u; i < n; i += stride) {
    if (i + 16u <= n) *(uint4*)((char*)a.cache + i) = *(const uint4*)((const char*)a.copy_from + i);
    else
      for (uint64_t k = i; k < n; k += 2u) *(uint16_t*)((char*)a.cache + k) = *(const uint16_t*)((const char*)a.copy_from + k);
  }
}

// Where token t goes: its position, and its row of the cache as page * rows + row; false: nowhere.
__device__ __forceinline__ bool place(const AppendArgs& a, uint32_t t, int32_t* position, uint32_t* page, uint32_t* row) {
  uint32_t s = t;
  int64_t pos;
  if (a.offsets) {
    // the last sequence that starts at or before t; between its neighbours' offsets, whatever they hold
    uint32_t lo = 0, hi = a.seqs;   // offsets[lo] <= t (or lo = 0), offsets[hi] > t (or hi = seqs)
    while (hi - lo > 1u) {
      const uint32_t mid = (lo + hi) / 2u;
      if (a.offsets[mid] <= (int64_t)t) lo = mid;
      else hi = mid;
    }
    s = lo;
    if (s >= a.seqs || (int64_t)a.offsets[s] > (int64_t)t || (int64_t)a.offsets[s + 1] <= (int64_t)t) return false;
    pos = (int64_t)a.lengths[s] - a.offsets[s + 1] + t;
  } else {
    pos = (int64_t)a.lengths[s] - 1;
  }
  if (pos < 0 || pos >= (int64_t)a.slots * a.rows.d) return false;
  const uint32_t slot = divide(a.rows, (uint32_t)pos);
  const int32_t p = a.table[(uint64_t)s * a.slots + slot];
  if (p < 0 || (uint32_t)p >= a.pages) return false;
  *position = (int32_t)pos;
  *page = (uint32_t)p;
  *row = (uint32_t)pos - slot * a.rows.d;
  return true;
}

template <typename C, typename T>
__global__ __launch_bounds__(kBlock) void lt_cache_append_kernel(const AppendArgs a) {
  const uint32_t half = a.rotary.dims / 2u, unit = a.dim - half;
  const uint64_t n = (uint64_t)a.tokens * 2u * a.heads * unit, stride = (uint64_t)gridDim.x * kBlock;
  for (uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += stride) {
    const uint32_t u = (uint32_t)(i % unit), h = (uint32_t)(i / unit % a.heads), kind = (uint32_t)(i / unit / a.heads % 2u), t = (uint32_t)(i / unit / a.heads / 2u);
    int32_t position;
    uint32_t page, row;
    if (!place(a, t, &position, &page, &row)) continue;
    const T* x = kind == 0u ? (const T*)a.k + (int64_t)t * a.k_token + (int64_t)h * a.k_head : (const T*)a.v + (int64_t)t * a.v_token + (int64_t)h * a.v_head;
    C* y = (C*)a.cache + ((((uint64_t)page * 2u + kind) * a.heads + h) * a.rows.d + row) * a.dim;
    if (u >= half) {
      y[half + u] = (C)to_float(x[half + u]);
      continue;
    }
    const uint32_t p = a.rotary.interleaved ? 2u * u : u, q = a.rotary.interleaved ? 2u * u + 1u : u + half;
    float v = to_float(x[p]), w = to_float(x[q]);
    if (kind == 0u) rotate(turn_of(a.rotary, position, u), v, w, &v, &w);
    y[p] = (C)v;
    y[q] = (C)w;
  }
}

hipError_t launch_append(const void* args, hipStream_t s) {
  const AppendArgs& a = *(const AppendArgs*)args;
  if (a.cache_elems == 0) return hipSuccess;
  if (!a.cache || a.rows.d == 0 || a.rotary.dims > a.dim || a.rotary.dims > 2u * kMaxPairs) return hipErrorInvalidValue;
  if (a.copy_from) {
    const uint64_t pieces = (a.cache_elems + 2047u) / 2048u;
    LT_LAUNCH(lt_cache_copy_kernel, dim3((uint32_t)(pieces < 16384u ? pieces : 16384u)), dim3(kBlock), s, a);
  }
  const uint64_t n = (uint64_t)a.tokens * 2u * a.heads * (a.dim - a.rotary.dims / 2u);
  if (n == 0 || a.seqs == 0 || a.slots == 0) return hipGetLastError();
  if (!a.k || !a.v || !a.lengths || !a.table) return hipErrorInvalidValue;
  const uint32_t grid = (uint32_t)((n + kBlock - 1) / kBlock < 65536u ? (n + kBlock - 1) / kBlock : 65536u);
  if (a.cache_dtype == kF32 && a.dtype == kF32) LT_LAUNCH((lt_cache_append_kernel<float, float>), dim3(grid), dim3(kBlock), s, a);
  else if (a.cache_dtype == kF32 && a.dtype == kBF16) LT_LAUNCH((lt_cache_append_kernel<float, __bf16>), dim3(grid), dim3(kBlock), s, a);
  else if (a.cache_dtype == kBF16 && a.dtype == kF32) LT_LAUNCH((lt_cache_append_kernel<__bf16, float>), dim3(grid), dim3(kBlock), s, a);
  else if (a.cache_dtype == kBF16 && a.dtype == kBF16) LT_LAUNCH((lt_cache_append_kernel<__bf16, __bf16>), dim3(grid), dim3(kBlock), s, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

// ---- attention of one new token -------------------------------------------------------------------
// One workgroup per sequence and query head; its four waves take every fourth key each, a lane four elements of the
// head, with a running maximum and sum; the waves' parts meet in LDS.
template <typename T>
__global__ __launch_bounds__(kBlock) void lt_paged_attention_kernel(const PagedArgs a) {
  const uint32_t s = blockIdx.x / a.heads, h = blockIdx.x % a.heads, kh = h / (a.heads / a.kv_heads);
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  int64_t len = a.lengths[s];
  len = len < 0 ? 0 : len > (int64_t)a.capacity ? (int64_t)a.capacity : len;
  const T* q = (const T*)a.q + (int64_t)s * a.q_seq + (int64_t)h * a.q_head;
  const float scale = a.scale * kLog2e;
  float qv[4], acc[4] = {0, 0, 0, 0}, top = -INFINITY, sum = 0.0f;
  for (uint32_t i = 0; i < 4u; ++i) qv[i] = lane + 64u * i < a.dim ? to_float(q[lane + 64u * i]) : 0.0f;
  for (uint32_t p = wave; p < (uint32_t)len; p += 4u) {
    const uint32_t slot = divide(a.rows, p);
    const int32_t page = a.table[(uint64_t)s * a.slots + slot];
    if (page < 0 || (uint32_t)page >= a.pages) continue;
    const T* k = (const T*)a.cache + (((uint64_t)page * 2u * a.kv_heads + kh) * a.rows.d + (p - slot * a.rows.d)) * a.dim;
    const T* v = k + (uint64_t)a.kv_heads * a.rows.d * a.dim;
    float dot = 0.0f;
    for (uint32_t i = 0; i < 4u; ++i)
      if (lane + 64u * i < a.dim) dot = fmaf(qv[i], to_float(k[lane + 64u * i]), dot);
    for (int m = 32; m >= 1; m >>= 1) dot += __shfl_xor(dot, m, 64);
    dot *= scale;
    const float t = fmaxf(top, dot), safe = t == -INFINITY ? 0.0f : t;
    const float keep = exp2f(top - safe), w = exp2f(dot - safe);
    top = t;
    sum = fmaf(sum, keep, w);
    for (uint32_t i = 0; i < 4u; ++i)
      if (lane + 64u * i < a.dim) acc[i] = fmaf(acc[i], keep, w * to_float(v[lane + 64u * i]));
  }
  __shared__ float tops[4], sums[4], parts[4][256];
  for (uint32_t i = 0; i < 4u; ++i) parts[wave][lane + 64u * i] = acc[i];
  if (lane == 0u) {
    tops[wave] = top;
    sums[wave] = sum;
  }
  __syncthreads();
  float all = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  if (all == -INFINITY) all = 0.0f;
  float total = 0.0f, o = 0.0f;
  for (int w = 0; w < 4; ++w) {
    const float f = exp2f(tops[w] - all);
    total = fmaf(sums[w], f, total);
    o = fmaf(parts[w][threadIdx.x], f, o);
  }
  if (threadIdx.x < a.dim) ((T*)a.out)[((uint64_t)s * a.heads + h) * a.dim + threadIdx.x] = (T)(total > 0.0f || total != total ? o / total : 0.0f);
}

hipError_t launch_paged(const void* args, hipStream_t s) {
  const PagedArgs& a = *(const PagedArgs*)args;
  if (a.seqs == 0) return hipSuccess;
  if (!a.q || !a.lengths || !a.out || (a.capacity > 0 && (!a.cache || !a.table)) || a.dim == 0 || a.dim > 256u || a.kv_heads == 0 || a.heads % a.kv_heads != 0 || a.rows.d == 0)
    return hipErrorInvalidValue;
  if (a.dtype == kF32) LT_LAUNCH(lt_paged_attention_kernel<float>, dim3(a.seqs * a.heads), dim3(kBlock), s, a);
  else if (a.dtype == kBF16) LT_LAUNCH(lt_paged_attention_kernel<__bf16>, dim3(a.seqs * a.heads), dim3(kBlock), s, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

const bool registered = set_operator(kOpCacheAppend, launch_append) && set_operator(kOpPagedAttention, launch_paged);

}  // namespace
}  // namespace ltk
