// Rows of a table by token, and the gradient of the table.
#include <hip/hip_runtime.h>

#include "lt_launch.h"

namespace ltk {
namespace {

constexpr uint32_t kBlock = 256;

// ---- lookup: one wave an output row -------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kBlock) void lt_embedding_kernel(const EmbedArgs a) {
  const uint32_t t = blockIdx.x * (kBlock / 64u) + threadIdx.x / 64u, lane = threadIdx.x & 63u;
  if (t >= a.tokens) return;
  const int32_t id = a.ids[t];
  const bool there = id >= 0 && (uint32_t)id < a.rows;
  const T* row = (const T*)a.table + (uint64_t)(there ? id : 0) * a.dim;
  T* out = (T*)a.out + (uint64_t)t * a.dim;
  for (uint32_t d = lane; d < a.dim; d += 64u) out[d] = there ? (T)((float)row[d] * a.scale) : (T)0.0f;
}

template <typename T>
hipError_t launch_lookup(const EmbedArgs& a, hipStream_t s) {
  LT_LAUNCH(lt_embedding_kernel<T>, dim3((a.tokens + kBlock / 64u - 1u) / (kBlock / 64u)), dim3(kBlock), s, a);
  return hipGetLastError();
}

hipError_t launch_embedding(const void* args, hipStream_t s) {
  const EmbedArgs& a = *(const EmbedArgs*)args;
  if (a.tokens == 0 || a.dim == 0) return hipSuccess;
  return a.dtype == kF32 ? launch_lookup<float>(a, s) : a.dtype == kBF16 ? launch_lookup<__bf16>(a, s) : hipErrorInvalidValue;
}

// ---- the gradient: tokens in the order of their ids ------------------------------------------------------
// A stable radix sort, a digit of the ids at a time, lowest first.  Workgroup b has tokens b * each to (b + 1) * each - 1 of the order
// so far, wave w of it a contiguous share.  Count: how many of each digit.  Move: a token's place is what stands before it: smaller
// digits anywhere, its own digit in earlier workgroups, in earlier waves of this one, and in this wave before it.
__device__ __forceinline__ uint32_t key_of(const EmbedGradArgs& a, uint32_t i) {
  if (a.key) return a.key[i];
  const int32_t id = a.ids[i];
  return id >= 0 && (uint32_t)id < a.rows ? (uint32_t)id : a.rows;
}

// one more in LDS (counts come out the same in any order)
__device__ __forceinline__ void one_more(uint32_t* n) { __hip_atomic_fetch_add(n, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

__global__ __launch_bounds__(kEmbedBlock) void lt_embedding_count_kernel(const EmbedGradArgs a) {
  __shared__ uint32_t hist[1u << kEmbedMaxBits];
  const uint32_t digits = 1u << a.bits;
  for (uint32_t d = threadIdx.x; d < digits; d += kEmbedBlock) hist[d] = 0u;
  if (a.named)   // (the first pass clears them)
    for (uint32_t i = blockIdx.x * kEmbedBlock + threadIdx.x; i <= a.rows / 32u; i += gridDim.x * kEmbedBlock) a.named[i] = 0u;
  __syncthreads();
  const uint32_t begin = blockIdx.x * a.each;
  for (uint32_t i = begin + threadIdx.x; i < begin + a.each && i < a.tokens; i += kEmbedBlock) one_more(&hist[(key_of(a, i) >> a.shift) & (digits - 1u)]);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kEmbedBlock) a.counts[d * a.blocks + blockIdx.x] = hist[d];
}

__global__ __launch_bounds__(kEmbedBlock) void lt_embedding_move_kernel(const EmbedGradArgs a) {
  constexpr uint32_t kWaves = kEmbedBlock / 64u;
  __shared__ uint32_t start[1u << kEmbedMaxBits];            // where this workgroup's tokens of a digit go
  __shared__ uint32_t mine[kWaves][1u << kEmbedMaxBits];     // a wave's tokens of a digit, then where they go
  __shared__ uint32_t waves[kWaves];
  const uint32_t digits = 1u << a.bits, lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
  for (uint32_t d = threadIdx.x; d < kWaves * digits; d += kEmbedBlock) mine[d / digits][d % digits] = 0u;
  // digit d = this thread's (at most as many digits as threads): all of it, and what earlier workgroups have
  uint32_t all = 0u, before = 0u;
  if (threadIdx.x < digits)
    for (uint32_t b = 0; b < a.blocks; ++b) {
      const uint32_t c = a.counts[threadIdx.x * a.blocks + b];
      all += c;
      before += b < blockIdx.x ? c : 0u;
    }
  uint32_t upto = all;   // inclusive scan over the workgroup
#pragma unroll
  for (uint32_t o = 1; o < 64u; o *= 2u) {
    const uint32_t v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 63u) waves[wave] = upto;
  __syncthreads();
  uint32_t smaller = upto - all;
  for (uint32_t w = 0; w < wave; ++w) smaller += waves[w];
  if (threadIdx.x < digits) start[threadIdx.x] = smaller + before;
  const uint32_t share = a.each / kWaves, begin = blockIdx.x * a.each + wave * share;
  for (uint32_t r = 0; r < share; r += 64u) {
    const uint32_t i = begin + r + lane;
    if (i < a.tokens) one_more(&mine[wave][(key_of(a, i) >> a.shift) & (digits - 1u)]);
  }
  __syncthreads();
  if (threadIdx.x < digits) {
    uint32_t at = start[threadIdx.x];
    for (uint32_t w = 0; w < kWaves; ++w) {
      const uint32_t c = mine[w][threadIdx.x];
      mine[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  for (uint32_t r = 0; r < share; r += 64u) {
    const uint32_t i = begin + r + lane;
    const bool there = i < a.tokens;
    const uint32_t key = there ? key_of(a, i) : 0u, digit = (key >> a.shift) & (digits - 1u);
    // the lanes with the same digit
    uint64_t same = __ballot(there);
    for (uint32_t b = 0; b < a.bits; ++b) {
      const uint64_t ones = __ballot((digit >> b) & 1u);
      same &= (digit >> b) & 1u ? ones : ~ones;
    }
    const uint32_t earlier = __popcll(same & (((uint64_t)1 << lane) - 1u));
    const uint32_t at = there ? mine[wave][digit] + earlier : 0u;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (there && earlier == 0u) mine[wave][digit] = at + (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (there) {
      a.key_to[at] = key;
      a.pos_to[at] = a.pos ? a.pos[i] : i;
      if (a.named && key < a.rows && !(a.named[key / 32u] >> (key % 32u) & 1u)) atomicOr(&a.named[key / 32u], 1u << (key % 32u));
    }
  }
}

// One thread a column of a piece: runs of one id, added up in order.  Blocks behind the pieces': rows that no id names.
template <typename T, typename O>
__global__ __launch_bounds__(kBlock) void lt_embedding_sum_kernel(const EmbedGradArgs a) {
  const uint32_t tiles = (a.dim + kBlock - 1u) / kBlock;
  uint32_t unit = blockIdx.x / tiles;
  const uint32_t d = (blockIdx.x % tiles) * kBlock + threadIdx.x;
  if (d >= a.dim) return;
  const O* base = (const O*)a.base;
  O* out = (O*)a.out;
  if (unit >= a.pieces) {   // sixteen rows
    if (a.in_place) return;
    for (uint32_t r = (unit - a.pieces) * 16u, end = min(r + 16u, a.rows); r < end; ++r)
      if (!a.named || !(a.named[r / 32u] >> (r % 32u) & 1u)) out[(uint64_t)r * a.dim + d] = base ? base[(uint64_t)r * a.dim + d] : (O)0.0f;
    return;
  }
  const uint32_t begin = unit * a.piece, end = min(begin + a.piece, a.tokens);
  float* parts = a.parts + (uint64_t)unit * 2u * a.dim + d;
  const O* from = a.in_place ? out : base;
  for (uint32_t i = begin; i < end;) {
    const uint32_t key = a.key[i];
    if (key >= a.rows) break;
    const bool begins = i > begin || begin == 0u || a.key[begin - 1u] != key;
    float sum = 0.0f;
    do sum += (float)((const T*)a.dy)[(uint64_t)a.pos[i] * a.dim + d];
    while (++i < end && a.key[i] == key);
    const bool ends = i < end || end == a.tokens || a.key[end] != key;
    const uint64_t at = (uint64_t)key * a.dim + d;
    if (begins && ends) out[at] = (O)((from ? (float)from[at] : 0.0f) + a.scale * sum);
    else parts[begins ? a.dim : 0u] = sum;
  }
}

// A row that a piece begins and shares with the next: the pieces' sums in order.
template <typename O>
__global__ __launch_bounds__(kBlock) void lt_embedding_join_kernel(const EmbedGradArgs a) {
  const uint32_t tiles = (a.dim + kBlock - 1u) / kBlock;
  const uint32_t piece = blockIdx.x / tiles, d = (blockIdx.x % tiles) * kBlock + threadIdx.x;
  const uint32_t begin = piece * a.piece;
  uint32_t next = begin + a.piece;
  if (d >= a.dim || next >= a.tokens) return;
  const uint32_t key = a.key[next];
  if (key >= a.rows || a.key[next - 1u] != key || (begin > 0u && a.key[begin] == key && a.key[begin - 1u] == key)) return;
  const float* parts = a.parts + (uint64_t)piece * 2u * a.dim + d;
  float sum = parts[a.dim];
  do {
    parts += 2u * a.dim;
    sum += parts[0];
    next += a.piece;
  } while (next < a.tokens && a.key[next] == key);
  O* out = (O*)a.out;
  const O* from = a.in_place ? out : (const O*)a.base;
  const uint64_t at = (uint64_t)key * a.dim + d;
  out[at] = (O)((from ? (float)from[at] : 0.0f) + a.scale * sum);
}

template <typename T, typename O>
hipError_t launch_sums(const EmbedGradArgs& a, hipStream_t s) {
  const uint64_t tiles = (a.dim + kBlock - 1u) / kBlock;
  if (a.pass == kEmbedJoin) {
    const uint64_t grid = tiles * a.pieces;
    if (grid * kBlock >= (uint64_t)1 << 32) return hipErrorInvalidValue;
    LT_LAUNCH(lt_embedding_join_kernel<O>, dim3((uint32_t)grid), dim3(kBlock), s, a);
    return hipGetLastError();
  }
  const uint64_t grid = tiles * (a.pieces + (a.in_place ? 0u : (a.rows + 15u) / 16u));
  if (grid == 0) return hipSuccess;
  if (grid * kBlock >= (uint64_t)1 << 32) return hipErrorInvalidValue;
  LT_LAUNCH((lt_embedding_sum_kernel<T, O>), dim3((uint32_t)grid), dim3(kBlock), s, a);
  return hipGetLastError();
}

hipError_t launch_embedding_grad(const void* args, hipStream_t s) {
  const EmbedGradArgs& a = *(const EmbedGradArgs*)args;
  if ((uint64_t)a.rows * a.dim == 0) return hipSuccess;
  if (a.pass == kEmbedCount || a.pass == kEmbedMove) {
    if (a.tokens == 0 || a.bits > kEmbedMaxBits || a.blocks == 0 || a.blocks > kEmbedBlocks || a.each % kEmbedBlock != 0 || (uint64_t)a.each * a.blocks < a.tokens) return hipErrorInvalidValue;
    if (a.pass == kEmbedCount) LT_LAUNCH(lt_embedding_count_kernel, dim3(a.blocks), dim3(kEmbedBlock), s, a);
    else LT_LAUNCH(lt_embedding_move_kernel, dim3(a.blocks), dim3(kEmbedBlock), s, a);
    return hipGetLastError();
  }
  if (a.dtype == kF32) return a.out_dtype == kF32 ? launch_sums<float, float>(a, s) : launch_sums<float, __bf16>(a, s);
  return a.out_dtype == kF32 ? launch_sums<__bf16, float>(a, s) : launch_sums<__bf16, __bf16>(a, s);
}

const bool registered = set_operator(kOpEmbedding, launch_embedding), registered_grad = set_operator(kOpEmbeddingGrad, launch_embedding_grad);

}  // namespace
}  // namespace ltk
