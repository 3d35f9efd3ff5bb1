// Rotary positions: out[t][h] = x[t][h] with its first n elements rotated, pair by pair, by an angle that the token's
// position and the pair's frequency give, and the rest as it is; the gradient turns back.
//
// Bound by memory: every element is read and written once.  16 bytes a lane where rows allow, up to four rows of a thread on
// their way while the workgroup computes its tokens' turns (lt_rotary.h).  65536 tokens of 32 x 128 bf16: 172 us, 6.2 TB/s (one thread
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

enum Past { kNothingPast, kReadsPast, kAllPast };

template <typename T, int V, bool IL, Past PAST>
__global__ __launch_bounds__(kRowBlock) void lt_rope_kernel(const RopeArgs a) {
  __shared__ Turn turns[kMaxTurns];
  const uint32_t pairs = a.rotary.dims / 2u, lane = divide(a.slots, threadIdx.x), u = threadIdx.x - lane * a.slots.d, lanes = kRowBlock / a.slots.d;
  const uint64_t row0 = (uint64_t)blockIdx.x * (lanes * a.rows_each), rows = a.tokens * a.heads.d;
  const uint32_t n = (uint32_t)(rows - row0 < (uint64_t)lanes * a.rows_each ? rows - row0 : (uint64_t)lanes * a.rows_each);
  const uint32_t token0 = rows < 0x7fffffffu ? divide(a.heads, (uint32_t)row0) : (uint32_t)(row0 / a.heads.d), head0 = (uint32_t)(row0 - (uint64_t)token0 * a.heads.d);
  bool turned;
  const uint32_t at = slot_at<V, IL>(a.rotary, u, &turned);
  Slot<T, V, IL> s[kMaxRows];
  uint32_t token[kMaxRows];
#pragma unroll
  for (int i = 0; i < kMaxRows; ++i) {
    const uint32_t r = lane + i * lanes;
    token[i] = divide(a.heads, head0 + r);   // (after the first)
    if (r >= n || lane >= lanes) continue;
    const uint32_t h = head0 + r - token[i] * a.heads.d, t = token0 + token[i], o = a.s_outer == 0 ? 0u : divide(a.inner, t);
    const T* row = (const T*)a.x + (int64_t)o * a.s_outer + (int64_t)(a.whole ? t : t - divide(a.inner, t) * a.inner.d) * a.s_inner + (int64_t)h * a.s_head;
    load_slot<T, V, IL, PAST != kNothingPast>(row, a.rotary, at, turned, &s[i]);
  }
  const uint32_t tokens = divide(a.heads, head0 + n - 1u) + 1u;
  for (uint32_t i = threadIdx.x; i < tokens * pairs; i += kRowBlock) {
    const uint32_t k = divide(a.pairs, i), t = token0 + k;
    turns[i] = turn_of(a.rotary, a.positions[t - divide(a.n_pos, t) * a.n_pos.d], i - k * pairs);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMaxRows; ++i) {
    const uint32_t r = lane + i * lanes;
    if (r >= n || lane >= lanes) continue;
    store_slot<T, T, V, IL, PAST == kAllPast>((T*)a.out + (row0 + r) * a.dim, a.rotary, at, turned, s[i], turns + token[i] * pairs);
  }
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
void launch_rows(const RopeArgs& a, uint32_t grid, Past past, hipStream_t s) {
  if (past == kAllPast) LT_LAUNCH((lt_rope_kernel<T, V, IL, kAllPast>), dim3(grid), dim3(kRowBlock), s, a);
  else if (past == kReadsPast) LT_LAUNCH((lt_rope_kernel<T, V, IL, kReadsPast>), dim3(grid), dim3(kRowBlock), s, a);
  else LT_LAUNCH((lt_rope_kernel<T, V, IL, kNothingPast>), dim3(grid), dim3(kRowBlock), s, a);
}

template <typename T>
hipError_t launch_rope_of(RopeArgs a, hipStream_t s) {
  const uint64_t rows = a.tokens * a.heads.d, aligned = row_alignment(a.x, sizeof(T), a.s_outer, a.s_inner, a.s_head);
  const uint32_t v = piece_of(a.rotary, a.dim, aligned, 16u / sizeof(T)), slots = v ? slots_of(a.rotary, a.dim, v) : 0u, pairs = a.rotary.dims / 2u;
  const uint64_t bytes = rows * a.dim * sizeof(T), cache = (uint64_t)256 << 20;
  const Past past = bytes >= cache ? kAllPast : 2 * bytes >= cache ? kReadsPast : kNothingPast;
  // rows a thread: four where that leaves four workgroups a compute unit, and the tokens' turns fit
  a.rows_each = past == kNothingPast ? kMaxRows : 2u;
  if (v && slots <= kRowBlock) {
    const uint32_t lanes = kRowBlock / slots;
    auto tokens = [&](uint32_t each) { return (lanes * each + a.heads.d - 2u) / a.heads.d + 1u; };
    while (a.rows_each > 1u && (rows / (lanes * a.rows_each) < 1024u || tokens(a.rows_each) * pairs > kMaxTurns)) a.rows_each /= 2u;
    if (tokens(a.rows_each) * pairs <= kMaxTurns) {
      a.slots.set(slots);
      a.pairs.set(pairs);
      const uint64_t grid = (rows + lanes * a.rows_each - 1) / (lanes * a.rows_each);
      if (grid < ((uint64_t)1 << 31)) {
        if (a.rotary.interleaved) {
          if (v * sizeof(T) == 16u) launch_rows<T, 16 / sizeof(T), true>(a, (uint32_t)grid, past, s);
          else if (v == 4u) launch_rows<T, 4, true>(a, (uint32_t)grid, past, s);
          else launch_rows<T, 2, true>(a, (uint32_t)grid, past, s);
        } else {
          if (v * sizeof(T) == 16u) launch_rows<T, 16 / sizeof(T), false>(a, (uint32_t)grid, past, s);
          else if (v == 4u) launch_rows<T, 4, false>(a, (uint32_t)grid, past, s);
          else if (v == 2u) launch_rows<T, 2, false>(a, (uint32_t)grid, past, s);
          else launch_rows<T, 1, false>(a, (uint32_t)grid, past, s);
        }
        return hipGetLastError();
      }
    }
  }
  const uint64_t n = (rows * (a.dim - pairs) + kRowBlock - 1) / kRowBlock;
  LT_LAUNCH(lt_rope_any_kernel<T>, dim3((uint32_t)(n < 65536u ? n : 65536u)), dim3(kRowBlock), s, a);
  return hipGetLastError();
}

hipError_t launch_rope(const void* args, hipStream_t s) {
  const RopeArgs& a = *(const RopeArgs*)args;
  if (a.tokens * a.heads.d * a.dim == 0) return hipSuccess;
  if (!a.x || !a.positions || !a.out || a.inner.d == 0 || a.n_pos.d == 0 || a.rotary.dims > a.dim || a.rotary.dims > 2u * kMaxPairs) return hipErrorInvalidValue;
  return a.dtype == kF32 ? launch_rope_of<float>(a, s) : a.dtype == kBF16 ? launch_rope_of<__bf16>(a, s) : hipErrorInvalidValue;
}

const bool registered = set_operator(kOpRope, launch_rope);

}  // namespace
}  // namespace ltk
