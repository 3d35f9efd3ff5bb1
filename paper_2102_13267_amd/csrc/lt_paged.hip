// A paged cache of keys and values: new rows written into it (the keys rotated by their positions on the way), and
// the attention of one new token a sequence over what the sequence has in it.
//
// The cache is [pages][2][key heads][rows][dim]; sequence s holds position p in row p % rows of page table[s][p / rows].
// What lengths and tables say is checked here, key by key: nothing outside the cache is read or written.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lt_launch.h"
#include "lt_interp.h"
#include "lt_reduce.h"
#include "lt_rotary.h"

namespace ltk {
namespace {

constexpr uint32_t kBlock = 256;
constexpr float kLog2e = 1.44269504088896340736f;

// ---- new rows ------------------------------------------------------------------------------------
// Bound by memory for prompts, by latency for single tokens: a workgroup has all rows (keys and values, head by head) of a few tokens
// on their way while it finds out where these go and computes their turns.  8 prompts of up to 2048 tokens, 8 key heads of 128 bf16,
// 49 MB: 11.7 us, 4.2 TB/s (one thread a pair, each with a search and a turn of its own, 42); 64 single tokens 4.3 us on the device, less
// than a call costs the host.
typedef uint32_t WordsAny __attribute__((ext_vector_type(4), aligned(2)));   // wherever a window of caches begins
__global__ __launch_bounds__(kBlock) void lt_cache_copy_kernel(const AppendArgs a) {
  const uint64_t n = a.cache_elems * (a.cache_dtype == kF32 ? 4u : 2u), stride = (uint64_t)gridDim.x * kBlock * 16u;
  for (uint64_t i = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) * 16u; i < n; i += stride) {
    if (i + 16u <= n) *(WordsAny*)((char*)a.cache + i) = *(const WordsAny*)((const char*)a.copy_from + i);
    else
      for (uint64_t k = i; k < n; k += 2u) *(uint16_t*)((char*)a.cache + k) = *(const uint16_t*)((const char*)a.copy_from + k);
  }
}

// The sequence that token t belongs to, found by a wave together: the last one whose offset is not behind t.  Offsets that decrease lead
// to some sequence, never out of the table.
__device__ __forceinline__ uint32_t sequence_of(const AppendArgs& a, uint32_t t) {
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t lo = 0, n = a.seqs + 1u;
  while (n > 1u) {
    const uint32_t step = (n + 63u) / 64u, j = lo + lane * step;
    const uint32_t before = (uint32_t)__popcll(__ballot(lane * step < n && (int64_t)a.offsets[lane * step < n ? j : lo] <= (int64_t)t));
    if (before == 0u) break;
    const uint32_t skip = (before - 1u) * step;
    lo += skip;
    n = min(step, n - skip);
  }
  return lo;
}

// Where token t of sequence s goes: its position, and the place of its first key in the cache (elements); false: nowhere.
__device__ __forceinline__ bool place(const AppendArgs& a, uint32_t t, uint32_t s, int32_t* position, int64_t* at) {
  if (s >= a.seqs) return false;
  int64_t pos = (int64_t)a.lengths[s] - 1;
  if (a.offsets) {
    const int64_t from = a.offsets[s], to = a.offsets[s + 1u];
    if ((int64_t)t < from || (int64_t)t >= to) return false;
    pos += 1 - to + t;
  }
  if (pos < 0 || pos >= (int64_t)a.slots * a.rows.d) return false;
  const uint32_t slot = divide(a.rows, (uint32_t)pos);
  const int32_t p = a.table[(uint64_t)s * a.slots + slot];
  if (p < 0 || (uint32_t)p >= a.pages) return false;
  *position = (int32_t)pos;
  *at = ((int64_t)p * 2 * a.heads * a.rows.d + ((uint32_t)pos - slot * a.rows.d)) * a.dim;
  return true;
}

constexpr uint32_t kMaxTokens = 256;   // of a workgroup

template <typename C, typename T, int V, bool IL>
__device__ __forceinline__ void append_rows(const AppendArgs& a, Turn* turns) {
  __shared__ int64_t to[kMaxTokens];
  __shared__ int32_t position[kMaxTokens];
  __shared__ uint32_t sequence[kMaxTokens];
  const uint32_t pairs = a.rotary.dims / 2u, lane = divide(a.slots_each, threadIdx.x), u = threadIdx.x - lane * a.slots_each.d, lanes = kBlock / a.slots_each.d;
  // rows: token by token its keys' heads, then its values'
  const uint64_t row0 = (uint64_t)blockIdx.x * (lanes * a.rows_each), rows = (uint64_t)a.tokens * a.token_rows.d;
  const uint32_t n = (uint32_t)(rows - row0 < (uint64_t)lanes * a.rows_each ? rows - row0 : (uint64_t)lanes * a.rows_each);
  const uint32_t token0 = rows < 0x7fffffffu ? divide(a.token_rows, (uint32_t)row0) : (uint32_t)(row0 / a.token_rows.d), first = (uint32_t)(row0 - (uint64_t)token0 * a.token_rows.d);
  const uint32_t tokens = divide(a.token_rows, first + n - 1u) + 1u;
  bool turned;
  const uint32_t at = slot_at<V, IL>(a.rotary, u, &turned);
  Slot<T, V, IL> s[kMaxRows];
  uint32_t token[kMaxRows], head[kMaxRows];
#pragma unroll
  for (int i = 0; i < kMaxRows; ++i) {
    const uint32_t r = first + lane + i * lanes;
    token[i] = divide(a.token_rows, r);   // (after the first)
    head[i] = r - token[i] * a.token_rows.d;
    if (lane + i * lanes >= n || lane >= lanes) continue;
    const int64_t t = token0 + token[i];
    const T* row = head[i] < a.heads ? (const T*)a.k + t * a.k_token + (int64_t)head[i] * a.k_head : (const T*)a.v + t * a.v_token + (int64_t)(head[i] - a.heads) * a.v_head;
    load_slot<T, V, IL, false>(row, a.rotary, at, turned, &s[i]);
  }
  if (a.offsets) {
    for (uint32_t i = threadIdx.x >> 6; i < tokens; i += kBlock / 64u) {
      const uint32_t q = sequence_of(a, token0 + i);
      if ((threadIdx.x & 63u) == 0u) sequence[i] = q;
    }
    __syncthreads();
  }
  for (uint32_t i = threadIdx.x; i < tokens; i += kBlock) {
    int32_t p = 0;
    int64_t where = -1;
    if (!place(a, token0 + i, a.offsets ? sequence[i] : token0 + i, &p, &where)) where = -1;
    position[i] = p;
    to[i] = where;
  }
  __syncthreads();
  if (pairs > 0u) {
    for (uint32_t i = threadIdx.x; i < tokens * pairs; i += kBlock) {
      const uint32_t k = divide(a.pairs, i);
      turns[i] = turn_of(a.rotary, position[k], i - k * pairs);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kMaxRows; ++i) {
    if (lane + i * lanes >= n || lane >= lanes) continue;
    const int64_t where = to[token[i]];
    if (where < 0) continue;
    // (a page's keys, head by head, are followed by its values)
    C* row = (C*)a.cache + where + (int64_t)head[i] * a.rows.d * a.dim;
    store_slot<C, T, V, IL, false>(row, a.rotary, at, turned, s[i], pairs > 0u && head[i] < a.heads ? turns + token[i] * pairs : nullptr);
  }
}

// RIDE: the workgroups behind the first `append_grid` rotate (AppendArgs::rope): a step for 32 sequences 27.6 us, in two launches 30.6.
template <typename C, typename T, int V, bool IL, bool RIDE>
__global__ __launch_bounds__(kBlock) void lt_cache_append_kernel(const AppendArgs a) {
  __shared__ Turn turns[kMaxTurns];
  if (!RIDE || blockIdx.x < a.append_grid) append_rows<C, T, V, IL>(a, turns);
  else if constexpr (RIDE) rope_rows<T, V, IL, kNothingPast>(a.rope, blockIdx.x - a.append_grid, turns);
}

// Rows that the above does not take: interleaved pairs at odd places, rows of very many slots.  One thread per pair (or element of the rest).
template <typename C, typename T>
__global__ __launch_bounds__(kBlock) void lt_cache_append_any_kernel(const AppendArgs a) {
  const uint32_t half = a.rotary.dims / 2u, unit = a.dim - half;
  const uint64_t n = (uint64_t)a.tokens * a.token_rows.d * unit, stride = (uint64_t)gridDim.x * kBlock;
  for (uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += stride) {
    const uint32_t u = (uint32_t)(i % unit), h = (uint32_t)(i / unit % a.token_rows.d), t = (uint32_t)(i / unit / a.token_rows.d);
    uint32_t lo = 0, hi = a.seqs;   // offsets[lo] <= t (or lo = 0), offsets[hi] > t (or hi = seqs)
    while (a.offsets && hi - lo > 1u) {
      const uint32_t mid = (lo + hi) / 2u;
      if ((int64_t)a.offsets[mid] <= (int64_t)t) lo = mid;
      else hi = mid;
    }
    int32_t position;
    int64_t where;
    if (!place(a, t, a.offsets ? lo : t, &position, &where)) continue;
    const T* x = h < a.heads ? (const T*)a.k + (int64_t)t * a.k_token + (int64_t)h * a.k_head : (const T*)a.v + (int64_t)t * a.v_token + (int64_t)(h - a.heads) * a.v_head;
    C* y = (C*)a.cache + where + (int64_t)h * a.rows.d * a.dim;
    if (u >= half) {
      y[half + u] = (C)to_float(x[half + u]);
      continue;
    }
    const uint32_t p = a.rotary.interleaved ? 2u * u : u, q = a.rotary.interleaved ? 2u * u + 1u : u + half;
    float v = to_float(x[p]), w = to_float(x[q]);
    if (h < a.heads) rotate(turn_of(a.rotary, position, u), v, w, &v, &w);
    y[p] = (C)v;
    y[q] = (C)w;
  }
}

template <typename C, typename T, int V, bool IL>
void launch_append_rows(const AppendArgs& a, bool ride, uint32_t workgroups, hipStream_t s) {
  if constexpr (sizeof(C) == sizeof(T)) {
    if (ride) {
      LT_LAUNCH((lt_cache_append_kernel<C, T, V, IL, true>), dim3(workgroups), dim3(kBlock), s, a);
      return;
    }
  }
  LT_LAUNCH((lt_cache_append_kernel<C, T, V, IL, false>), dim3(workgroups), dim3(kBlock), s, a);
}

template <typename C, typename T>
hipError_t launch_append_of(AppendArgs a, bool* rode, hipStream_t s) {
  constexpr uint32_t kMost = 16u / (sizeof(C) > sizeof(T) ? sizeof(C) : sizeof(T));
  const uint64_t rows = (uint64_t)a.tokens * a.token_rows.d;
  const uint64_t aligned =
      std::min(row_alignment(a.cache, sizeof(C), 0, 0, 0), std::min(row_alignment(a.k, sizeof(T), a.k_token, a.k_head, 0), row_alignment(a.v, sizeof(T), a.v_token, a.v_head, 0)));
  const uint32_t v = piece_of(a.rotary, a.dim, aligned, kMost), slots = v ? slots_of(a.rotary, a.dim, v) : 0u, pairs = a.rotary.dims / 2u;
  a.rows_each = kMaxRows;
  if (v && slots <= kBlock) {
    const uint32_t lanes = kBlock / slots;
    auto tokens = [&](uint32_t each) { return (lanes * each + a.token_rows.d - 2u) / a.token_rows.d + 1u; };
    auto fits = [&](uint32_t each) { return tokens(each) * pairs <= kMaxTurns && tokens(each) <= kMaxTokens; };
    while (a.rows_each > 1u && (rows / (lanes * a.rows_each) < kRowGrid || !fits(a.rows_each))) a.rows_each /= 2u;
    const uint64_t grid = (rows + lanes * a.rows_each - 1) / (lanes * a.rows_each);
    if (fits(a.rows_each) && grid < kMostGrid) {
      a.slots_each.set(slots);
      a.pairs.set(pairs ? pairs : 1u);
      a.append_grid = (uint32_t)grid;
      // a rotation of the same type and layout, in pieces of the same size, takes the launch's other workgroups
      RopeLayout l{};
      if constexpr (sizeof(C) == sizeof(T))
        *rode = a.rope.out && a.rope.dtype == a.dtype && a.rope.rotary.interleaved == a.rotary.interleaved && fit_to_run(a.rope) &&
                lay_out(&a.rope, sizeof(T), &l) && l.v == v && l.past == kNothingPast && grid + l.grid < kMostGrid;
      const uint32_t workgroups = a.append_grid + (*rode ? l.grid : 0u);
      if (a.rotary.interleaved) {
        if (v == kMost) launch_append_rows<C, T, kMost, true>(a, *rode, workgroups, s);
        else if (v == 4u) launch_append_rows<C, T, 4, true>(a, *rode, workgroups, s);
        else launch_append_rows<C, T, 2, true>(a, *rode, workgroups, s);
      } else {
        if (v == kMost) launch_append_rows<C, T, kMost, false>(a, *rode, workgroups, s);
        else if (v == 4u) launch_append_rows<C, T, 4, false>(a, *rode, workgroups, s);
        else if (v == 2u) launch_append_rows<C, T, 2, false>(a, *rode, workgroups, s);
        else launch_append_rows<C, T, 1, false>(a, *rode, workgroups, s);
      }
      return hipGetLastError();
    }
  }
  const uint64_t n = (rows * (a.dim - pairs) + kBlock - 1) / kBlock;
  LT_LAUNCH((lt_cache_append_any_kernel<C, T>), dim3((uint32_t)(n < 65536u ? n : 65536u)), dim3(kBlock), s, a);
  return hipGetLastError();
}

hipError_t launch_new_rows(const AppendArgs& a, bool* rode, hipStream_t s) {
  if (a.cache_elems == 0) return hipSuccess;
  if (!a.cache || a.rows.d == 0 || a.token_rows.d != 2u * a.heads || a.rotary.dims > a.dim || a.rotary.dims > 2u * kMaxPairs) return hipErrorInvalidValue;
  if (a.copy_from) {
    const uint64_t pieces = (a.cache_elems + 2047u) / 2048u;
    LT_LAUNCH(lt_cache_copy_kernel, dim3((uint32_t)(pieces < 16384u ? pieces : 16384u)), dim3(kBlock), s, a);
  }
  if (a.tokens == 0 || a.seqs == 0 || a.slots == 0) return hipGetLastError();
  if (!a.k || !a.v || !a.lengths || !a.table) return hipErrorInvalidValue;
  if (a.cache_dtype == kF32 && a.dtype == kF32) return launch_append_of<float, float>(a, rode, s);
  if (a.cache_dtype == kF32 && a.dtype == kBF16) return launch_append_of<float, __bf16>(a, rode, s);
  if (a.cache_dtype == kBF16 && a.dtype == kF32) return launch_append_of<__bf16, float>(a, rode, s);
  if (a.cache_dtype == kBF16 && a.dtype == kBF16) return launch_append_of<__bf16, __bf16>(a, rode, s);
  return hipErrorInvalidValue;
}

// (a rotation that cannot share the launch gets its own)
hipError_t launch_append(const void* args, hipStream_t s) {
  const AppendArgs& a = *(const AppendArgs*)args;
  bool rode = false;
  const hipError_t e = launch_new_rows(a, &rode, s);
  if (e != hipSuccess || rode || !a.rope.out) return e;
  return launch_operator(kOpRope, &a.rope, s);
}

// ---- attention of one new token -------------------------------------------------------------------
// Every key and value is read once, for all query heads of its key head together: what bounds it is memory, so that the arithmetic is
// given to the matrix cores, where sixteen heads cost what one does, and nothing goes through LDS on its way there.
//
// A wave takes steps of WK keys (bf16 32, fp32 16).  Scores transposed, s = K q^T (MFMA 16x16: A 16 keys, B 16 query heads, which stay in
// registers): lane (n, g), n = lane & 15, g = lane / 16, reads 16-byte pieces of key n's row, and of the result holds keys
// 4 g .. 4 g + 3 of a tile for head n.  So a head's maximum is a maximum over registers and two exchanges between lanes, and o = V^T p takes
// the weights as they lie: which key an MFMA's k stands for is free as long as both operands agree, so lane (n, g) holds in B what it
// computed and reads for A the rows of the same keys, 1 / 16 of a row of dim elements each (bf16: two rows' halves are put together by
// v_perm_b32).  The accumulator has head n in lane n, so that rescaling by a new maximum is a product in place.  K of the
// next step is on its way while this one's weights are computed, V of this one too.
//
// The matrix cores take bf16 weights with bf16 values, so a weight meets its value as two numbers, its upper half and what that leaves, rounded: 2^-15
// of it is lost, 1 / 128 of what rounding the result may lose (one rounded number, 2^-8: the largest error of the results 0.0021 instead of 0.0017; us with
// one / two: one sequence of 300 7.3 / 7.5, 60 ragged 74.2 / 74.2, one of 131072 86.7 / 86.8, a step for 32 sequences 27.6 / 27.8).
//
// Four waves share a tile of 4 WK keys; their maxima, sums and products meet in LDS at the end.
//
// A workgroup has one chunk of a sequence, for one block of up to 16 NH query heads of a key head (PagedArgs has how long chunks are).
// A sequence's chunks are of equal length, so that a long one among short ones holds nobody up.  Pieces of a block meet in memory
// (relaxed accesses of device scope, as the reductions exchange theirs), and whoever comes last joins them in their order: up
// to 32 at once, more in groups of about their root, whose last ones then join the groups.  So results do not depend on
// who comes when.
//
// 32 query heads, 8 key heads of 128 bf16: one sequence of 131072 keys, 537 MB, 86 us, 6.2 TB/s; 60 sequences of 256 to 4096 74 us, 4.7 TB/s
// (workgroups whose waves happen to run late hold up the end, 15 to 20 us of it); one of 300 7.5 us, of which the chain length, page, keys,
// softmax, join takes most.  fp32, 7 sequences of up to 3001, 4 key heads of 80: 13.0 us.  One workgroup per sequence and query head: 63749, 2070, 70 and 805.
template <typename T, int DP, int NH> struct Geo {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int KT = BF ? 2 : 1;              // tiles of 16 keys in a wave's step
  static constexpr int WK = 16 * KT, TILE = 4 * WK;
  static constexpr int CE = 16 / (int)sizeof(T);     // elements of 16 bytes
  static constexpr int NC = DP / (4 * CE);           // 16-byte pieces of a key's row per lane
  static constexpr int NV = DP / 16;                 // elements of a value's row per lane
  // bytes of a piece of it (96 and 160: of two elements, so that none ends behind a head of an even number of them), their number, and dwords of one
  static constexpr int VB = DP == 32 || DP == 96 || DP == 160 ? 2 * (int)sizeof(T) : NV * (int)sizeof(T) % 16 == 0 ? 16 : 8;
  static constexpr int NP = NV * (int)sizeof(T) / VB, DW = VB / 4;
  static constexpr int PITCH = DP + 4;
};

typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef uint32_t U2 __attribute__((ext_vector_type(2)));
typedef float F4 __attribute__((ext_vector_type(4)));
typedef float F2 __attribute__((ext_vector_type(2)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef __bf16 B2 __attribute__((ext_vector_type(2)));

constexpr int kSlots = 1024;   // page numbers of a stretch of a sequence that a workgroup holds

// PAST: read past the last-level cache, for what will not be found there the next time either
template <int BYTES, bool PAST = false> __device__ __forceinline__ U4 load_bytes(const void* p) {
  U4 r = {0u, 0u, 0u, 0u};
  if constexpr (BYTES == 16) r = PAST ? __builtin_nontemporal_load((const U4*)p) : *(const U4*)p;
  else if constexpr (BYTES == 8) {
    const U2 t = PAST ? __builtin_nontemporal_load((const U2*)p) : *(const U2*)p;
    r.x = t.x;
    r.y = t.y;
  } else r.x = PAST ? __builtin_nontemporal_load((const uint32_t*)p) : *(const uint32_t*)p;
  return r;
}

typedef U4 U4Any __attribute__((aligned(2)));   // wherever elements are
typedef U2 U2Any __attribute__((aligned(2)));
typedef uint32_t U1Any __attribute__((aligned(2)));

// BYTES of a row from element d on.  AL 16: a row is made of such pieces; what is behind its end is read from its beginning.  kWide: a row of 16 bytes and
// more that starts anywhere and ends inside a piece; KEY: read across the row's end, as values lie behind every key (otherwise from further
// back, so that the last row's end is the last that is read, and moved down).  Elements behind dim are anything.  2 or 4: row by element.
constexpr int kWide = 0;
template <typename T, int BYTES, int AL, bool KEY>
__device__ __forceinline__ U4 load_piece(const T* row, uint32_t d, uint32_t dim) {
  if constexpr (AL >= BYTES) return load_bytes<BYTES>(row + (d < dim ? d : 0u));
  U4 r = {0u, 0u, 0u, 0u};
  if constexpr (AL == kWide && KEY) r = *(const U4Any*)(row + (d < dim ? d : 0u));
  else if constexpr (AL == kWide && BYTES == 4) {
    constexpr uint32_t kEach = 4 / sizeof(T);
    const uint32_t at = min(d, dim - kEach), back = (d - at) * 8u * (uint32_t)sizeof(T);
    r.x = *(const U1Any*)(row + at) >> (back & 31u);
  } else if constexpr (AL == kWide) {
    constexpr uint32_t kEach = 8 / sizeof(T);
#pragma unroll
    for (uint32_t i = 0; i < BYTES / 8u; ++i) {
      const uint32_t e = d + i * kEach, at = min(e, dim - kEach), back = (e - at) * 8u * (uint32_t)sizeof(T);
      const U2 t = *(const U2Any*)(row + at);
      const uint64_t v = ((uint64_t)t.y << 32 | t.x) >> (back & 63u);
      r[2 * i] = (uint32_t)v;
      r[2 * i + 1] = (uint32_t)(v >> 32);
    }
  } else {
#pragma unroll
    for (int i = 0; i < BYTES / AL; ++i) {
      const uint32_t e = d + (uint32_t)(i * AL / (int)sizeof(T));
      const T* p = row + (e < dim ? e : 0u);
      if constexpr (AL == 4) r[i] = *(const uint32_t*)p;
      else r[i / 2] |= (uint32_t)*(const uint16_t*)p << (16 * (i & 1));
    }
  }
  return r;
}

// Zeros in place of the elements from dim on: they count nothing, next to infinities too.
template <typename T, int AL>
__device__ __forceinline__ U4 cut(U4 v, uint32_t d, uint32_t dim) {
  constexpr uint32_t kEach = 4 / sizeof(T);
  if constexpr (AL == 16) return d < dim ? v : U4{0u, 0u, 0u, 0u};
#pragma unroll
  for (uint32_t e = 0; e < 4u; ++e) {
    if (d + e * kEach >= dim) v[e] = 0u;
    else if (kEach == 2u && d + e * kEach + 1u >= dim) v[e] &= 0xFFFFu;
  }
  return v;
}

// Over the four rows of 16 lanes: neighbouring rows trade places, then halves of the wave.
__device__ __forceinline__ float max_over_groups(float v) {
  auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
  t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}
__device__ __forceinline__ float sum_over_groups(float v) {
  auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(t[0]) + __uint_as_float(t[1]);
  t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}
__device__ __forceinline__ float power2(float v) { return __builtin_amdgcn_exp2f(v); }

__device__ __forceinline__ uint32_t length_of(const PagedArgs& a, uint32_t s) {
  const int32_t n = a.lengths[s];
  return n < 0 ? 0u : (uint32_t)n > a.capacity ? a.capacity : (uint32_t)n;
}

// Tiles of a sequence, one at least: an empty one has zeros to write.
template <uint32_t TILE> __device__ __forceinline__ uint32_t tiles_of(uint32_t len) { return len == 0u ? 1u : (len - 1u) / TILE + 1u; }

// Inclusive sums over the wave, every lane active: shifts inside rows of 16 lanes, then the rows' last lanes.
__device__ __forceinline__ uint32_t sums_over_wave(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);
  return v;
}

__device__ __forceinline__ uint32_t chunk_of(const PagedArgs& a, uint32_t all) { return max(a.least, (all * a.pairs + a.chunks - 1u) / a.chunks); }
__device__ __forceinline__ uint32_t chunks_of(const PagedArgs& a, uint32_t tiles, uint32_t c) { return tiles <= a.whole ? 1u : (tiles + c - 1u) / c; }

// A workgroup's share.
struct Chunk {
  uint32_t seq, len, tiles;      // tiles: of the whole sequence
  uint32_t pair;                 // its block of query heads
  uint32_t part, parts, piece0;  // part of `parts`, whose pieces lie from piece0 on
};

// Found by every wave for itself (four waves that meet at barriers took longer), as sums over the sequences, up to four of them a lane;
// false: there is none for this workgroup.
template <uint32_t TILE>
__device__ __forceinline__ bool find_chunk(const PagedArgs& a, Chunk* w) {
  static_assert(kPagedFind <= 4 * 64, "lengths stay in registers");
  const uint32_t lane = threadIdx.x & 63u, each = (a.seqs + 63u) / 64u, from = lane * each;
  uint32_t len[4], tiles = 0;
#pragma unroll
  for (uint32_t i = 0; i < 4u; ++i) len[i] = i < each && from + i < a.seqs ? length_of(a, from + i) : 0u;
  const uint32_t mine = from < a.seqs ? min(each, a.seqs - from) : 0u;
#pragma unroll
  for (uint32_t i = 0; i < 4u; ++i) tiles += i < mine ? tiles_of<TILE>(len[i]) : 0u;
  const uint32_t c = chunk_of(a, (uint32_t)__builtin_amdgcn_readlane((int)sums_over_wave(tiles), 63));
  uint32_t k[4], chunks = 0, split = 0;
#pragma unroll
  for (uint32_t i = 0; i < 4u; ++i) {
    k[i] = i < mine ? chunks_of(a, tiles_of<TILE>(len[i]), c) : 0u;
    chunks += k[i];
    split += k[i] > 1u ? k[i] : 0u;
  }
  uint32_t before = sums_over_wave(chunks) - chunks, split_before = sums_over_wave(split) - split;
  const uint32_t at = blockIdx.x;
  const uint64_t here = __ballot(before * a.pairs <= at && at < (before + chunks) * a.pairs);
  if (here == 0u) return false;
  uint32_t i = 0, n = len[0], parts = k[0];
#pragma unroll
  for (uint32_t j = 1; j < 4u; ++j) {
    const bool behind = j < mine && at >= (before + parts) * a.pairs;   // (stays false once it is)
    before += behind ? parts : 0u;
    split_before += behind && parts > 1u ? parts : 0u;
    i = behind ? j : i;
    n = behind ? len[j] : n;
    parts = behind ? k[j] : parts;
  }
  const int owner = __ffsll((unsigned long long)here) - 1;
  auto of_owner = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, owner); };
  w->seq = of_owner(from + i);
  w->len = of_owner(n);
  w->tiles = tiles_of<TILE>(w->len);
  w->parts = of_owner(parts);
  const uint32_t rel = at - of_owner(before) * a.pairs;
  w->pair = rel / w->parts;
  w->part = rel - w->pair * w->parts;
  w->piece0 = of_owner(split_before) * a.pairs + w->pair * w->parts;
  return true;
}

// Of more than kPagedFind sequences one workgroup writes down the chunks, for every chunk (of all blocks of heads) what the above finds: sequence, length, its
// first chunk's number, and its parts together with the pieces before them in 16 bits each (at most 2 kPagedChunks).  No parts:
// behind the last chunk.
constexpr uint32_t kListBlock = 1024;
__global__ __launch_bounds__(kListBlock) void lt_paged_list_kernel(const PagedArgs a) {
  __shared__ uint32_t sums[3][kListBlock / 64];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, each = (a.seqs + kListBlock - 1u) / kListBlock;
  const uint32_t from = (uint32_t)min((uint64_t)threadIdx.x * each, (uint64_t)a.seqs), to = min(a.seqs, from + each), most = a.listed;
  uint4* list = (uint4*)a.list;
  auto tiles_at = [&](uint32_t s, uint32_t* len) {
    *len = length_of(a, s);
    return *len == 0u ? 1u : (*len - 1u) / a.tile + 1u;
  };
  // what the threads before this one have, and all of them together
  auto before = [&](uint32_t v, uint32_t which, uint32_t* all) {
    const uint32_t sum = sums_over_wave(v);
    if (lane == 63u) sums[which][wave] = sum;
    __syncthreads();
    uint32_t b = 0;
    *all = 0;
#pragma unroll
    for (uint32_t i = 0; i < kListBlock / 64u; ++i) {
      if (i < wave) b += sums[which][i];
      *all += sums[which][i];
    }
    return b + sum - v;
  };
  uint32_t len, tiles = 0, all, chunks = 0, split = 0, total, ignored;
#pragma unroll 4
  for (uint32_t s = from; s < to; ++s) tiles += tiles_at(s, &len);
  before(tiles, 0, &all);
  const uint32_t c = chunk_of(a, all);
#pragma unroll 4
  for (uint32_t s = from; s < to; ++s) {
    const uint32_t k = chunks_of(a, tiles_at(s, &len), c);
    chunks += k;
    split += k > 1u ? k : 0u;
  }
  uint32_t at = before(chunks, 1, &total), pieces = before(split, 2, &ignored);
#pragma unroll 4
  for (uint32_t s = from; s < to; ++s) {
    const uint32_t k = chunks_of(a, tiles_at(s, &len), c);
    for (uint32_t i = 0; i < k; ++i)
      if (at + i < most) list[at + i] = make_uint4(s, len, at, k | pieces << 16);
    at += k;
    pieces += k > 1u ? k : 0u;
  }
  for (uint32_t i = total + threadIdx.x; i < most; i += kListBlock) list[i] = make_uint4(0u, 0u, 0u, 0u);
}

template <uint32_t TILE>
__device__ __forceinline__ bool read_chunk(const PagedArgs& a, Chunk* w) {
  const uint4 e = ((const uint4*)a.list)[blockIdx.x / a.pairs];
  w->parts = e.w & 0xFFFFu;
  if (w->parts == 0u) return false;
  w->seq = e.x;
  w->len = e.y;
  w->tiles = tiles_of<TILE>(w->len);
  const uint32_t rel = blockIdx.x - e.z * a.pairs;
  w->pair = rel / w->parts;
  w->part = rel - w->pair * w->parts;
  w->piece0 = (e.w >> 16) * a.pairs + w->pair * w->parts;
  return true;
}

// A piece: [16 NH heads][DP] sums of weights times values, [16 NH] maxima, [16 NH] sums of weights.
template <int DP, int NH> constexpr uint32_t kPieceFloats = 16 * NH * DP + 32 * NH;
constexpr uint32_t kMostPieces = 32;   // at once; in two steps at most 23 (the root of 512)

// Whether the calling workgroup is the last of `count` to come here.
__device__ __forceinline__ bool last_of(uint32_t* ticket, uint32_t count, uint32_t* flag) {
  all_published();
  __syncthreads();
  if (threadIdx.x == 0u) {
    const bool last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == count - 1u;
    if (last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last ? 1u : 0u;
  }
  __syncthreads();
  return *flag != 0u;
}

// (Waves a SIMD: as many as an instance's registers leave room for without spilling; heads of 256 in half of them: 5000 keys 20.5 -> 23.5 us.)
template <typename T, int DP, int NH, bool PG, int AL, bool PAST>
__global__ __launch_bounds__(kBlock, NH == 1 && (AL == 16 || AL == kWide) ? (DP <= 64 ? 4 : DP <= 128 ? 3 : DP == 160 ? 2 : 1) : 1) void lt_paged_attention_kernel(const PagedArgs a) {
  using G = Geo<T, DP, NH>;
  constexpr int KT = G::KT, NC = G::NC, NV = G::NV, NP = G::NP;
  constexpr uint32_t kSize = sizeof(T);
  __shared__ int32_t pages[PG ? 1 : kSlots];
  __shared__ uint32_t last_flag;
  __shared__ float tops[4][16 * NH], sums[4][16 * NH], factor[kMostPieces][16 * NH], weight_of[kMostPieces][16 * NH], total_of[16 * NH];
  __shared__ __attribute__((aligned(16))) float meet[4][16 * G::PITCH];
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15u, g = lane >> 4;

  Chunk w;
  uint32_t t0, t1;
  if (a.split) {
    if (!(a.listed > 0u ? read_chunk<G::TILE>(a, &w) : find_chunk<G::TILE>(a, &w))) return;
    const uint32_t even = w.tiles / w.parts, odd = w.tiles - even * w.parts;
    t0 = w.part * even + min(w.part, odd);
    t1 = t0 + even + (w.part < odd ? 1u : 0u);
  } else {
    w.seq = blockIdx.x / a.pairs;
    w.pair = blockIdx.x - w.seq * a.pairs;
    w.len = length_of(a, w.seq);
    w.tiles = tiles_of<G::TILE>(w.len);
    w.part = w.piece0 = 0u;
    w.parts = 1u;
    t0 = 0u;
    t1 = w.tiles;
  }
  // PG: the page numbers of a wave's next 64 tiles of 16 keys lie in its lanes, lane KT s + t those of tile t of its step s; the first are
  // asked for before the sequence's length has to be known
  auto pages_from = [&](uint32_t key0) {
    const uint32_t k = key0 + lane / KT * G::TILE + lane % KT * 16u;
    return k < a.capacity ? a.table[(uint64_t)w.seq * a.slots + divide(a.rows, k)] : -1;
  };
  int32_t pages_next = PG ? pages_from(t0 * G::TILE + wave * G::WK) : -1;
  const uint32_t group = a.heads / a.kv_heads, blocks = a.pairs / a.kv_heads, kh = w.pair / blocks, h0 = kh * group + (w.pair - kh * blocks) * 16u * NH,
                 heads = min(16u * NH, (kh + 1u) * group - h0);
  const uint32_t key_end = (uint32_t)min((uint64_t)t1 * G::TILE, (uint64_t)w.len);
  const int64_t value = (int64_t)a.kv_heads * a.rows.d * a.dim;   // from a key to its value

  // B of the scores: lane (n, g) has head n's elements (4 c + g) CE .. + CE - 1; zeros behind the last head and the last element
  U4 q[NH][NC];
#pragma unroll
  for (int b = 0; b < NH; ++b) {
    const uint32_t h = 16u * b + n, to = h < heads ? a.dim : 0u;
    const T* row = (const T*)a.q + (int64_t)w.seq * a.q_seq + (int64_t)(h0 + (h < heads ? h : 0u)) * a.q_head;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const uint32_t d = (4u * c + g) * G::CE;
      if (a.q_whole) q[b][c] = cut<T, 16>(load_piece<T, 16, 16, true>(row, d, to), d, to);
      else q[b][c] = cut<T, (int)sizeof(T)>(load_piece<T, 16, (int)sizeof(T), true>(row, d, to), d, to);
    }
  }

  F4 acc[NH][NV];
  float top[NH], sum[NH];
#pragma unroll
  for (int b = 0; b < NH; ++b) {
    top[b] = -INFINITY;
    sum[b] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) acc[b][j] = F4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const float scale = a.scale * kLog2e;
  // Weights are 2^-spread at most, so that those of all `len` keys add up to less than one, and no sum of theirs with values passes the largest of these.  bf16: the
  // exponents are that much smaller (rounded, 2^-20 of a weight); fp32: the powers are.
  const uint32_t spread = 32u - (uint32_t)__builtin_clz(w.len | 1u);
  const float shift = G::BF ? (float)spread : 0.0f, share = __uint_as_float((127u - spread) << 23);
  // (PG) bytes from a tile's first row to what this lane reads of its own
  const uint32_t key_at = (n * a.dim + g * G::CE) * kSize, key_at0 = g * 16u, value_at0 = (n * NV < a.dim ? n * NV : 0u) * kSize;

  // Where a step's keys lie.  PG: a page holds whole tiles of 16, so a tile has one page: its first row, and how many of its keys there are.
  // Otherwise every lane finds its own keys, and a stretch's page numbers lie in LDS.
  const uint32_t stretch = PG ? 0x7fffffffu / G::TILE : (uint32_t)min((uint64_t)(kSlots - 2) * a.rows.d / G::TILE, (uint64_t)0x7fffffffu / G::TILE);
  for (uint32_t first = t0; first < t1; first += stretch) {
    const uint32_t k0 = first * G::TILE, k1 = (uint32_t)min((uint64_t)first * G::TILE + (uint64_t)stretch * G::TILE, (uint64_t)key_end);
    if (k0 >= k1) break;   // (an empty sequence)
    const uint32_t slot0 = divide(a.rows, k0);
    if constexpr (!PG) {
      const uint32_t n_slots = divide(a.rows, k1 - 1u) - slot0 + 1u;
      if (first != t0) __syncthreads();       // (the stretch before has been read)
      for (uint32_t i = threadIdx.x; i < n_slots; i += kBlock) {
        const int32_t p = a.table[(uint64_t)w.seq * a.slots + slot0 + i];
        pages[i] = p >= 0 && (uint32_t)p < a.pages ? p : -1;
      }
      __syncthreads();
    }
    const uint32_t wave0 = k0 + wave * G::WK;
    int32_t pages_now = -1;
    const char* tile[KT];
    uint32_t there[KT], step = 0;
    auto find_tiles = [&](uint32_t key0) {
      if (step % (64 / KT) == 0u) {
        pages_now = pages_next >= 0 && (uint32_t)pages_next < a.pages ? pages_next : -1;
        pages_next = pages_from(key0 + 64 / KT * G::TILE);
      }
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        const uint32_t k = key0 + 16u * t;
        const int32_t p = __builtin_amdgcn_readlane(pages_now, (int)(step % (64 / KT) * KT + t));
        there[t] = p >= 0 && k < k1 ? min(16u, k1 - k) : 0u;
        tile[t] = (const char*)a.cache + (there[t] > 0u ? (((int64_t)p * 2 * a.kv_heads + kh) * a.rows.d + (k - divide(a.rows, k) * a.rows.d)) * a.dim * kSize : (int64_t)0);
      }
      ++step;
    };
    auto find_row = [&](uint32_t key, bool* ok) {
      const uint32_t slot = divide(a.rows, key);
      const int32_t p = key < k1 ? pages[slot - slot0] : -1;
      *ok = p >= 0;
      return p >= 0 ? (((int64_t)p * 2 * a.kv_heads + kh) * a.rows.d + (key - slot * a.rows.d)) * a.dim : (int64_t)0;
    };
    U4 k[KT][NC];
    // (PG: a piece behind the row's end is the next row's, or the values' behind the last one)
    auto load_keys = [&](uint32_t key0) {
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        if constexpr (PG) {
          const uint32_t at = n < there[t] ? key_at : key_at0;
#pragma unroll
          for (int c = 0; c < NC; ++c) k[t][c] = load_bytes<16, PAST>(tile[t] + at + c * 64);
        } else {
          bool ok;
          const T* row = (const T*)a.cache + find_row(key0 + 16u * t + n, &ok);
#pragma unroll
          for (int c = 0; c < NC; ++c) k[t][c] = load_piece<T, 16, AL, true>(row, (4u * c + g) * G::CE, a.dim);
        }
      }
    };

    uint32_t key0 = wave0;
    if (key0 < k1) {
      if constexpr (PG) find_tiles(key0);
      load_keys(key0);
    }
    for (; key0 < k1; key0 += G::TILE) {
      U4 v[4 * KT][NP];
      uint32_t mine = 0u;   // which of this lane's keys there are
#pragma unroll
      for (int i = 0; i < 4 * KT; ++i) {
        const uint32_t t = i >> 2, r = 4u * g + (i & 3u);
        bool ok;
        if constexpr (PG) {
          ok = r < there[t];
          const uint32_t at = (ok ? r * a.dim * kSize : 0u) + value_at0;
          const char* row = tile[t] + value * kSize;
#pragma unroll
          for (int p = 0; p < NP; ++p) v[i][p] = load_bytes<G::VB, PAST>(row + at + (NP == 1 || n * NV + p * (G::VB / kSize) < a.dim ? p * G::VB : 0));
        } else {
          const T* row = (const T*)a.cache + value + find_row(key0 + 16u * t + r, &ok);
#pragma unroll
          for (int p = 0; p < NP; ++p) v[i][p] = load_piece<T, G::VB, AL, false>(row, n * NV + p * (G::VB / kSize), a.dim);   // (what is behind the end is not stored)
        }
        mine |= ok ? 1u << i : 0u;
      }
      // ---- scores
      if (a.dim != DP) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int c = 0; c < NC; ++c) k[t][c] = cut<T, AL>(k[t][c], (4u * c + g) * G::CE, a.dim);
      }
      F4 s[NH][KT];
#pragma unroll
      for (int b = 0; b < NH; ++b)
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          s[b][t] = F4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if constexpr (G::BF) {
              s[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, k[t][c]), __builtin_bit_cast(B8, q[b][c]), s[b][t], 0, 0, 0);
            } else if (c * 4 * G::CE < (int)a.dim) {   // (pieces wholly behind the head are not multiplied)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                s[b][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[t][c][e]), __uint_as_float(q[b][c][e]), s[b][t], 0, 0, 0);
            }
          }
        }
      if (key0 + G::TILE < k1) {
        if constexpr (PG) find_tiles(key0 + G::TILE);
        load_keys(key0 + G::TILE);
      }
      // ---- weights
      const bool all = __all(mine == (1u << (4 * KT)) - 1u);
#pragma unroll
      for (int b = 0; b < NH; ++b) {
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[b][t][r] *= scale;
            mx = fmaxf(mx, s[b][t][r]);
          }
        if (!all) {
          mx = -INFINITY;
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              s[b][t][r] = mine >> (4 * t + r) & 1u ? s[b][t][r] : -INFINITY;
              mx = fmaxf(mx, s[b][t][r]);
            }
        }
        const float fresh = fmaxf(top[b], max_over_groups(mx) + shift), safe = fresh == -INFINITY ? 0.0f : fresh, keep = power2(top[b] - safe);
        top[b] = fresh;
        float part = 0.0f;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[b][t][r] = power2(s[b][t][r] - safe);
            if constexpr (!G::BF) s[b][t][r] *= share;
            part += s[b][t][r];
          }
        sum[b] = fmaf(sum[b], keep, part);
#pragma unroll
        for (int j = 0; j < NV; ++j) acc[b][j] *= keep;
      }
      // ---- products
      if (!all) {
#pragma unroll
        for (int i = 0; i < 4 * KT; ++i)
#pragma unroll
          for (int p = 0; p < NP; ++p)
            if (!(mine >> i & 1u)) v[i][p] = U4{0u, 0u, 0u, 0u};
      }
      if constexpr (G::BF) {
        B8 weight[NH], rest[NH];
#pragma unroll
        for (int b = 0; b < NH; ++b)
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float x = s[b][i >> 2][i & 3], y = s[b][i >> 2][(i & 3) + 1];
            // (2^-20 of the weight on top: what is left is above zero where the weight is, so that an infinite value stays one)
            const uint32_t hx = __float_as_uint(x) & 0xFFFF0000u, hy = __float_as_uint(y) & 0xFFFF0000u;
            const B2 high = __builtin_bit_cast(B2, __builtin_amdgcn_perm(hy, hx, 0x07060302u));
            weight[b][i] = high[0];
            weight[b][i + 1] = high[1];
            rest[b][i] = (__bf16)fmaf(x, 1.0f + 0x1p-20f, -__uint_as_float(hx));
            rest[b][i + 1] = (__bf16)fmaf(y, 1.0f + 0x1p-20f, -__uint_as_float(hy));
          }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          constexpr uint32_t kLow = 0x05040100u, kHigh = 0x07060302u;
          U4 f;
#pragma unroll
          for (int p = 0; p < 4; ++p)
            f[p] = __builtin_amdgcn_perm(v[2 * p + 1][j / 2 / G::DW][j / 2 % G::DW], v[2 * p][j / 2 / G::DW][j / 2 % G::DW], (j & 1) ? kHigh : kLow);
#pragma unroll
          for (int b = 0; b < NH; ++b) {
            acc[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, f), weight[b], acc[b][j], 0, 0, 0);
            acc[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, f), rest[b], acc[b][j], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int b = 0; b < NH; ++b) acc[b][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[r][j / G::DW][j % G::DW]), s[b][0][r], acc[b][j], 0, 0, 0);
      }
    }
  }

  // ---- the four waves' parts
#pragma unroll
  for (int b = 0; b < NH; ++b) {
    const float all = sum_over_groups(sum[b]);
    if (g == 0u) {
      tops[wave][16 * b + n] = top[b];
      sums[wave][16 * b + n] = all;
    }
  }
  __syncthreads();
  const bool whole = w.parts == 1u;
  auto piece = [&](uint32_t i) { return a.parts + (uint64_t)(w.piece0 + i) * kPieceFloats<DP, NH>; };
  auto put = [&](uint32_t hh, uint32_t d, const F4& o, float total) {
    const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
    T* y = (T*)a.out + ((uint64_t)w.seq * a.heads + h0 + hh) * a.dim + d;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (d + e < a.dim) y[e] = (T)(o[e] * inv);
  };
  auto common = [&](uint32_t h) { return fmaxf(fmaxf(tops[0][h], tops[1][h]), fmaxf(tops[2][h], tops[3][h])); };
  auto safe_of = [](float t) { return t == -INFINITY ? 0.0f : t; };
  auto total_at = [&](uint32_t h) {
    const float t = safe_of(common(h));
    float total = 0.0f;
#pragma unroll
    for (int x = 0; x < 4; ++x) total = fmaf(sums[x][h], power2(tops[x][h] - t), total);
    return total;
  };
#pragma unroll
  for (int b = 0; b < NH; ++b) {
    const float f = power2(top[b] - safe_of(common(16u * b + n)));
    if (b > 0) __syncthreads();
    if (16u * b + n < heads)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < NV; j += 2) *(F2*)&meet[wave][n * G::PITCH + (4u * g + r) * NV + j] = F2{acc[b][j][r] * f, acc[b][j + 1][r] * f};
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 16u * DP / 4u; i += kBlock) {
      const uint32_t h = i / (DP / 4u), d = i % (DP / 4u) * 4u, hh = 16u * b + h;
      if (hh >= heads || d >= a.dim) continue;
      F4 o = *(const F4*)&meet[0][h * G::PITCH + d];
#pragma unroll
      for (int x = 1; x < 4; ++x) o += *(const F4*)&meet[x][h * G::PITCH + d];
      if (whole) put(hh, d, o, total_at(hh));
      else publish4(piece(w.part) + hh * DP + d, make_float4(o[0], o[1], o[2], o[3]));
    }
  }
  if (whole) return;
  if (threadIdx.x < heads) {
    publish(piece(w.part) + 16 * NH * DP + threadIdx.x, common(threadIdx.x));
    publish(piece(w.part) + 16 * NH * DP + 16 * NH + threadIdx.x, total_at(threadIdx.x));
  }
  // pieces first, first + step, ... : joined, into the output or into the first one's place.  A lane has four elements of a head; where the heads
  // leave lanes over, several share an element's pieces.  Eight of a lane's pieces are on their way at once, the first of them
  // together with the maxima.
  const uint32_t units = heads * (DP / 4u), ways = units <= kBlock ? kBlock / units : 1u;
  auto join = [&](uint32_t first, uint32_t step, uint32_t count, bool out) {
    for (uint32_t i = threadIdx.x; i < count * 16u * NH; i += kBlock) {
      const uint32_t p = i / (16u * NH), h = i % (16u * NH);
      if (h >= heads) continue;
      factor[p][h] = published(piece(first + p * step) + 16 * NH * DP + h);
      weight_of[p][h] = published(piece(first + p * step) + 16 * NH * DP + 16 * NH + h);
    }
    const uint32_t way = ways == 1u ? 0u : threadIdx.x / units;
    for (uint32_t u = threadIdx.x - way * units; u < units || u < kBlock; u += kBlock) {
      const uint32_t hh = u / (DP / 4u), d = u % (DP / 4u) * 4u;
      const bool mine = u < units && way < ways && d < a.dim;
      float4 t[8];
      auto load = [&](uint32_t p0) {
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i)
          if (mine && p0 + i * ways < count) t[i] = published4(piece(first + (p0 + i * ways) * step) + hh * DP + d);
      };
      load(way);
      if (u < kBlock) {   // (the first time round)
        __syncthreads();
        if (threadIdx.x < heads) {
          const uint32_t h = threadIdx.x;
          float most = -INFINITY, total = 0.0f;
          for (uint32_t p = 0; p < count; ++p) most = fmaxf(most, factor[p][h]);
          for (uint32_t p = 0; p < count; ++p) {
            const float f = power2(factor[p][h] - safe_of(most));
            factor[p][h] = f;
            total = fmaf(weight_of[p][h], f, total);
          }
          total_of[h] = total;
          if (!out) {
            publish(piece(first) + 16 * NH * DP + h, most);
            publish(piece(first) + 16 * NH * DP + 16 * NH + h, total);
          }
        }
        __syncthreads();
      }
      F4 o = {0.0f, 0.0f, 0.0f, 0.0f};
      for (uint32_t p0 = way; mine && p0 < count; p0 += 8u * ways) {
        if (p0 != way) load(p0);
#pragma unroll
        for (uint32_t i = 0; i < 8u; ++i)
          if (p0 + i * ways < count) {
            const float f = factor[p0 + i * ways][hh];
            o = F4{fmaf(t[i].x, f, o[0]), fmaf(t[i].y, f, o[1]), fmaf(t[i].z, f, o[2]), fmaf(t[i].w, f, o[3])};
          }
      }
      if (ways > 1u) {   // (once round: units <= kBlock)
        float* shared = &meet[0][0];   // (all four waves' of it)
        *(F4*)(shared + threadIdx.x * 4u) = o;
        __syncthreads();
        if (way != 0u) continue;
        for (uint32_t x = 1; mine && x < ways; ++x) o += *(const F4*)(shared + (x * units + u) * 4u);
      }
      if (!mine) continue;
      if (out) put(hh, d, o, total_of[hh]);
      else publish4(piece(first) + hh * DP + d, make_float4(o[0], o[1], o[2], o[3]));
    }
  };
  // (24 pieces at once and in two steps: 7 sequences of up to 3001 keys 12.9 / 15.1 us; 64, where one of 131072 has 64 chunks a
  // key head: 95.4 / 91.4)
  uint32_t each = w.parts;
  if (w.parts > kMostPieces)
    for (each = 3u; each * each < w.parts;) ++each;
  const uint32_t first = w.part / each * each, groups = (w.parts + each - 1u) / each;
  if (!last_of(a.tickets + w.piece0 + first, min(each, w.parts - first), &last_flag)) return;
  join(first, 1u, min(each, w.parts - first), groups == 1u);
  // (the second piece begins no group: its ticket is that of the groups)
  if (groups > 1u && last_of(a.tickets + w.piece0 + 1u, groups, &last_flag)) join(0u, each, groups, true);
}

template <typename T, int DP, int NH>
hipError_t launch_paged_as(const PagedArgs& a, hipStream_t s) {
  const uint32_t row = a.dim * (uint32_t)sizeof(T);
  const bool whole = row % 16u == 0u && (uintptr_t)a.cache % 16u == 0u;
  // Read past the last-level cache (one block of query heads a key head: others read the same keys) where the pages that the table can name are half of it and more: the next
  // layer's cache and weights would push them out, and what they push out has to be written back if it is new.  us through it / past it, the same cache
  // again, eight of them in turn, each behind 600 MB read, behind 600 MB written, 8 key heads of 128 bf16:
  //   20 MB of keys and values (16 sequences of 300) 8.0 / 9.1, 8.8 / 10.1, 13.3 / 13.7, 14.7 / 13.8; 45 MB (64 of 32 to 512) - , 14.9 / 15.3, 18.4 / 19.1, 22.8 / 19.3;
  //   82 MB (one of 20000) 22.0 / 22.0, 25.0 / 23.6, 28.2 / 27.3, 36.9 / 27.6; 93 MB (32 of 128 to 2048) 22.7 / 24.5, 26.5 / 26.2, 29.9 / 30.2, 38.7 / 30.3;
  //   188 MB (one of 46000) 36.8 / 38.3, 42.7 / 40.0, 45.8 / 43.8, 65.6 / 43.9; 345 MB (60 of 256 to 4096) 64.3 / 66.5, 71.9 / 68.7, 75.5 / 73.3, 104.8 / 74.2;
  //   537 MB (one of 131072) 100 / 88, 100 / 90, 104 / 94, 138 / 94.
  // (What is read in the end, lengths say, on the device alone; a table as wide as the longest context names all of its pool, and short sequences lose up to 1.5 us by it.)
  const bool past = a.reach() * 2u * a.kv_heads * a.rows.d * row >= ((uint64_t)128 << 20) && a.pairs == a.kv_heads;
  if (whole && a.rows.d % 16u == 0u && past) LT_LAUNCH((lt_paged_attention_kernel<T, DP, NH, true, 16, true>), dim3(a.workgroups), dim3(kBlock), s, a);
  else if (whole && a.rows.d % 16u == 0u) LT_LAUNCH((lt_paged_attention_kernel<T, DP, NH, true, 16, false>), dim3(a.workgroups), dim3(kBlock), s, a);
  else if (whole) LT_LAUNCH((lt_paged_attention_kernel<T, DP, NH, false, 16, false>), dim3(a.workgroups), dim3(kBlock), s, a);
  else if (row >= 16u) LT_LAUNCH((lt_paged_attention_kernel<T, DP, NH, false, kWide, false>), dim3(a.workgroups), dim3(kBlock), s, a);
  else if constexpr (DP == 32) LT_LAUNCH((lt_paged_attention_kernel<T, DP, NH, false, (int)sizeof(T), false>), dim3(a.workgroups), dim3(kBlock), s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_paged_of(const PagedArgs& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2u) {
    if (a.blocks_of == 32u) return a.padded == 32u ? launch_paged_as<T, 32, 2>(a, s) : launch_paged_as<T, 64, 2>(a, s);
  }
  if (a.padded == 32u) return launch_paged_as<T, 32, 1>(a, s);
  if (a.padded == 64u) return launch_paged_as<T, 64, 1>(a, s);
  if (a.padded == 96u) return launch_paged_as<T, 96, 1>(a, s);
  if (a.padded == 128u) return launch_paged_as<T, 128, 1>(a, s);
  if (a.padded == 160u) return launch_paged_as<T, 160, 1>(a, s);
  return launch_paged_as<T, 256, 1>(a, s);
}

hipError_t launch_paged(const void* args, hipStream_t s) {
  PagedArgs a = *(const PagedArgs*)args;
  if (a.seqs == 0) return hipSuccess;
  if (!a.q || !a.lengths || !a.out || (a.capacity > 0 && (!a.cache || !a.table)) || a.dim == 0 || a.dim > a.padded || a.kv_heads == 0 || a.heads % a.kv_heads != 0 ||
      a.rows.d == 0 || a.workgroups == 0 || (a.split && (!a.parts || !a.tickets || a.least == 0 || a.chunks == 0 || a.chunks > kPagedChunks)) || a.tile != (a.dtype == kF32 ? 64u : 128u) ||
      (a.blocks_of != 16u && (a.blocks_of != 32u || a.padded > 64u || a.dtype == kF32)) ||
      (a.split && a.seqs > kPagedFind && a.listed != (a.workgroups + a.pairs - 1u) / a.pairs))
    return hipErrorInvalidValue;
  const int64_t size = a.dtype == kF32 ? 4 : 2;
  if (a.listed > 0u) {
    a.list = a.parts + (uint64_t)a.pieces * a.part_floats();
    LT_LAUNCH(lt_paged_list_kernel, dim3(1), dim3(kListBlock), s, a);
  }
  a.q_whole = (uintptr_t)a.q % 16u == 0u && a.q_seq * size % 16 == 0 && a.q_head * size % 16 == 0 && a.dim * size % 16 == 0;
  return a.dtype == kF32 ? launch_paged_of<float>(a, s) : a.dtype == kBF16 ? launch_paged_of<__bf16>(a, s) : hipErrorInvalidValue;
}

const bool registered = set_operator(kOpCacheAppend, launch_append) && set_operator(kOpPagedAttention, launch_paged);

}  // namespace
}  // namespace ltk
