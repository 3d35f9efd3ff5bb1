// What the kernels of rotary positions share: a pair's turn, and rows of heads that are read, rotated and written in
// pieces.
//
// A row (a token's head) is made of slots, a thread each: rotated ones first, then the rest.  Half layout: a slot has V elements at
// V i and their partners at n / 2 + V i; interleaved: V / 2 pairs at V i.  A workgroup takes rows in a row, so that all heads of a token
// share its turns: they are computed once a workgroup, into LDS, while the rows are on their way.
#ifndef LT_ROTARY_H_
#define LT_ROTARY_H_

#include <hip/hip_runtime.h>

#include "lt_kernels.h"

namespace ltk {

constexpr uint32_t kRowBlock = 256;       // threads of a workgroup
constexpr uint32_t kMaxTurns = 4096;      // of its tokens' pairs: 32 KB of LDS
constexpr int kMaxRows = 4;               // of a thread, all of them on their way at once
// Workgroups that are worth more than further rows a thread: two a compute unit (at least 256 / 512 / 1024, us: 8 prompts of up to 2048 tokens appended
// 11.6 / 11.6 / 12.8, of 512 each 10.3 / 10.2 / 9.8; fp32 rotation of 5331 x 12 x 80 18.6 / 18.6 / 19.4; of one row a thread always 14.0 and 20.0).
constexpr uint32_t kRowGrid = 512;
constexpr uint64_t kMostGrid = (uint64_t)1 << 24;   // workgroups are below that: a launch holds less than 2^32 threads

struct __attribute__((aligned(8))) Turn {
  float c, s;   // amplitude * cos, amplitude * sin
};

// The turn of a pair at a position.  Quarter turns in 64 bits: the whole ones go, their last two bits are the quadrant,
// and the rest, half a quarter at most, is left without another rounding.  On |x| <= pi / 4 the
// Taylor polynomials to x^13 and x^14 err by 2e-14 and 1e-15, so that what they and the amplitude give is rounded to 32 bits once.
// (Remainder, polynomials and amplitude in 32 bits: a sine off by up to three times as much; us so / as it is: 8 prompts of up to 2048 tokens appended
// 11.5 / 11.7, rotation and gradient of 8 x 2048 x 16 x 64 33.7 / 33.9, others alike.)
__device__ __forceinline__ Turn turn_of(const Rotary& r, int32_t position, uint32_t pair) {
  const double q = (double)position * r.turns[pair];
  const double whole = rint(q);
  const int quadrant = (int)whole;
  const double x = (q - whole) * 1.57079632679489662, xx = x * x;
  const double s = x * fma(xx, fma(xx, fma(xx, fma(xx, fma(xx, fma(xx, 1.0 / 6227020800.0, -1.0 / 39916800.0), 1.0 / 362880.0), -1.0 / 5040.0), 1.0 / 120.0), -1.0 / 6.0), 1.0);
  const double c = fma(xx, fma(xx, fma(xx, fma(xx, fma(xx, fma(xx, fma(xx, -1.0 / 87178291200.0, 1.0 / 479001600.0), -1.0 / 3628800.0), 1.0 / 40320.0), -1.0 / 720.0), 1.0 / 24.0), -0.5), 1.0);
  const double sn = (quadrant & 1) ? c : s, cs = (quadrant & 1) ? s : c;
  const bool flip_s = (quadrant & 2) != 0, flip_c = ((quadrant + 1) & 2) != 0;
  Turn t;
  t.c = (float)(r.amplitude * (flip_c ? -cs : cs));
  t.s = (float)(r.amplitude * ((flip_s != (r.back != 0u)) ? -sn : sn));
  return t;
}

__device__ __forceinline__ void rotate(const Turn& t, float x, float y, float* a, float* b) {
  *a = fmaf(x, t.c, -(y * t.s));
  *b = fmaf(y, t.c, x * t.s);
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__bf16 v) { return (float)v; }

__host__ __device__ inline uint32_t divide(const Divider& d, uint32_t n) { return (uint32_t)(((uint64_t)n * d.magic) >> (31u + d.shift)); }

// V elements that lie next to each other, as they are in memory.
template <typename T, int V> struct Piece { typedef T type __attribute__((ext_vector_type(V))); };
template <typename T> struct Piece<T, 1> { typedef T type; };

template <typename T, int V> __device__ __forceinline__ float element(const typename Piece<T, V>::type& p, int i) {
  if constexpr (V == 1) return to_float(p);
  else return to_float(p[i]);
}
template <typename T, int V> __device__ __forceinline__ typename Piece<T, V>::type rounded(const float (&v)[V]) {
  typename Piece<T, V>::type p;
  if constexpr (V == 1) p = (T)v[0];
  else
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = (T)v[i];
  return p;
}

// A slot of a row on its way: its elements and, in the half layout, their partners.
template <typename T, int V, bool IL> struct Slot {
  typename Piece<T, V>::type a, b;
};

// Where slot u of a row is: its first element, and (half layout) its partners' first.
template <int V, bool IL> __device__ __forceinline__ uint32_t slot_at(const Rotary& r, uint32_t u, bool* turned) {
  const uint32_t rotated = IL ? r.dims / V : r.dims / 2u / V;
  *turned = u < rotated;
  return *turned ? u * V : r.dims + (u - rotated) * V;
}

// PAST: what does not fit the last-level cache together with its result is read past it
template <typename T, int V, bool IL, bool PAST> __device__ __forceinline__ void load_slot(const T* row, const Rotary& r, uint32_t at, bool turned, Slot<T, V, IL>* s) {
  typedef typename Piece<T, V>::type P;
  if constexpr (PAST) {
    s->a = __builtin_nontemporal_load((const P*)(row + at));
    if (!IL && turned) s->b = __builtin_nontemporal_load((const P*)(row + at + r.dims / 2u));
  } else {
    s->a = *(const P*)(row + at);
    if (!IL && turned) s->b = *(const P*)(row + at + r.dims / 2u);
  }
}

// turns: those of the row's token, one for each pair; null: nothing is rotated.  PAST: results larger than the last-level cache
// are stored past it.
template <typename C, typename T, int V, bool IL, bool PAST>
__device__ __forceinline__ void store_slot(C* row, const Rotary& r, uint32_t at, bool turned, const Slot<T, V, IL>& s, const Turn* turns) {
  typedef typename Piece<C, V>::type P;
  float a[V], b[V];
#pragma unroll
  for (int i = 0; i < V; ++i) a[i] = element<T, V>(s.a, i);
  if (!IL && turned) {
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = element<T, V>(s.b, i);
  }
  if (turned && turns) {
    if constexpr (IL) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) rotate(turns[at / 2u + i], a[2 * i], a[2 * i + 1], &a[2 * i], &a[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) rotate(turns[at + i], a[i], b[i], &a[i], &b[i]);
    }
  }
  const P p = rounded<C, V>(a);
  if constexpr (PAST) __builtin_nontemporal_store(p, (P*)(row + at));
  else *(P*)(row + at) = p;
  if (!IL && turned) {
    const P q = rounded<C, V>(b);
    if constexpr (PAST) __builtin_nontemporal_store(q, (P*)(row + at + r.dims / 2u));
    else *(P*)(row + at + r.dims / 2u) = q;
  }
}

// Elements of a piece: the most, up to `most`, that row starts (all multiples of `aligned` elements apart and from 16 bytes),
// the rotated part and the rest are made of; 0: not even one piece fits the layout (interleaved pairs at odd places).
inline uint32_t piece_of(const Rotary& r, uint32_t dim, uint64_t aligned, uint32_t most) {
  uint32_t v = most;
  const uint32_t part = r.interleaved ? r.dims : r.dims / 2u;
  while (v > 1u && (part % v != 0u || (dim - r.dims) % v != 0u || aligned % v != 0u)) v /= 2u;
  return r.interleaved && v < 2u ? 0u : v;
}
inline uint32_t slots_of(const Rotary& r, uint32_t dim, uint32_t v) { return (r.interleaved ? r.dims / v : r.dims / 2u / v) + (dim - r.dims) / v; }

// The largest power of two, up to 16, that divides all of a row's strides (in elements) and, in bytes, its address.
inline uint64_t row_alignment(const void* p, uint64_t size, int64_t s0, int64_t s1, int64_t s2) {
  uint64_t bits = (uint64_t)s0 | (uint64_t)s1 | (uint64_t)s2 | 16u | ((uint64_t)(uintptr_t)p / size);
  if ((uintptr_t)p % size != 0u) return 1;
  return bits & (~bits + 1u);
}

enum Past { kNothingPast, kReadsPast, kAllPast };

// Workgroup `block` of a rotation: its rows (see above).
template <typename T, int V, bool IL, Past PAST>
__device__ __forceinline__ void rope_rows(const RopeArgs& a, uint32_t block, Turn* turns) {
  const uint32_t pairs = a.rotary.dims / 2u, lane = divide(a.slots, threadIdx.x), u = threadIdx.x - lane * a.slots.d, lanes = kRowBlock / a.slots.d;
  const uint64_t row0 = (uint64_t)block * (lanes * a.rows_each), rows = a.tokens * a.heads.d;
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

// How a rotation's rows are laid out over workgroups: the launcher's part of its arguments, the elements of a piece, and the grid.
// false: rows that the above does not take (interleaved pairs at odd places, rows of very many slots).
struct RopeLayout {
  uint32_t v, grid;
  Past past;
};
inline bool lay_out(RopeArgs* a, uint32_t size, RopeLayout* l) {
  const uint64_t rows = a->tokens * a->heads.d, in = row_alignment(a->x, size, a->s_outer, a->s_inner, a->s_head), out = row_alignment(a->out, size, 0, 0, 0);
  const uint64_t aligned = in < out ? in : out;
  const uint32_t v = piece_of(a->rotary, a->dim, aligned, 16u / size), slots = v ? slots_of(a->rotary, a->dim, v) : 0u, pairs = a->rotary.dims / 2u;
  if (v == 0 || slots > kRowBlock) return false;
  const uint64_t bytes = rows * a->dim * size, cache = (uint64_t)256 << 20;
  l->past = bytes >= cache ? kAllPast : 2 * bytes >= cache ? kReadsPast : kNothingPast;
  // rows a thread: four where that leaves kRowGrid workgroups, and the tokens' turns fit
  a->rows_each = l->past == kNothingPast ? kMaxRows : 2u;
  const uint32_t lanes = kRowBlock / slots;
  auto tokens = [&](uint32_t each) { return (lanes * each + a->heads.d - 2u) / a->heads.d + 1u; };
  while (a->rows_each > 1u && (rows / (lanes * a->rows_each) < kRowGrid || tokens(a->rows_each) * pairs > kMaxTurns)) a->rows_each /= 2u;
  const uint64_t grid = (rows + lanes * a->rows_each - 1) / (lanes * a->rows_each);
  if (tokens(a->rows_each) * pairs > kMaxTurns || grid >= kMostGrid) return false;
  a->slots.set(slots);
  a->pairs.set(pairs);
  l->v = v;
  l->grid = (uint32_t)grid;
  return true;
}

inline bool fit_to_run(const RopeArgs& a) {
  return a.x && a.positions && a.out && a.inner.d > 0 && a.n_pos.d > 0 && a.rotary.dims <= a.dim && a.rotary.dims <= 2u * kMaxPairs;
}

}  // namespace ltk
#endif
