// Rows of a table by token, y[n] = scale * table[id[n]], and the gradient of the table, base[v] + scale * sum over id[n] = v of dy[n].
//
// Both are bound by memory.  The lookup reads the rows and writes them once: 16384 x 1024 bf16 of 50000 rows 10.6 us, 6.3 TB/s.
// The gradient sorts the tokens by id first, a stable radix sort, so that a row's sum is taken in ascending order of its tokens, in fp32, rounded
// once, the same on every run, whatever the number of tokens of an id (a text's most frequent one is a tenth of it); atomic adds would
// be neither the same on every run nor quick on that row.  The sorted tokens are then cut into pieces of equal length, so a frequent id's sum is shared
// by many waves, and joined.  Its own bytes: dy once, the gradient once, and the rows that it is added to.  16384 x 1024 bf16, 50000 rows: sort
// 2.8 + 4.9 us for each of two digits, sums 22 (132 MB, 6 TB/s), join 7.8; into rows in place 32768 x 2048: sort 9.8 x 2, sums 39, join 10.8;
// 5331 tokens: sorted by one workgroup in 13.6.  Rows that are no multiple of 16 bytes go by shorter pieces, one element where their number is odd.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lt_launch.h"

namespace ltk {
namespace {

constexpr uint32_t kBlock = 256;

__device__ __forceinline__ uint32_t divide(uint32_t n, const Divider& by) { return (uint32_t)(((uint64_t)n * by.magic) >> 31) >> by.shift; }

// V elements that are moved at once.
template <typename T, int V>
struct Piece {
  typedef T Vec __attribute__((ext_vector_type(V), aligned(V * sizeof(T) < 16 ? V * sizeof(T) : 16)));
  Vec v;
  __device__ __forceinline__ void load(const T* p) { v = *(const Vec*)p; }
  __device__ __forceinline__ void store(T* p) const { *(Vec*)p = v; }
  __device__ __forceinline__ float get(int j) const { return (float)v[j]; }
  __device__ __forceinline__ void set(int j, float x) { v[j] = (T)x; }
};
template <typename T>
struct Piece<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = v; }
  __device__ __forceinline__ float get(int) const { return (float)v; }
  __device__ __forceinline__ void set(int, float x) { v = (T)x; }
};

// ---- lookup: one thread a piece of an output row, two of them where there are many ---------------------------
// (two: four workgroups a compute unit and more.  us with one / two: 16384 x 1024 bf16 11.5 / 10.9, x 4096 48.8 / 45.3, 32768 x 203 fp32
// 15.2 / 12.4, 2048 x 1024 5.4 / 5.2)
template <typename T, int V, int N>
__global__ __launch_bounds__(kBlock) void lt_embedding_kernel(const EmbedArgs a) {
  const uint32_t units = a.tokens * a.row.d, first = blockIdx.x * (kBlock * N) + threadIdx.x;
  Piece<T, V> p[N];
  bool there[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t u = min(first + k * kBlock, units - 1u), t = divide(u, a.row);
    const int32_t id = a.ids[t];
    there[k] = (uint32_t)id < a.rows;   // (a negative one is a large number)
    if (a.rows > 0u) p[k].load((const T*)a.table + (uint64_t)(there[k] ? id : 0) * a.dim + (u - t * a.row.d) * V);
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t u = first + k * kBlock;
    if (u >= units) return;
#pragma unroll
    for (int j = 0; j < V; ++j) p[k].set(j, there[k] ? p[k].get(j) * a.scale : 0.0f);
    p[k].store((T*)a.out + (uint64_t)u * V);
  }
}

template <typename T, int V>
hipError_t launch_pieces(EmbedArgs a, hipStream_t s) {
  const uint64_t units = (uint64_t)a.tokens * (a.dim / V);
  if (units >= (uint64_t)1 << 31) return hipErrorInvalidValue;
  a.row.set(a.dim / V);
  if (units > 1024u * 2u * kBlock) LT_LAUNCH((lt_embedding_kernel<T, V, 2>), dim3((uint32_t)((units + 2u * kBlock - 1u) / (2u * kBlock))), dim3(kBlock), s, a);
  else LT_LAUNCH((lt_embedding_kernel<T, V, 1>), dim3((uint32_t)((units + kBlock - 1u) / kBlock)), dim3(kBlock), s, a);
  return hipGetLastError();
}

// as many elements at once as rows, and where the tensors start, allow
uint32_t widest(uint32_t elem, uint32_t dim, uintptr_t starts) {
  uint32_t v = 16u / elem;
  while (v > 1u && (dim % v != 0u || starts % (v * elem) != 0u)) v /= 2u;
  return v;
}

// (a result of 2^31 pieces and more in parts of whole rows)
template <typename T>
hipError_t launch_lookup(const EmbedArgs& a, hipStream_t s) {
  const uint32_t v = widest(sizeof(T), a.dim, (uintptr_t)a.table | (uintptr_t)a.out);
  const uint32_t most = (uint32_t)std::max<uint64_t>(1u, (((uint64_t)1 << 31) - 1u) / (a.dim / v));
  EmbedArgs part = a;
  for (uint32_t t = 0; t < a.tokens; t += part.tokens) {
    part.tokens = std::min(most, a.tokens - t);
    part.ids = a.ids + t;
    part.out = (T*)a.out + (uint64_t)t * a.dim;
    hipError_t e;
    if (v == 8u) e = launch_pieces<T, 16 / sizeof(T)>(part, s);   // (eight bf16; fp32 has four at most)
    else if (v == 4u) e = launch_pieces<T, 4>(part, s);
    else if (v == 2u) e = launch_pieces<T, 2>(part, s);
    else e = launch_pieces<T, 1>(part, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_embedding(const void* args, hipStream_t s) {
  const EmbedArgs& a = *(const EmbedArgs*)args;
  if (a.tokens == 0 || a.dim == 0) return hipSuccess;
  return a.dtype == kF32 ? launch_lookup<float>(a, s) : a.dtype == kBF16 ? launch_lookup<__bf16>(a, s) : hipErrorInvalidValue;
}

// ---- the gradient: tokens in the order of their ids ------------------------------------------------------
// A stable radix sort, a digit of the ids at a time, lowest first.  (Counting the next digit while tokens are moved was slower: a frequent id's
// digit is one counter in memory for all of them.)
__device__ __forceinline__ uint32_t key_of(const EmbedGradArgs& a, uint32_t i) {
  if (a.key) return a.key[i];
  const int32_t id = a.ids[i];
  return (uint32_t)id < a.rows ? (uint32_t)id : a.rows;
}

// one more in LDS (counts come out the same in any order)
__device__ __forceinline__ void one_more(uint32_t* n) { __hip_atomic_fetch_add(n, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

// How many of a wave's tokens with this digit came before this one: those of earlier rounds, which `so_far` counts (a wave's own), and
// those of lower lanes.
template <uint32_t BITS>   // (a digit's, at most)
__device__ __forceinline__ uint32_t place(uint32_t* so_far, uint32_t digit, bool there, uint32_t lane) {
  const uint64_t all = __ballot(there);
  uint32_t low = (uint32_t)all, high = (uint32_t)(all >> 32);   // the lanes with the same digit
#pragma unroll
  for (uint32_t b = 0; b < BITS; ++b) {
    const uint64_t ones = __ballot(digit >> b & 1u);
    const uint32_t mine = (uint32_t)((int32_t)(digit << (31u - b)) >> 31);
    low &= ~((uint32_t)ones ^ mine);
    high &= ~((uint32_t)(ones >> 32) ^ mine);
  }
  const uint64_t same = (uint64_t)high << 32 | low;
  const uint32_t earlier = __builtin_amdgcn_mbcnt_hi(high, __builtin_amdgcn_mbcnt_lo(low, 0u));
  const uint32_t at = there ? so_far[digit] + earlier : 0u;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (there && earlier == 0u) so_far[digit] = at + (uint32_t)__popcll(same);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return at;
}

// The sum of what the threads before this one have.
__device__ __forceinline__ uint32_t sum_before(uint32_t mine, uint32_t* waves) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
  uint32_t upto = mine;
#pragma unroll
  for (uint32_t o = 1; o < 64u; o *= 2u) {
    const uint32_t v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 63u) waves[wave] = upto;
  __syncthreads();
  uint32_t before = upto - mine;
#pragma unroll
  for (uint32_t w = 0; w < kEmbedBlock / 64u; ++w) before += w < wave ? waves[w] : 0u;
  return before;
}

// Few tokens: one workgroup, an id and its token in a word, sixteen of them a thread at most.
__global__ __launch_bounds__(kEmbedBlock) void lt_embedding_sort_kernel(const EmbedGradArgs a) {
  constexpr uint32_t kWaves = kEmbedBlock / 64u;
  __shared__ uint32_t items[kEmbedFew];
  __shared__ uint32_t counts[kWaves][1u << kEmbedFewBits];
  __shared__ uint32_t start[1u << kEmbedFewBits];
  __shared__ uint32_t waves[kWaves];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
  const uint32_t rounds = (a.tokens + kEmbedBlock - 1u) / kEmbedBlock, begin = wave * rounds * 64u + lane;
  uint32_t item[kEmbedFew / kEmbedBlock], at[kEmbedFew / kEmbedBlock];
#pragma unroll
  for (uint32_t r = 0; r < kEmbedFew / kEmbedBlock; ++r) {
    const uint32_t i = begin + r * 64u;
    if (r < rounds && i < a.tokens) item[r] = key_of(a, i) * kEmbedFew + i;
  }
  for (uint32_t shift = 0; shift < a.bits; shift += kEmbedFewBits) {
    const uint32_t bits = min(kEmbedFewBits, a.bits - shift), digits = 1u << bits;
    for (uint32_t d = threadIdx.x; d < kWaves * digits; d += kEmbedBlock) counts[d / digits][d % digits] = 0u;
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < kEmbedFew / kEmbedBlock; ++r)
      if (r < rounds) at[r] = place<kEmbedFewBits>(counts[wave], (item[r] / kEmbedFew >> shift) & (digits - 1u), begin + r * 64u < a.tokens, lane);
    __syncthreads();
    uint32_t all = 0u;
    if (threadIdx.x < digits) {
      uint32_t c[kWaves];
#pragma unroll
      for (uint32_t w = 0; w < kWaves; ++w) c[w] = counts[w][threadIdx.x];
#pragma unroll
      for (uint32_t w = 0; w < kWaves; ++w) {
        counts[w][threadIdx.x] = all;
        all += c[w];
      }
    }
    const uint32_t smaller = sum_before(all, waves);
    if (threadIdx.x < digits) start[threadIdx.x] = smaller;
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < kEmbedFew / kEmbedBlock; ++r)
      if (r < rounds && begin + r * 64u < a.tokens) {
        const uint32_t digit = (item[r] / kEmbedFew >> shift) & (digits - 1u);
        items[start[digit] + counts[wave][digit] + at[r]] = item[r];
      }
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < kEmbedFew / kEmbedBlock; ++r)
      if (r < rounds && begin + r * 64u < a.tokens) item[r] = items[begin + r * 64u];
  }
#pragma unroll
  for (uint32_t r = 0; r < kEmbedFew / kEmbedBlock; ++r)
    if (r < rounds && begin + r * 64u < a.tokens) {
      a.key_to[begin + r * 64u] = item[r] / kEmbedFew;
      a.pos_to[begin + r * 64u] = item[r] % kEmbedFew;
    }
}

// Many: workgroup b has tokens b * each to (b + 1) * each - 1 of the order so far, wave w of it a contiguous share.  Count: how many of each digit
// a workgroup has.  Move: a token's place is what stands before it: smaller digits anywhere, its own digit in earlier workgroups, in
// earlier waves of this one, and in this wave before it.
__global__ __launch_bounds__(kEmbedBlock) void lt_embedding_count_kernel(const EmbedGradArgs a) {
  __shared__ uint32_t hist[1u << kEmbedMaxBits];
  const uint32_t digits = 1u << a.bits;
  for (uint32_t d = threadIdx.x; d < digits; d += kEmbedBlock) hist[d] = 0u;
  __syncthreads();
  const uint32_t begin = blockIdx.x * a.each;
  for (uint32_t i = begin + threadIdx.x; i < begin + a.each && i < a.tokens; i += kEmbedBlock) one_more(&hist[(key_of(a, i) >> a.shift) & (digits - 1u)]);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kEmbedBlock) a.counts[blockIdx.x * digits + d] = hist[d];
}

__global__ __launch_bounds__(kEmbedBlock) void lt_embedding_move_kernel(const EmbedGradArgs a) {
  constexpr uint32_t kWaves = kEmbedBlock / 64u;
  __shared__ uint32_t mine[kWaves][1u << kEmbedMaxBits];     // a wave's tokens of a digit, then where they go
  __shared__ uint32_t waves[kWaves];
  const uint32_t digits = 1u << a.bits, lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
  const uint32_t share = a.each / kWaves, begin = blockIdx.x * a.each + wave * share;
  uint32_t key = begin + lane < a.tokens ? key_of(a, begin + lane) : 0u;   // of the first round
  for (uint32_t d = threadIdx.x; d < kWaves * digits; d += kEmbedBlock) mine[d / digits][d % digits] = 0u;
  // digit d = this thread's: all of it, and what earlier workgroups have
  uint32_t all = 0u, before = 0u;
  if (threadIdx.x < digits) {
#pragma unroll 16
    for (uint32_t b = 0; b < a.blocks; ++b) {
      const uint32_t c = a.counts[b * digits + threadIdx.x];
      all += c;
      before += b < blockIdx.x ? c : 0u;
    }
  }
  const uint32_t smaller = sum_before(all, waves);   // (its barrier also tells that `mine` is clear)
  for (uint32_t r = 0; r < share; r += 64u) {
    const uint32_t i = begin + r + lane;
    if (i < a.tokens) one_more(&mine[wave][((r == 0u ? key : key_of(a, i)) >> a.shift) & (digits - 1u)]);
  }
  __syncthreads();
  if (threadIdx.x < digits) {
    uint32_t at = smaller + before, c[kWaves];
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) c[w] = mine[w][threadIdx.x];
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
      mine[w][threadIdx.x] = at;
      at += c[w];
    }
  }
  __syncthreads();
  for (uint32_t r = 0; r < share; r += 64u) {
    const uint32_t i = begin + r + lane;
    const bool there = i < a.tokens;
    if (r > 0u) key = there ? key_of(a, i) : 0u;
    const uint32_t at = place<kEmbedMaxBits>(mine[wave], (key >> a.shift) & (digits - 1u), there, lane);
    if (!there) continue;
    a.key_to[at] = key;
    a.pos_to[at] = a.pos ? a.pos[i] : i;
  }
}

// The first of the sorted tokens whose id is `key` or more: a wave asks 64 at a time.
__device__ __forceinline__ uint32_t first_of(const EmbedGradArgs& a, uint32_t key, uint32_t from, uint32_t lane) {
  uint32_t low = from, high = a.tokens;   // it is in low .. high
  while (high - low > 64u) {
    const uint32_t step = (high - low + 63u) / 64u, at = low + lane * step;
    const uint32_t below = __popcll(__ballot(at < high && a.key[at] < key));   // lanes whose token is before it
    if (below == 0u) return low;
    high = min(high, low + below * step);
    low += (below - 1u) * step + 1u;
  }
  return low + __popcll(__ballot(low + lane < high && a.key[low + lane] < key));
}

// which wave this is of all of a launch's (many_workgroups)
__device__ __forceinline__ uint32_t wave_of_many() { return __builtin_amdgcn_readfirstlane((blockIdx.y * gridDim.x + blockIdx.x) * (kBlock / 64u) + threadIdx.x / 64u); }

// A wave has a piece of the sorted tokens and 64 pieces of their rows: runs of one id are added up in order, eight rows on their way.  A
// run that is whole is written; what is shared with another piece of tokens is left in `parts`.  Waves behind the pieces': sixteen rows
// of the table each, those that no id names.
template <typename T, typename O, int V>
__global__ __launch_bounds__(kBlock) void lt_embedding_sum_kernel(const EmbedGradArgs a) {
  const uint32_t lane = threadIdx.x & 63u, unit = wave_of_many();
  const uint32_t tiles = (a.dim / V + 63u) / 64u, index = unit / tiles, d = ((unit % tiles) * 64u + lane) * V;
  const O* const base = (const O*)a.base;
  O* const out = (O*)a.out;
  const bool active = d < a.dim;
  if (index >= a.pieces) {
    if (a.in_place) return;
    uint32_t row = (index - a.pieces) * kEmbedRows;
    const uint32_t end = min(row + kEmbedRows, a.rows);
    if (row >= end) return;
    uint32_t named = 0u;   // a bit a row
    for (uint32_t at = first_of(a, row, 0u, lane); at < a.tokens;) {
      const uint32_t key = at + lane < a.tokens ? a.key[at + lane] : a.rows;
      uint32_t bit = key < end ? 1u << (key - row) : 0u;
#pragma unroll
      for (uint32_t o = 32u; o > 0u; o /= 2u) bit |= __shfl_xor(bit, o);
      named |= bit;
      const uint32_t last = __shfl(key, 63);
      if (last + 1u >= end) break;   // (past these rows, or the last one found)
      at = first_of(a, last + 1u, at, lane);
    }
    named = __builtin_amdgcn_readfirstlane(named);
    if (!active) return;
    for (uint32_t bit = 1u; row < end; ++row, bit *= 2u) {
      if (named & bit) continue;
      Piece<O, V> p;
      if (base) p.load(base + (uint64_t)row * a.dim + d);
      else
#pragma unroll
        for (int j = 0; j < V; ++j) p.set(j, 0.0f);
      p.store(out + (uint64_t)row * a.dim + d);
    }
    return;
  }
  constexpr uint32_t kWay = 8;
  const uint32_t begin = index * a.piece, end = min(begin + a.piece, a.tokens);
  const O* const from = a.in_place ? out : base;
  float* const parts = a.parts + (uint64_t)index * 2u * a.dim + d;
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.0f;
  bool begins = begin == 0u || a.key[begin - 1u] != a.key[begin];
  for (uint32_t i0 = begin; i0 < end; i0 += 64u) {
    // 64 tokens' ids and places, a lane each; a bit for each that is the last of a run, and of the rows that exist
    const uint32_t i = i0 + lane;
    const uint32_t key = i < end ? a.key[i] : a.rows, pos = i < end ? a.pos[i] : 0u;
    const uint32_t after = i + 1u < a.tokens ? a.key[i + 1u] : a.rows;
    const uint64_t last = __ballot(i < end && (i + 1u == a.tokens || after != key)), counts = __ballot(i < end && key < a.rows);
    if (counts == 0u) return;
    const uint32_t n = (uint32_t)__popcll(counts);   // (the ids that are no rows stand at the end)
    for (uint32_t k0 = 0; k0 < n; k0 += kWay) {
      Piece<T, V> p[kWay];
      Piece<O, V> q[kWay];
#pragma unroll
      for (uint32_t k = 0; k < kWay; ++k) {
        const uint32_t at = __builtin_amdgcn_readlane(pos, min(k0 + k, 63u)), row = __builtin_amdgcn_readlane(key, min(k0 + k, 63u));
        if (k0 + k >= n || !active) continue;
        p[k].load((const T*)a.dy + (uint64_t)at * a.dim + d);
        if (from && (last >> (k0 + k) & 1u)) q[k].load(from + (uint64_t)row * a.dim + d);
      }
#pragma unroll
      for (uint32_t k = 0; k < kWay; ++k) {
        if (k0 + k >= n) break;
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += p[k].get(j);
        const bool ends = last >> (k0 + k) & 1u;
        if (!ends && i0 + k0 + k + 1u < end) continue;
        if (active) {
          if (begins && ends) {
            Piece<O, V> r;
#pragma unroll
            for (int j = 0; j < V; ++j) r.set(j, (from ? q[k].get(j) : 0.0f) + a.scale * sum[j]);
            r.store(out + (uint64_t)__builtin_amdgcn_readlane(key, k0 + k) * a.dim + d);
          } else {
            Piece<float, V> r;
#pragma unroll
            for (int j = 0; j < V; ++j) r.set(j, sum[j]);
            r.store(parts + (begins ? a.dim : 0u));
          }
        }
        begins = true;
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] = 0.0f;
      }
    }
    if (n < 64u) return;
  }
}

// A row that a piece begins and shares with the next: the pieces' sums in order, sixteen on their way.
template <typename O, int V>
__global__ __launch_bounds__(kBlock) void lt_embedding_join_kernel(const EmbedGradArgs a) {
  const uint32_t lane = threadIdx.x & 63u, unit = wave_of_many();
  const uint32_t tiles = (a.dim / V + 63u) / 64u, index = unit / tiles, d = ((unit % tiles) * 64u + lane) * V;
  if (index + 1u >= a.pieces) return;
  const uint32_t begin = index * a.piece, next = begin + a.piece;
  const uint32_t key = a.key[next];
  if (key >= a.rows || a.key[next - 1u] != key || (begin > 0u && a.key[begin] == key && a.key[begin - 1u] == key)) return;
  // how many pieces further it goes
  uint32_t more = 0u;
  for (;;) {
    const uint32_t at = index + 1u + more + lane;
    const uint64_t same = __ballot(at < a.pieces && a.key[at * a.piece] == key);
    if (same == ~(uint64_t)0) {
      more += 64u;
      continue;
    }
    more += (uint32_t)__builtin_ctzll(~same);
    break;
  }
  if (d >= a.dim) return;
  constexpr uint32_t kWay = 16;
  O* const out = (O*)a.out;
  const O* const from = a.in_place ? out : (const O*)a.base;
  const uint64_t at = (uint64_t)key * a.dim + d;
  Piece<O, V> r;
  if (from) r.load(from + at);
  const float* parts = a.parts + (uint64_t)index * 2u * a.dim + d;
  Piece<float, V> sum;
  sum.load(parts + a.dim);
  for (uint32_t k0 = 1u; k0 <= more; k0 += kWay) {
    Piece<float, V> p[kWay];
#pragma unroll
    for (uint32_t k = 0; k < kWay; ++k) p[k].load(parts + (uint64_t)min(k0 + k, more) * 2u * a.dim);
#pragma unroll
    for (uint32_t k = 0; k < kWay; ++k)
      if (k0 + k <= more)
#pragma unroll
        for (int j = 0; j < V; ++j) sum.set(j, sum.get(j) + p[k].get(j));
  }
#pragma unroll
  for (int j = 0; j < V; ++j) r.set(j, (from ? r.get(j) : 0.0f) + a.scale * sum.get(j));
  r.store(out + at);
}

template <typename T, typename O, int V>
hipError_t launch_wide(const EmbedGradArgs& a, hipStream_t s) {
  const uint64_t n = a.workgroups(V);
  if (n == 0) return hipSuccess;
  if (n >= kMostWorkgroups) return hipErrorInvalidValue;
  const ManyWorkgroups many = many_workgroups(n);
  const dim3 grid(many.x, many.y);
  if (a.pass == kEmbedJoin) LT_LAUNCH((lt_embedding_join_kernel<O, V>), grid, dim3(kBlock), s, a);
  else LT_LAUNCH((lt_embedding_sum_kernel<T, O, V>), grid, dim3(kBlock), s, a);
  return hipGetLastError();
}

template <typename T, typename O>
hipError_t launch_sums(const EmbedGradArgs& a, hipStream_t s) {
  // (`parts` starts at 256 bytes)
  auto fits = [&](uint32_t v) {
    auto lies = [&](const void* p, uint32_t elem) { return (uintptr_t)p % std::min(16u, v * elem) == 0; };
    return a.dim % v == 0 && lies(a.dy, sizeof(T)) && lies(a.base, sizeof(O)) && lies(a.out, sizeof(O));
  };
  if constexpr (sizeof(T) == 2 && sizeof(O) == 2)
    if (fits(8u)) return launch_wide<T, O, 8>(a, s);
  if (fits(4u)) return launch_wide<T, O, 4>(a, s);
  if (fits(2u)) return launch_wide<T, O, 2>(a, s);
  return launch_wide<T, O, 1>(a, s);
}

hipError_t launch_embedding_grad(const void* args, hipStream_t s) {
  const EmbedGradArgs& a = *(const EmbedGradArgs*)args;
  if ((uint64_t)a.rows * a.dim == 0) return hipSuccess;
  if (a.pass == kEmbedSort) {
    if (a.tokens == 0 || a.tokens > kEmbedFew || a.rows >= 1u << (2u * kEmbedFewBits) || a.bits > 2u * kEmbedFewBits) return hipErrorInvalidValue;
    LT_LAUNCH(lt_embedding_sort_kernel, dim3(1), dim3(kEmbedBlock), s, a);
    return hipGetLastError();
  }
  if (a.pass == kEmbedCount || a.pass == kEmbedMove) {
    if (a.tokens == 0 || a.bits > kEmbedMaxBits || a.blocks == 0 || a.blocks > kEmbedBlocks || a.each % kEmbedBlock != 0 || (uint64_t)a.each * a.blocks < a.tokens)
      return hipErrorInvalidValue;
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
