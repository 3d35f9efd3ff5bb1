// Softmax cross entropy over a vocabulary, l = x w^T: lse = log sum exp l, loss = lse - l[label], and its gradient, g = (exp(l - lse) - [label]) dloss,
// dx = g w, dw = g^T x, with no more of l or g in memory than a piece of the vocabulary's: 128 MB of long bf16 rows, up to 512 of short ones, up to
// 1 GB in fp32 (twice that where bf16 logits are kept for the gradient), and 4096 rows at least, so that a small vocabulary is one piece.
//
// Bound by the matrix units: 2 N V D operations for the losses, 6 N V D for the gradient (the logits again), 4 where they are kept.
// The losses leave every tile of l as a maximum and a sum of exponentials for each of its tokens, which are joined; g is written in
// bf16 (or fp32), a piece at a time, and read by two products that add to dx in fp32 and make the piece's rows of dw.
// Every product is one kernel: bf16 tiles of 256 x 256 over eight waves, each with 128 x 64 of it, two slabs of 64 of k in LDS (128 KB), which the
// memory system fills by itself while the slab before is multiplied (v_mfma_f32_16x16x32_bf16); the fragments of a quarter of a slab are read under the
// products of the quarter before, and the next tile's first slab comes in under the results of this one.  (Four waves of 128 x 128 were
// slower: nothing is left to run while one waits; 32x32x16 products were 1 % slower.)
// fp32: tiles of 128 x 128, v_mfma_f32_32x32x2_f32.
//
// 8192 tokens, nine tenths of them with a label, x 131072 rows x 4096 bf16 (7.9 Tflop a product): logits 5.6 ms, 1.41 PFLOP/s; sixteen pieces of g 6.0, of dx 7.0
// (its sums in fp32 are read and written once a piece), of dw 5.8 ms, where a library's product of that size reaches 1.5: the chip lowers its
// clock under this load.  2048 x 32768 x 1024: 113 us a product, 1.2 PFLOP/s, as the library's.
// fp32 4096 x 16384 x 2048: 1.98 ms a product, 139 TFLOP/s; 1024 x 16000 x 768: 220 to 230 us, 112, the last round of tiles half empty; kept logits to g 21 us where forming them again takes 230.
// One token x 131072 x 4096: 190 us, 5.6 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>

#include "lt_dma.h"
#include "lt_launch.h"

namespace ltk {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;

// ---- which tokens count ------------------------------------------------------------------------------
// One workgroup.  A wave has a contiguous share of the tokens: it counts those whose label is a row, and, once all waves'
// counts are known, writes them down one behind the other.
constexpr uint32_t kTokensBlock = 1024;
__global__ __launch_bounds__(kTokensBlock) void lt_vocab_tokens_kernel(const VocabArgs a) {
  __shared__ uint32_t counts[kTokensBlock / 64];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
  const uint32_t share = ((a.tokens + kTokensBlock - 1u) / kTokensBlock) * 64u, begin = min(a.tokens, wave * share), end = min(a.tokens, begin + share);
  uint32_t mine = 0u;
  for (uint32_t i = begin + lane; i < end; i += 64u) mine += (uint32_t)a.labels[i] < a.vocab ? 1u : 0u;
#pragma unroll
  for (uint32_t o = 32u; o > 0u; o /= 2u) mine += __shfl_xor(mine, o);
  if (lane == 0u) counts[wave] = mine;
  __syncthreads();
  uint32_t at = 0u, all = 0u;
  for (uint32_t w = 0; w < kTokensBlock / 64u; ++w) {
    at += w < wave ? counts[w] : 0u;
    all += counts[w];
  }
  for (uint32_t r = begin; r < end; r += 64u) {
    const uint32_t i = r + lane;
    const int32_t label = i < end ? a.labels[i] : -1;
    const bool there = (uint32_t)label < a.vocab;   // (a negative one is a large number)
    const uint64_t which = __ballot(there);
    const uint32_t p = at + (uint32_t)__popcll(which & (((uint64_t)1 << lane) - 1u));
    at += (uint32_t)__popcll(which);
    if (i >= end) continue;
    a.packed_of[i] = there ? (int32_t)p : -1;
    if (there) {
      a.row_of[p] = (int32_t)i;
      a.label[p] = label;
      if (a.lse) a.lse_of[p] = a.lse[i];
    } else {
      if (a.loss) a.loss[i] = 0.0f;
      if (a.lse_out) a.lse_out[i] = 0.0f;
    }
  }
  for (uint32_t p = all + threadIdx.x; p < a.padded; p += kTokensBlock) {
    a.label[p] = -1;
    a.row_of[p] = 0;
    a.lse_of[p] = 0.0f;
  }
  if (threadIdx.x == 0u) *a.count = all;
}

// What a maximum takes from logits before their exponentials: nothing if it is infinite (the sum is then 0, or infinite, and no NaN).
__device__ __forceinline__ float finite_or_0(float top) { return fabsf(top) == INFINITY ? 0.0f : top; }

// the losses' gradient where it is one number
__device__ __forceinline__ float one_dloss(const VocabArgs& a) { return a.dloss ? a.dloss[0] : a.dloss_value; }

// ---- rows one behind the other, padded to whole slabs: one wave a row ------------------------------------
constexpr uint32_t kRowsBlock = 256;
// which wave this is of all of a launch's (many_workgroups)
__device__ __forceinline__ uint32_t wave_of_many() { return (blockIdx.y * gridDim.x + blockIdx.x) * (kRowsBlock / 64u) + threadIdx.x / 64u; }
template <typename T, bool VEC>
__global__ __launch_bounds__(kRowsBlock) void lt_vocab_pack_kernel(const VocabArgs a) {
  const uint32_t row = wave_of_many(), lane = threadIdx.x & 63u;
  const T* src;
  if (a.pack_w) {
    if (row >= a.rows) return;
    src = (const T*)a.w + (uint64_t)row * a.dim;
  } else {
    const uint32_t n = *a.count;
    if (row >= ((n + kVocabTile - 1u) & ~(kVocabTile - 1u))) return;
    src = row < n ? (const T*)a.x + (uint64_t)a.row_of[row] * a.dim : nullptr;
  }
  T* out = (T*)a.packed + (uint64_t)row * a.width;
  if (a.weigh) {   // (times dloss, rounded: the products are of this type)
    const float weight = src ? a.dloss[a.row_of[row]] : 0.0f;
    for (uint32_t d = lane * 2u; d < a.width; d += 128u) {   // (a width is whole slabs)
      out[d] = src && d < a.dim ? (T)((float)src[d] * weight) : (T)0.0f;
      out[d + 1u] = src && d + 1u < a.dim ? (T)((float)src[d + 1u] * weight) : (T)0.0f;
    }
    return;
  }
  if (VEC) {
    constexpr uint32_t V = 16 / sizeof(T);
    for (uint32_t d = lane * V; d < a.width; d += 64u * V) *(uint4*)(out + d) = src && d < a.dim ? *(const uint4*)(src + d) : make_uint4(0u, 0u, 0u, 0u);
  } else {
    for (uint32_t d = lane; d < a.width; d += 64u) out[d] = src && d < a.dim ? src[d] : (T)0.0f;
  }
}

// ---- the products -------------------------------------------------------------------------------------
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4s* lds_v4s_ptr;

// An operand's slab: BX rows (or columns) of the product by 128 bytes of k, as it arrives from memory.
//   KC, k contiguous: [x][k], rows of 128 bytes, 16-byte chunk c of row x at place c ^ ((x >> 1) & 7);
//   otherwise x contiguous: [k][x], chunk c of row k at place c ^ ((k & 3) << 2).
// Either way what one cycle of a fragment read touches lies in different banks.
template <typename T, int BX, bool KC>
struct Slab {
  static constexpr uint32_t kK = 128 / sizeof(T);
  static constexpr uint32_t kBytes = BX * 128;
  static constexpr bool kAlongK = KC;
  static constexpr uint32_t kPerRow = KC ? 8 : BX * sizeof(T) / 16;
  __host__ __device__ static constexpr uint32_t swz(uint32_t row) { return KC ? (row >> 1) & 7u : (row & 3u) << 2; }
};

// What a wave's matrix instructions take and give: blocks of kX rows (columns), kSteps of them for a slab of k; a lane's results are kQuads times
// four consecutive rows, 8 q + 4 * (lane / kX) on, of column lane % kX.
template <typename T> struct Mma;
template <> struct Mma<__bf16> {
  typedef v8bf Frag;
  typedef v4f Acc;
  static constexpr uint32_t kX = 16, kSteps = 2, kQuads = 1, kProducts = 1, kReadsAcross = 2;
  template <int BX, bool KC>
  static __device__ __forceinline__ Frag read(const char* tile, uint32_t x0, uint32_t kk, uint32_t lane) {
    typedef Slab<__bf16, BX, KC> S;
    if constexpr (KC) {
      const uint32_t row = x0 + (lane & 15u), c = kk * 4u + (lane >> 4);
      return *(const v8bf*)(tile + row * 128u + ((c ^ S::swz(row)) << 4));
    } else {
      // the hardware's transposing read: lane i of sixteen gets element i of each of four rows of k
      const uint32_t i16 = lane & 15u, k = kk * 32u + (lane >> 4) * 8u + (i16 >> 2);
      const uint32_t col = (x0 + 4u * (i16 & 3u)) * 2u;
      const char* p = tile + k * (BX * 2u) + (((col >> 4) ^ S::swz(k)) << 4) + (col & 15u);
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)p);
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(p + 4 * BX * 2));   // (k + 4: the same swizzle)
      const v8s r = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(v8bf, r);
    }
  }
  static __device__ __forceinline__ Acc mma(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<float> {
  typedef v4f Frag;   // k (2 kk + lane / 32) * 4 + j, j = 0 .. 3, of both operands: one product each
  typedef v16f Acc;
  static constexpr uint32_t kX = 32, kSteps = 4, kQuads = 4, kProducts = 4, kReadsAcross = 4;
  template <int BX, bool KC>
  static __device__ __forceinline__ Frag read(const char* tile, uint32_t x0, uint32_t kk, uint32_t lane) {
    typedef Slab<float, BX, KC> S;
    const uint32_t x = x0 + (lane & 31u), c = kk * 2u + (lane >> 5);
    if constexpr (KC) {
      return *(const v4f*)(tile + x * 128u + ((c ^ S::swz(x)) << 4));
    } else {
      Frag f;
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j) f[j] = *(const float*)(tile + (c * 4u + j) * (BX * 4u) + (((x >> 2) ^ S::swz(j)) << 4) + (x & 3u) * 4u);
      return f;
    }
  }
  static __device__ __forceinline__ Acc mma(Frag a, Frag b, Acc c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

typedef uint32_t AnyWhere __attribute__((ext_vector_type(4), aligned(2)));

template <int N> struct Num {
  static constexpr int value = N;
};

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// C = A B over tiles of BM x BN, WM x WN waves.
//   kVocabLogits, kVocabGrad  A: rows of w [x][k], B: packed tokens [x][k], k = width; a lane has sixteen rows of one token
//   kVocabDx                  A: rows of w [k][x] (columns of dim), B: g [token][row]: [x][k], k = rows of the piece
//   kVocabDw                  A: packed tokens (times dloss, where they have one each) [k][x] (columns of dim), B: g [k][x] (rows of w), k = tokens; a lane has sixteen columns of one row
template <typename T, int BM, int BN, int WM, int WN, uint32_t PASS>
__global__ __launch_bounds__(WM * WN * 64, 2) void lt_vocab_product_kernel(const VocabArgs a) {
  constexpr bool kLogit = PASS == kVocabLogits || PASS == kVocabGrad, kAK = kLogit, kBK = PASS != kVocabDw;
  constexpr uint32_t kThreads = WM * WN * 64;
  typedef Mma<T> M;
  constexpr uint32_t X = M::kX;
  constexpr int MB = BM / WM / X, NB = BN / WN / X;
  typedef Slab<T, BM, kAK> SA;
  typedef Slab<T, BN, kBK> SB;
  constexpr uint32_t kStage = SA::kBytes + SB::kBytes, kPad = BM + 16 / sizeof(T);
  // results that go through LDS leave the first stage to the next tile's first slab: half of the columns at a time behind it
  constexpr uint32_t kHalf = BN / 2, kOut = PASS == kVocabGrad || PASS == kVocabDw ? kHalf * kPad * sizeof(T) : 0u;
  __shared__ __attribute__((aligned(16))) char smem[kStage + (kStage > kOut ? kStage : kOut)];
  __shared__ float2 red[PASS == kVocabLogits ? WM * BN : 1];

  const uint32_t n_tokens = __builtin_amdgcn_readfirstlane(*a.count);
  const uint32_t m = kLogit ? a.rows : a.width, n = PASS == kVocabDw ? a.rows : n_tokens;
  const uint32_t k = kLogit ? a.width : PASS == kVocabDx ? (a.rows + SA::kK - 1u) / SA::kK * SA::kK : (n_tokens + SA::kK - 1u) / SA::kK * SA::kK;
  // as many tiles as there are tokens for (of dx: times the splits of k), an even and contiguous share for each of the eight dies (one set of
  // panels in its cache), walked eight rows of tiles at a time, by as many workgroups as there are
  const uint32_t tiles_m = (m + BM - 1u) / BM, tiles_n = (n + BN - 1u) / BN, tiles = tiles_m * tiles_n, nt = PASS == kVocabDx ? tiles * a.splits : tiles;
  const uint32_t die = blockIdx.x & 7u, own = nt / 8u + (die < nt % 8u ? 1u : 0u), first_own = die * (nt / 8u) + min(die, nt % 8u);
  const uint32_t all_slabs = k / SA::kK, per = PASS == kVocabDx ? uniform((all_slabs + a.splits - 1u) / a.splits) : all_slabs;
  struct Tile {
    uint32_t m, n, split, first_slab, slabs;
  };
  auto tile_at = [&](uint32_t index) {
    Tile r;
    uint32_t t = first_own + index;
    r.split = PASS == kVocabDx ? uniform(t / tiles) : 0u;
    t -= r.split * tiles;
    const uint32_t strip = uniform(t / (8u * tiles_n)), strip_rows = min(8u, tiles_m - strip * 8u), in_strip = t - strip * 8u * tiles_n;
    r.n = uniform(in_strip / strip_rows) * BN;
    r.m = (strip * 8u + uniform(in_strip % strip_rows)) * BM;
    r.first_slab = min(all_slabs, r.split * per);
    r.slabs = min(all_slabs - r.first_slab, per);
    return r;
  };
  uint32_t index = blockIdx.x / 8u;
  if (index >= own) return;

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid / 64u), wm = wave / WN, wn = wave % WN;
  const void* const A = PASS == kVocabDw ? a.x : a.w;
  const void* const B = kLogit ? a.x : a.g;
  const uint64_t lda = (PASS == kVocabDw ? a.width : a.w_stride) * sizeof(T), ldb = (kLogit ? a.width : a.stride) * sizeof(T);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // a slab of an operand of nx rows or columns and nk of k, from x0 on: what is behind either is a copy of the last (of a result never
  // stored, of k met by zeros)
  auto copy = [&](auto slab_type, const void* base, uint64_t ld, uint32_t x0, uint32_t nx, uint32_t nk, uint32_t slab, uint32_t to) __attribute__((always_inline)) {
    typedef decltype(slab_type) S;
    constexpr bool KC = S::kAlongK;
    constexpr uint32_t kInstr = S::kBytes / 16 / kThreads;
    const uint64_t start = (uint64_t)base + (KC ? (uint64_t)x0 * ld + (uint64_t)slab * 128u : (uint64_t)slab * S::kK * ld + (uint64_t)x0 * sizeof(T));
    const char* const from = (const char*)((uint64_t)uniform((uint32_t)(start >> 32)) << 32 | uniform((uint32_t)start));
    const uint32_t place = uniform(to + wave * 1024u);
    // (rows of a copy are kThreads / kPerRow apart, so a lane's chunk is the same one in all of them)
    static_assert(S::swz(kThreads / S::kPerRow) == 0u && S::swz(2u * kThreads / S::kPerRow) == 0u, "the same place in every row");
    const uint32_t row0 = tid / S::kPerRow, c = (tid % S::kPerRow) ^ S::swz(row0);
    const uint32_t col = KC ? c * 16u : min(c * (uint32_t)(16 / sizeof(T)), nx - x0 - (uint32_t)(16 / sizeof(T))) * (uint32_t)sizeof(T), left = KC ? nx - 1u - x0 : nk - 1u - slab * S::kK;
#pragma unroll
    for (uint32_t it = 0; it < kInstr; ++it)
      copy_1k(from, min(row0 + it * (kThreads / S::kPerRow), left) * (uint32_t)ld + col, place + it * kThreads * 16u);
  };
  // rows that exist: w's of the piece; packed tokens and rows of g up to whole tiles
  const uint32_t ax = kLogit ? a.rows : PASS == kVocabDx ? a.w_stride : a.width, bx = PASS == kVocabDw ? a.stride : a.padded;
  const uint32_t ak = PASS == kVocabDx ? a.rows : a.padded, bk = a.padded;
  auto stage = [&](const Tile& t, uint32_t slab, uint32_t which) __attribute__((always_inline)) {
    copy(SA(), A, lda, t.m, ax, ak, t.first_slab + slab, lds0 + which * kStage);
    copy(SB(), B, ldb, t.n, bx, bk, t.first_slab + slab, lds0 + which * kStage + SA::kBytes);
  };

  typename M::Acc acc[MB][NB];
  // fp32: a sum of 256 products at most, and the sum of those sums (one chain of 4096 has three times the error)
  constexpr uint32_t kChain = 8;
  constexpr bool kChains = sizeof(T) == 4;
  typename M::Acc total[kChains ? MB : 1][kChains ? NB : 1];
  auto join_chain = [&]() __attribute__((always_inline)) {
    if constexpr (kChains) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          total[i][j] += acc[i][j];
          acc[i][j] = {};
        }
    }
  };
  // The products of a slab in parts: a step of k, half of the wave's rows.  The fragments of the next part (its rows', and with a new
  // step its columns') are read while the products of one are formed, evenly among them.
  constexpr int kHalves = MB >= 4 ? 2 : 1, kRows = MB / kHalves, kParts = (int)M::kSteps * kHalves;
  typename M::Frag fa[kRows], fb[NB];
  auto read_rows = [&](uint32_t which, uint32_t part, typename M::Frag(&f)[kRows]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) f[i] = M::template read<BM, kAK>(smem + which * kStage, wm * (BM / WM) + (part % kHalves * kRows + i) * X, part / kHalves, lane);
  };
  auto read_columns = [&](uint32_t which, uint32_t part, typename M::Frag(&f)[NB]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NB; ++j) f[j] = M::template read<BN, kBK>(smem + which * kStage + SA::kBytes, wn * (BN / WN) + j * X, part / kHalves, lane);
  };
  // part P, and the reads of part NEXT of the slab in stage `which` (none: kParts)
  auto part = [&](auto p, auto then, uint32_t which) __attribute__((always_inline)) {
    constexpr int P = (int)decltype(p)::value, NEXT = (int)decltype(then)::value;
    constexpr bool columns = NEXT < kParts && NEXT % kHalves == 0;
    typename M::Frag ga[kRows], gb[NB];
    if constexpr (columns) read_columns(which, NEXT, gb);
    if constexpr (NEXT < kParts) read_rows(which, NEXT, ga);
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[P % kHalves * kRows + i][j] = M::mma(fa[i], fb[j], acc[P % kHalves * kRows + i][j]);
    if constexpr (NEXT < kParts) {
      constexpr int kReads = (kAK ? 1 : M::kReadsAcross) * kRows + (columns ? (kBK ? 1 : M::kReadsAcross) * NB : 0), kProducts = kRows * NB * M::kProducts;
#pragma unroll
      for (int q = 0; q < kProducts; ++q) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if ((q + 1) * kReads / kProducts > q * kReads / kProducts) __builtin_amdgcn_sched_group_barrier(0x100, (kReads + kProducts - 1) / kProducts, 0);
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) fa[i] = ga[i];
      if constexpr (columns)
#pragma unroll
        for (int j = 0; j < NB; ++j) fb[j] = gb[j];
    }
  };
  auto parts_but_last = [&](uint32_t which) __attribute__((always_inline)) {
    part(Num<0>(), Num<1>(), which);
    part(Num<1>(), Num<2>(), which);
    part(Num<2>(), Num<3>(), which);
  };
  static_assert(kParts == 4, "four parts");
  Tile next = tile_at(index);
  if (next.slabs > 0u) stage(next, 0u, 0u);
  for (;;) {
  const Tile tile = next;
  const uint32_t tile_m = tile.m, tile_n = tile.n, slabs = tile.slabs;
  // what the results of this tile's tokens will ask for: on its way under the products
  uint32_t label[NB];
  float lse[NB];
#pragma unroll
  for (int j = 0; kLogit && j < NB; ++j) {
    const uint32_t token = tile_n + wn * (BN / WN) + lane % X + j * X;
    label[j] = (uint32_t)a.label[token] - (a.first + tile_m) - wm * (BM / WM);   // (of this wave's rows)
    lse[j] = PASS == kVocabGrad ? a.lse_of[token] : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (uint32_t r = 0; r < 4u * M::kQuads; ++r) {
        acc[i][j][r] = 0.0f;
        if constexpr (kChains) total[i][j][r] = 0.0f;
      }
  landed<0>();
  __syncthreads();   // the first slab is there for every wave, and every wave is done with the tile before
  if (slabs > 0u) {
    read_columns(0u, 0u, fb);
    read_rows(0u, 0u, fa);
    for (uint32_t s = 0; s + 1u < slabs; ++s) {
      const uint32_t which = s & 1u;
      stage(tile, s + 1u, which ^ 1u);
      parts_but_last(which);
      // behind the barrier the next slab has landed for every wave, and every wave has read this one, whose place the one after takes
      landed_and_read<0>();
      __syncthreads();
      part(Num<kParts - 1>(), Num<0>(), which ^ 1u);
      if (kChains && s % kChain == kChain - 1u) join_chain();
    }
    parts_but_last((slabs - 1u) & 1u);
    landed_and_read<0>();
    __syncthreads();
    part(Num<kParts - 1>(), Num<kParts>(), 0u);
    if constexpr (kChains) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] += total[i][j];
    }
  }
  // the next tile's first slab is on its way under this one's results
  index += gridDim.x / 8u;
  const bool more = index < own;
  if (more) {
    next = tile_at(index);
    if (next.slabs > 0u) stage(next, 0u, 0u);
  }

  // a lane's results: column y = wn .. + j * X + lane % X, rows x = wm .. + i * X + 8 * q + 4 * (lane / X) + 0 .. 3
  // (where they go is worked out anew for every tile: kept from one to the next it would take registers that the products need)
  uint32_t own_lane = lane;
  asm volatile("" : "+v"(own_lane));
  const uint32_t own_tid = wave * 64u + own_lane;
  const uint32_t y0 = wn * (BN / WN) + own_lane % X, x0 = wm * (BM / WM) + 4u * (own_lane / X);
  auto each_quad = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (uint32_t q = 0; q < M::kQuads; ++q) f(i, q, x0 + i * X + 8u * q);
  };

  if constexpr (PASS == kVocabLogits) {
    const bool edge = tile_m + BM > m;
    if (a.logits) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        float* const row = a.logits + (uint64_t)(tile_n + y0 + j * X) * a.stride + tile_m;
        each_quad([&](int i, uint32_t q, uint32_t x) { *(v4f*)(row + x) = v4f{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]}; });
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const uint32_t y = y0 + j * X, token = tile_n + y;
      if (__ballot(label[j] < (uint32_t)(BM / WM)) != 0u) {
        float hit = 0.0f;
        bool mine = false;
        each_quad([&](int i, uint32_t q, uint32_t x) {
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r) {
            const bool here = x + r - wm * (BM / WM) == label[j];
            hit = here ? acc[i][j][4 * q + r] : hit;
            mine = mine || here;
          }
        });
        if (mine) a.picked[token] = hit;
      }
      if (edge)
        each_quad([&](int i, uint32_t q, uint32_t x) {
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r)
            if (tile_m + x + r >= m) acc[i][j][4 * q + r] = -INFINITY;
        });
      float top = -INFINITY, sum = 0.0f;
      each_quad([&](int i, uint32_t q, uint32_t) {
#pragma unroll
        for (uint32_t r = 0; r < 4u; ++r) top = fmaxf(top, acc[i][j][4 * q + r]);
      });
#pragma unroll
      for (uint32_t o = X; o < 64u; o *= 2u) top = fmaxf(top, __shfl_xor(top, o));
      const float from = finite_or_0(top);
      each_quad([&](int i, uint32_t q, uint32_t) {
#pragma unroll
        for (uint32_t r = 0; r < 4u; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][4 * q + r] - from) * kLog2e);
      });
#pragma unroll
      for (uint32_t o = X; o < 64u; o *= 2u) sum += __shfl_xor(sum, o);
      if (lane < X) red[wm * BN + y] = make_float2(top, sum);
    }
    __syncthreads();
    float* const parts = a.parts + (uint64_t)(tile_m / BM) * 2u * a.padded + tile_n;
    for (uint32_t y = own_tid; y < (uint32_t)BN; y += kThreads) {
      float top = red[y].x, sum = 0.0f;
#pragma unroll
      for (int w = 1; w < WM; ++w) top = fmaxf(top, red[w * BN + y].x);
      const float from = finite_or_0(top);
#pragma unroll
      for (int w = 0; w < WM; ++w) sum += red[w * BN + y].y * __builtin_amdgcn_exp2f((red[w * BN + y].x - from) * kLog2e);
      parts[y] = top;
      parts[a.padded + y] = sum;
    }
  } else if constexpr (PASS == kVocabDx) {
    // four columns of a token at a time, all of a block of tokens' on their way when they are added to
    float* const sums = a.sums + ((uint64_t)tile.split * a.padded + tile_n) * a.width + tile_m;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      float* const row = sums + (uint64_t)(y0 + j * X) * a.width;
      if (a.add) {
        v4f old[MB][M::kQuads];
        each_quad([&](int i, uint32_t q, uint32_t x) {
          if (tile_m + x < m) old[i][q] = *(const v4f*)(row + x);
        });
        each_quad([&](int i, uint32_t q, uint32_t) {
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r) acc[i][j][4 * q + r] += old[i][q][r];
        });
      }
      each_quad([&](int i, uint32_t q, uint32_t x) {
        if (tile_m + x < m) *(v4f*)(row + x) = v4f{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
      });
    }
  } else {
    // through LDS, [y][x], to whole rows in memory
    T* const out = (T*)(smem + kStage);
    const bool edge = tile_m + BM > m || tile_n + BN > n;
    constexpr uint32_t V = 16 / sizeof(T), kChunks = BM / V;
    if constexpr (PASS == kVocabGrad) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        each_quad([&](int i, uint32_t q, uint32_t) {
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r) acc[i][j][4 * q + r] = __builtin_amdgcn_exp2f((acc[i][j][4 * q + r] - lse[j]) * kLog2e);
        });
        if (__ballot(label[j] < (uint32_t)(BM / WM)) != 0u)
          each_quad([&](int i, uint32_t q, uint32_t x) {
#pragma unroll
            for (uint32_t r = 0; r < 4u; ++r) acc[i][j][4 * q + r] -= x + r - wm * (BM / WM) == label[j] ? 1.0f : 0.0f;
          });
        if (edge)
          each_quad([&](int i, uint32_t q, uint32_t x) {
#pragma unroll
            for (uint32_t r = 0; r < 4u; ++r)
              if (tile_m + x + r >= m || tile_n + y0 + j * X >= n) acc[i][j][4 * q + r] = 0.0f;
          });
      }
    }
    // (where no token counts, dw is 0 whatever dloss is: as the mean over none it is infinite)
    const float factor = PASS == kVocabDw && a.rank0 && n_tokens > 0u ? one_dloss(a) : 1.0f;
#pragma unroll
    for (uint32_t half = 0; half < 2u; ++half) {
      if (half > 0u) __syncthreads();   // (the first half's rows have been read)
      if (wn / (WN / 2) == half) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
          each_quad([&](int i, uint32_t q, uint32_t x) {
            T* const at = out + (y0 + j * X - half * kHalf) * kPad + x;
            v4f v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            if constexpr (PASS == kVocabDw) v *= factor;
            if constexpr (sizeof(T) == 4) *(v4f*)at = v;
            else *(v4bf*)at = v4bf{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
          });
      }
      __syncthreads();
      const uint32_t from = tile_n + half * kHalf;
      if constexpr (PASS == kVocabGrad) {
        T* const g = (T*)a.g + (uint64_t)from * a.stride + tile_m;
#pragma unroll 4
        for (uint32_t e = own_tid; e < kHalf * kChunks; e += kThreads) *(uint4*)(g + (uint64_t)(e / kChunks) * a.stride + e % kChunks * V) = *(const uint4*)(out + e / kChunks * kPad + e % kChunks * V);
      } else {
        const uint32_t rows = min(kHalf, n > from ? n - from : 0u), cols = min((uint32_t)BM, a.dim > tile_m ? a.dim - tile_m : 0u);
        T* const dw = (T*)a.dw + (uint64_t)from * a.dim + tile_m;
        // (sixteen bytes wherever they start: the hardware takes them)
        for (uint32_t e = own_tid; e < rows * kChunks; e += kThreads) {
          const uint32_t y = e / kChunks, x = e % kChunks * V;
          if (x >= cols) continue;
          T* const to = dw + (uint64_t)y * a.dim + x;
          if (x + V <= cols) *(AnyWhere*)to = *(const AnyWhere*)(out + y * kPad + x);
          else
            for (uint32_t k = 0; x + k < cols; ++k) to[k] = out[y * kPad + x + k];
        }
      }
    }
  }
  if (!more) return;
  }
}

// ---- few tokens: w goes by once, straight into registers --------------------------------------------------
// The tokens' rows of x stay in LDS, sixteen tokens a block (chunk c of token t at place c ^ (t & 15)); a wave takes sixteen rows of w at a time, eight steps of k on their way
// while eight are multiplied, and on to its next rows.  A lane has four rows of one token of a block: it keeps a running maximum and sum.
//   kVocabLogits  x and labels as they are, a maximum and a sum a workgroup and token;   kVocabGrad  packed tokens, g
template <typename T> struct Narrow;
template <> struct Narrow<__bf16> {
  typedef v8bf Frag;
  static constexpr uint32_t kStep = 32;   // of k
  static __device__ __forceinline__ v4f mma(Frag a, Frag b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Narrow<float> {
  typedef v4f Frag;
  static constexpr uint32_t kStep = 16;
  static __device__ __forceinline__ v4f mma(Frag a, Frag b, v4f c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);   // (k 4 (lane / 16) + j of both)
    return c;
  }
};

constexpr uint32_t kFewBlock = 512, kFewWaves = kFewBlock / 64;
template <typename T, int TB, uint32_t PASS>
__global__ __launch_bounds__(kFewBlock, 2) void lt_vocab_few_kernel(const VocabArgs a) {
  typedef Narrow<T> M;
  typedef typename M::Frag Frag;
  constexpr uint32_t kWay = 8, V = 16 / sizeof(T);
  __shared__ __attribute__((aligned(16))) char xs[kVocabFewBytes];
  __shared__ float2 red[PASS == kVocabLogits ? kFewWaves * TB * 16 : 1];
  const uint32_t n = PASS == kVocabLogits ? a.tokens : __builtin_amdgcn_readfirstlane(*a.count);
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid / 64u), t16 = lane & 15u, group = lane >> 4;
  const uint32_t row_bytes = (a.width * (uint32_t)sizeof(T) + 255u) & ~255u, chunks = a.width / V;
  for (uint32_t e = tid; e < n * chunks; e += kFewBlock) {
    const uint32_t t = e / chunks, c = e - t * chunks;
    *(uint4*)(xs + t * row_bytes + ((c ^ (t & 15u)) << 4)) = *(const uint4*)((const T*)a.x + (uint64_t)t * a.width + c * V);
  }
  float top[TB], sum[TB], lse[TB];
  uint32_t label[TB];
  const uint32_t last_token = max(n, 1u) - 1u;   // (columns behind the last token: the last one's again, of results never used)
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const uint32_t t = b * 16u + t16;
    top[b] = -INFINITY;
    sum[b] = 0.0f;
    label[b] = t < n ? (uint32_t)(PASS == kVocabLogits ? a.labels[t] : a.label[t]) - a.first : ~0u;
    lse[b] = PASS == kVocabGrad && t < n ? a.lse_of[t] : 0.0f;
  }
  uint32_t at[TB], key[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const uint32_t t = min(b * 16u + t16, last_token);
    at[b] = t * row_bytes;
    key[b] = t & 15u;
  }
  __syncthreads();
  const uint32_t steps = a.width / M::kStep, units = ((PASS == kVocabGrad ? a.stride : a.rows) + 15u) / 16u, all = gridDim.x * kFewWaves;
  // (rows of g up to its stride are zeros, and tokens up to a whole slab of them)
  if constexpr (PASS == kVocabGrad && TB * 16 < 128 / sizeof(T)) {
    const uint32_t each = a.stride / V, many = ((uint32_t)(128 / sizeof(T)) - TB * 16u) * each;
    for (uint32_t e = blockIdx.x * kFewBlock + tid; e < many; e += gridDim.x * kFewBlock) *(uint4*)((T*)a.g + (uint64_t)(TB * 16u) * a.stride + (uint64_t)e * V) = make_uint4(0u, 0u, 0u, 0u);
  }
  auto fetch = [&](uint32_t unit, uint32_t s0, Frag(&f)[kWay]) __attribute__((always_inline)) {
    const T* const row = (const T*)a.w + (uint64_t)min(unit * 16u + t16, a.rows - 1u) * a.width + group * V;
#pragma unroll
    for (uint32_t k = 0; k < kWay; ++k)
      if (s0 + k < steps) f[k] = *(const Frag*)(row + (s0 + k) * M::kStep);
  };
  uint32_t unit = blockIdx.x * kFewWaves + wave, s0 = 0u;
  Frag f[kWay], g[kWay];
  constexpr bool kChains = sizeof(T) == 4;   // (sums of 128 products, and their sum)
  v4f acc[TB], total[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) acc[b] = total[b] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  if (unit < units) fetch(unit, 0u, f);
  while (unit < units) {
    const bool last = s0 + kWay >= steps;
    const uint32_t next = last ? unit + all : unit, next_s = last ? 0u : s0 + kWay;
    if (next < units) fetch(next, next_s, g);
#pragma unroll
    for (uint32_t k = 0; k < kWay; ++k) {
      if (s0 + k >= steps) break;
      const uint32_t c = (s0 + k) * 4u + group;
#pragma unroll
      for (int b = 0; b < TB; ++b) acc[b] = M::mma(f[k], *(const Frag*)(xs + at[b] + ((c ^ key[b]) << 4)), acc[b]);
    }
    if constexpr (kChains) {
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        total[b] += acc[b];
        acc[b] = last ? total[b] : v4f{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    if (last) {
      const uint32_t row = unit * 16u + group * 4u;
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        if constexpr (PASS == kVocabLogits) {
          float here = top[b];
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r) {
            if (row + r == label[b] && row + r < a.rows) a.picked[b * 16u + t16] = acc[b][r];
            if (row + r >= a.rows) acc[b][r] = -INFINITY;
            here = fmaxf(here, acc[b][r]);
          }
          const float from = finite_or_0(here);
          sum[b] *= __builtin_amdgcn_exp2f((top[b] - from) * kLog2e);
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r) sum[b] += __builtin_amdgcn_exp2f((acc[b][r] - from) * kLog2e);
          top[b] = here;
        } else {
          const uint32_t t = b * 16u + t16;
          float v[4];
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r) {
            v[r] = __builtin_amdgcn_exp2f((acc[b][r] - lse[b]) * kLog2e) - (row + r == label[b] ? 1.0f : 0.0f);
            if (row + r >= a.rows || t >= n) v[r] = 0.0f;
          }
          T* const at = (T*)a.g + (uint64_t)t * a.stride + row;
          if constexpr (sizeof(T) == 4) *(v4f*)at = v4f{v[0], v[1], v[2], v[3]};
          else *(v4bf*)at = v4bf{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        }
        acc[b] = total[b] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    unit = next;
    s0 = next_s;
#pragma unroll
    for (uint32_t k = 0; k < kWay; ++k) f[k] = g[k];
  }
  if constexpr (PASS == kVocabLogits) {
#pragma unroll
    for (int b = 0; b < TB; ++b) {
#pragma unroll
      for (uint32_t o = 16u; o < 64u; o *= 2u) {
        const float other = __shfl_xor(top[b], o), more = __shfl_xor(sum[b], o), both = fmaxf(top[b], other), from = finite_or_0(both);
        sum[b] = sum[b] * __builtin_amdgcn_exp2f((top[b] - from) * kLog2e) + more * __builtin_amdgcn_exp2f((other - from) * kLog2e);
        top[b] = both;
      }
      if (group == 0u) red[(wave * TB + b) * 16u + t16] = make_float2(top[b], sum[b]);
    }
    __syncthreads();
    if (tid < TB * 16u) {
      float most = -INFINITY, total = 0.0f;
#pragma unroll
      for (uint32_t w = 0; w < kFewWaves; ++w) most = fmaxf(most, red[w * TB * 16u + tid].x);
      const float from = finite_or_0(most);
#pragma unroll
      for (uint32_t w = 0; w < kFewWaves; ++w) total += red[w * TB * 16u + tid].y * __builtin_amdgcn_exp2f((red[w * TB * 16u + tid].x - from) * kLog2e);
      float* const parts = a.parts + (uint64_t)blockIdx.x * 2u * a.padded;
      parts[tid] = most;
      parts[a.padded + tid] = total;
    }
  }
}

// ---- losses: a token's maxima and sums of all tiles, sixty-four tokens a workgroup, a sixteenth of the tiles a thread --------
constexpr uint32_t kLossBlock = 1024;
__global__ __launch_bounds__(kLossBlock) void lt_vocab_loss_kernel(const VocabArgs a) {
  constexpr uint32_t kShares = kLossBlock / 64u, kWay = 8;
  __shared__ float2 red[kShares][64];
  const uint32_t lane = threadIdx.x & 63u, share = threadIdx.x / 64u, token = blockIdx.x * 64u + lane;
  const uint32_t n = a.few ? a.tokens : *a.count;
  if (blockIdx.x * 64u >= n) return;
  float top = -INFINITY, sum = 0.0f;
  if (token < n)
    for (uint32_t t0 = share + (a.add ? 0u : 1u); t0 <= a.tiles; t0 += kShares * kWay) {
      float m[kWay], s[kWay];
#pragma unroll
      for (uint32_t k = 0; k < kWay; ++k) {   // (behind the last tile: nothing)
        const uint32_t t = t0 + k * kShares;
        m[k] = t <= a.tiles ? a.parts[(uint64_t)t * 2u * a.padded + token] : -INFINITY;
        s[k] = t <= a.tiles ? a.parts[((uint64_t)t * 2u + 1u) * a.padded + token] : 0.0f;
      }
      float both = top;
#pragma unroll
      for (uint32_t k = 0; k < kWay; ++k) both = fmaxf(both, m[k]);
      const float from = finite_or_0(both);
      sum *= __builtin_amdgcn_exp2f((top - from) * kLog2e);
#pragma unroll
      for (uint32_t k = 0; k < kWay; ++k) sum += s[k] * __builtin_amdgcn_exp2f((m[k] - from) * kLog2e);
      top = both;
    }
  red[share][lane] = make_float2(top, sum);
  __syncthreads();
  if (share != 0u || token >= n) return;
  for (uint32_t w = 0; w < kShares; ++w) top = fmaxf(top, red[w][lane].x);
  const float from = finite_or_0(top);
  sum = 0.0f;
  for (uint32_t w = 0; w < kShares; ++w) sum += red[w][lane].y * __builtin_amdgcn_exp2f((red[w][lane].x - from) * kLog2e);
  if (!a.last) {
    a.parts[token] = top;
    a.parts[a.padded + token] = sum;
    return;
  }
  const float lse = from + kLn2 * __builtin_amdgcn_logf(sum);
  const uint32_t i = a.few ? token : (uint32_t)a.row_of[token];
  const bool counts = !a.few || (uint32_t)a.labels[i] < a.vocab;
  if (!a.few) a.lse_of[token] = lse;   // (for a gradient that shares the lists)
  if (a.loss) a.loss[i] = counts ? lse - a.picked[token] : 0.0f;
  if (a.lse_out) a.lse_out[i] = counts ? lse : 0.0f;
}

// ---- g from logits that were kept: one wave 256 of a token's, up to whole tiles of tokens and rows -------------------
template <typename T>
__global__ __launch_bounds__(kRowsBlock) void lt_vocab_kept_kernel(const VocabArgs a) {
  const uint32_t tiles = a.stride / 256u, unit = wave_of_many(), lane = threadIdx.x & 63u;
  const uint32_t token = unit / tiles, row = (unit - token * tiles) * 256u + lane * 4u, n = *a.count;
  if (token >= ((n + kVocabTile - 1u) & ~(kVocabTile - 1u))) return;
  const uint64_t at = (uint64_t)token * a.stride + row;
  v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (token < n) {
    const v4f l = *(const v4f*)(a.logits + at);
    const uint32_t label = (uint32_t)a.label[token] - a.first;
    const float lse = a.lse_of[token];
#pragma unroll
    for (uint32_t r = 0; r < 4u; ++r)
      if (row + r < a.rows) v[r] = __builtin_amdgcn_exp2f((l[r] - lse) * kLog2e) - (row + r == label ? 1.0f : 0.0f);
  }
  if constexpr (sizeof(T) == 4) *(v4f*)((float*)a.g + at) = v;
  else *(v4bf*)((__bf16*)a.g + at) = v4bf{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
}

// ---- dx: the workgroups' sums of a token, four columns a thread (packed rows are whole slabs), one wave a row -----------------
template <typename T>
__global__ __launch_bounds__(kRowsBlock) void lt_vocab_dx_kernel(const VocabArgs a) {
  const uint32_t i = wave_of_many(), lane = threadIdx.x & 63u;
  if (i >= a.tokens) return;
  const int32_t p = a.packed_of[i];
  T* const out = (T*)a.dx + (uint64_t)i * a.dim;
  const bool whole = a.dim % 4u == 0u && ((uintptr_t)a.dx & 15u) == 0u;
  const float weight = p < 0 ? 0.0f : a.rank0 ? one_dloss(a) : a.dloss[i];
  for (uint32_t d = lane * 4u; d < a.dim; d += 256u) {
    v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p >= 0) {
      const float* from = a.sums + (uint64_t)p * a.width + d;
#pragma unroll 8
      for (uint32_t s = 0; s < a.splits; ++s, from += (uint64_t)a.padded * a.width) v += *(const v4f*)from;
      v *= weight;
    }
    if (whole) {
      if constexpr (sizeof(T) == 4) *(v4f*)(out + d) = v;
      else *(v4bf*)(out + d) = v4bf{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    } else {
#pragma unroll
      for (uint32_t r = 0; r < 4u; ++r)
        if (d + r < a.dim) out[d + r] = (T)v[r];
    }
  }
}

template <typename T, int BM, int BN, int WM, int WN, uint32_t PASS>
hipError_t launch_tiles(const VocabArgs& a, hipStream_t s) {
  const uint64_t m = PASS == kVocabDx || PASS == kVocabDw ? a.width : a.rows, n = PASS == kVocabDw ? a.rows : a.tokens;
  const uint64_t tiles = (m + BM - 1) / BM * ((n + BN - 1) / BN) * (PASS == kVocabDx ? a.splits : 1u);
  if (tiles == 0) return hipSuccess;
  if (tiles >= (uint64_t)1 << 31) return hipErrorInvalidValue;
  // as many workgroups as run at once: one a compute unit, or two where LDS holds two
  const uint64_t grid = std::min<uint64_t>((tiles + 7) / 8 * 8, BM == 256 ? 256 : 512);
  if (((uintptr_t)a.x & 15u) || ((uintptr_t)a.w & 15u) || ((uintptr_t)a.g & 15u)) return hipErrorInvalidValue;
  LT_LAUNCH((lt_vocab_product_kernel<T, BM, BN, WM, WN, PASS>), dim3((uint32_t)grid), dim3(WM * WN * 64), s, a);
  static const char* const names[] = {"", "", "logits", "", "grad", "dx", "dw"};
  char name[48];
  snprintf(name, sizeof(name), "lt_vocab_product_kernel<%s,%d,%d,%s>", sizeof(T) == 4 ? "f32" : "bf16", BM, BN, names[PASS]);
  note_kernel(name);
  return hipGetLastError();
}

template <typename T, int B, int WM, int WN, uint32_t PASS>
hipError_t launch_product(const VocabArgs& a, hipStream_t s) {
  // fp32 and up to 64 tokens: tiles of 128 x 64, half of a square one's columns would be of no token (64 x 131072 x 4096: losses 997 / 602 us; with a
  // gradient 22 2730 / 1811).  In bf16 such products are bound by w's bytes already.
  if constexpr (sizeof(T) == 4 && PASS != kVocabDw)
    if (a.tokens <= 64u) return launch_tiles<T, B, 64, WM, WN, PASS>(a, s);
  return launch_tiles<T, B, B, WM, WN, PASS>(a, s);
}

template <typename T, uint32_t PASS>
hipError_t launch_few(const VocabArgs& a, hipStream_t s) {
  const uint32_t blocks = vocab_few_blocks(a.tokens);
  if (a.tokens == 0u) return hipSuccess;
  if (!vocab_few(a.tokens, a.width, sizeof(T)) || a.width % (128 / sizeof(T)) != 0u || a.w_stride != a.width) return hipErrorInvalidValue;
  if (((uintptr_t)a.x & 15u) || ((uintptr_t)a.w & 15u) || ((uintptr_t)a.g & 15u)) return hipErrorInvalidValue;
  if (blocks == 1u) LT_LAUNCH((lt_vocab_few_kernel<T, 1, PASS>), dim3(kVocabFewGrid), dim3(kFewBlock), s, a);
  else if (blocks == 2u) LT_LAUNCH((lt_vocab_few_kernel<T, 2, PASS>), dim3(kVocabFewGrid), dim3(kFewBlock), s, a);
  else LT_LAUNCH((lt_vocab_few_kernel<T, 4, PASS>), dim3(kVocabFewGrid), dim3(kFewBlock), s, a);
  return hipGetLastError();
}

template <typename T, int B, int WM, int WN>
hipError_t launch_of(const VocabArgs& a, hipStream_t s) {
  const ManyWorkgroups many = many_workgroups(a.workgroups());
  const dim3 grid(many.x, many.y), block(kRowsBlock);
  switch (a.pass) {
    case kVocabPack: {
      if (many.x == 0) return hipSuccess;
      const bool vec = (((uintptr_t)(a.pack_w ? a.w : a.x)) & 15u) == 0 && a.dim * sizeof(T) % 16 == 0;
      if (vec) LT_LAUNCH((lt_vocab_pack_kernel<T, true>), grid, block, s, a);
      else LT_LAUNCH((lt_vocab_pack_kernel<T, false>), grid, block, s, a);
      return hipGetLastError();
    }
    case kVocabLogits:
      if (a.few) return launch_few<T, kVocabLogits>(a, s);
      return launch_product<T, B, WM, WN, kVocabLogits>(a, s);
    case kVocabGrad:
      if (a.few) return launch_few<T, kVocabGrad>(a, s);
      return launch_product<T, B, WM, WN, kVocabGrad>(a, s);
    case kVocabDx: return launch_product<T, B, WM, WN, kVocabDx>(a, s);
    case kVocabDw: return launch_product<T, B, WM, WN, kVocabDw>(a, s);
    case kVocabKept:
      if (a.workgroups() >= kMostWorkgroups) return hipErrorInvalidValue;
      if (many.x > 0) LT_LAUNCH(lt_vocab_kept_kernel<T>, grid, block, s, a);
      return hipGetLastError();
    case kVocabDxOut:
      if (many.x > 0) LT_LAUNCH(lt_vocab_dx_kernel<T>, grid, block, s, a);
      return hipGetLastError();
  }
  return hipErrorInvalidValue;
}

hipError_t launch_vocab(const void* args, hipStream_t s) {
  const VocabArgs& a = *(const VocabArgs*)args;
  if (a.pass == kVocabTokens) {
    LT_LAUNCH(lt_vocab_tokens_kernel, dim3(1), dim3(kTokensBlock), s, a);
    return hipGetLastError();
  }
  if (a.pass == kVocabLoss) {
    if (a.padded > 0) LT_LAUNCH(lt_vocab_loss_kernel, dim3(a.padded / 64u), dim3(kLossBlock), s, a);
    return hipGetLastError();
  }
  if (a.dtype == kBF16) return a.tile == 256u ? launch_of<__bf16, 256, 2, 4>(a, s) : launch_of<__bf16, 128, 2, 2>(a, s);
  return a.dtype == kF32 ? launch_of<float, 128, 2, 2>(a, s) : hipErrorInvalidValue;
}

const bool registered = set_operator(kOpVocab, launch_vocab);

}  // namespace
}  // namespace ltk
