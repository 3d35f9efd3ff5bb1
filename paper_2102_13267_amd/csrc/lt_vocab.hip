// Softmax cross entropy over a vocabulary, l = x w^T, and its gradient, without the logits ever being in memory as a whole.
#include <hip/hip_runtime.h>

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
      if (a.lse) a.dloss_of[p] = a.dloss ? a.dloss[a.rank0 ? 0u : i] : a.dloss_value;
    } else {
      if (a.loss) a.loss[i] = 0.0f;
      if (a.lse_out) a.lse_out[i] = 0.0f;
    }
  }
  for (uint32_t p = all + threadIdx.x; p < a.padded; p += kTokensBlock) {
    a.label[p] = -1;
    if (a.lse) a.lse_of[p] = a.dloss_of[p] = 0.0f;
  }
  if (threadIdx.x == 0u) *a.count = all;
}

// ---- rows one behind the other, padded to whole slabs: one wave a row ------------------------------------
constexpr uint32_t kRowsBlock = 256;
template <typename T, bool VEC>
__global__ __launch_bounds__(kRowsBlock) void lt_vocab_pack_kernel(const VocabArgs a) {
  const uint32_t row = blockIdx.x * (kRowsBlock / 64u) + threadIdx.x / 64u, lane = threadIdx.x & 63u;
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
  __device__ static __forceinline__ uint32_t swz(uint32_t row) { return KC ? (row >> 1) & 7u : (row & 3u) << 2; }
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

// C = A B over tiles of BM x BN, WM x WN waves.
//   kVocabLogits, kVocabGrad  A: rows of w [x][k], B: packed tokens [x][k], k = width; a lane has sixteen rows of one token
//   kVocabDx                  A: g [token][row]: [x][k], B: rows of w: [k][x], k = rows of the piece
//   kVocabDw                  A: packed tokens [k][x] (columns of dim), B: g [k][x] (rows of w), k = tokens; a lane has sixteen columns of one row
template <typename T, int BM, int BN, int WM, int WN, uint32_t PASS>
__global__ __launch_bounds__(WM * WN * 64, 2) void lt_vocab_product_kernel(const VocabArgs a) {
  constexpr bool kLogit = PASS == kVocabLogits || PASS == kVocabGrad, kAK = PASS != kVocabDw, kBK = kLogit;
  constexpr uint32_t kThreads = WM * WN * 64;
  typedef Mma<T> M;
  constexpr uint32_t X = M::kX;
  constexpr int MB = BM / WM / X, NB = BN / WN / X;
  typedef Slab<T, BM, kAK> SA;
  typedef Slab<T, BN, kBK> SB;
  constexpr uint32_t kStage = SA::kBytes + SB::kBytes, kPad = BM + 16 / sizeof(T);
  constexpr size_t kOut = PASS == kVocabGrad || PASS == kVocabDw ? (size_t)BN * kPad * sizeof(T) : 0;
  __shared__ __attribute__((aligned(16))) char smem[2 * kStage > kOut ? 2 * kStage : kOut];
  __shared__ float2 red[PASS == kVocabLogits ? WM * BN : 1];

  const uint32_t n_tokens = *a.count;
  const uint32_t m = kLogit ? a.rows : PASS == kVocabDx ? n_tokens : a.width, n = kLogit ? n_tokens : PASS == kVocabDx ? a.width : a.rows;
  const uint32_t k = kLogit ? a.width : PASS == kVocabDx ? (a.rows + SA::kK - 1u) / SA::kK * SA::kK : (n_tokens + SA::kK - 1u) / SA::kK * SA::kK;
  // as many tiles as there are tokens for, an even and contiguous share for each of the eight dies (one set of panels in its cache),
  // walked eight rows of tiles at a time
  const uint32_t tiles_m = (m + BM - 1u) / BM, tiles_n = (n + BN - 1u) / BN, nt = tiles_m * tiles_n;
  const uint32_t die = blockIdx.x & 7u, own = nt / 8u + (die < nt % 8u ? 1u : 0u);
  if (blockIdx.x / 8u >= own) return;
  const uint32_t t = die * (nt / 8u) + min(die, nt % 8u) + blockIdx.x / 8u;
  const uint32_t strip = t / (8u * tiles_n), strip_rows = min(8u, tiles_m - strip * 8u), in_strip = t - strip * 8u * tiles_n;
  const uint32_t tile_n = in_strip / strip_rows * BN, tile_m = (strip * 8u + in_strip % strip_rows) * BM;

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid / 64u), wm = wave / WN, wn = wave % WN;
  const void* const A = kLogit ? a.w : PASS == kVocabDx ? a.g : a.x;
  const void* const B = kLogit ? a.x : PASS == kVocabDx ? a.w : a.g;
  const uint64_t lda = (kLogit ? a.w_stride : PASS == kVocabDx ? a.stride : a.width) * sizeof(T), ldb = (kLogit ? a.width : PASS == kVocabDx ? a.w_stride : a.stride) * sizeof(T);
  // the slabs of this workgroup's share of k
  const uint32_t all_slabs = k / SA::kK, per = PASS == kVocabDx ? (all_slabs + a.splits - 1u) / a.splits : all_slabs;
  const uint32_t first_slab = PASS == kVocabDx ? min(all_slabs, blockIdx.y * per) : 0u, slabs = min(all_slabs - first_slab, per);

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // a slab of an operand of nx rows or columns and nk of k, from x0 on: what is behind either is a copy of the last (of a result never
  // stored, of k met by zeros)
  auto copy = [&](auto slab_type, const void* base, uint64_t ld, uint32_t x0, uint32_t nx, uint32_t nk, uint32_t slab, uint32_t to) __attribute__((always_inline)) {
    typedef decltype(slab_type) S;
    constexpr bool KC = S::kAlongK;
    constexpr uint32_t kInstr = S::kBytes / 16 / kThreads;
    const char* const from = (const char*)base + (KC ? (uint64_t)x0 * ld + (uint64_t)slab * 128u : (uint64_t)slab * S::kK * ld + (uint64_t)x0 * sizeof(T));
#pragma unroll
    for (uint32_t it = 0; it < kInstr; ++it) {
      const uint32_t e = it * kThreads + tid, row = e / S::kPerRow, c = (e % S::kPerRow) ^ S::swz(row);
      const uint32_t off = KC ? min(row, nx - 1u - x0) * (uint32_t)ld + c * 16u
                              : min(row, nk - 1u - slab * S::kK) * (uint32_t)ld + min(c * (uint32_t)(16 / sizeof(T)), nx - x0 - (uint32_t)(16 / sizeof(T))) * (uint32_t)sizeof(T);
      copy_1k(from, off, to + (it * kThreads + wave * 64u) * 16u);
    }
  };
  // rows that exist: w's of the piece; packed tokens and rows of g up to whole tiles
  const uint32_t ax = kLogit ? a.rows : PASS == kVocabDx ? a.padded : a.width, bx = kLogit ? a.padded : PASS == kVocabDx ? a.w_stride : a.stride;
  const uint32_t ak = a.padded, bk = PASS == kVocabDx ? a.rows : a.padded;
  auto stage = [&](uint32_t slab, uint32_t which) __attribute__((always_inline)) {
    copy(SA(), A, lda, tile_m, ax, ak, first_slab + slab, lds0 + which * kStage);
    copy(SB(), B, ldb, tile_n, bx, bk, first_slab + slab, lds0 + which * kStage + SA::kBytes);
  };

  typename M::Acc acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (uint32_t r = 0; r < 4u * M::kQuads; ++r) acc[i][j][r] = 0.0f;
  // A step of k of every fragment at a time, read while the products of the one before are formed.
  struct Frags {
    typename M::Frag a[MB], b[NB];
  };
  auto read = [&](uint32_t which, uint32_t kk) __attribute__((always_inline)) {
    const char* const As = smem + which * kStage;
    const char* const Bs = As + SA::kBytes;
    Frags f;
#pragma unroll
    for (int j = 0; j < NB; ++j) f.b[j] = M::template read<BN, kBK>(Bs, wn * (BN / WN) + j * X, kk, lane);
#pragma unroll
    for (int i = 0; i < MB; ++i) f.a[i] = M::template read<BM, kAK>(As, wm * (BM / WM) + i * X, kk, lane);
    return f;
  };
  auto multiply = [&](const Frags& f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) acc[i][j] = M::mma(f.a[i], f.b[j], acc[i][j]);
    // the reads of the next step among the products, evenly
    constexpr int kReads = (kAK ? 1 : M::kReadsAcross) * MB + (kBK ? 1 : M::kReadsAcross) * NB, kProducts = MB * NB * M::kProducts;
#pragma unroll
    for (int q = 0; q < kProducts; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if ((q + 1) * kReads / kProducts > q * kReads / kProducts) __builtin_amdgcn_sched_group_barrier(0x100, (kReads + kProducts - 1) / kProducts, 0);
    }
  };
  if (slabs > 0u) {
    stage(0u, 0u);
    landed<0>();
    __syncthreads();
    Frags f = read(0u, 0u);
    for (uint32_t s = 0; s < slabs; ++s) {
      const uint32_t which = s & 1u;
      if (s + 1u < slabs) stage(s + 1u, which ^ 1u);
#pragma unroll
      for (uint32_t kk = 1; kk < M::kSteps; ++kk) {
        const Frags g = read(which, kk);
        multiply(f);
        f = g;
      }
      // behind the barrier the next slab has landed for every wave, and every wave has read this one, whose place the one after takes
      landed_and_read<0>();
      __syncthreads();
      const Frags g = read(which ^ 1u, 0u);   // (behind the last slab: what is there, unused)
      multiply(f);
      f = g;
    }
  }
  __syncthreads();

  // a lane's results: column y = wn .. + j * X + lane % X, rows x = wm .. + i * X + 8 * q + 4 * (lane / X) + 0 .. 3
  const uint32_t y0 = wn * (BN / WN) + lane % X, x0 = wm * (BM / WM) + 4u * (lane / X);
  auto each_quad = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (uint32_t q = 0; q < M::kQuads; ++q) f(i, q, x0 + i * X + 8u * q);
  };
  if constexpr (PASS == kVocabLogits) {
    const bool edge = tile_m + BM > m;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const uint32_t y = y0 + j * X, token = tile_n + y;
      const uint32_t label = (uint32_t)a.label[token] - (a.first + tile_m) - wm * (BM / WM);   // (of this wave's rows)
      if (__ballot(label < (uint32_t)(BM / WM)) != 0u)
        each_quad([&](int i, uint32_t q, uint32_t x) {
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r)
            if (x + r - wm * (BM / WM) == label) a.picked[token] = acc[i][j][4 * q + r];
        });
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
      const float from = top == -INFINITY ? 0.0f : top;
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
    for (uint32_t y = tid; y < (uint32_t)BN; y += kThreads) {
      float top = red[y].x, sum = 0.0f;
#pragma unroll
      for (int w = 1; w < WM; ++w) top = fmaxf(top, red[w * BN + y].x);
      const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (int w = 0; w < WM; ++w) sum += red[w * BN + y].y * __builtin_amdgcn_exp2f((red[w * BN + y].x - from) * kLog2e);
      parts[y] = top;
      parts[a.padded + y] = sum;
    }
  } else if constexpr (PASS == kVocabDx) {
    float* const sums = a.sums + (uint64_t)blockIdx.y * a.padded * a.width;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const uint32_t d = tile_n + y0 + j * X;
      if (d >= n) continue;
      each_quad([&](int i, uint32_t q, uint32_t x) {
#pragma unroll
        for (uint32_t r = 0; r < 4u; ++r) {
          float* const at = sums + (uint64_t)(tile_m + x + r) * a.width + d;
          *at = a.add ? *at + acc[i][j][4 * q + r] : acc[i][j][4 * q + r];
        }
      });
    }
  } else {
    // through LDS, [y][x], to whole rows in memory
    T* const out = (T*)smem;
    const bool edge = tile_m + BM > m || tile_n + BN > n;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const uint32_t y = y0 + j * X, token = tile_n + y;
      if constexpr (PASS == kVocabGrad) {
        const float lse = a.lse_of[token], dloss = a.dloss_of[token];
        const uint32_t label = (uint32_t)a.label[token] - (a.first + tile_m) - wm * (BM / WM);
        each_quad([&](int i, uint32_t q, uint32_t) {
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r) acc[i][j][4 * q + r] = __builtin_amdgcn_exp2f((acc[i][j][4 * q + r] - lse) * kLog2e);
        });
        if (__ballot(label < (uint32_t)(BM / WM)) != 0u)
          each_quad([&](int i, uint32_t q, uint32_t x) {
#pragma unroll
            for (uint32_t r = 0; r < 4u; ++r) acc[i][j][4 * q + r] -= x + r - wm * (BM / WM) == label ? 1.0f : 0.0f;
          });
        each_quad([&](int i, uint32_t q, uint32_t) {
#pragma unroll
          for (uint32_t r = 0; r < 4u; ++r) acc[i][j][4 * q + r] *= dloss;
        });
        if (edge)
          each_quad([&](int i, uint32_t q, uint32_t x) {
#pragma unroll
            for (uint32_t r = 0; r < 4u; ++r)
              if (tile_m + x + r >= m || token >= n) acc[i][j][4 * q + r] = 0.0f;
          });
      }
      each_quad([&](int i, uint32_t q, uint32_t x) {
        const v4f v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        if constexpr (sizeof(T) == 4) *(v4f*)(out + y * kPad + x) = v;
        else *(v4bf*)(out + y * kPad + x) = v4bf{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
      });
    }
    __syncthreads();
    constexpr uint32_t V = 16 / sizeof(T), kChunks = BM / V;
    if constexpr (PASS == kVocabGrad) {
      T* const g = (T*)a.g + (uint64_t)tile_n * a.stride + tile_m;
      for (uint32_t e = tid; e < BN * kChunks; e += kThreads) *(uint4*)(g + (uint64_t)(e / kChunks) * a.stride + e % kChunks * V) = *(const uint4*)(out + e / kChunks * kPad + e % kChunks * V);
    } else {
      const uint32_t rows = min((uint32_t)BN, n - tile_n), cols = min((uint32_t)BM, a.dim > tile_m ? a.dim - tile_m : 0u);
      T* const dw = (T*)a.dw + (uint64_t)tile_n * a.dim + tile_m;
      if (((uintptr_t)a.dw & 15u) == 0u && a.dim % V == 0u) {
        for (uint32_t e = tid; e < rows * kChunks; e += kThreads)
          if (e % kChunks * V < cols) *(uint4*)(dw + (uint64_t)(e / kChunks) * a.dim + e % kChunks * V) = *(const uint4*)(out + e / kChunks * kPad + e % kChunks * V);
      } else {
        for (uint32_t e = tid; e < rows * BM; e += kThreads)
          if (e % BM < cols) dw[(uint64_t)(e / BM) * a.dim + e % BM] = out[e / BM * kPad + e % BM];
      }
    }
  }
}

// ---- losses: a token's maxima and sums of all tiles, sixty-four tokens a workgroup, a sixteenth of the tiles a thread --------
constexpr uint32_t kLossBlock = 1024;
__global__ __launch_bounds__(kLossBlock) void lt_vocab_loss_kernel(const VocabArgs a) {
  constexpr uint32_t kShares = kLossBlock / 64u;
  __shared__ float2 red[kShares][64];
  const uint32_t lane = threadIdx.x & 63u, share = threadIdx.x / 64u, token = blockIdx.x * 64u + lane;
  const uint32_t n = *a.count;
  if (blockIdx.x * 64u >= n) return;
  float top = -INFINITY, sum = 0.0f;
  if (token < n)
    for (uint32_t t = share; t < a.tiles_all; t += kShares) {
      const float m = a.parts[(uint64_t)t * 2u * a.padded + token], s = a.parts[((uint64_t)t * 2u + 1u) * a.padded + token];
      const float both = fmaxf(top, m), from = both == -INFINITY ? 0.0f : both;
      sum = sum * __builtin_amdgcn_exp2f((top - from) * kLog2e) + s * __builtin_amdgcn_exp2f((m - from) * kLog2e);
      top = both;
    }
  red[share][lane] = make_float2(top, sum);
  __syncthreads();
  if (share != 0u || token >= n) return;
  for (uint32_t w = 0; w < kShares; ++w) top = fmaxf(top, red[w][lane].x);
  const float from = top == -INFINITY ? 0.0f : top;
  sum = 0.0f;
  for (uint32_t w = 0; w < kShares; ++w) sum += red[w][lane].y * __builtin_amdgcn_exp2f((red[w][lane].x - from) * kLog2e);
  const float lse = from + kLn2 * __builtin_amdgcn_logf(sum);
  const uint32_t i = (uint32_t)a.row_of[token];
  if (a.loss) a.loss[i] = lse - a.picked[token];
  if (a.lse_out) a.lse_out[i] = lse;
}

// ---- dx: the workgroups' sums of a token, one wave a row ---------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kRowsBlock) void lt_vocab_dx_kernel(const VocabArgs a) {
  const uint32_t i = blockIdx.x * (kRowsBlock / 64u) + threadIdx.x / 64u, lane = threadIdx.x & 63u;
  if (i >= a.tokens) return;
  const int32_t p = a.packed_of[i];
  T* out = (T*)a.dx + (uint64_t)i * a.dim;
  for (uint32_t d = lane; d < a.dim; d += 64u) {
    float v = 0.0f;
    if (p >= 0)
      for (uint32_t s = 0; s < a.splits; ++s) v += a.sums[((uint64_t)s * a.padded + (uint32_t)p) * a.width + d];
    out[d] = (T)v;
  }
}

template <typename T, int B, int WM, int WN, uint32_t PASS>
hipError_t launch_product(const VocabArgs& a, hipStream_t s) {
  const uint64_t m = PASS == kVocabDx ? a.padded : PASS == kVocabDw ? a.width : a.rows, n = PASS == kVocabDx ? a.width : PASS == kVocabDw ? a.rows : a.padded;
  const uint64_t tiles = (m + B - 1) / B * ((n + B - 1) / B), grid = (tiles + 7) / 8 * 8;
  if (tiles == 0) return hipSuccess;
  if (grid * WM * WN * 64 >= (uint64_t)1 << 32) return hipErrorInvalidValue;
  if (((uintptr_t)a.x & 15u) || ((uintptr_t)a.w & 15u) || ((uintptr_t)a.g & 15u)) return hipErrorInvalidValue;
  LT_LAUNCH((lt_vocab_product_kernel<T, B, B, WM, WN, PASS>), dim3((uint32_t)grid, PASS == kVocabDx ? a.splits : 1u), dim3(WM * WN * 64), s, a);
  static const char* const names[] = {"", "", "logits", "", "grad", "dx", "dw"};
  char name[48];
  snprintf(name, sizeof(name), "lt_vocab_product_kernel<%s,%d,%s>", sizeof(T) == 4 ? "f32" : "bf16", B, names[PASS]);
  note_kernel(name);
  return hipGetLastError();
}

template <typename T, int B, int WM, int WN>
hipError_t launch_of(const VocabArgs& a, hipStream_t s) {
  const dim3 block(kRowsBlock);
  switch (a.pass) {
    case kVocabPack: {
      const uint32_t rows = a.pack_w ? a.rows : a.padded;
      if (rows == 0) return hipSuccess;
      const bool vec = (((uintptr_t)(a.pack_w ? a.w : a.x)) & 15u) == 0 && a.dim * sizeof(T) % 16 == 0;
      if (vec) LT_LAUNCH((lt_vocab_pack_kernel<T, true>), dim3((rows + 3u) / 4u), block, s, a);
      else LT_LAUNCH((lt_vocab_pack_kernel<T, false>), dim3((rows + 3u) / 4u), block, s, a);
      return hipGetLastError();
    }
    case kVocabLogits: return launch_product<T, B, WM, WN, kVocabLogits>(a, s);
    case kVocabGrad: return launch_product<T, B, WM, WN, kVocabGrad>(a, s);
    case kVocabDx: return launch_product<T, B, WM, WN, kVocabDx>(a, s);
    case kVocabDw: return launch_product<T, B, WM, WN, kVocabDw>(a, s);
    case kVocabDxOut:
      if (a.tokens > 0) LT_LAUNCH(lt_vocab_dx_kernel<T>, dim3((a.tokens + 3u) / 4u), block, s, a);
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
  if (a.dtype == kBF16) return launch_of<__bf16, 256, 2, 4>(a, s);
  return a.dtype == kF32 ? launch_of<float, 128, 2, 2>(a, s) : hipErrorInvalidValue;
}

const bool registered = set_operator(kOpVocab, launch_vocab);

}  // namespace
}  // namespace ltk
