// Kernel argument blocks shared by the host lowering pass and the HIP kernels.
//
// Every fused region is run by one kernel family.  What varies per region -- the
// elementwise chain -- is not compiled: it is a small bytecode program that lives in
// the kernel-argument segment (read through scalar loads) and is interpreted with the
// value slots held in vector registers.  The paper leaves code generation to its
// backend compiler (section 4, "lowering"); this build replaces that compiler with an
// interpreter so that a cache miss costs microseconds, not a JIT run.
#ifndef LT_KERNELS_H_
#define LT_KERNELS_H_

#include <stdint.h>

namespace ltk {

constexpr int kMaxIn = 8;       // array inputs of one program
constexpr int kMaxOut = 8;      // outputs of one program
constexpr int kMaxScal = 32;    // scalar table: dynamic scalars and immediates
constexpr int kMaxCode = 48;    // instructions
constexpr int kSlots = 32;      // value slots a program may name (kernels hold 16 or 32)
constexpr int kVec = 4;         // elements handled per lane and interpreted instruction

// device dtypes of loads / stores
enum : uint32_t { kF32 = 0, kBF16 = 1, kI32 = 2, kI64 = 3 };

// how an input is addressed from the flat index i of the iteration space [rows, cols]
enum : uint32_t {
  kFull = 0,     // element i
  kRowVec = 1,   // element i % cols   (a vector broadcast along rows, e.g. a bias)
  kColVec = 2,   // element i / cols   (one value per row)
  kScalar = 3,   // element 0
  kStrided = 4   // sum_k coord_k(i) * stride[k] over the (<= 4-d) iteration space
};

// interpreter opcodes.  Unary ops come first: the interpreter reads operand b only for
// op >= kAdd.  Operand a is always a value slot; a scalar-table operand can only be b (or c of
// kFma), so non-commutative ops have a reversed form ("kRsub": b - a).
enum : uint32_t {
  kMov = 0, kNeg, kAbs, kExp, kLog, kTanh, kSqrt, kRsqrt, kRecip, kRelu, kGelu, kSquare,
  kSigmoid, kRoundBf16,
  kAdd, kSub, kRsub, kMul, kDiv, kRdiv, kMax, kMin,
  kReluGrad,     // b > 0 ? a : 0     (a = dy, b = x)
  kRreluGrad,    // a > 0 ? b : 0
  kGeluGrad,     // a * gelu'(b)
  kRgeluGrad,    // b * gelu'(a)
  kFma,          // a*b + c
  kSplat,        // b (a scalar-table entry) replicated
  kNumOps
};

// instruction word: op[7:0] dst[12:8] a[18:13] b[24:19] c[30:25];
// operand < 32: value slot; operand >= 32: scal[operand - 32]
inline uint32_t encode(uint32_t op, uint32_t dst, uint32_t a, uint32_t b = 0, uint32_t c = 0) {
  return op | (dst << 8) | (a << 13) | (b << 19) | (c << 25);
}

// how the kernels fetch an input on their fast path (full 4-vectors)
enum : uint32_t {
  kFetchVec4 = 0,   // one 16-byte (8-byte for bf16) load of four consecutive elements
  kFetchBcast = 1,  // one element, replicated to the four lanes
  kFetchSlow = 2    // element by element through the general addressing code
};

struct EwIn {
  const void* ptr;
  uint32_t mode;
  uint32_t dtype;
  uint32_t fetch;      // kFetch*: decided by the host from mode, cols and alignment
  uint32_t pad;
  int64_t stride[4];   // kStrided only, in elements
};

struct EwOut {
  void* ptr;
  uint32_t dtype;
  uint32_t slot;       // value slot stored
  uint32_t scalar;     // 1: a rank-0 result, written once (by flat index 0)
  uint32_t pad;
};

struct EwProg {
  uint32_t n_in, n_out, n_code, anchor_slot;  // anchor_slot: where a reduction / GEMM result enters
  uint32_t vec_ok;     // 1: cols % 4 == 0, so a 4-vector never straddles a row
  uint32_t full_vec_ok;  // 1: every 4-vector of the flat space starts at a multiple of 4
  uint32_t cols;       // last dimension of the iteration space (>= 1)
  uint32_t n_slots;    // value slots the program uses (selects the 16- or 32-slot kernel)
  uint32_t needs_divmod;  // 1: some input is addressed by i / cols or i % cols
  uint32_t fast;       // 1: n % 4 == 0, every input fetches as vec4 / broadcast, outputs contiguous
  uint32_t all_f32;    // 1: every input and output is fp32
  uint32_t pad2;
  uint64_t n;          // elements of the iteration space
  uint32_t dims[4];    // iteration space collapsed to 4 dims (kStrided addressing)
  EwIn in[kMaxIn];
  EwOut out[kMaxOut];
  float scal[kMaxScal];
  uint32_t code[kMaxCode];
};

// ---- elementwise region -----------------------------------------------------------
struct EwArgs {
  EwProg prog;
};

// ---- reductions ---------------------------------------------------------------------
enum : uint32_t { kRedSum = 0, kRedMax = 1, kRedMean = 2 };

// row reduction: out[r] = post(reduce_c pro(x[r, c]))
struct RowArgs {
  EwProg pro;          // iteration space [rows, cols]; its result is slot pro.anchor_slot
  EwProg post;         // iteration space [rows]
  uint32_t rows, cols, red, threads_per_row;
  // filled in by launch_row_reduce for the streamed variant: input numbers of the (up to two) fp32
  // inputs read in full and of the (up to one) fp32 vector broadcast along rows; counts
  uint32_t vin[2], rin, n_vin, n_rin, pad;
};

// global reduction, single launch: per-workgroup partials, the last workgroup to finish
// combines them, then runs the post program (scalar epilogue and optional finaliser)
struct AllArgs {
  EwProg pro;          // iteration space = the reduced tensor, flat
  EwProg post;         // iteration space: 1 element, or the finaliser's shape
  float* partials;     // [gridDim.x]
  uint32_t* ticket;    // zero before launch; reset by the kernel
  uint32_t red, pad;
  uint64_t count;      // elements reduced (for mean)
};

// column reduction over axis 0 of [rows, cols]
struct ColArgs {
  EwProg pro;          // iteration space [rows, cols]
  EwProg post;         // iteration space [cols]
  float* partials;     // [gridDim.y, cols]
  uint32_t* tickets;   // [gridDim.x], zero before launch; reset by the kernel
  uint32_t rows, cols, red;
  uint32_t narrow;     // set by launch_col_reduce: at most 64 columns and 65536 elements, one workgroup (see the kernel)
  // filled in by launch_col_reduce for the streamed variants (by the lowering if norm_grad): input
  // numbers of the (up to two) inputs read in full and of the (up to two) per-row inputs (kColVec),
  // padded with the first
  uint32_t vin[2], cin[2];
  // 1: the program is input vin[0] * ((input vin[1] - input cin[0]) * input cin[1]), a layer norm's
  // weight gradient before its sum, and is not interpreted
  uint32_t norm_grad;
  // 1 (with norm_grad and a sum): the column sums of input vin[0] (the norm's bias gradient) ride along;
  // their partials follow the others', post2 runs on them
  uint32_t sum2;
  EwProg post2;        // iteration space [cols]
  // Not null: the launch that computed the norm's gradient, or a contraction that reads the summed tensor, has left
  // `parts_rows` partial sums of every column here (rows of [1 + sum2][cols] floats: a norm's weight gradient's, then its
  // bias gradient's), and this one only adds them up.
  const float* parts;
  uint32_t parts_rows, pad;
};

// ---- row operators with a fixed body ---------------------------------------------------
enum : uint32_t { kSoftmax = 0, kSoftmaxGrad, kLayerNorm, kLayerNormGrad, kXent, kXentGrad };

struct RowOpArgs {
  uint32_t op, rows, cols, threads_per_row;
  const void* in[5];
  uint32_t in_dtype[5];
  void* out[3];        // (out[1] of xent_grad: null, or the losses, which ride along)
  uint32_t out_dtype[3];
  float eps;           // layer norm
  float scale;         // xent_grad
  // layer_norm_grad: column sums that ride along (0 none, 1 of dy * xhat, 2 of dy as well); col_rows workgroups leave theirs in
  // col_parts, a row of [col_sums][cols] floats each (ColArgs::parts)
  uint32_t col_sums, col_rows;
  float* col_parts;
  // xent and xent_grad: the sum or mean (kRedSum, kRedMean) of the losses goes to `total` as well; the workgroups exchange
  // theirs through total_parts[gridDim.x] and the ticket (zero before the launch; reset by the kernel)
  uint32_t has_total, total_red;
  float* total;
  float* total_parts;
  uint32_t* total_ticket;
};

// ---- contraction ------------------------------------------------------------------------
// C[b] = post(A[b] * B[b]); A is M x K, B is K x N, element (i, j) of an operand is at
// base + b0*sb0 + b1*sb1 + i*s_row + j*s_col (element strides), so transposes, batched
// operands and head-split layouts are all addressing, never copies.
struct GemmOperand {
  const void* ptr;
  int64_t s_row, s_col, s_b0, s_b1;
};

//
// A post program that is a chain -- one running value per element, each step combining it with nothing, a scalar
// or an input, results stored on the way -- is also laid out as such.  The epilogues then evaluate it with the
// running values in registers the compiler has numbered: no slot is looked up, copied out or copied back, and
// 32 elements of a lane share the decoding of a step.
constexpr int kMaxChain = 8;
enum : uint32_t { kSrcNone = 0, kSrcScal, kSrcRow0, kSrcRow1, kSrcFull0, kSrcFull1 };
constexpr uint32_t kNoOut = 0xff;
// step word: op[7:0] src[11:8] scal[19:12] out[27:20].  With v the running value, s the source and c the scalar: an op's
// first operand is v, its second s, and its reversed form takes them the other way round; kFma: v * c + s, kRfma: s * c + v.
constexpr uint32_t kRfma = kNumOps;
struct Chain {
  uint32_t n;                  // steps + 1; 0: the program is no chain
  uint32_t n_row, n_full;      // inputs addressed by column, inputs addressed like the output (up to two of each),
  uint32_t row[2], full[2];    // their input numbers
  uint32_t first_out;          // the output that is the product itself, or kNoOut
  uint32_t step[kMaxChain];    // out: the output that is the running value after the step, or kNoOut
};

struct GemmArgs {
  GemmOperand a, b;
  uint32_t m, n, k;
  uint32_t batch0, batch1;   // batch = batch0 * batch1 (b = b0 * batch1 + b1)
  uint32_t in_dtype;         // kF32 or kBF16 (both operands)
  uint32_t tiles_m, tiles_n;
  // where output element (b0, b1, row, col) goes: b0*o_b0 + b1*o_b1 + row*o_row + col (elements).
  // Contiguous [batch, m, n] by default; a permuted layout when the product's only reader is a
  // permutation (head merge), which then costs nothing.
  int64_t o_b0, o_b1, o_row;
  // Split-K (the LDS-staged kernels): `splits` workgroups share an output tile, each contracting a
  // slice of k and leaving its fp32 partial product, row major, in split_ws[split]; the post
  // program then runs in a second launch (SplitPostArgs) that adds the partials up in split order.
  // With splits = 1 and split_ws set the product goes there as it is, for the second launch.
  // Workgroup tile: bf16 128 x 128 or 128 x 64; fp32 128 x 128 or 64 x 64, and for direct = 1, the one-launch
  // kernel for small products, 16 x 16, 16 x 64, 32 x 32 or 64 x 32.
  // halves = 2 (the LDS-staged kernels): a workgroup of twice the size, each half of it contracting half of the
  // workgroup's k; the two products meet in LDS.
  uint32_t splits, tile_m, tile_n, halves;
  uint32_t direct;
  float* split_ws;           // [splits][batch * m * n] floats
  // The one-launch small kernel (direct = 1) with splits > 1: `splits` workgroups share a tile;
  // split_ws then holds [tile][split][tile_m x tile_n] partial tiles and tickets[tile]
  // counts the workgroups that have left theirs (zero before the launch; the last one adds the
  // partials up in split order, runs the post program and resets the ticket).
  uint32_t* tickets;
  EwProg post;               // iteration space = the output
  // post as a chain, for the LDS-staged kernels: every input and output has the operands' type, columns come in
  // whole 16-byte chunks
  Chain chain;
  // The one-launch small kernel can carry the column sums of its B operand ([k, n], rows
  // contiguous) along: a weight gradient x^T dy and the bias gradient sum_rows(dy) read the same
  // dy.  col_sum = 1: the workgroups of the first tile row add up the columns of B they fetch
  // anyway (col_red: kRedSum or kRedMean) and run col_post on them, iteration space [n].
  // The LDS-staged kernels do so too where A is [k, m] and B [k, n], rows contiguous, in an unbatched product (bf16: tiles of 128
  // columns).  With col_parts set (k splits; n a multiple of four) each split leaves its sums there, [splits][n], for
  // ColArgs::parts, and col_post is not used.
  uint32_t col_sum, col_red;
  float* col_parts;
  EwProg col_post;
};

// second launch of a split-K contraction: anchor = sum over splits of ws[split][i], then the
// contraction's post program over the flat output, exactly like an elementwise region
struct SplitPostArgs {
  EwProg prog;
  const float* ws;
  uint32_t splits, pad;
  uint64_t stride;           // floats between consecutive splits (= elements of the output)
};

// ---- attention core ------------------------------------------------------------------------
// o = softmax(q k^T) v over batch0 x batch1 heads, q and o [sq, d], k and v [sk, d], and its gradients
// for dy [sq, d].  Rows contiguous (s_col = 1), any row and head strides.
enum : uint32_t { kAttnForward = 0, kAttnDq, kAttnDkv };

struct AttnArgs {
  uint32_t pass, dtype, d, sq, sk, batch0, batch1, pad;
  // q is taken as q * q_scale, rounded to its type; dq, rounded, is stored times dq_scale
  float q_scale, dq_scale;
  GemmOperand q, k, v, o, dy;
  GemmOperand dq, dk, dv;
  // [3][batch0 * batch1 * sq]: row maxima and reciprocal row sums (written by the forward pass unless
  // null), row sums of p * (dy v^T) (written by kAttnDq, read by kAttnDkv)
  float* stats;
};

// ---- window update -------------------------------------------------------------------------
// out = base with the window [start, start + len) along one axis replaced by upd.  The tensors are
// seen as [outer, dim, inner] (base, out) and [outer, len, inner] (upd), dense.  window_only: out
// is base's own buffer (updated in place), so only the window is written.
struct SliceArgs {
  const void* base;
  const void* upd;
  void* out;
  uint64_t n;              // elements this launch walks: the window (window_only) or all of out
  uint64_t dim, inner, start, len;
  uint32_t elem_bytes;     // 2, 4 or 8
  uint32_t window_only;
};

// ---- rotary positions, and a paged cache of keys and values ------------------------------------
// Quarter turns per position of every rotated pair (frequency * 2 / pi), in 64 bits: it and position * turns are rounded six times, 2^-50 of
// the quarter turns together, which is 2^-20 of one at the largest position; their fraction is what is left to compute a sine of.
constexpr uint32_t kMaxPairs = 128;
struct Rotary {
  double turns[kMaxPairs];
  double amplitude;
  uint32_t dims, interleaved;   // dims 0: nothing is rotated
  uint32_t back, pad;           // back: turn the other way
};

// n / d for n < 2^31, 1 <= d <= 2^31: the product with ceil(2^(31 + shift) / d), shift = ceil(log2 d)
struct Divider {
  uint32_t d, magic, shift;
  void set(uint32_t div) {
    d = div;
    shift = 0;
    while (shift < 31u && (1u << shift) < div) ++shift;
    magic = (uint32_t)((((uint64_t)1 << (31u + shift)) + div - 1u) / div);
  }
};

// out[t][h] = x[t][h] rotated by positions[t % n_pos].  Token t of x is at (t / inner) * s_outer + (t % inner) * s_inner,
// its head h s_head further, elements contiguous; out is dense.
struct RopeArgs {
  const void* x;
  const int32_t* positions;
  void* out;
  uint64_t tokens;              // below 2^31
  uint32_t dtype, dim;
  Divider heads, inner, n_pos;
  uint32_t whole;               // inner is all of the tokens
  int64_t s_outer, s_inner, s_head;
  Divider slots, pairs;         // of a row: these three are the launcher's
  uint32_t rows_each, pad;
  Rotary rotary;
};

// New rows of a paged cache [pages][2][heads][rows][dim].  copy_from: the cache to copy to `cache` first
// (null: `cache` holds it already).  offsets null: token t is sequence t's.
struct AppendArgs {
  void* cache;
  const void* copy_from;
  const void* k;
  const void* v;
  const int32_t* lengths;
  const int32_t* table;
  const int32_t* offsets;
  uint64_t cache_elems;
  uint32_t cache_dtype, dtype, tokens, seqs, slots, pages, heads, dim;
  Divider rows, token_rows;     // of a page; of a token: 2 heads
  uint32_t rows_each, append_grid;   // (these two, and the next two, are the launcher's)
  Divider slots_each, pairs;
  int64_t k_token, k_head, v_token, v_head;   // element strides
  Rotary rotary;
  // a rotation that shares the launch (the queries of the tokens whose keys are appended); rope.out null: none
  RopeArgs rope;
};

// out[s][h] = softmax(scale q K^T) V over sequence s's keys in the paged cache.  Work is counted in tiles of `tile` keys for
// blocks of `blocks_of` query heads of one key head; `pairs` such blocks a sequence.  split: sequences of more than `whole` tiles are cut into chunks of c
// tiles, c = max(least, all sequences' tiles / chunks), a workgroup each, and what several of them have of a block meets in `parts`, with a ticket a
// piece (zero before and after a launch).  A sequence of t > c tiles has ceil(t / c) < 2 t / c chunks, so there are fewer than 2 `chunks` pieces.
// Otherwise a workgroup has a block of a sequence.
//
// Fewer blocks than compute units: one chunk a compute unit, of two tiles at least, but up to five tiles of bf16 stay whole, which a join would take as long as
// (chunks 256 / 512, us, 8 key heads of 128 bf16: one sequence of 131072 keys 86.2 / 91.1, of 20000 24.4 / 28.8, 4 of 5000 21.9 / 25.5; least two / four tiles:
// one of 3000 11.3 / 13.4, of 1500 11.1 / 12.9; of 600, five tiles, 10.4 in three parts, 9.8 whole; fp32 7 of up to 3001 13.5 so, 12.9 cut).  Otherwise two chunks a compute unit, of four
// tiles (fp32, tiles of 64 keys: two) at least, so that short ones fill up beside long ones (256 / 512: 60 sequences of 256 to 4096 84 / 74, 32 of up to 2048
// with their append 29.6 / 27.6; least two / four: 28.9 / 27.6).  More chunks gain nothing (768: one of 131072 96, 60 of up to 4096 76.5).
constexpr uint32_t kPagedFull = 256;            // blocks, a workgroup each, that leave no compute unit without one
constexpr uint32_t kPagedChunks = 512;
// Up to so many sequences a workgroup finds its chunk by itself; of more a list of them is written first (lengths of 100 to 1000, 2 key heads of
// 128 bf16, by themselves / from a list, us: 128 sequences 22.7 / 25.2, 256 31.0 / 33.3, 1024 143 / 111, 16384 10870 / 1492).
constexpr uint32_t kPagedFind = 256;
struct PagedArgs {
  const void* q;
  const void* cache;
  const int32_t* lengths;
  const int32_t* table;
  void* out;
  uint32_t dtype, seqs, heads, kv_heads, dim, slots, pages;
  uint32_t capacity;            // most keys of a sequence: slots * rows of a page (0 without pages)
  Divider rows;                 // of a page
  float scale;
  int64_t q_seq, q_head;        // element strides
  float* parts;
  uint32_t* tickets;
  uint32_t padded, blocks_of, pairs, tile;   // padded: the kernel instance's head size
  uint32_t workgroups, split, least, whole, chunks;
  uint32_t listed;              // entries of the list, one for each chunk there can be (0: none is written)
  void* list;                   // behind the pieces (the launcher sets it)
  uint32_t pieces, q_whole;     // pieces: that parts and tickets are for.  q_whole: rows of q are whole 16-byte pieces (the launcher sets it)

  // pages that the table can name: the pool may be far larger
  uint64_t reach() const { return (uint64_t)seqs * slots < pages ? (uint64_t)seqs * slots : pages; }
  uint64_t part_floats() const { return (uint64_t)blocks_of * padded + 2u * blocks_of; }
  // The instance, and how the work is shared out; `capacity` and what comes before it are set.  Tiles of all sequences must be below 2^32.
  void share_out() {
    const uint32_t group = heads / kv_heads;
    // (heads of 80 in the instance of 96 12.9 us, of 128 14.6; 148 short sequences with 8 key heads of 160 in that of 160 14.9, of 256 29.2; 75 with 4 of 20
    // and their append in that of 32 16.4, of 64 18.3)
    padded = dim <= 32u ? 32u : dim <= 64u ? 64u : dim <= 96u ? 96u : dim <= 128u ? 128u : dim <= 160u ? 160u : 256u;
    // Two blocks of 16 in one read keys once for more heads, but a workgroup takes longer: in bf16, for heads of up to 64, where there are many and long ones (us, in 16s /
    // 32s, 32 query heads a key head, sequences x key heads of up to so many keys, heads of 32: 64 x 2048 10.3 / 10.4, 64 x 8192 17.5 / 16.0, 256 x 512 7.1 / 8.3, 256 x
    // 1024 11.7 / 12.3, 256 x 2048 15.1 / 14.8, 1024 x 1024 24.2 / 19.2, but 1024 x 300 11.0 / 9.3; of 64: 32 x 4096 12.7 / 16.3, 64 x 4096 16.8 / 16.7, 64 x 8192 24.8 / 23.7, 512 x 600 14.0 / 15.2, 128 x
    // 2048 15.2 / 15.4, 256 x 2048 22.7 / 20.2, 1600 x 300 24.2 / 26.7, 1600 x 1000 52.3 / 43.9; 64 heads on one of 64 128 x 4096 35.2 / 28.9).  Heads of 96 and 128 leave 32s two waves a SIMD and one: of 128
    // 256 x 2048 37.1 / 39.0, 1024 x 300 28.6 / 38.7, 1600 x 300 41.0 / 61.4, although 64 x 8192 43.4 / 39.2, 256 x 4096 62.8 / 58.4; fp32 is slower in 32s everywhere (128 x 4096 of 64 38.9 / 41.9,
    // of 128 77.3 / 83.5).  One sequence of 20000 keys on one head of 128: 19.6 / 30.0.
    const uint64_t rowsets = (uint64_t)seqs * kv_heads;
    blocks_of = group <= 16u || dtype == kF32 || padded > 64u || rowsets < 64u || capacity < 512u || rowsets * capacity < (1u << 19) ? 16u : 32u;
    pairs = kv_heads * ((group + blocks_of - 1u) / blocks_of);
    tile = dtype == kF32 ? 64u : 128u;
    const uint64_t most = capacity == 0 ? 1 : (capacity - 1u) / tile + 1u, all = (uint64_t)seqs * pairs;
    const bool few = all < kPagedFull;
    chunks = few ? kPagedFull : kPagedChunks;
    least = few || dtype == kF32 ? 2u : 4u;
    whole = few && dtype != kF32 ? 5u : least;
    split = most > whole ? 1u : 0u;
    const uint64_t each = (most + least - 1u) / least;   // chunks of a sequence at most
    workgroups = (uint32_t)(split ? (all + chunks < all * each ? all + chunks : all * each) : all);
    pieces = (uint32_t)(split ? (2u * chunks < all * each ? 2u * chunks : all * each) : 0u);
    listed = split && seqs > kPagedFind ? (workgroups + pairs - 1u) / pairs : 0u;
  }
  uint64_t parts_bytes() const { return (uint64_t)pieces * part_floats() * sizeof(float) + 16u * (uint64_t)listed; }
};

// Argument blocks travel by value in the kernel argument segment, which holds 4 KiB.
static_assert(sizeof(EwArgs) <= 4096 && sizeof(RowArgs) <= 4096 && sizeof(AllArgs) <= 4096 && sizeof(ColArgs) <= 4096 &&
                  sizeof(GemmArgs) <= 4096 && sizeof(SplitPostArgs) <= 4096 && sizeof(SliceArgs) <= 4096 &&
                  sizeof(AttnArgs) <= 4096 && sizeof(RopeArgs) <= 4096 && sizeof(AppendArgs) <= 4096 && sizeof(PagedArgs) <= 4096,
              "a kernel's argument block must fit the kernel argument segment");

}  // namespace ltk
#endif  // LT_KERNELS_H_
