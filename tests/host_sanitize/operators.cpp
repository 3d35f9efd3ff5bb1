// Rotary positions and the paged cache on the null device, built with -fsanitize=address,undefined
// (tests/test_operators_sanitized.py): recording, refusals, plans of the ordinary and the degenerate sizes, and how an attention
// over a paged cache is shared out, for random sizes and lengths.  Exit code 0 = every expectation held.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <limits>
#include <random>
#include <string>
#include <vector>

#include "../../include/lt.h"
#include "../../paper_2102_13267_amd/csrc/lt_kernels.h"

#define CHECK(cond)                                                         \
  do {                                                                      \
    if (!(cond)) {                                                          \
      std::fprintf(stderr, "%s:%d: CHECK failed: %s\n", __FILE__, __LINE__, #cond); \
      std::exit(1);                                                         \
    }                                                                       \
  } while (0)

static lt_ctx* ctx;

static lt_tensor dev(std::vector<int64_t> dims, lt_dtype dt, bool donatable = false) {
  lt_tensor t = 0;
  CHECK(lt_tensor_from_device(ctx, nullptr, dt, (int)dims.size(), dims.data(), donatable ? LT_DONATABLE : 0, &t) == LT_OK);
  return t;
}
static lt_status op(uint16_t code, std::vector<lt_tensor> in, std::vector<lt_attr> attrs, lt_tensor* out) {
  return lt_op(ctx, code, in.data(), (int)in.size(), attrs.data(), (int)attrs.size(), out, 1);
}
static lt_attr integer(uint16_t key, int64_t v) {
  lt_attr a{};
  a.key = key;
  a.v.i = v;
  return a;
}
static lt_attr real(uint16_t key, double v) {
  lt_attr a{};
  a.key = key;
  a.is_float = 1;
  a.v.f = v;
  return a;
}

// One step of decoding and one of a prompt: rotation, append (in place and copied), attention.
static void steps(int64_t seqs, int64_t tokens, int64_t heads, int64_t kv, int64_t dim, int64_t rows, int64_t slots, int64_t pages, lt_dtype dt) {
  const lt_tensor cache = dev({pages, 2, kv, rows, dim}, dt, true), lengths = dev({seqs}, LT_I32), table = dev({seqs, slots}, LT_I32), offsets = dev({seqs + 1}, LT_I32);
  const lt_tensor q = dev({seqs, heads, dim}, dt), k = dev({seqs, kv, dim}, dt), positions = dev({seqs}, LT_I32), ks = dev({tokens, kv, dim}, dt);
  std::vector<lt_attr> turn;
  if (dim >= 2) turn = {integer(LT_ATTR_ROPE_DIMS, dim / 2 * 2 > 256 ? 256 : dim / 2 * 2), integer(LT_ATTR_ROPE_INTERLEAVED, rows % 2)};
  for (int round = 0; round < 2; ++round) {
    lt_tensor a = 0, b = 0, r = q, o = 0;
    CHECK(op(LT_OP_CACHE_APPEND, {cache, ks, ks, lengths, table, offsets}, turn, &a) == LT_OK);
    CHECK(lt_assign(ctx, cache, a) == LT_OK);
    CHECK(lt_release(ctx, a) == LT_OK);
    if (round == 0) CHECK(lt_barrier(ctx, 1, nullptr) == LT_OK);
    CHECK(op(LT_OP_CACHE_APPEND, {cache, k, k, lengths, table}, turn, &b) == LT_OK);
    if (!turn.empty()) CHECK(op(round ? LT_OP_ROPE_GRAD : LT_OP_ROPE, {q, positions}, turn, &r) == LT_OK);
    CHECK(op(LT_OP_PAGED_ATTENTION, {r, b, lengths, table}, {}, &o) == LT_OK);
    CHECK(lt_barrier(ctx, 1, nullptr) == LT_OK);
    size_t n = 0;
    CHECK(lt_dump_plan(ctx, nullptr, 0, &n) == LT_OK && lt_dump_schedule(ctx, nullptr, 0, &n) == LT_OK && lt_dump_ir(ctx, nullptr, 0, &n) == LT_OK);
    CHECK(lt_release(ctx, b) == LT_OK && lt_release(ctx, o) == LT_OK);
    if (r != q) CHECK(lt_release(ctx, r) == LT_OK);
  }
  for (lt_tensor t : {cache, lengths, table, offsets, q, k, positions, ks}) CHECK(lt_release(ctx, t) == LT_OK);
}

static void refusals() {
  const double inf = std::numeric_limits<double>::infinity(), nan = std::nan("");
  const lt_tensor x = dev({3, 2, 8}, LT_F32), p = dev({3}, LT_I32), cache = dev({4, 2, 2, 16, 8}, LT_F32, true), l = dev({3}, LT_I32), t = dev({3, 5}, LT_I32);
  lt_tensor out = 0;
  for (double v : {inf, -inf, nan, -1.0, 0.0, 0.5}) {
    CHECK(op(LT_OP_ROPE, {x, p}, {real(LT_ATTR_ROPE_BASE, v)}, &out) == LT_ERR_ARG);
    CHECK(op(LT_OP_ROPE_GRAD, {x, p}, {real(LT_ATTR_ROPE_FACTOR, v)}, &out) == LT_ERR_ARG);
    CHECK(op(LT_OP_CACHE_APPEND, {cache, x, x, l, t}, {real(LT_ATTR_ROPE_HIGH, v)}, &out) == LT_ERR_ARG);
  }
  for (int64_t v : {INT64_MIN, (int64_t)-2, (int64_t)0, (int64_t)1, (int64_t)3, (int64_t)10, INT64_MAX})
    CHECK(op(LT_OP_ROPE, {x, p}, {integer(LT_ATTR_ROPE_DIMS, v)}, &out) == LT_ERR_ARG);
  for (double v : {inf, nan, 1e300, 3e38, -3e38}) CHECK(op(LT_OP_PAGED_ATTENTION, {x, cache, l, t}, {real(LT_ATTR_SCALE, v)}, &out) == LT_ERR_ARG);
  CHECK(op(LT_OP_PAGED_ATTENTION, {x, cache, l}, {}, &out) == LT_ERR_ARG && op(LT_OP_CACHE_APPEND, {cache, x, x, l}, {}, &out) == LT_ERR_ARG && op(LT_OP_ROPE, {x}, {}, &out) == LT_ERR_ARG);
  CHECK(op(LT_OP_PAGED_ATTENTION, {x, x, l, t}, {}, &out) == LT_ERR_SHAPE && op(LT_OP_ROPE, {x, x}, {}, &out) == LT_ERR_DTYPE);
  // sizes whose products pass 63 bits
  const lt_tensor huge = dev({(int64_t)1 << 40, 2, 1, 1, 1}, LT_F32), wide = dev({3, (int64_t)1 << 31}, LT_I32), one = dev({3, 1, 1}, LT_F32);
  CHECK(op(LT_OP_PAGED_ATTENTION, {one, huge, l, t}, {}, &out) == LT_ERR_SHAPE && op(LT_OP_CACHE_APPEND, {cache, x, x, l, wide}, {}, &out) == LT_ERR_SHAPE);
  for (lt_tensor h : {x, p, cache, l, t, huge, wide, one}) CHECK(lt_release(ctx, h) == LT_OK);
}

// More blocks than a launch has threads for, and more tiles than 31 bits count.
static void too_large(int64_t seqs, int64_t kv, int64_t slots, int64_t rows, lt_status expected) {
  const lt_tensor q = dev({seqs, kv, 4}, LT_F32), cache = dev({9, 2, kv, rows, 4}, LT_F32), l = dev({seqs}, LT_I32), t = dev({seqs, slots}, LT_I32);
  lt_tensor out = 0;
  CHECK(op(LT_OP_PAGED_ATTENTION, {q, cache, l, t}, {}, &out) == LT_OK);
  CHECK(lt_barrier(ctx, 1, nullptr) == expected);
  for (lt_tensor h : {q, cache, l, t, out}) CHECK(lt_release(ctx, h) == LT_OK);
}

// What workgroups of an attention take: every tile of every block once, and never more pieces, workgroups or entries than there is room for.
static void shares(std::mt19937& rng) {
  auto pick = [&](int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); };
  ltk::PagedArgs a{};
  a.dtype = pick(0, 1) ? ltk::kF32 : ltk::kBF16;
  a.seqs = (uint32_t)(1u << pick(0, 11)) + (uint32_t)pick(0, 5);
  a.kv_heads = (uint32_t)pick(1, 9);
  a.heads = a.kv_heads * (uint32_t)(pick(0, 3) ? pick(1, 8) : pick(15, 70));
  a.dim = (uint32_t)pick(1, 256);
  a.rows.set((uint32_t)pick(1, 64));
  a.slots = (uint32_t)(1u << pick(0, 10));
  a.capacity = a.slots * a.rows.d;
  a.share_out();
  CHECK(a.dim <= a.padded && a.pairs * a.blocks_of >= a.heads && a.workgroups >= a.seqs * a.pairs);
  if (!a.split) {
    CHECK(a.workgroups == a.seqs * a.pairs && a.pieces == 0 && a.listed == 0 && a.parts_bytes() == 0);
    return;
  }
  const int64_t skew = pick(1, 12);
  std::vector<uint64_t> tiles(a.seqs);
  uint64_t all = 0;
  for (uint64_t& t : tiles) {
    const uint64_t n = (uint64_t)(a.capacity * std::pow(pick(0, 1000) / 1000.0, (double)skew));
    t = n == 0 ? 1 : (n - 1) / a.tile + 1;
    all += t;
  }
  const uint64_t c = std::max<uint64_t>(a.least, (all * a.pairs + a.chunks - 1) / a.chunks);
  uint64_t chunks = 0, pieces = 0;
  for (uint64_t t : tiles) {
    const uint64_t k = t <= a.whole ? 1 : (t + c - 1) / c;
    chunks += k;
    if (k > 1) pieces += k;
    CHECK(k < 65536);
  }
  CHECK(chunks * a.pairs <= a.workgroups && pieces * a.pairs <= a.pieces && a.pieces <= 2 * a.chunks && a.chunks <= ltk::kPagedChunks);
  CHECK((a.listed != 0) == (a.seqs > ltk::kPagedFind) && (a.listed == 0 || ((uint64_t)a.listed * a.pairs >= a.workgroups && chunks <= a.listed)));
  CHECK(a.parts_bytes() % 16 == 0 && a.parts_bytes() >= 4 * a.pieces * a.part_floats());
}

int main() {
  CHECK(lt_init(-1, nullptr, nullptr, 0, &ctx) == LT_OK);
  refusals();
  for (lt_dtype dt : {LT_F32, LT_BF16}) {
    steps(3, 7, 4, 2, 8, 4, 5, 7, dt);
    steps(1, 1, 1, 1, 1, 1, 1, 1, dt);
    steps(400, 900, 8, 2, 128, 16, 300, 5000, dt);
    steps(64, 1 << 20, 32, 8, 128, 16, 1000, 100000, dt);
    steps(2, 3, 70, 1, 255, 7, 2, 4, dt);
    steps(3, 4, 6, 3, 20, 5, 3, 0, dt);    // no pages
    steps(3, 4, 6, 3, 20, 5, 0, 4, dt);    // no slots
    steps(3, 0, 6, 3, 20, 5, 2, 4, dt);    // no new tokens
    steps(0, 0, 6, 3, 20, 5, 2, 4, dt);    // no sequences
    steps(0, 5, 6, 3, 20, 5, 2, 4, dt);
  }
  too_large((int64_t)1 << 24, 1, 1, 1, LT_ERR_UNSUPPORTED);
  too_large(((int64_t)1 << 24) - 1, 1, 1, 1, LT_OK);
  too_large(((int64_t)1 << 24) - 1, 1, 1000, 1, LT_ERR_UNSUPPORTED);
  too_large((int64_t)1 << 20, 8, 2, 1, LT_OK);
  too_large((int64_t)1 << 20, 16, 2, 1, LT_ERR_UNSUPPORTED);
  too_large(64, 1, ((int64_t)1 << 31) - 1, 1, LT_ERR_UNSUPPORTED);
  std::mt19937 rng(1);
  for (int i = 0; i < 4000; ++i) shares(rng);
  CHECK(lt_shutdown(ctx) == LT_OK);
  std::puts("operators: ok");
  return 0;
}
