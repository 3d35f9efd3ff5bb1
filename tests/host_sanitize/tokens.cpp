// Table lookups, dropout and the cross entropy over a vocabulary on the null device, built with -fsanitize=address,undefined
// (tests/test_token_operators_sanitized.py): plans of ordinary and degenerate sizes, in one barrier and in several, refusals, and how a table's
// gradient and a few tokens are shared out, for random sizes.  Exit code 0 = every expectation held.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
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
static lt_status op(uint16_t code, std::vector<lt_tensor> in, std::vector<lt_attr> attrs, lt_tensor* out, int n_out = 1) {
  return lt_op(ctx, code, in.data(), (int)in.size(), attrs.data(), (int)attrs.size(), out, n_out);
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
static void dumps() {
  size_t n = 0;
  CHECK(lt_dump_plan(ctx, nullptr, 0, &n) == LT_OK && lt_dump_schedule(ctx, nullptr, 0, &n) == LT_OK && lt_dump_ir(ctx, nullptr, 0, &n) == LT_OK);
}

// A step of training at a model's two ends, the losses' gradient one number or one a token; the second one in a barrier for each operator.
static void steps(int64_t tokens, int64_t vocab, int64_t dim, lt_dtype dt, bool xent) {
  const lt_tensor table = dev({vocab, dim}, dt, true), ids = dev({tokens}, LT_I32), state = dev({2}, LT_I64), weights = dev({tokens}, LT_F32), mean = dev({}, LT_F32);
  for (int round = 0; round < 4; ++round) {
    const bool apart = round & 1;
    std::vector<lt_tensor> made;
    auto keep = [&](lt_tensor t) {
      made.push_back(t);
      if (apart) CHECK(lt_barrier(ctx, 1, nullptr) == LT_OK);
      return t;
    };
    lt_tensor y = 0, x = 0, both[2] = {}, grads[2] = {}, back = 0, grad = 0;
    CHECK(op(LT_OP_EMBEDDING, {table, ids}, {real(LT_ATTR_SCALE, 2.0)}, &y) == LT_OK);
    keep(y);
    CHECK(op(LT_OP_DROPOUT, {y, state, y}, {real(LT_ATTR_RATE, 0.1), integer(LT_ATTR_SITE, 3)}, &x) == LT_OK);
    keep(x);
    if (xent) {
      CHECK(op(LT_OP_LINEAR_XENT, {x, table, ids}, {}, both, 2) == LT_OK);
      keep(both[0]);
      keep(both[1]);
      CHECK(op(LT_OP_LINEAR_XENT_GRAD, {x, table, ids, both[1], round & 2 ? weights : mean}, {}, grads, 2) == LT_OK);
      keep(grads[0]);
      keep(grads[1]);
    } else {
      grads[0] = x;
      CHECK(op(LT_OP_EMBEDDING_GRAD, {x, ids}, {integer(LT_ATTR_ROWS, vocab)}, &grads[1]) == LT_OK);
      keep(grads[1]);
    }
    CHECK(op(LT_OP_DROPOUT, {grads[0], state}, {real(LT_ATTR_RATE, 0.1), integer(LT_ATTR_SITE, 3)}, &back) == LT_OK);
    keep(back);
    CHECK(op(LT_OP_EMBEDDING_GRAD, {back, ids, grads[1]}, {real(LT_ATTR_SCALE, 2.0)}, &grad) == LT_OK);
    keep(grad);
    if (round & 2) CHECK(lt_assign(ctx, table, grad) == LT_OK);
    CHECK(lt_barrier(ctx, 1, nullptr) == LT_OK);
    dumps();
    for (lt_tensor t : made) CHECK(lt_release(ctx, t) == LT_OK);
  }
  // a result alone
  lt_tensor both[2] = {}, grads[2] = {};
  for (int keep = 0; xent && keep < 4; ++keep) {
    CHECK(op(LT_OP_LINEAR_XENT, {op(LT_OP_EMBEDDING, {table, ids}, {}, &grads[0]) == LT_OK ? grads[0] : 0, table, ids}, {}, both, 2) == LT_OK);
    const lt_tensor x = grads[0];
    CHECK(op(LT_OP_LINEAR_XENT_GRAD, {x, table, ids, both[1], mean}, {}, grads, 2) == LT_OK);
    const lt_tensor all[4] = {both[0], both[1], grads[0], grads[1]};
    for (int i = 0; i < 4; ++i)
      if (i != keep) CHECK(lt_release(ctx, all[i]) == LT_OK);
    CHECK(lt_release(ctx, x) == LT_OK);
    CHECK(lt_barrier(ctx, 1, nullptr) == LT_OK);
    dumps();
    CHECK(lt_release(ctx, all[keep]) == LT_OK);
  }
  for (lt_tensor t : {table, ids, state, weights, mean}) CHECK(lt_release(ctx, t) == LT_OK);
}

static void refusals() {
  const lt_tensor table = dev({7, 8}, LT_F32), ids = dev({3}, LT_I32), x = dev({3, 8}, LT_F32), b = dev({3, 8}, LT_BF16), state = dev({2}, LT_I64), l = dev({3}, LT_F32), longer = dev({4}, LT_F32);
  lt_tensor out[2] = {};
  for (double rate : {-0.1, 1.0, 2.0, (double)INFINITY, (double)NAN}) CHECK(op(LT_OP_DROPOUT, {x, state}, {real(LT_ATTR_RATE, rate)}, out) == LT_ERR_ARG);
  CHECK(op(LT_OP_DROPOUT, {x, ids}, {real(LT_ATTR_RATE, 0.1)}, out) != LT_OK);
  CHECK(op(LT_OP_DROPOUT, {x, state, b}, {real(LT_ATTR_RATE, 0.1)}, out) != LT_OK);
  CHECK(op(LT_OP_EMBEDDING, {ids, ids}, {}, out) != LT_OK);
  CHECK(op(LT_OP_EMBEDDING, {table, l}, {}, out) != LT_OK);
  CHECK(op(LT_OP_EMBEDDING_GRAD, {x, ids}, {}, out) != LT_OK);
  CHECK(op(LT_OP_EMBEDDING_GRAD, {x, ids}, {integer(LT_ATTR_ROWS, -1)}, out) != LT_OK);
  CHECK(op(LT_OP_EMBEDDING_GRAD, {x, ids}, {integer(LT_ATTR_ROWS, (int64_t)1 << 40)}, out) != LT_OK);
  CHECK(op(LT_OP_EMBEDDING_GRAD, {x, ids, ids}, {}, out) != LT_OK);
  CHECK(op(LT_OP_LINEAR_XENT, {x, table, ids}, {}, out, 1) != LT_OK);
  CHECK(op(LT_OP_LINEAR_XENT, {b, table, ids}, {}, out, 2) != LT_OK);
  CHECK(op(LT_OP_LINEAR_XENT, {x, table, l}, {}, out, 2) != LT_OK);
  CHECK(op(LT_OP_LINEAR_XENT_GRAD, {x, table, ids, l}, {}, out, 2) != LT_OK);
  CHECK(op(LT_OP_LINEAR_XENT_GRAD, {x, table, ids, l, longer}, {}, out, 2) != LT_OK);
  CHECK(op(LT_OP_LINEAR_XENT_GRAD, {x, table, ids, longer, l}, {}, out, 2) != LT_OK);
  for (lt_tensor t : {table, ids, x, b, state, l, longer}) CHECK(lt_release(ctx, t) == LT_OK);
}

static void shares(std::mt19937& rng) {
  auto pick = [&](uint32_t most) { return (uint32_t)std::exp(std::uniform_real_distribution<double>(0.0, std::log((double)most))(rng)); };
  ltk::EmbedGradArgs a{};
  a.tokens = pick((1u << 27) - 1u);
  a.rows = pick((1u << 27) - 1u);
  a.share_out();
  CHECK(a.blocks >= 1 && a.blocks <= ltk::kEmbedBlocks && a.each % ltk::kEmbedBlock == 0 && (uint64_t)a.each * a.blocks >= a.tokens);
  CHECK((uint64_t)a.piece * a.pieces >= a.tokens && (uint64_t)a.piece * (a.pieces - 1) < a.tokens && a.pieces <= 4096 + 1);
  CHECK(a.rows >> a.bits == 0);
  if (a.few()) CHECK(a.tokens <= ltk::kEmbedFew && ((uint64_t)a.rows + 1) * ltk::kEmbedFew <= (uint64_t)1 << 32);
  const uint32_t n = pick(100), width = 32 * pick(1u << 15);
  if (ltk::vocab_few(n, width, 4)) CHECK(n <= 16 * ltk::vocab_few_blocks(n) && (uint64_t)n * ((width * 4ull + 255) & ~255ull) <= ltk::kVocabFewBytes);
}

int main() {
  CHECK(lt_init(-1, nullptr, nullptr, 0, &ctx) == LT_OK);
  refusals();
  for (lt_dtype dt : {LT_F32, LT_BF16}) {
    for (int64_t tokens : {1, 64, 65, 5331})
      for (int64_t vocab : {1, 4097, 300000})
        for (int64_t dim : {33, 2048}) steps(tokens, vocab, dim, dt, true);
    steps(8192, 131072, 256, dt, true);
    steps(1 << 20, 1000, 8, dt, false);
    steps(1000, 1 << 20, 8, dt, false);
    steps(0, 5, 8, dt, true);
    steps(0, 5, 8, dt, false);
    steps(5, 0, 8, dt, false);
    steps(5, 3, 0, dt, false);
  }
  std::mt19937 rng(1);
  for (int i = 0; i < 20000; ++i) shares(rng);
  CHECK(lt_shutdown(ctx) == LT_OK);
  std::puts("tokens: ok");
  return 0;
}
