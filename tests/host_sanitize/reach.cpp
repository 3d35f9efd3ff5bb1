// How many threads the launches of the token operators have, at the largest sizes that are accepted, planned on the null device
// (tests/test_token_operators_reach.py): below 2^32 along x, and as many workgroups as there is work for.  Exit code 0 = every expectation held.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../include/lt.h"
#include "../../paper_2102_13267_amd/csrc/lt_core.h"

#define CHECK(cond)                                                         \
  do {                                                                      \
    if (!(cond)) {                                                          \
      std::fprintf(stderr, "%s:%d: CHECK failed: %s\n", __FILE__, __LINE__, #cond); \
      std::exit(1);                                                         \
    }                                                                       \
  } while (0)

static lt_ctx* ctx;

static lt_tensor dev(std::vector<int64_t> dims, lt_dtype dt) {
  lt_tensor t = 0;
  CHECK(lt_tensor_from_device(ctx, nullptr, dt, (int)dims.size(), dims.data(), 0, &t) == LT_OK);
  return t;
}
static void op(uint16_t code, std::vector<lt_tensor> in, std::vector<lt_attr> attrs, lt_tensor* out, int n_out) {
  CHECK(lt_op(ctx, code, in.data(), (int)in.size(), attrs.data(), (int)attrs.size(), out, n_out) == LT_OK);
}

static void holds(uint64_t workgroups, uint64_t at_least) {
  CHECK(workgroups >= at_least && workgroups < ltk::kMostWorkgroups);
  const ltk::ManyWorkgroups grid = ltk::many_workgroups(workgroups);
  CHECK((uint64_t)grid.x * 256u < (uint64_t)1 << 32 && grid.y <= 65535u && (uint64_t)grid.x * grid.y >= workgroups);
  CHECK((uint64_t)grid.x * grid.y * 4u < (uint64_t)1 << 32);   // (waves are counted in 32 bits)
}

// every launch of the plan; the passes of a cross entropy that were seen, a bit each
static uint32_t look(uint32_t v) {
  uint32_t seen = 0;
  for (const lt::Launch& l : ctx->last_plan->launches) {
    if (l.kind == lt::L_EMBEDGRAD) {
      const ltk::EmbedGradArgs& a = *(const ltk::EmbedGradArgs*)l.args.data();
      if (a.pass == ltk::kEmbedSum || a.pass == ltk::kEmbedJoin) holds(a.workgroups(v), 1);
      else CHECK(a.blocks <= ltk::kEmbedBlocks);
    } else if (l.kind == lt::L_VOCAB) {
      const ltk::VocabArgs& a = *(const ltk::VocabArgs*)l.args.data();
      seen |= 1u << a.pass;
      if (a.pass == ltk::kVocabPack) holds(a.workgroups(), ((a.pack_w ? a.rows : a.tokens) + 3u) / 4u);
      if (a.pass == ltk::kVocabDxOut) holds(a.workgroups(), (a.tokens + 3u) / 4u);
      if (a.pass == ltk::kVocabKept) holds(a.workgroups(), ((uint64_t)a.tokens * a.rows + 1023u) / 1024u);
      if (a.pass == ltk::kVocabLoss) CHECK((uint64_t)(a.padded / 64u) * 1024u < (uint64_t)1 << 32);
    }
  }
  return seen;
}

static uint32_t entropy(int64_t tokens, int64_t vocab, int64_t dim, lt_dtype dt, bool each) {
  const lt_tensor x = dev({tokens, dim}, dt), w = dev({vocab, dim}, dt), labels = dev({tokens}, LT_I32), dloss = each ? dev({tokens}, LT_F32) : dev({}, LT_F32);
  lt_tensor both[2], grads[2];
  op(LT_OP_LINEAR_XENT, {x, w, labels}, {}, both, 2);
  op(LT_OP_LINEAR_XENT_GRAD, {x, w, labels, both[1], dloss}, {}, grads, 2);
  CHECK(lt_barrier(ctx, 1, nullptr) == LT_OK);
  const uint32_t seen = look(1);
  for (lt_tensor t : {x, w, labels, dloss, both[0], both[1], grads[0], grads[1]}) CHECK(lt_release(ctx, t) == LT_OK);
  return seen;
}

static void gradient(int64_t tokens, int64_t rows, int64_t dim, uint32_t v) {
  const lt_tensor dy = dev({tokens, dim}, LT_BF16), ids = dev({tokens}, LT_I32);
  lt_attr n{};
  n.key = LT_ATTR_ROWS;
  n.v.i = rows;
  lt_tensor out = 0;
  op(LT_OP_EMBEDDING_GRAD, {dy, ids}, {n}, &out, 1);
  CHECK(lt_barrier(ctx, 1, nullptr) == LT_OK);
  look(v);
  for (lt_tensor t : {dy, ids, out}) CHECK(lt_release(ctx, t) == LT_OK);
}

int main() {
  CHECK(lt_init(-1, nullptr, nullptr, 0, &ctx) == LT_OK);
  const int64_t most = ((int64_t)1 << 27) - 1;
  const uint32_t rows = 1u << ltk::kVocabPack | 1u << ltk::kVocabDxOut, kept = 1u << ltk::kVocabKept;
  for (lt_dtype dt : {LT_F32, LT_BF16})
    for (bool each : {false, true})
      for (int64_t tokens : {most, (int64_t)1 << 26, ((int64_t)1 << 26) - 1, (int64_t)1 << 25}) CHECK((entropy(tokens, 200, 8, dt, each) & rows) == rows);
  CHECK(entropy(1 << 23, 2048, 128, LT_F32, false) & kept);   // (69 GB of logits)
  CHECK(entropy((1 << 23) - 1, 4000, 128, LT_F32, true) & kept);
  // tables of 200 GB, and few rows that are long, element by element and eight at once
  gradient(1000, ((int64_t)1 << 21) - 1, 50001, 1);
  gradient(1000, ((int64_t)1 << 21) - 1, 50000, 8);
  gradient(4096, 8, ((int64_t)1 << 23) + 1, 1);
  gradient(40000, 3, ((int64_t)1 << 21) + 1, 1);
  gradient(4096, 8, (int64_t)1 << 24, 8);
  gradient(most, most, 1, 1);
  gradient(most, most, 512, 8);
  CHECK(lt_shutdown(ctx) == LT_OK);
  std::puts("reach: ok");
  return 0;
}
