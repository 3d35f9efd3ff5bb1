"""Table lookups, dropout and the cross entropy over a vocabulary together, as a language model's step has them at its two ends, and in the ways a step is run:
captured and replayed, as HIP graphs, through the static barrier, over streams, from windows and views, on another stream, far out in large tensors."""
import numpy as np
import pytest
import torch

from oracle.numeric import Eager, round_to_bf16
from paper_2102_13267_amd import Context
from test_gpu_token_operators import E24, HALF, TINY, context, data, entropy_bounds, entropy_case, grad_bound, grads_bound, within

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


class Step:
    """Lookup, dropout, cross entropy with the same table, backward to the one gradient of that table, which is updated in place."""

    def __init__(self, ctx, dtype, tokens=70, vocab=500, dim=64, seed=0):
        rg = np.random.default_rng(seed)
        self.ctx, self.dtype, self.vocab, self.rg = ctx, dtype, vocab, rg
        self.table = torch.tensor(data(rg, (vocab, dim), dtype, 3.0 / np.sqrt(dim)), device="cuda").to(TORCH[dtype])
        self.ids, self.labels = (torch.tensor(rg.integers(-1, vocab, tokens).astype(np.int32), device="cuda") for _ in range(2))
        self.state = torch.tensor([12345 + seed, 7], dtype=torch.int64, device="cuda")
        self.T = ctx.tensor(self.table, donatable=True)
        self.I, self.L, self.S = ctx.tensor(self.ids), ctx.tensor(self.labels), ctx.tensor(self.state)

    def record(self, B=None, lr=0.25):
        B = B or self.ctx
        if B is self.ctx:
            T, I, L, S = self.T, self.I, self.L, self.S
        else:
            T, I, L, S = B.tensor(self.table.float().cpu().numpy(), self.dtype), B.tensor(self.ids.cpu().numpy()), B.tensor(self.labels.cpu().numpy()), B.tensor(self.state.cpu().numpy())
        x = B.dropout(B.embedding(T, I, scale=4.0), S, 0.1, site=3)
        loss, lse = B.linear_xent(x, T, L)
        dx, dw = B.linear_xent_grad(x, T, L, lse, 1.0 / 70)
        grad = B.embedding_grad(B.dropout_grad(dx, S, 0.1, site=3), I, into=dw, scale=4.0)
        B.assign(T, B.sub(T, B.mul(grad, lr)))
        return T, loss, grad

    def next(self):
        """other tokens, another step of the generator"""
        n = self.ids.numel()
        self.ids.copy_(torch.tensor(self.rg.integers(-1, self.vocab, n).astype(np.int32)))
        self.labels.copy_(torch.tensor(self.rg.integers(-1, self.vocab, n).astype(np.int32)))
        self.state[1] += 1
        torch.cuda.synchronize()

    def expected(self):
        """what a step makes of what is there now, op by op with the types' roundings"""
        E = Eager()
        T, loss, grad = self.record(E)
        return [E.fetch(t) for t in (T, loss, grad)]

    def check(self, want, loss, grad=None):
        """Of fp32: the ops' own roundings add up to a few hundred halves of a step of what is summed; of bf16: each of the four values of that type between
        the table and its gradient (x, dx, dw, the sum) is off by a rounding or two."""
        tol = 2e-5 if self.dtype == "f32" else 2e-2
        got = [self.table.float().cpu().numpy(), self.ctx.fetch(loss)] + ([] if grad is None else [self.ctx.fetch(grad)])
        for g, w in zip(got, want):
            assert np.linalg.norm(g - w) <= tol * np.linalg.norm(w), (np.linalg.norm(g - w), np.linalg.norm(w))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,dim", [(70, 500, 64), (333, 1500, 128), (1, 9, 8), (40, 2000, 100)])
def test_steps_with_one_table_at_both_ends(dtype, tokens, vocab, dim):
    ctx = context()
    s = Step(ctx, dtype, tokens, vocab, dim)
    for _ in range(3):
        want = s.expected()
        _, loss, grad = s.record()
        ctx.barrier()
        assert ctx.device_ptr(s.T) == s.table.data_ptr()               # updated in place
        s.check(want, loss, grad)
        s.next()
    ctx.close()


@pytest.mark.parametrize("fusion", [True, False])
def test_one_region_per_op_gives_the_same(fusion):
    outs = []
    for on in (True, fusion):
        ctx = context()
        ctx.set_fusion(on)
        s = Step(ctx, "f32", 50, 300, 64)
        _, loss, grad = s.record()
        outs.append([ctx.fetch(t) for t in (loss, grad)] + [s.table.cpu().numpy()])
        ctx.close()
    for a, b in zip(*outs):
        assert np.linalg.norm(a - b) <= 1e-5 * np.linalg.norm(a)       # (logits kept from one to the other, or formed twice: the same sums)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_step_and_graphs(dtype):
    ctx = context()
    ctx.set_graphs(True)
    s = Step(ctx, dtype)
    want = s.expected()
    _, loss, grad = s.record()
    ctx.barrier()
    step = ctx.capture_step()
    s.check(want, loss, grad)
    for i in range(7):
        s.next()
        want = s.expected()
        step.replay()
        if i % 3 == 1:
            torch.randn(1 << 20, device="cuda").sum()
        s.check(want, loss, grad)
    assert ctx.stats().graph_launches > 0
    ctx.close()


def test_a_step_through_the_static_barrier_and_in_a_captured_graph():
    stream = torch.cuda.Stream(device=0)
    ctx = context(stream=stream)
    s = Step(ctx, "bf16")
    torch.cuda.synchronize()
    want = s.expected()
    _, loss, grad = s.record()
    ctx.barrier_static()
    s.check(want, loss, grad)
    s.next()
    graph = torch.cuda.CUDAGraph()
    before = s.table.clone()
    with torch.cuda.graph(graph, stream=stream):
        _, loss, grad = s.record()
        ctx.barrier_static(False)
    s.table.copy_(before)
    for i in range(6):
        s.next()
        want = s.expected()
        if i % 2:
            torch.randn(1 << 20, device="cuda").sum()
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        s.check(want, loss, grad)
    del graph
    ctx.close()


def test_operators_spread_over_streams():
    """steps that do not depend on each other, whose temporaries must not meet"""
    runs = []
    for streams in (1, 4):
        ctx = context(workspace_bytes=1 << 30)
        ctx.set_streams(streams)
        steps = [Step(ctx, "bf16", 2000 + 300 * i, 9000 + 100 * i, 128, seed=i) for i in range(3)]
        for _ in range(3):
            outs = [s.record() for s in steps]
            ctx.barrier()
            assert (ctx.plan_streams() > 1) == (streams > 1)
            runs.append([ctx.fetch(o[1]) for o in outs] + [s.table.float().cpu().numpy() for s in steps])
            del outs
        ctx.close()
    for a, b in zip(runs[:3], runs[3:]):
        for x, y in zip(a, b):
            assert np.array_equal(x, y)


def test_two_contexts_on_streams_of_their_own():
    streams = [torch.cuda.Stream(device=0) for _ in range(2)]
    ctxs = [context(stream=st) for st in streams]
    steps = [Step(c, "bf16", 300, 3000, 64, seed=i) for i, c in enumerate(ctxs)]
    torch.cuda.synchronize()
    for _ in range(3):
        wants = [s.expected() for s in steps]
        outs = [s.record() for s in steps]
        for c in ctxs:
            c.barrier(False)
        for s, w, o in zip(steps, wants, outs):
            s.check(w, o[1], o[2])
            s.next()
        del outs
    for c in ctxs:
        c.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_kept_for_the_gradient_are_those_formed_again(dtype):
    """next to a gradient of other operands, which forms them itself"""
    rg = np.random.default_rng(1)
    tokens, vocab, dim = 300, 900, 2048
    x, w, labels = entropy_case(rg, (tokens,), vocab, dim, dtype)
    weight = rg.random(tokens).astype(np.float32)
    ctx = context()
    X, W, L, D = ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels), ctx.tensor(weight)
    loss, lse = ctx.linear_xent(X, W, L)
    together = ctx.linear_xent_grad(X, W, L, lse, D)
    ctx.barrier()
    apart = ctx.linear_xent_grad(X, W, L, lse, D)
    ctx.barrier()
    for a, b in zip(together, apart):
        a, b = ctx.fetch(a), ctx.fetch(b)
        assert np.linalg.norm(a - b) <= (1e-6 if dtype == "f32" else 1e-3) * np.linalg.norm(b)
    E = Eager("f64")
    lse32 = ctx.fetch(lse)
    rx, rw = (t.data for t in E.linear_xent_grad(E.tensor(x, dtype), E.tensor(w, dtype), E.tensor(labels), E.tensor(lse32), E.tensor(weight)))
    there, bx, bw = grads_bound(x, w, labels, lse32, weight, dtype)
    within(ctx.fetch(together[0])[there], rx[there], bx)
    within(ctx.fetch(together[1]), rw, bw)
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,dim,least", [(9000, 9001, 40, 8), (200, 600001, 8, 12)])
def test_many_pieces_of_the_vocabulary(tokens, vocab, dim, least, dtype):
    """so many tokens, or rows, that g is large or takes several pieces, the last of them short"""
    rg = np.random.default_rng(2)
    x, w, labels = entropy_case(rg, (tokens,), vocab, dim, dtype)
    ctx, E = context(workspace_bytes=1 << 30), Eager("f64")
    X, W, L = ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)
    loss, lse = ctx.linear_xent(X, W, L)
    dx, dw = ctx.linear_xent_grad(X, W, L, lse, 0.5)
    ctx.barrier()
    assert sum(line.split()[1] == "VOCAB" for line in ctx.dump_schedule().splitlines()) > least
    lse32 = ctx.fetch(lse)
    ref = [t.data for t in E.linear_xent(E.tensor(x, dtype), E.tensor(w, dtype), E.tensor(labels))]
    there, dlse, dloss = entropy_bounds(x, w, labels, dtype)
    within(lse32[there], ref[1][there], dlse)
    within(ctx.fetch(loss)[there], ref[0][there], dloss)
    rx, rw = (t.data for t in E.linear_xent_grad(E.tensor(x, dtype), E.tensor(w, dtype), E.tensor(labels), E.tensor(lse32), E.tensor(np.float32(0.5))))
    there, bx, bw = grads_bound(x, w, labels, lse32, np.float32(0.5), dtype)
    within(ctx.fetch(dx)[there], rx[there], bx)
    within(ctx.fetch(dw), rw, bw)
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_smaller_pieces_where_memory_is_short(dtype):
    """the same step in a workspace that holds pieces of g of 128 MB, but none as large as it would take"""
    rg = np.random.default_rng(16)
    x, w, labels = entropy_case(rg, (9000,), 9001, 136, dtype)
    got = []
    # (g in one piece: 9216 x 9216, 170 MB in bf16 and 340 in fp32, next to some 50 of sums and packed rows; 140 in pieces of 128)
    for room in (1 << 30, (210 if dtype == "bf16" else 300) << 20):
        ctx = context(workspace_bytes=room)
        X, W, L = ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)
        loss, lse = ctx.linear_xent(X, W, L)
        dx, dw = ctx.linear_xent_grad(X, W, L, lse, 0.5)
        ctx.barrier()
        got.append(([ctx.fetch(t) for t in (loss, lse, dx, dw)], sum(line.split()[1] == "VOCAB" for line in ctx.dump_schedule().splitlines())))
        ctx.close()
    assert got[0][1] < got[1][1]
    for a, b in zip(got[0][0], got[1][0]):
        assert np.linalg.norm(a - b) <= (1e-6 if dtype == "f32" else 1e-3) * np.linalg.norm(b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_losses_of_so_many_tokens_that_they_are_joined_piece_by_piece(dtype):
    rg = np.random.default_rng(3)
    tokens, vocab, dim = 300000, 9001, 8
    x, w, labels = entropy_case(rg, (tokens,), vocab, dim, dtype, ignored=0.0)
    ctx = context(workspace_bytes=1 << 30)
    loss, lse = ctx.linear_xent(ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels))
    ctx.barrier()
    assert sum(line.split()[1] == "VOCAB" for line in ctx.dump_schedule().splitlines()) > 4
    some = rg.integers(0, tokens, 500)
    E = Eager("f64")
    ref = [t.data for t in E.linear_xent(E.tensor(x[some], dtype), E.tensor(w, dtype), E.tensor(labels[some]))]
    _, dlse, dloss = entropy_bounds(x[some], w, labels[some], dtype)
    within(ctx.fetch(lse)[some], ref[1], dlse)
    within(ctx.fetch(loss)[some], ref[0], dloss)
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 20, 33])
def test_views_of_every_operand(dtype, dim):
    """windows along the first axis that start anywhere are read where they lie; other windows, permutations and broadcasts are copied"""
    rg = np.random.default_rng(4)
    ctx, E = context(), Eager("f64")

    def both(a, *kind):
        return [(B, B.tensor(a, *kind)) for B in (ctx, E)]
    big, ids, st, res = both(data(rg, (3, 31, dim), dtype), dtype), both(rg.integers(-1, 32, 61).astype(np.int32)), both(np.array([[1, 2], [3, 4], [5, 6]], np.int64)), both(data(rg, (1, dim), dtype), dtype)
    wide = both(data(rg, (12, dim + 9), dtype), dtype)
    outs = []
    for (B, b), (_, i), (_, s), (_, r), (_, z) in zip(big, ids, st, res, wide):
        table = B.reshape(B.narrow(b, 0, 1, 1), (31, dim))
        t = B.narrow(table, 0, 5, 25)
        j = B.narrow(i, 0, 7, 12)
        e = B.embedding(t, j, scale=2.0)
        x = B.narrow(z, 1, 3, dim)
        d = B.dropout(B.narrow(z, 0, 1, 11), B.reshape(B.narrow(s, 0, 1, 1), (2,)), 0.3, residual=B.narrow(z, 0, 0, 11))
        f = B.dropout(x, B.reshape(B.narrow(s, 0, 2, 1), (2,)), 0.3, residual=B.expand(r, (12, dim)))
        loss, lse = B.linear_xent(x, t, j)
        each = B.expand(B.tensor(np.array([0.3], np.float32)), (12,))
        dx, dw = B.linear_xent_grad(x, t, j, lse, each)
        g = B.embedding_grad(B.expand(B.reshape(r, (dim,)), (12, dim)), j, rows=25)
        h = B.embedding_grad(B.reshape(B.expand(B.narrow(B.reshape(x, (3, 4, dim)), 1, 1, 1), (3, 4, dim)), (12, dim)), j, into=t)
        p = B.embedding(B.permute(B.tensor(np.zeros((dim, 9), np.float32) + np.arange(9, dtype=np.float32)), (1, 0)), B.reshape(B.narrow(i, 0, 1, 6), (2, 3)))
        outs.append([B.fetch(v) for v in (e, d, f, loss, dx, dw, g, h, p)])
    for k, (a, b) in enumerate(zip(*outs)):
        assert a.shape == b.shape and np.linalg.norm(a - b) <= (1e-5 if dtype == "f32" else 1e-2) * np.linalg.norm(b), k
    ctx.close()


def test_a_rank_0_gradient_on_the_device():
    rg = np.random.default_rng(5)
    ctx = context()
    x, w, labels = entropy_case(rg, (90,), 400, 64, "f32")
    X, W, L = ctx.tensor(x), ctx.tensor(w), ctx.tensor(labels)
    loss, lse = ctx.linear_xent(X, W, L)
    scale = ctx.tensor(np.array([0.5], np.float32))
    for d in (ctx.mean(scale), ctx.scalar(0.5), 0.5, ctx.expand(ctx.scalar(0.5), (90,)), ctx.expand(scale, (90,))):
        got = [ctx.fetch(t) for t in ctx.linear_xent_grad(X, W, L, lse, d)]
        one = [ctx.fetch(t) for t in ctx.linear_xent_grad(X, W, L, lse, 1.0)]
        for a, b in zip(got, one):
            assert np.array_equal(a, b * np.float32(0.5))
    nothing = [ctx.fetch(t) for t in ctx.linear_xent_grad(X, W, L, lse, 0.0)]
    assert all((t == 0).all() for t in nothing)
    ctx.close()


def test_runs_are_the_same_bits():
    rg = np.random.default_rng(6)
    ctx = context(workspace_bytes=512 << 20)
    for dtype in ("f32", "bf16"):
        x, w, labels = entropy_case(rg, (700,), 5000, 192, dtype)
        X, W, L = ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)
        first = None
        for _ in range(4):
            loss, lse = ctx.linear_xent(X, W, L)
            dx, dw = ctx.linear_xent_grad(X, W, L, lse, 0.1)
            now = [ctx.fetch(t) for t in (loss, lse, dx, dw)]
            first = first or now
            assert all(np.array_equal(a, b) for a, b in zip(first, now))
    ctx.close()


def test_a_table_longer_than_32_bits_reach():
    """rows at the far end of a table of 2^32 elements and more"""
    dim = 4096
    rows = 2 ** 32 // dim + 1000
    table = torch.empty((rows, dim), dtype=torch.bfloat16, device="cuda")
    end = torch.randn((900, dim), device="cuda").to(torch.bfloat16)
    table[-900:] = end
    ids = torch.tensor([rows - 1, rows - 900, 2 ** 31 - 1, rows, rows - 450], dtype=torch.int32, device="cuda")
    ctx = context()
    T, I = ctx.tensor(table, donatable=True), ctx.tensor(ids)
    y = ctx.fetch(ctx.embedding(T, I))
    want = torch.stack([end[-1], end[0], torch.zeros_like(end[0]), torch.zeros_like(end[0]), end[450]]).float().cpu().numpy()
    assert np.array_equal(y, want)
    dy = torch.ones((5, dim), dtype=torch.bfloat16, device="cuda")
    ctx.assign(T, ctx.embedding_grad(ctx.tensor(dy), I, into=T))
    ctx.barrier()
    assert ctx.device_ptr(T) == table.data_ptr()
    after = end.clone()
    for k in (899, 0, 450):
        after[k] = (after[k].float() + 1).to(torch.bfloat16)
    assert torch.equal(table[-900:], after)
    # its last rows as a vocabulary's: the logits of the far rows are those of the same rows by themselves
    ctx.close()
    del table, dy


def test_a_vocabulary_longer_than_32_bits_reach():
    dim = 1024
    rows = 2 ** 32 // dim + 700
    w = torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda")
    w[-700:] = (torch.randn((700, dim), device="cuda") / 8).to(torch.bfloat16)
    for tokens in (5, 300):                                             # few, whose rows stay in LDS, and tiles of them
        x = torch.randn((tokens, dim), device="cuda").to(torch.bfloat16)
        labels = torch.randint(rows - 700, rows, (tokens,), dtype=torch.int32, device="cuda")
        ctx = context(workspace_bytes=(30 << 30) if tokens == 5 else (16 << 30))
        loss, lse = (ctx.fetch(t) for t in ctx.linear_xent(ctx.tensor(x), ctx.tensor(w), ctx.tensor(labels)))
        l = (x.double() @ w[-700:].double().t()).cpu().numpy()
        want = np.log(np.exp(l).sum(-1) + (rows - 700.0))
        assert np.allclose(lse, want, atol=1e-4)
        assert np.allclose(loss, want - l[np.arange(tokens), labels.cpu().numpy() - (rows - 700)], atol=1e-3)
        if tokens == 5:
            dw = ctx.linear_xent_grad(ctx.tensor(x), ctx.tensor(w), ctx.tensor(labels), ctx.tensor(lse), 1.0)[1]
            tail = ctx.fetch(ctx.narrow(dw, 0, rows - 700, 700))
            p = np.exp(l - want[:, None])
            p[np.arange(tokens), labels.cpu().numpy() - (rows - 700)] -= 1
            ref = p.T @ x.double().cpu().numpy()
            assert np.linalg.norm(tail - ref) <= 1e-2 * np.linalg.norm(ref)
        ctx.close()
    del w


def test_dropout_of_more_than_32_bits_of_elements():
    n = 2 ** 32 + 24
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    st = np.array([77, 1], np.int64)
    ctx = context(workspace_bytes=(9 << 30))
    y = ctx.dropout(ctx.tensor(x), ctx.tensor(st), 0.5, 9)
    tail = ctx.fetch(ctx.narrow(y, 0, n - 100, 100))
    assert np.array_equal(tail == 0, Eager.random_bits(100, st, 9, first=n - 100) < 32768)
    ctx.close()
    del x


def test_gradients_of_one_leaf_in_a_graph_while_others_live():
    """a captured backward pass next to an eager one of the same tensors"""
    ctx = context()
    ctx.set_graphs(True)
    rg = np.random.default_rng(8)
    x, w, labels = entropy_case(rg, (64,), 300, 64, "bf16")
    X, W, L = ctx.tensor(x, "bf16"), ctx.tensor(w, "bf16"), ctx.tensor(labels)
    held = []
    for i in range(6):
        loss, lse = ctx.linear_xent(X, W, L)
        held.append(ctx.linear_xent_grad(X, W, L, lse, 1.0))
        ctx.barrier()
        if i > 3:
            held.pop(0)
    first = [ctx.fetch(t) for t in held[0]]
    for h in held[1:]:
        assert all(np.array_equal(ctx.fetch(a), b) for a, b in zip(h, first))
    ctx.close()


def test_lookups_of_tied_rows_in_bf16_round_once():
    """a base and many small sums: one rounding of the whole, not one a term"""
    ctx, E = context(), Eager("f64")
    rg = np.random.default_rng(9)
    base = round_to_bf16(np.full((3, 16), 256.0, np.float32))
    dy, ids = data(rg, (5000, 16), "bf16", 0.01), np.ones(5000, np.int32)
    got = ctx.fetch(ctx.embedding_grad(ctx.tensor(dy, "bf16"), ctx.tensor(ids), into=ctx.tensor(base, "bf16")))
    ref = E.embedding_grad(E.tensor(dy, "bf16"), E.tensor(ids), into=E.tensor(base, "bf16")).data
    within(got, ref, grad_bound(dy, ids, 3, 1.0, ref, "bf16"))
    ctx.close()


@pytest.mark.parametrize("tokens", [3, 17, 90])
def test_long_sums_in_fp32(tokens):
    """all terms of one sign, 4096 of them: a sum is of sums of 256 at most, each off by as many half steps as it has terms"""
    rg = np.random.default_rng(11)
    ctx = context()
    dim, vocab = 4096, 300
    x, w = rg.uniform(0.5, 1.0, (tokens, dim)).astype(np.float32), (rg.uniform(0.5, 1.0, (vocab, dim)) / 512).astype(np.float32)
    labels = rg.integers(0, vocab, tokens).astype(np.int32)
    X, W, L = ctx.tensor(x), ctx.tensor(w), ctx.tensor(labels)
    loss, lse = ctx.linear_xent(X, W, L)
    dx, dw = ctx.linear_xent_grad(X, W, L, lse, 1.0)
    logits = x.astype(np.float64) @ w.astype(np.float64).T
    top = logits.max(-1)
    want = np.log(np.exp(logits - top[:, None]).sum(-1)) + top
    dl = (256 + dim / 256 + 2) * E24 * top
    dlse = dl + (3 * (top - logits.min(-1)) + 96 + vocab / 2048 + 8) * E24 + 3 * E24 * want
    got = ctx.fetch(lse)
    within(got, want, dlse, "lse")
    within(ctx.fetch(loss), want - logits[np.arange(tokens), labels], 2 * dlse, "loss")
    # the gradient's terms have both signs: what the logits are off goes through p, what the sums of 300 and of the tokens are off is by their terms
    g = np.exp(logits - want[:, None])
    dg = g * (dl + dlse)[:, None] + g * (3 * np.abs(logits - want[:, None]) + 4) * E24
    g[np.arange(tokens), labels] -= 1
    dg += E24 * np.abs(g)
    within(ctx.fetch(dx), g @ w, dg @ w + (256 + 8) * E24 * (np.abs(g) @ w) + TINY, "dx")
    within(ctx.fetch(dw), g.T @ x, dg.T @ x + (tokens + 8) * E24 * (np.abs(g).T @ x) + TINY, "dw")
    ctx.close()


@pytest.mark.parametrize("tokens", [2, 70])
def test_infinite_logits(tokens):
    """a logit of +inf makes its token's lse +inf, and its loss where that row is not the label's"""
    ctx = context()
    x, w = np.zeros((tokens, 64), np.float32), np.zeros((300, 64), np.float32)
    x[:, 0] = 1.0
    w[:, 0] = np.linspace(-1, 1, 300)
    w[7, 1], w[8, 1] = 3e38, -3e38
    x[0, 1], x[1, 1] = 10.0, -10.0       # token 0: +inf at row 7, -inf at row 8; token 1 the other way round
    labels = np.full(tokens, 5, np.int32)
    want = np.array([np.inf, np.inf] + [np.log(np.exp(np.float64(w[:, 0])).sum())] * (tokens - 2))
    loss, lse = (ctx.fetch(t) for t in ctx.linear_xent(ctx.tensor(x), ctx.tensor(w), ctx.tensor(labels)))
    assert np.isposinf(lse[:2]).all() and np.isposinf(loss[:2]).all()
    assert np.allclose(lse[2:], want[2:], rtol=0, atol=1e-4) and np.allclose(loss[2:], want[2:] - w[5, 0], rtol=0, atol=1e-4)
    ctx.close()


@pytest.mark.parametrize("dtype,tokens,dim", [("f32", 9, 4096), ("f32", 8, 2080), ("f32", 19, 2048), ("bf16", 2, 16384), ("bf16", 3, 30016), ("bf16", 40, 1920)])
def test_few_tokens_of_long_rows(dtype, tokens, dim):
    """rows of x that fit in shared memory, or just do not"""
    rg = np.random.default_rng(12)
    ctx, E = context(), Eager("f64")
    x, w, labels = entropy_case(rg, (tokens,), 1003, dim, dtype)
    there, dlse, dloss = entropy_bounds(x, w, labels, dtype)
    ref = [t.data for t in E.linear_xent(E.tensor(x, dtype), E.tensor(w, dtype), E.tensor(labels))]
    loss, lse = ctx.linear_xent(ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels))
    within(ctx.fetch(lse)[there], ref[1][there], dlse, "lse")
    within(ctx.fetch(loss)[there], ref[0][there], dloss, "loss")
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [33, 200])
def test_rows_packed_once(dtype, dim):
    """rows of w that are no whole slabs, a cross entropy and its gradient in one trace and in two: the same bits"""
    rg = np.random.default_rng(13)
    ctx = context()
    x, w, labels = entropy_case(rg, (130,), 700, dim, dtype)
    X, W, L = ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)
    loss, lse = ctx.linear_xent(X, W, L)
    dx, dw = ctx.linear_xent_grad(X, W, L, lse, 0.25)
    one = [ctx.fetch(t) for t in (loss, lse, dx, dw)]
    loss, lse = ctx.linear_xent(X, W, L)
    two = [ctx.fetch(loss), ctx.fetch(lse)]
    two += [ctx.fetch(t) for t in ctx.linear_xent_grad(X, W, L, lse, 0.25)]
    for a, b in zip(one, two):
        assert np.array_equal(a, b)
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_added_where_they_lie(dtype):
    """chains of table gradients on top of a cross entropy's: the same bits as one barrier after the other, whatever else reads them or is kept"""
    rg = np.random.default_rng(14)
    ctx = context()
    x, w, labels = entropy_case(rg, (130,), 700, 64, dtype)
    X, W, L = ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)
    I, J, N = (ctx.tensor(rg.integers(-1, 701, n).astype(np.int32)) for n in (90, 300, 0))
    Y, Z = ctx.tensor(data(rg, (90, 64), dtype), dtype), ctx.tensor(data(rg, (300, 64), dtype), dtype)
    none = ctx.tensor(np.zeros((0, 64), np.float32), dtype)

    def program(after, keep):
        loss, lse = ctx.linear_xent(X, W, L)
        after(lse)
        dx, dw = ctx.linear_xent_grad(X, W, L, lse, 0.25)
        after(dw)
        one = ctx.embedding_grad(Y, I, into=dw)
        after(one)
        two = ctx.embedding_grad(Z, J, into=one, scale=0.5)
        after(two)
        three = ctx.embedding_grad(none, N, into=two)
        after(three)
        r = dict(dx=dx, dw=dw, one=one, two=two, three=three)
        if keep == "read":
            r = dict(three=three, more=ctx.add(dw, one))
        elif keep == "itself":
            r = dict(again=ctx.embedding_grad(ctx.narrow(one, 0, 3, 90), I, into=one))
        elif keep != "all":
            r = {k: r[k] for k in keep.split()}
        return r
    for keep in ("three", "all", "dx three", "dw three", "one three", "two", "read", "itself"):
        lazy = {k: ctx.fetch(t) for k, t in program(lambda t: None, keep).items()}
        eager = {k: ctx.fetch(t) for k, t in program(ctx.fetch, keep).items()}
        for k in lazy:
            assert np.array_equal(lazy[k], eager[k]), (keep, k)
    ctx.close()


@pytest.mark.parametrize("streams", [1, 4])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_table_updated_in_place_behind_its_readers(dtype, streams):
    """the table that a step looks up, multiplies by and differentiates is added to in place at its end: every reader sees the old one"""
    rg = np.random.default_rng(15)
    ctx = context()
    ctx.set_streams(streams)
    table, ids, labels = data(rg, (300, 64), dtype, 0.25), rg.integers(-1, 300, 200).astype(np.int32), rg.integers(-1, 300, 200).astype(np.int32)
    given = torch.tensor(table, device="cuda").to(TORCH[dtype])
    T, I, L = ctx.tensor(given, donatable=True), ctx.tensor(ids), ctx.tensor(labels)
    S = ctx.tensor(table, dtype)   # the same, a step of which is a barrier an operator
    for step in range(5):
        x = ctx.embedding(T, I, scale=2.0)
        loss, lse = ctx.linear_xent(x, T, L)
        dx, dw = ctx.linear_xent_grad(x, T, L, lse, 0.5)
        if step % 2:
            ctx.assign(T, ctx.embedding_grad(dx, I, into=T, scale=-0.25))
        else:
            ctx.assign(T, ctx.sub(T, ctx.embedding_grad(dx, I, into=dw)))
        y = ctx.embedding(T, I)    # (the new one)
        ctx.barrier()
        u = ctx.embedding(S, I, scale=2.0)
        ctx.barrier()
        loss2, lse2 = ctx.linear_xent(u, S, L)
        ctx.barrier()
        du, dw2 = ctx.linear_xent_grad(u, S, L, lse2, 0.5)
        ctx.barrier()
        if step % 2:
            S = ctx.embedding_grad(du, I, into=S, scale=-0.25)
        else:
            g = ctx.embedding_grad(du, I, into=dw2)
            ctx.barrier()
            S = ctx.sub(S, g)
        ctx.barrier()
        for a, b in ((loss, loss2), (lse, lse2), (T, S), (y, ctx.embedding(S, I))):
            assert np.array_equal(ctx.fetch(a), ctx.fetch(b)), step
        assert np.array_equal(given.float().cpu().numpy(), ctx.fetch(T))
    ctx.close()
