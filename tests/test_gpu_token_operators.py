"""Table lookup by token and its gradient, dropout, and the cross entropy over a vocabulary, against the oracle in 64 bits.

Tolerances, from the arithmetic.  E = 2^-24 is half a step of fp32, R half a step of the result's type (2^-24, bf16 2^-8).
Lookup: a product and a rounding: (E + R) |ref|.  Its gradient: a sum of n terms, times the scale, plus the base: |scale| (n + 2) E sum |dy| + E |ref| + R |ref|.
Dropout: the factor's rounding, the product's, the sum's: 2 E |x factor| + (E + R) |ref|; which elements are kept is exact.
Cross entropy: a logit is a sum of dim products: dl = (dim + 1) E max_v sum |x w| off at most.  exp(l - top) has its argument rounded
three times (the difference, the factor, the product): 3 E |l - top|, at most 3 E span, and two roundings of its own; a sum's path has 64 additions in a lane, a tile's
few, and one per 16 tiles of 128: depth = 96 + V / 2048.  So lse is off by dl + (3 span + depth + 8) E + 3 E |lse| (its logarithm's), called dlse, and
loss by dlse + dl + E |loss|.  The gradient takes lse as given: p is off by p (dl + (3 |l - lse| + 4) E), p - [label] by that, a rounding E and one to
the type R, and g by |dloss| times that; dx and dw by |dg| |w| + (n + 2) E |g| |w| + R |ref|, n the length of the sum, and dw, where every token has a dloss of its own
and x dloss is rounded, by R |g| |x| more."""
import numpy as np
import pytest
import torch

from oracle.numeric import Eager, round_to_bf16
from paper_2102_13267_amd import Context

pytestmark = pytest.mark.gpu
E24 = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TINY = 1e-37


def context(**kw):
    return Context(device=0, workspace_bytes=kw.pop("workspace_bytes", 256 << 20), **kw)


def data(rg, shape, dtype, scale=1.0):
    x = (rg.standard_normal(shape) * scale).astype(np.float32)
    return round_to_bf16(x) if dtype == "bf16" else x


def within(got, ref, bound, what=""):
    assert got.shape == ref.shape, what
    off = np.abs(got - ref) - bound
    assert (off <= 0).all(), (what, float(np.max(off)), float(np.max(np.abs(got - ref))))


# ---- lookup ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ids,rows,dim", [((1,), 1, 1), ((8,), 100, 4096), ((3, 5), 17, 7), ((2, 1, 9), 33, 64), ((1000,), 50, 200), ((70,), 300, 331), ((257,), 5, 1024)])
def test_embedding(ids, rows, dim, dtype):
    rg = np.random.default_rng(1)
    ctx, E = context(), Eager("f64")
    table, i = data(rg, (rows, dim), dtype), rg.integers(0, rows, ids).astype(np.int32)
    i.reshape(-1)[::3] = rg.choice([-1, rows, -2 ** 31, 2 ** 31 - 1, 0, rows - 1], i.reshape(-1)[::3].shape)
    for scale in (1.0, -22.6):
        ref = E.embedding(E.tensor(table, dtype), E.tensor(i), scale).data
        got = ctx.fetch(ctx.embedding(ctx.tensor(table, dtype), ctx.tensor(i), scale))
        within(got, ref, (E24 + HALF[dtype]) * np.abs(ref) + TINY)
        assert (got[(i < 0) | (i >= rows)] == 0).all()
        if scale == 1.0:
            assert np.array_equal(got[(i >= 0) & (i < rows)], table[i[(i >= 0) & (i < rows)]])
    ctx.close()


def grad_bound(dy, ids, rows, scale, ref, out_dtype):
    n, total = np.zeros(rows), np.zeros((rows, dy.shape[-1]))
    there = (ids >= 0) & (ids < rows)
    np.add.at(n, ids[there], 1)
    np.add.at(total, ids[there], np.abs(dy[there].astype(np.float64)))
    return abs(scale) * (n[:, None] + 2) * E24 * total + (E24 + HALF[out_dtype]) * np.abs(ref) + TINY


GRADS = [((1,), 1, 1), ((1,), 1000, 8), ((31,), 4, 5), ((32,), 1, 64), ((33,), 40, 64), ((3, 100), 7, 130), ((5000,), 3000, 72), ((4097,), 2, 257), ((9000,), 100000, 8), ((2, 40), 70001, 64),
         ((20000,), 33, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ids,rows,dim", GRADS)
def test_embedding_grad(ids, rows, dim, dtype):
    rg = np.random.default_rng(2)
    ctx, E = context(workspace_bytes=512 << 20), Eager("f64")
    dy, i = data(rg, ids + (dim,), dtype), rg.integers(-1, rows + 1, ids).astype(np.int32)
    ref = E.embedding_grad(E.tensor(dy, dtype), E.tensor(i), rows=rows, scale=3.0).data
    got = ctx.fetch(ctx.embedding_grad(ctx.tensor(dy, dtype), ctx.tensor(i), rows=rows, scale=3.0))
    within(got, ref, grad_bound(dy, i, rows, 3.0, ref, dtype))
    for base_dtype in ("f32", "bf16"):
        base = data(rg, (rows, dim), base_dtype)
        ref = E.embedding_grad(E.tensor(dy, dtype), E.tensor(i), into=E.tensor(base, base_dtype)).data
        bound = grad_bound(dy, i, rows, 1.0, ref, base_dtype)
        B, D, I = ctx.tensor(base, base_dtype), ctx.tensor(dy, dtype), ctx.tensor(i)
        out = ctx.embedding_grad(D, I, into=B)
        within(ctx.fetch(out), ref, bound)
        assert np.array_equal(ctx.fetch(B), base)                                # (a copy: the base stays)
        held = torch.tensor(base, device="cuda").to(torch.bfloat16 if base_dtype == "bf16" else torch.float32)
        P = ctx.tensor(held, donatable=True)
        ctx.assign(P, ctx.embedding_grad(D, I, into=P))
        ctx.barrier()
        assert ctx.device_ptr(P) == held.data_ptr()                              # in place
        now = held.float().cpu().numpy()
        within(now, ref, bound)
        untouched = np.setdiff1d(np.arange(rows), i)
        assert np.array_equal(now[untouched], base[untouched])
    ctx.close()


def test_embedding_grad_of_one_token_everywhere_and_of_none():
    rg = np.random.default_rng(3)
    for n, rows, dim in ((10000, 50, 33), (10000, 200000, 33)):
        for which in ("one", "none", "two", "last"):
            ctx, E = context(), Eager("f64")
            dy = data(rg, (n, dim), "f32")
            i = np.full(n, {"one": 7, "none": -1, "two": 7, "last": rows - 1}[which], np.int32)
            if which == "two":
                i[n // 2:] = 8
            ref = E.embedding_grad(E.tensor(dy), E.tensor(i), rows=rows).data
            first, second = (ctx.fetch(ctx.embedding_grad(ctx.tensor(dy), ctx.tensor(i), rows=rows)) for _ in range(2))
            within(first, ref, grad_bound(dy, i, rows, 1.0, ref, "f32"), which)
            assert np.array_equal(first, second)
            ctx.close()


def test_embedding_grad_gives_the_same_bits_every_time():
    rg = np.random.default_rng(4)
    ctx = context()
    n, rows = 30000, 5000
    i = np.clip((rows ** rg.random(n)).astype(np.int64) - 1, 0, rows - 1).astype(np.int32)
    D, I = ctx.tensor(data(rg, (n, 96), "f32")), ctx.tensor(i)
    runs = [ctx.fetch(ctx.embedding_grad(D, I, rows=rows)) for _ in range(4)]
    assert all(np.array_equal(runs[0], r) for r in runs[1:])
    ctx.close()


def test_lookups_of_nothing():
    ctx = context()
    none = ctx.tensor(torch.empty(0, dtype=torch.int32, device="cuda"))
    table = ctx.tensor(np.ones((5, 8), np.float32))
    assert ctx.fetch(ctx.embedding(table, none)).shape == (0, 8)
    assert np.array_equal(ctx.fetch(ctx.embedding_grad(ctx.tensor(torch.empty((0, 8), device="cuda")), none, rows=5)), np.zeros((5, 8)))
    assert np.array_equal(ctx.fetch(ctx.embedding_grad(ctx.tensor(torch.empty((0, 8), device="cuda")), none, into=table)), np.ones((5, 8)))
    empty = ctx.tensor(torch.empty((0, 8), device="cuda"))
    some = ctx.tensor(np.array([0, 3, -1], np.int32))
    assert np.array_equal(ctx.fetch(ctx.embedding(empty, some)), np.zeros((3, 8)))
    assert ctx.fetch(ctx.embedding_grad(ctx.tensor(np.ones((3, 8), np.float32)), some, rows=0)).shape == (0, 8)
    ctx.close()


# ---- dropout --------------------------------------------------------------------------------------------
def test_random_words_are_the_published_ones():
    """The known answers that go with the generator's publication: of zeros, of ones, of the digits of pi."""
    for counter, key, want in (((0,) * 4, (0,) * 2, (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(Eager.random_words(counter, key)) == want


STATES = [(0, 0), (1, 2), (-1, -1), (2 ** 63 - 1, 2 ** 40 + 3), (0x299f31d0a4093822, 0x0370734413198a2e)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5, 7), (64, 33), (1000, 8), (257, 100), (2, 3, 4, 5, 6)])
def test_dropout(shape, dtype):
    rg = np.random.default_rng(5)
    ctx, E = context(), Eager("f64")
    x, res = data(rg, shape, dtype), data(rg, shape, dtype)
    x.reshape(-1)[x.reshape(-1) == 0] = 1.0
    X, RES = ctx.tensor(x, dtype), ctx.tensor(res, dtype)
    for k, (rate, site) in enumerate(((0.0, 0), (0.1, 3), (0.5, 2 ** 31 - 1), (0.99998, 1), (2.0 ** -18, 5))):
        st = np.array(STATES[k], np.int64)
        S = ctx.tensor(st)
        factor = 65536.0 / (65536 - int(np.rint(rate * 65536)))
        for residual in (None, res):
            ref = E.dropout(E.tensor(x, dtype), E.tensor(st), rate, site, None if residual is None else E.tensor(res, dtype)).data
            got = ctx.fetch(ctx.dropout(X, S, rate, site, None if residual is None else RES))
            within(got, ref, 2 * E24 * np.abs(x) * factor + (E24 + HALF[dtype]) * np.abs(ref) + TINY)
            if residual is None:
                assert np.array_equal(got == 0, ref == 0)
                assert np.array_equal(got, ctx.fetch(ctx.dropout_grad(X, S, rate, site)))
    ctx.close()


def test_dropout_drops_what_is_not_finite_and_keeps_the_mean():
    ctx = context()
    n = 1 << 20
    x = np.full(n, np.nan, np.float32)
    x[::2] = np.inf
    st = np.array([123, 9], np.int64)
    got = ctx.fetch(ctx.dropout(ctx.tensor(x), ctx.tensor(st), 0.25))
    kept = Eager.random_bits(4096, st, 0) >= 16384
    assert np.array_equal(got[:4096] == 0, ~kept) and not np.isfinite(got[:4096][kept]).any()
    # how many of n are kept has a deviation of sqrt(n / 4 * 3 / 4): within six of them
    assert abs((got == 0).sum() - n / 4) < 6 * (n * 3 / 16) ** 0.5
    ones = ctx.fetch(ctx.dropout(ctx.tensor(np.ones(n, np.float32)), ctx.tensor(st), 0.25))
    assert set(np.unique(ones)) == {np.float32(0), np.float32(4 / 3)}
    # other sites, steps and seeds: other masks, half of which agree
    half = [ctx.fetch(ctx.dropout(ctx.tensor(np.ones(n, np.float32)), ctx.tensor(np.array(s, np.int64)), 0.5, site)) for s, site in (((1, 1), 0), ((1, 1), 1), ((1, 2), 0), ((2, 1), 0), ((1 + 2 ** 32, 1), 0), ((1, 1 + 2 ** 32), 0))]
    for i in range(len(half)):
        for j in range(i):
            assert abs((half[i] == half[j]).sum() - n / 2) < 6 * (n / 4) ** 0.5
    ctx.close()


def test_dropout_of_a_long_tensor_reaches_its_end():
    ctx = context(workspace_bytes=1 << 30)
    n = (1 << 26) + 13
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    st = np.array([5, 6], np.int64)
    y = ctx.dropout(ctx.tensor(x), ctx.tensor(st), 0.5, 2)
    tail = ctx.fetch(ctx.narrow(y, 0, n - 1000, 1000))
    assert np.array_equal(tail == 0, Eager.random_bits(1000, st, 2, first=n - 1000) < 32768)
    ctx.close()


# ---- cross entropy over a vocabulary ----------------------------------------------------------------------
def entropy_case(rg, lead, vocab, dim, dtype, spread=3.0, ignored=0.3):
    x, w = data(rg, lead + (dim,), dtype), data(rg, (vocab, dim), dtype, spread / np.sqrt(dim))
    labels = rg.integers(0, vocab, lead).astype(np.int32)
    off = rg.random(lead) < ignored
    labels[off] = rg.choice([-1, vocab, -100, 2 ** 31 - 1, -2 ** 31], off.sum())
    return x, w, labels


def entropy_bounds(x, w, labels, dtype):
    """Of loss and lse, by token."""
    there = (labels >= 0) & (labels < len(w))
    X, W = x[there].astype(np.float64), w.astype(np.float64)
    logits = X @ W.T
    dl = (x.shape[-1] + 1) * E24 * (np.abs(X) @ np.abs(W).T).max(-1)
    top, low = logits.max(-1), logits.min(-1)
    lse = np.log(np.exp(logits - top[:, None]).sum(-1)) + top
    dlse = dl + (3 * (top - low) + 96 + len(w) / 2048 + 8) * E24 + 3 * E24 * np.abs(lse)
    loss = lse - logits[np.arange(len(lse)), labels[there]]
    return there, dlse, dlse + dl + E24 * np.abs(loss)


def grads_bound(x, w, labels, lse, dloss, dtype):
    there = (labels >= 0) & (labels < len(w))
    X, W, s, d = x[there].astype(np.float64), w.astype(np.float64), lse[there].astype(np.float64)[:, None], np.broadcast_to(dloss, labels.shape)[there].astype(np.float64)[:, None]
    logits = X @ W.T
    dl = (x.shape[-1] + 1) * E24 * (np.abs(X) @ np.abs(W).T)
    p = np.exp(logits - s)
    g = p.copy()
    g[np.arange(len(g)), labels[there]] -= 1
    g *= d
    dg = np.abs(d) * p * (dl + (3 * np.abs(logits - s) + 4) * E24) + (E24 + (HALF[dtype] if dtype == "bf16" else 0)) * np.abs(g)
    bx = dg @ np.abs(W) + (len(w) + 2) * E24 * (np.abs(g) @ np.abs(W)) + HALF[dtype] * np.abs(g @ W) + TINY
    bw = dg.T @ np.abs(X) + ((len(g) + 2) * E24 + (HALF[dtype] if np.ndim(dloss) else 0)) * (np.abs(g).T @ np.abs(X)) + HALF[dtype] * np.abs(g.T @ X) + TINY
    return there, bx, bw


ENTROPIES = [((1,), 1, 1), ((1,), 2, 3), ((1,), 300, 64), ((3,), 257, 8), ((2, 3), 1000, 100), ((16,), 4000, 256), ((17,), 513, 96), ((5, 13), 255, 331), ((300,), 700, 200), ((257,), 256, 64),
             ((64,), 10007, 72), ((600,), 300, 520), ((33,), 9000, 1024), ((1,), 5003, 1024), ((16,), 777, 128), ((17,), 4100, 192), ((40,), 3000, 512), ((64,), 20000, 64), ((65,), 1000, 64), ((5,), 9, 2048)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lead,vocab,dim", ENTROPIES)
def test_linear_xent(lead, vocab, dim, dtype):
    rg = np.random.default_rng(6)
    ctx, E = context(), Eager("f64")
    x, w, labels = entropy_case(rg, lead, vocab, dim, dtype)
    X, W, L = ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)
    loss, lse = ctx.linear_xent(X, W, L)
    ref = [t.data for t in E.linear_xent(E.tensor(x, dtype), E.tensor(w, dtype), E.tensor(labels))]
    there, dlse, dloss = entropy_bounds(x, w, labels, dtype)
    got = ctx.fetch(loss), ctx.fetch(lse)
    assert got[0].shape == lead and got[1].shape == lead
    within(got[1][there], ref[1][there], dlse, "lse")
    within(got[0][there], ref[0][there], dloss, "loss")
    assert (got[0][~there] == 0).all() and (got[1][~there] == 0).all()
    lse32 = got[1]
    for weight in (np.float32(0.37), (rg.random(lead) - 0.3).astype(np.float32)):
        D = float(weight) if weight.ndim == 0 else ctx.tensor(weight)
        dx, dw = ctx.linear_xent_grad(X, W, L, ctx.tensor(lse32), D)
        rx, rw = (t.data for t in E.linear_xent_grad(E.tensor(x, dtype), E.tensor(w, dtype), E.tensor(labels), E.tensor(lse32), E.tensor(weight)))
        there, bx, bw = grads_bound(x, w, labels, lse32, weight, dtype)
        ax, aw = ctx.fetch(dx), ctx.fetch(dw)
        within(ax[there], rx[there], bx, "dx")
        within(aw, rw, bw, "dw")
        assert (ax[~there] == 0).all()
    ctx.close()


def test_linear_xent_gradients_are_its_differences():
    """Central differences of the summed loss, in fp32: a step of 2^-6 leaves at most h^2 / 6 max |third derivative| and the losses' own errors over h."""
    rg = np.random.default_rng(7)
    ctx = context()
    x, w, labels = entropy_case(rg, (5,), 40, 16, "f32", ignored=0.2)
    weight = rg.random(5).astype(np.float32)
    L, D = ctx.tensor(labels), ctx.tensor(weight)

    def total(x, w):
        return float((ctx.fetch(ctx.linear_xent(ctx.tensor(x), ctx.tensor(w), L)[0]).astype(np.float64) * weight).sum())
    loss, lse = ctx.linear_xent(ctx.tensor(x), ctx.tensor(w), L)
    dx, dw = (ctx.fetch(t) for t in ctx.linear_xent_grad(ctx.tensor(x), ctx.tensor(w), L, lse, D))
    h = 2.0 ** -6
    for array, grad, other in ((x, dx, np.abs(w).max()), (w, dw, np.abs(x).max())):
        for at in [tuple(rg.integers(0, s) for s in array.shape) for _ in range(12)]:
            up, down = array.copy(), array.copy()
            up[at] += h
            down[at] -= h
            step = float(up[at]) - float(down[at])
            diff = ((total(up, w) - total(down, w)) if array is x else (total(x, up) - total(x, down))) / step
            # the third derivative of a log-sum-exp along a direction that moves logits by at most c: 2 c^3; five losses of up to 1e-5 error each
            assert abs(diff - grad[at]) <= h * h / 6 * 2 * (other ** 3) * 5 + 2e-5 * 5 / step, (at, diff, grad[at])
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_xent_does_not_look_at_tokens_that_do_not_count(dtype):
    rg = np.random.default_rng(8)
    ctx = context()
    x, w, labels = entropy_case(rg, (40,), 300, 64, dtype, ignored=0.5)
    off = (labels < 0) | (labels >= 300)
    assert off.any() and not off.all()
    bad = x.copy()
    bad[off] = rg.choice([np.nan, np.inf, -np.inf], bad[off].shape)
    dloss = rg.random(40).astype(np.float32)
    bad_dloss = np.where(off, np.nan, dloss).astype(np.float32)
    W, L = ctx.tensor(w, dtype), ctx.tensor(labels)
    results = []
    for xx, dd in ((x, dloss), (bad, bad_dloss)):
        X = ctx.tensor(xx, dtype)
        loss, lse = ctx.linear_xent(X, W, L)
        lse_in = np.where(off, np.nan if xx is bad else 0.0, ctx.fetch(lse)).astype(np.float32)
        dx, dw = ctx.linear_xent_grad(X, W, L, ctx.tensor(lse_in), ctx.tensor(dd))
        results.append([ctx.fetch(t) for t in (loss, lse, dx, dw)])
    for a, b in zip(*results):
        assert np.isfinite(a).all() and np.array_equal(a, b)
    none = ctx.tensor(np.full(40, -1, np.int32))
    loss, lse = ctx.linear_xent(ctx.tensor(bad, dtype), W, none)
    dx, dw = ctx.linear_xent_grad(ctx.tensor(bad, dtype), W, none, lse, 1.0)
    for t in (loss, lse, dx, dw):
        assert (ctx.fetch(t) == 0).all()
    ctx.close()


def test_linear_xent_of_what_is_not_finite():
    """A NaN row of w reaches every token; an infinite logit makes the loss NaN or infinite, as the formulas have it; large logits do not overflow."""
    rg = np.random.default_rng(9)
    for dtype in ("f32", "bf16"):
        ctx = context()
        x, w, labels = entropy_case(rg, (7,), 400, 64, dtype, ignored=0.0)
        for scale in (1e4, 1e15):
            big = round_to_bf16(x * np.float32(scale)) if dtype == "bf16" else x * np.float32(scale)
            loss, lse = (ctx.fetch(t) for t in ctx.linear_xent(ctx.tensor(big, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)))
            l = big.astype(np.float64) @ w.astype(np.float64).T
            slack = 65 * E24 * (np.abs(big).astype(np.float64) @ np.abs(w).astype(np.float64).T).max(-1) + 8 * E24 * np.abs(l.max(-1)) + np.log(400)
            assert (np.abs(lse - l.max(-1)) <= slack).all()
            assert (np.abs(loss - (l.max(-1) - l[np.arange(7), labels])) <= 2 * slack + E24 * np.abs(loss)).all()
        w[123, 5] = np.nan
        loss, lse = (ctx.fetch(t) for t in ctx.linear_xent(ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)))
        assert np.isnan(loss).all() and np.isnan(lse).all()
        x[3] = np.nan
        w[123, 5] = 0.0
        loss, lse = (ctx.fetch(t) for t in ctx.linear_xent(ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)))
        assert np.array_equal(np.isnan(loss), np.arange(7) == 3) and np.array_equal(np.isnan(lse), np.arange(7) == 3)
        ctx.close()


def test_linear_xent_of_no_tokens():
    ctx = context()
    w = ctx.tensor(np.ones((300, 64), np.float32))
    x, labels = ctx.tensor(torch.empty((0, 64), device="cuda")), ctx.tensor(torch.empty(0, dtype=torch.int32, device="cuda"))
    loss, lse = ctx.linear_xent(x, w, labels)
    dx, dw = ctx.linear_xent_grad(x, w, labels, lse, 1.0)
    assert ctx.fetch(loss).shape == (0,) and ctx.fetch(dx).shape == (0, 64) and np.array_equal(ctx.fetch(dw), np.zeros((300, 64)))
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_only_the_gradient_that_is_used(dtype):
    rg = np.random.default_rng(10)
    ctx = context()
    x, w, labels = entropy_case(rg, (50,), 600, 128, dtype)
    X, W, L = ctx.tensor(x, dtype), ctx.tensor(w, dtype), ctx.tensor(labels)
    loss, lse = ctx.linear_xent(X, W, L)
    both = [ctx.fetch(t) for t in ctx.linear_xent_grad(X, W, L, lse, 1.0)]
    for slot in range(2):
        alone = ctx.linear_xent_grad(X, W, L, lse, 1.0)[slot]
        assert np.array_equal(ctx.fetch(alone), both[slot])
    assert np.array_equal(ctx.fetch(ctx.linear_xent(X, W, L)[1]), ctx.fetch(lse))
    ctx.close()
