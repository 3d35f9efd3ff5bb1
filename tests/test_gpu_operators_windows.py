"""Windows and broadcasts as operands of the operators that read a paged cache: the bits of the same operators on tensors of their own."""
import numpy as np
import pytest

from oracle.numeric import Eager
from paper_2102_13267_amd import Context, Rotary
from test_gpu_operators import compare_attention, data, ints, paged_case

pytestmark = pytest.mark.gpu


def context():
    return Context(device=0, workspace_bytes=256 << 20)


def test_copies_of_integers_move_words():
    """small ones (numbers below the smallest of fp32), large and negative ones, those that fp32 could not hold"""
    rg = np.random.default_rng(1)
    ctx = context()
    x = ints(rg.integers(-2 ** 31, 2 ** 31, (37, 24)))
    x[0, :8] = [0, 1, -1, 5, (1 << 24) + 1, 2 ** 31 - 1, -2 ** 31, 0x7F800001]
    X, one, row = ctx.tensor(x), ctx.tensor(x[0, 4:5]), ctx.tensor(x[:1])
    outs = [(ctx.narrow(X, 0, 3, 20), x[3:23]), (ctx.narrow(X, 1, 1, 20), x[:, 1:21]), (ctx.narrow(X, 1, 3, 1), x[:, 3:4]), (ctx.permute(X, (1, 0)), x.T), (ctx.reshape(X, (24, 37)), x.reshape(24, 37)),
            (ctx.expand(one, (1001,)), np.repeat(x[0, 4:5], 1001)), (ctx.expand(row, (40, 24)), np.repeat(x[:1], 40, 0))]
    big = ints(rg.integers(-2 ** 31, 2 ** 31, (2051, 2048)))
    B = ctx.tensor(big)
    outs += [(ctx.narrow(B, 0, 1, 2048), big[1:2049]), (ctx.narrow(B, 1, 4, 2000), big[:, 4:2004]), (ctx.reshape(B, (2048, 2051)), big.reshape(2048, 2051)),
             (ctx.expand(ctx.tensor(big[5:6]), (999, 2048)), np.repeat(big[5:6], 999, 0))]
    for got, ref in outs:
        assert np.array_equal(ctx.fetch(got), ref)
    ctx.close()


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f32", 10), ("bf16", 9)])
def test_some_sequences_of_a_batch(dtype, dim):
    """windows of lengths, table, positions and offsets, and their copies"""
    rg = np.random.default_rng(2)
    lens, kv, rows, r = [40, 9, 1, 700, 0, 33], 2, 16, Rotary(dims=8)
    cache, table = paged_case(rg, lens, kv, rows, dim, dtype)
    q, k, v = (data(rg, (3, h, dim), dtype) for h in (4, kv, kv))
    positions = ints(np.array([5, 2 ** 24 + 1, 8, 0, 699, 3]))
    offsets = ints([9, 0, 1, 2, 3, 7])
    wide = np.concatenate([table, np.full((6, 3), -1, np.int32)], 1)
    outs = []
    for own in (True, False):
        ctx = context()
        part = lambda a: ctx.tensor(np.ascontiguousarray(a[1:4])) if own else ctx.narrow(ctx.tensor(a), 0, 1, 3)     # noqa: E731,B023
        L, T, P = part(ints(lens)), part(table), part(positions)
        W = ctx.tensor(np.ascontiguousarray(wide[1:4, :table.shape[1]])) if own else ctx.narrow(part(wide), 1, 0, table.shape[1])
        O = ctx.tensor(offsets[1:5]) if own else ctx.narrow(ctx.tensor(offsets), 0, 1, 4)     # noqa: E741
        C, K, V, Q = ctx.tensor(cache, dtype, donatable=True), ctx.tensor(k, dtype), ctx.tensor(v, dtype), ctx.tensor(q, dtype)
        ctx.assign(C, ctx.cache_append(C, K, V, L, T, offsets=O, rotary=r))
        y = ctx.rope(Q, P, r)
        o, w = ctx.paged_attention(y, C, L, T), ctx.paged_attention(y, C, L, W)
        outs.append([ctx.fetch(t) for t in (C, y, o, w)])
        ctx.close()
    for a, b in zip(*outs):
        assert np.array_equal(a, b)
    assert np.array_equal(outs[0][2], outs[0][3])


@pytest.mark.parametrize("dtype,rows,dim", [("bf16", 16, 64), ("f32", 5, 20), ("bf16", 3, 7), ("bf16", 8, 20)])
def test_one_layer_of_a_tensor_of_layers(dtype, rows, dim):
    """a cache inside a larger tensor, also off 16 bytes: read where it lies, and the layers beside it as they were behind an append"""
    rg = np.random.default_rng(3)
    lens, kv = [40, 9, 1, 300], 1
    cache, table = paged_case(rg, lens, kv, rows, dim, dtype, fill=0.0)
    layers = data(rg, (3, *cache.shape), dtype)
    layers[0] = layers[2] = np.nan
    layers[1] = cache
    q, k, v = (data(rg, (4, h, dim), dtype) for h in (3, kv, kv))
    ctx, E = context(), Eager("f64")
    pool = ctx.tensor(layers, dtype)
    C = ctx.reshape(ctx.narrow(pool, 0, 1, 1), cache.shape)
    L, T, Q = ctx.tensor(ints(lens)), ctx.tensor(table), ctx.tensor(q, dtype)
    o = ctx.paged_attention(Q, C, L, T)
    new = ctx.cache_append(C, ctx.tensor(k, dtype), ctx.tensor(v, dtype), L, T)
    after = ctx.paged_attention(Q, new, L, T)
    del C                # (a window that is still held would be a result)
    ctx.barrier()
    assert " EW " not in ctx.dump_plan()
    e = [E.tensor(cache, dtype), E.tensor(ints(lens)), E.tensor(table)]
    appended = E.fetch(E.cache_append(e[0], E.tensor(k, dtype), E.tensor(v, dtype), e[1], e[2])).astype(np.float32)
    compare_attention(ctx.fetch(o), E.fetch(E.paged_attention(E.tensor(q, dtype), *e)), q, cache, lens, table, dtype)
    assert np.array_equal(ctx.fetch(new), appended) and np.array_equal(ctx.fetch(pool), layers, equal_nan=True)
    compare_attention(ctx.fetch(after), E.fetch(E.paged_attention(E.tensor(q, dtype), E.tensor(appended, dtype), *e[1:])), q, appended, lens, table, dtype)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_length_position_and_table_for_all(dtype):
    rg = np.random.default_rng(4)
    kv, rows, dim, n = 2, 16, 64, 75
    cache, table = paged_case(rg, [n], kv, rows, dim, dtype)
    q = data(rg, (5, 4, dim), dtype)
    for p in (7, (1 << 24) + 1):
        outs = []
        for own in (True, False):
            ctx = context()
            all_ = lambda a, shape: ctx.tensor(np.ascontiguousarray(np.broadcast_to(a, shape))) if own else ctx.expand(ctx.tensor(a), shape)     # noqa: E731,B023
            y = ctx.rope(ctx.tensor(q, dtype), all_(ints([p]), (5,)))
            outs.append([ctx.fetch(t) for t in (y, ctx.paged_attention(y, ctx.tensor(cache, dtype), all_(ints([n]), (5,)), all_(table, (5, table.shape[1]))))])
            ctx.close()
        for a, b in zip(*outs):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f32", 7)])
def test_broadcasts_of_heads(dtype, dim):
    rg = np.random.default_rng(6)
    r, p = Rotary(dims=6), ints([3, 1, 4, 100, 5])
    cases = [((2, 1, 5, 3, dim), (2, 4, 5, 3, dim), None), ((2, 5, 1, dim), (4, 2, 5, 3, dim), None), ((1, 2, 1, 3, dim), (4, 2, 5, 3, dim), None), ((2, 1, 5, 3, dim), (2, 4, 5, 3, dim), (3, 1, 2)),
             ((2, 1, 1, 1, 1, dim), (2, 3, 1, 5, 2, dim), None), ((3, 1, 2, 5, 2, dim), (3, 4, 2, 5, 2, dim), (4, 1, 1))]
    for frm, to, window in cases:
        x = data(rg, frm, dtype)
        outs = []
        for own in (True, False):
            ctx = context()
            if own:
                a = np.broadcast_to(x, to)
                X = ctx.tensor(np.ascontiguousarray(a if window is None else np.take(a, range(window[1], window[1] + window[2]), axis=window[0])), dtype)
            else:
                X = ctx.expand(ctx.tensor(x, dtype), to)
                X = X if window is None else ctx.narrow(X, *window)
            y = ctx.rope(X, ctx.tensor(p), r)
            del X
            ctx.barrier()
            outs.append(ctx.fetch(y))
            ctx.close()
        assert np.array_equal(*outs)


def test_positions_that_all_tokens_share_in_the_tokens_shape():
    rg = np.random.default_rng(5)
    x, p = data(rg, (10, 3, 4, 8), "bf16"), ints(rg.integers(0, 2 ** 26, (2, 1, 3)))
    outs = []
    for own in (True, False):
        ctx = context()
        P = ctx.tensor(np.repeat(p, 5, 1).reshape(10, 3)) if own else ctx.reshape(ctx.expand(ctx.tensor(p), (2, 5, 3)), (10, 3))
        outs.append(ctx.fetch(ctx.rope(ctx.tensor(x, "bf16"), P)))
        ctx.close()
    assert np.array_equal(*outs)
