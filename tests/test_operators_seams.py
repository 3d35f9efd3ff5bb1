"""That an attention over a paged cache counts every key once: a key that is lost, or counted twice, where chunks, tiles, stretches of pages or the
pieces of a join meet, changes the results that are looked at here by more than the comparison lets pass.

Values are 0 but for those of a few windows of positions, which are 1 in one element of one key head each, so that every result is the sum of a few
weights.  The keys' scores are m ln 2, m = 0 to 3, so that weights are powers of two (largest and smallest ones take turns along the sequence).

Tolerances: E = 2^-24.  scale and its product with log2(e) round three times, m <= 3 times that is an exponent's error (9 E ln 2), the power's own 2 E;
sums of n terms err by n E at most, numerator and denominator; bf16 values meet weights that are 2^-15 + 2^-18 off at most, and the result is rounded
to its type: |got - ref| <= (2 (11 E + n E) + W + R) ref, W = 2^-14 (bf16; fp32 0), R = 2^-8 (2^-24).  A class has at most 7 keys, one of which has
weight 1 of at most 1 + 6 * 8: a lost key changes the result by 1 / 49 = 5.2 * 2^-8 of it, more than 2 tolerances, and so does one that is counted twice."""
import math

import numpy as np
import pytest

from paper_2102_13267_amd import Context

E24 = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
WEIGHT = {"f32": 0.0, "bf16": 2.0 ** -14}
KEYS = 7   # of a class
CASES = [([20000], 8, 1, 64, 128), ([9001], 4, 4, 16, 64), ([5003], 12, 2, 24, 80), ([3333], 2, 1, 7, 256), ([6007], 40, 1, 16, 128), ([6001, 4, 0, 129, 2500, 1, 640, 128], 4, 2, 16, 64),
         ([8192], 1, 1, 1, 32), ([4097], 2, 2, 3, 10), ([600, 700, 641, 640, 5 * 128, 5 * 128 + 1], 4, 4, 16, 128)]


def powers(n):
    return np.arange(n) // 53 % 4


def class_of(n, kv, dim, round_):
    """the class of each position (a key head's element), -1: its value is nothing in this round"""
    p = np.arange(n)
    return np.where(p // (kv * dim) // KEYS == round_, p % (kv * dim), -1)


def expected(n, heads, kv, dim, round_, keep=None):
    """[heads, dim]; keep: how often each key counts (1)"""
    w = 2.0 ** powers(n) * (1.0 if keep is None else keep)
    c = class_of(n, kv, dim, round_)
    out = np.bincount(c[c >= 0], weights=w[c >= 0], minlength=kv * dim)[:kv * dim] / w.sum()
    return np.repeat(out.reshape(kv, dim), heads // kv, 0)


def agrees(got, ref, n, dtype):
    return bool((np.abs(got - ref) <= (2 * (11 + n) * E24 + WEIGHT[dtype] + HALF[dtype]) * ref).all())


def rounds(lens, kv, dim):
    return -(-max(lens) // (kv * dim * KEYS))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,heads,kv,rows,dim", CASES)
def test_the_comparison_sees_every_key(lens, heads, kv, rows, dim, dtype):
    """a key left out, or counted twice, anywhere"""
    rg = np.random.default_rng(1)
    for n in lens:
        if n == 0:
            continue
        refs = [expected(n, heads, kv, dim, r) for r in range(-(-n // (kv * dim * KEYS)))]
        assert all(agrees(r, r, n, dtype) for r in refs)
        for at in {0, n - 1, n // 2, n // 128 * 128 % n, *(int(i) for i in rg.integers(0, n, 20))}:
            for times in (0.0, 2.0) if n > 1 else (2.0,):
                keep = np.ones(n)
                keep[at] = times
                r = at // (kv * dim) // KEYS
                wrong = expected(n, heads, kv, dim, r, keep)
                if n == 1:
                    continue      # (one key is all of it, however often it counts)
                assert not agrees(wrong, refs[r], n, dtype), (n, at, times)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,heads,kv,rows,dim", CASES)
def test_every_key_counts_once(lens, heads, kv, rows, dim, dtype):
    rg = np.random.default_rng(2)
    need = [-(-n // rows) for n in lens]
    pages, slots = sum(need) + 2, max(need) + 1
    order, table, at = rg.permutation(pages), np.full((len(lens), slots), -1, np.int32), 0
    for s, k in enumerate(need):
        table[s, :k] = order[at:at + k]
        at += k
    cache = np.full((pages, 2, kv, rows, dim), np.nan, np.float32)       # what no sequence holds
    q = np.zeros((len(lens), heads, dim), np.float32)
    q[:, :, 0] = 1.0
    for s, n in enumerate(lens):
        p = np.arange(n)
        cache[table[s, p // rows], :, :, p % rows] = 0.0
        cache[table[s, p // rows], 0, :, p % rows, 0] = powers(n)[:, None]
    ctx = Context(device=0, workspace_bytes=256 << 20)
    Q, N, T = ctx.tensor(q, dtype), ctx.tensor(np.asarray(lens, np.int32)), ctx.tensor(table)
    for r in range(rounds(lens, kv, dim)):
        marked = cache.copy()
        for s, n in enumerate(lens):
            c = class_of(n, kv, dim, r)
            p = np.flatnonzero(c >= 0)
            marked[table[s, p // rows], 1, c[p] // dim, p % rows, c[p] % dim] = 1.0
        got = ctx.fetch(ctx.paged_attention(Q, ctx.tensor(marked, dtype), N, T, scale=math.log(2.0)))
        for s, n in enumerate(lens):
            if n == 0:
                assert not got[s].any()
            else:
                assert agrees(got[s], expected(n, heads, kv, dim, r), n, dtype), (r, s)
    ctx.close()
