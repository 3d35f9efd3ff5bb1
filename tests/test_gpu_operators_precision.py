"""How exact the operators are where the type of their data does not limit them, against 64 bits.

Tolerances, from the arithmetic.  E = 2^-24 is half a step of fp32, R half a step of the result's type (2^-24, bf16 2^-8).
Attention: ds = (dim + 8) E scale max_k sum_d |q_d k_d| bounds a score's error, which puts exp(score) 2 ds + 4 E off; sums of n terms
err by n E of their magnitudes, numerator and denominator each.  A weight meets bf16 values as two bf16 numbers: what the first one
leaves is below 2^-7 of it and is rounded by 2^-8 of itself (2^-15), the second one is made 2^-20 of the weight larger, and the exponent is
rounded where it is below 64 (2^-19, times ln 2): below W = 2^-14 together.  |got - ref| <= (2 (2 ds + 4 E + n E) + W) sum_k p |v| + R |ref|.
Rotation: a turn is the product of amplitude and a sine of 64 bits, rounded once (E of each product); y s and the sum are rounded once
each: |got - ref| <= E (|x c| + 2 |y s| + |ref|) + A (|x| + |y|), where A is what 64 bits lose of an angle: position 2^-50 (its product and the
frequency's roundings) + 2^-40 (what the polynomials leave out, the terms of E^2)."""
import math

import numpy as np
import pytest

from oracle.numeric import Eager, round_to_bf16
from paper_2102_13267_amd import Context, Rotary
from test_gpu_operators import data, ints, paged_case

pytestmark = pytest.mark.gpu
E24 = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
WEIGHT = {"f32": 0.0, "bf16": 2.0 ** -14}


def attend(cache, table, lens, q, dtype, scale=None):
    ctx = Context(device=0, workspace_bytes=256 << 20)
    got = ctx.fetch(ctx.paged_attention(ctx.tensor(q, dtype), ctx.tensor(cache, dtype), ctx.tensor(ints(lens)), ctx.tensor(table), scale=scale))
    ctx.close()
    return got


def check(got, cache, table, lens, q, dtype):
    seqs, heads, dim = q.shape
    rows, group = cache.shape[3], heads // cache.shape[2]
    scale = 1 / math.sqrt(dim)
    for s, n in enumerate(lens):
        if n == 0:
            assert not got[s].any()
            continue
        pos = np.arange(n)
        for h in range(heads):
            k, v = (cache[table[s, pos // rows], i, h // group, pos % rows].astype(np.float64) for i in (0, 1))
            qq = q[s, h].astype(np.float64)
            ds = (dim + 8) * E24 * scale * (np.abs(k) @ np.abs(qq)).max()
            e = np.exp(k @ qq * scale - (k @ qq * scale).max())
            p = e / e.sum()
            ref = p @ v
            tol = (2 * (2 * ds + 4 * E24 + n * E24) + WEIGHT[dtype]) * (p @ np.abs(v)) + HALF[dtype] * np.abs(ref) + 1e-37
            assert (np.abs(got[s, h] - ref) <= tol).all(), (s, h, np.max(np.abs(got[s, h] - ref) / tol))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,rows,dim", [(8, 2, 16, 128), (4, 4, 16, 64), (6, 2, 5, 96), (5, 1, 16, 32), (3, 3, 8, 20), (2, 1, 16, 256), (4, 2, 24, 160)])
def test_weights_are_not_rounded_to_the_cache_s_type(heads, kv, rows, dim, dtype):
    rg = np.random.default_rng(dim)
    lens = [2, 3, 17, 40, 100, 200, 0, 77]
    cache, table = paged_case(rg, lens, kv, rows, dim, dtype)
    q = data(rg, (len(lens), heads, dim), dtype)
    check(attend(cache, table, lens, q, dtype), cache, table, lens, q, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim", [(16, 64), (16, 32), (5, 64), (8, 24), (16, 20), (3, 50), (16, 5), (7, 3), (16, 128), (16, 96)])
@pytest.mark.parametrize("wide", [False, True])
def test_weights_of_many_heads_a_key_head_are_not_rounded(wide, rows, dim, dtype):
    """with a table for long sequences two blocks of 16 heads are taken at once"""
    rg = np.random.default_rng(1)
    lens = [int(n) for n in rg.integers(0, 90, 70)] + [700]
    cache, table = paged_case(rg, lens, 1, rows, dim, dtype, slots=8000 // rows if wide else None, fill=np.nan)
    q = data(rg, (len(lens), 24, dim), dtype)
    check(attend(cache, table, lens, q, dtype), cache, table, lens, q, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [16, 5])
def test_an_infinite_value_that_counts_is_the_result(rows, dtype):
    """also where its weight is a number of few bits, whose rest is nothing"""
    rg = np.random.default_rng(2)
    lens = [1, 2, 8, 40]
    cache, table = paged_case(rg, lens, 1, rows, 64, dtype)
    for s in range(len(lens)):
        cache[table[s, 0], 1, 0, 0, 3], cache[table[s, 0], 1, 0, 0, 60] = np.inf, -np.inf
    q = data(rg, (len(lens), 4, 64), dtype)
    for scale in (0.0, None):
        got = attend(cache, table, lens, q, dtype, scale)
        assert (got[..., 3] == np.inf).all() and (got[..., 60] == -np.inf).all() and np.isfinite(np.delete(got, (3, 60), axis=-1)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim", [(16, 64), (24, 80)])
def test_an_average_of_values_near_the_largest_is_finite(rows, dim, dtype):
    """of one chunk and of several, of all signs"""
    rg = np.random.default_rng(3)
    lens = [1, 2, 3, 64, 200, 300, 0]
    for more in ([], [5000]):
        at = lens + more
        cache, table = paged_case(rg, at, 2, rows, dim, dtype)
        v = np.float32(2.0 ** 127) * rg.uniform(1.0, 1.984375, cache[:, 1].shape).astype(np.float32)
        v[..., ::2] *= rg.choice([-1.0, 1.0], v[..., ::2].shape).astype(np.float32)
        cache[:, 1] = round_to_bf16(v) if dtype == "bf16" else v
        q = data(rg, (len(at), 4, dim), dtype)
        got = attend(cache, table, at, q, dtype)
        assert np.isfinite(got).all()
        check(got, cache, table, at, q, dtype)


@pytest.mark.parametrize("r", [Rotary(), Rotary(interleaved=True), Rotary(factor=8.0, original=8192.0, amplitude=1.3), Rotary(dims=32, base=500000.0, amplitude=-0.7)])
def test_sines_are_rounded_once(r):
    rg = np.random.default_rng(4)
    tokens, heads, dim = 700, 3, 64
    p = ints(np.concatenate([np.arange(300), rg.integers(-(1 << 17), 1 << 17, tokens - 300)]))
    a, first, second = Eager._angles(p, r, dim)
    ctx = Context(device=0, workspace_bytes=64 << 20)
    one, other, some = np.zeros((tokens, heads, dim), np.float32), np.zeros((tokens, heads, dim), np.float32), rg.standard_normal((tokens, heads, dim)).astype(np.float32)
    one[..., first] = 1.0
    other[..., second] = 1.0
    for sign, op in ((1.0, ctx.rope), (-1.0, ctx.rope_grad)):
        c, s = (r.amplitude * f(a)[:, None] for f in (np.cos, lambda z: np.sin(sign * z)))      # noqa: B023
        for x in (one, other, some):
            got = ctx.fetch(op(ctx.tensor(x), ctx.tensor(p), r)).astype(np.float64)
            u, w = x[..., first].astype(np.float64), x[..., second].astype(np.float64)
            lost = (np.abs(p)[:, None, None] * 2.0 ** -50 + 2.0 ** -40) * abs(r.amplitude) * (np.abs(u) + np.abs(w))
            for at, y, z in ((first, u * c, -w * s), (second, w * c, u * s)):
                tol = E24 * (np.abs(y) + 2 * np.abs(z) + np.abs(y + z)) + lost
                if x is not some:      # a product with one and a sum with nothing are exact
                    tol = E24 * np.abs(y + z) + lost
                assert (np.abs(got[..., at] - (y + z)) <= tol).all(), np.max(np.abs(got[..., at] - (y + z)) / tol)
    ctx.close()
