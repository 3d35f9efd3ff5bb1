"""Windows and broadcasts as operands of the operators that read a paged cache, without a GPU: what is read where it lies, what is written out first,
and what is refused, against the structural oracle."""
import pytest

from oracle.structural import Tracer
from paper_2102_13267_amd import Context
from test_operators_host import ROT, UNSUPPORTED, kinds, paged, refused, zeros


def windows_of_integers(B):
    """some of the sequences of a batch: their lengths, rows of the table, positions and offsets"""
    t = paged(B)
    lengths, table, positions = B.narrow(zeros(B, (9,), "s32"), 0, 2, 3), B.narrow(zeros(B, (9, 5), "s32"), 0, 2, 3), B.narrow(zeros(B, (7,), "s32"), 0, 4, 3)
    offsets = B.narrow(zeros(B, (9,), "s32"), 0, 1, 4)
    B.assign(t["cache"], B.cache_append(t["cache"], t["k"], t["v"], lengths, table, offsets=offsets, rotary=ROT))
    return t, B.paged_attention(B.rope(t["q"], positions, ROT), t["cache"], lengths, table)


def layers_of_one_tensor(B):
    """one layer's cache out of a tensor of all layers' caches"""
    t = paged(B)
    pool, many = zeros(B, (3, 7, 2, 2, 4, 8)), zeros(B, (21, 2, 2, 4, 8))
    a, b = B.reshape(B.narrow(pool, 0, 1, 1), (7, 2, 2, 4, 8)), B.narrow(many, 0, 7, 7)
    return t, [B.paged_attention(t["q"], c, t["lengths"], t["table"]) for c in (a, b)]


def appended_layers(B):
    """rows that go into the copy of one layer"""
    t = paged(B)
    pool = zeros(B, (3, 7, 2, 2, 4, 8))
    a = B.cache_append(B.reshape(B.narrow(pool, 0, 1, 1), (7, 2, 2, 4, 8)), t["k"], t["v"], t["lengths"], t["table"])
    return t, a, B.paged_attention(t["q"], a, t["lengths"], t["table"])


def broadcasts(B):
    """one length, position and row of the table for all sequences"""
    t = paged(B)
    lengths, table = B.expand(zeros(B, (1,), "s32"), (3,)), B.expand(zeros(B, (1, 5), "s32"), (3, 5))
    B.assign(t["cache"], B.cache_append(t["cache"], t["k"], t["v"], lengths, table))
    return t, B.paged_attention(B.rope(t["q"], B.expand(zeros(B, (1,), "s32"), (3,)), ROT), t["cache"], lengths, table)


def broadcasts_reshaped(B):
    """positions that all tokens share, in the shape of the tokens"""
    p = B.reshape(B.expand(zeros(B, (2, 1, 3), "s32"), (2, 5, 3)), (10, 3))
    return p, B.rope(zeros(B, (10, 3, 4, 8)), p, ROT), B.rope(zeros(B, (2, 3, 4, 8)), B.reshape(B.expand(zeros(B, (1,), "s32"), (6,)), (2, 3)), ROT)


def broadcasts_of_heads(B):
    """axes before the heads that two strides reach, and such that they do not"""
    p, r = zeros(B, (5,), "s32"), ROT
    y = zeros(B, (2, 1, 5, 3, 8))
    return [B.rope(B.expand(zeros(B, (2, 5, 1, 8)), (4, 2, 5, 3, 8)), p, r), B.rope(B.expand(zeros(B, (2, 5, 1, 1, 8)), (2, 5, 4, 3, 8)), zeros(B, (2, 5, 4), "s32"), r),
            B.rope(B.expand(y, (2, 4, 5, 3, 8)), p, r), B.rope_grad(B.narrow(B.expand(y, (2, 4, 5, 3, 8)), 3, 1, 2), p, r),
            B.rope(B.expand(B.expand(zeros(B, (5, 1, 8)), (2, 1, 5, 3, 8)), (3, 2, 7, 5, 3, 8)), p, r), B.rope(B.expand(B.expand(zeros(B, (2, 1, 1, 3, 8)), (2, 1, 5, 3, 8)), (2, 4, 5, 3, 8)), p, r),
            B.rope(B.expand(zeros(B, (1, 2, 1, 3, 8)), (4, 2, 5, 3, 8)), p, r)]


def copies_of_integers(B):
    """columns of a table, a window that is a result, and one behind a broadcast; copies of integers that share nothing with each other or with what reads them"""
    t = paged(B)
    wide = zeros(B, (3, 8), "s32")
    table = B.narrow(wide, 1, 2, 5)
    lengths = B.narrow(B.expand(zeros(B, (1,), "s32"), (9,)), 0, 4, 3)
    shown = B.narrow(zeros(B, (9,), "s32"), 0, 2, 3)
    same = B.narrow(zeros(B, (2, 3), "s32"), 1, 0, 3)
    return t, shown, same, B.cast(lengths, "f32"), B.add(t["q"], 1.0), B.paged_attention(t["q"], t["cache"], lengths, table), B.paged_attention(t["q"], t["cache"], shown, table)


@pytest.mark.parametrize("program", [windows_of_integers, layers_of_one_tensor, appended_layers, broadcasts, broadcasts_reshaped, broadcasts_of_heads, copies_of_integers])
def test_plans_equal_the_structural_oracles(program):
    ctx, ref = Context(), Tracer()
    keep = program(ctx), program(ref)
    for _ in range(2):
        info, want = ctx.barrier(), ref.barrier()
        assert info.hash == want["hash"] and ctx.dump_plan() == want["plan"]
        keep = (program(ctx), program(ref), keep)


def test_windows_are_read_where_they_lie():
    for program, launches in ((windows_of_integers, ["APPEND", "PAGED"]), (layers_of_one_tensor, ["PAGED", "PAGED"]), (appended_layers, ["APPEND", "PAGED"])):
        c = Context()
        keep = program(c)     # noqa: F841
        c.barrier()
        assert kinds(c) == launches and " EW " not in c.dump_plan()


def test_broadcasts_of_integers_are_written_out():
    c = Context()
    keep = broadcasts(c)     # noqa: F841
    c.barrier()
    assert kinds(c).count("EW") == 3


def test_broadcasts_of_heads_are_read_where_they_lie_if_two_strides_do():
    c = Context()
    keep = broadcasts_of_heads(c)     # noqa: F841
    c.barrier()
    assert kinds(c).count("EW") == 3


def test_a_window_that_an_elementwise_operation_reads_through_a_reshape_is_copied():
    c = Context()
    t = paged(c)
    w = c.reshape(c.narrow(zeros(c, (3, 7, 2, 2, 4, 8)), 0, 1, 1), (7, 2, 2, 4, 8))
    o = c.paged_attention(t["q"], w, t["lengths"], t["table"]), c.add(w, 1.0)      # noqa: F841
    c.barrier()
    assert kinds(c).count("EW") == 2


def test_what_stays_refused():
    """host scalars, and one entry for every slot of a table"""
    for build in (lambda c, t: c.paged_attention(t["q"], t["cache"], c.expand(c.scalar(4, "s32"), (3,)), t["table"]),
                  lambda c, t: c.paged_attention(t["q"], t["cache"], t["lengths"], c.expand(zeros(c, (1, 1), "s32"), (3, 5))),
                  lambda c, t: c.expand(c.scalar(4, "s32"), (3,))):
        c = Context()
        t = paged(c)
        out = build(c, t)      # noqa: F841
        refused(UNSUPPORTED, c.barrier)
