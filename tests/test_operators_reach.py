"""What an attention over a paged cache is taken to read, by the scheduler: no more pages than its table can name, however large the pool is."""
import pytest

from paper_2102_13267_amd import Context
from test_operators_host import zeros


def schedule(pages, slots=4, seqs=64, layers=8):
    """layers of attentions and products beside each other"""
    c = Context()
    c.set_streams(4)
    wide, heads, kv, dim, rows = 4096, 32, 8, 128, 16
    x, w = zeros(c, (seqs, wide), "bf16"), c.from_device(0, "bf16", (wide, wide))
    n, t = zeros(c, (seqs,), "s32"), zeros(c, (seqs, slots), "s32")
    for _ in range(layers):
        cache = c.from_device(0, "bf16", (pages, 2, kv, rows, dim))
        o = c.paged_attention(c.reshape(c.matmul(x, w), (seqs, heads, dim)), cache, n, t)
        x = c.add(c.matmul(c.reshape(o, (seqs, wide)), w), c.matmul(x, w))
    c.barrier()
    return c.plan_streams(), c.dump_schedule()


@pytest.mark.parametrize("slots", [1, 4])
def test_a_larger_pool_changes_no_schedule(slots):
    small = schedule(64 * slots, slots)
    for pages in (64 * slots + 44, 2048, 100000):
        assert schedule(pages, slots) == small
