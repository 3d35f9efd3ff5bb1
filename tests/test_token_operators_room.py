"""Cross entropies over a vocabulary in little memory: what a plan takes for speed it does without where there is no room.  Null device, then (-m gpu) values."""
import numpy as np
import pytest

from paper_2102_13267_amd import Context
from test_token_operators_host import zeros

MB = 1 << 20


def library_bytes():
    c = Context(workspace_bytes=64 * MB)
    n = c.stats().arena_bytes_in_use
    c.close()
    return n


# tokens, rows, dim, type; which results; megabytes that are enough, and that a plan with room would take more than
SPLIT = (1035, 131072, 4096, "f32", "dx", 215)       # g 128, x 21, sums 21 (of one split), dx 17
PACKED = (300, 131072, 1001, "bf16", "losses", 160)  # w packed in pieces of 128
MAXIMA = (40000, 200000, 64, "f32", "losses", 215)   # maxima and sums in pieces of 128
BOTH = (300, 131072, 1001, "bf16", "dx", 290)        # w packed in pieces of 128, g of as many rows


def results(c, case, x, w, labels, lse=None):
    if case[4] == "losses":
        return c.linear_xent(x, w, labels)
    return c.linear_xent_grad(x, w, labels, lse, 0.5)[:1]


@pytest.mark.parametrize("fusion", [True, False])
@pytest.mark.parametrize("case", [SPLIT, PACKED, MAXIMA, BOTH])
def test_what_a_plan_takes_for_speed_it_does_without(case, fusion):
    tokens, rows, dim, dtype, _, room = case
    sizes = []
    for n in (2048, room):
        c = Context(workspace_bytes=library_bytes() + n * MB)
        c.set_fusion(fusion)
        x, w = c.from_device(0, dtype, (tokens, dim)), c.from_device(0, dtype, (rows, dim))
        out = results(c, case, x, w, zeros(c, (tokens,), "s32"), zeros(c, (tokens,)))
        c.barrier()
        sizes.append((c.stats().arena_bytes_in_use, c.dump_schedule()))
        del out
        c.close()
    assert sizes[0][1] != sizes[1][1] or (not fusion and case is SPLIT)    # (whose splits are all that differs: one launch either way)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [SPLIT, PACKED, MAXIMA, BOTH])
def test_values(case):
    """the same with room and without: sums in fp32 in another order"""
    import torch
    tokens, rows, dim, dtype, which, room = case
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    x, w = torch.randn((tokens, dim), device="cuda").to(kind), (torch.randn((rows, dim), device="cuda") * (3.0 / dim ** 0.5)).to(kind)
    labels = torch.randint(-1, rows, (tokens,), dtype=torch.int32, device="cuda")
    lse = None
    if which == "dx":
        lse = torch.logsumexp((x[:, :dim].float() @ w.float().t()), -1)
    got = []
    for n in (2048 * MB, library_bytes() + room * MB):
        c = Context(device=0, workspace_bytes=n)
        got.append([c.fetch(t) for t in results(c, case, c.tensor(x), c.tensor(w), c.tensor(labels), None if lse is None else c.tensor(lse))])
        c.close()
    for a, b in zip(*got):
        assert np.linalg.norm(a - b) <= (2e-6 if dtype == "f32" or which == "losses" else 2e-3) * np.linalg.norm(a)
