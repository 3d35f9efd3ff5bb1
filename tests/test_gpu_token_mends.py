"""Calls of the token operators that were answered wrongly once, each beside what is right by the formulas."""
import numpy as np
import pytest
import torch

from test_gpu_token_operators import context, data

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,dim", [(0, 300, 64), (7, 300, 64), (40, 300, 33), (300, 900, 64), (300, 900, 2048)])
def test_a_gradient_that_no_token_adds_to(tokens, vocab, dim, dtype):
    """g is 0 for a token whose label is no row, whatever dloss is: the mean over no tokens has 1 / 0 there"""
    rg = np.random.default_rng(1)
    ctx = context()
    x, w = torch.tensor(data(rg, (tokens, dim), dtype), device="cuda"), data(rg, (vocab, dim), dtype)
    X, W, L = ctx.tensor(x.to(torch.bfloat16) if dtype == "bf16" else x), ctx.tensor(w, dtype), ctx.tensor(torch.full((tokens,), -1, dtype=torch.int32, device="cuda"))
    for value in (np.inf, -np.inf, np.nan):
        for dloss in (value, ctx.mean(ctx.tensor(np.array([value], np.float32))), ctx.tensor(torch.full((tokens,), value, device="cuda"))):
            loss, lse = ctx.linear_xent(X, W, L)
            dx, dw = ctx.linear_xent_grad(X, W, L, lse, dloss)
            assert all((ctx.fetch(t) == 0).all() for t in (loss, lse, dx, dw)), value
    ctx.close()
