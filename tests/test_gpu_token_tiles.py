"""The cross entropy over a vocabulary at sizes whose products are whole rounds of tiles of 256 x 256, with rows of many slabs: losses and every element of both gradients
against sums in 64 bits, with the bounds of test_gpu_token_operators."""
import pytest
import torch

from test_gpu_token_operators import E24, HALF, TINY, context

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("tokens,vocab,dim", [(4096, 16384, 1024), (4000, 20011, 1100), (2048, 32768, 2048)])
def test_losses_and_gradients(tokens, vocab, dim, each):
    """the second: edges in every direction, packed rows; the third: logits that are kept"""
    torch.manual_seed(tokens + vocab)
    half = HALF["bf16"]
    x, w = torch.randn((tokens, dim), device="cuda").to(torch.bfloat16), (torch.randn((vocab, dim), device="cuda") * (3.0 / dim ** 0.5)).to(torch.bfloat16)
    labels = torch.randint(0, vocab, (tokens,), dtype=torch.int32, device="cuda")
    labels[::17] = -1
    weight = torch.rand(tokens, device="cuda") - 0.3 if each else torch.full((tokens,), 0.37, device="cuda")
    ctx = context(workspace_bytes=4 << 30)
    X, W, L = ctx.tensor(x), ctx.tensor(w), ctx.tensor(labels)
    loss, lse = ctx.linear_xent(X, W, L)
    dx, dw = ctx.linear_xent_grad(X, W, L, lse, ctx.tensor(weight) if each else float(weight[0]))
    ctx.barrier()
    loss, lse, dx, dw = (torch.tensor(ctx.fetch(t), device="cuda").double() for t in (loss, lse, dx, dw))
    there = labels >= 0
    assert all((t[~there] == 0).all() for t in (loss, lse, dx))
    x, w, s, d, hit = x[there].double(), w.double(), lse[there][:, None], weight[there].double()[:, None], labels[there].long()[:, None]
    logits, terms = x @ w.t(), x.abs() @ w.abs().t()
    dl = (dim + 1) * E24 * terms
    want = torch.logsumexp(logits, -1)
    dlse = dl.amax(-1) + (3 * (logits.amax(-1) - logits.amin(-1)) + 96 + vocab / 2048 + 8) * E24 + 3 * E24 * want.abs()
    picked = logits.gather(1, hit)[:, 0]
    assert ((s[:, 0] - want).abs() <= dlse).all()
    assert ((loss[there] - (want - picked)).abs() <= dlse + dl.amax(-1) + E24 * (want - picked).abs()).all()
    # the gradient takes lse as given
    p = torch.exp(logits - s)
    g = p.clone().scatter_add_(1, hit, torch.full_like(s, -1.0)) * d
    dg = d.abs() * p * (dl + (3 * (logits - s).abs() + 4) * E24) + (E24 + half) * g.abs()
    for got, ref, bound, n, more in ((dx[there], g @ w, dg @ w.abs(), vocab, g.abs() @ w.abs()), (dw, g.t() @ x, dg.t() @ x.abs(), len(g), g.abs().t() @ x.abs())):
        off = (got - ref).abs() - bound - ((n + 2) * E24 + (half if each and got is dw else 0)) * more - half * ref.abs() - TINY
        assert (off <= 0).all(), float(off.max())
    # and by their norms: as many roundings at random leave a hundredth of what they could add up to
    assert torch.linalg.norm(dx[there] - g @ w) <= half * torch.linalg.norm(g @ w) and torch.linalg.norm(dw - g.t() @ x) <= 2 * half * torch.linalg.norm(g.t() @ x)
    ctx.close()
