"""The largest sizes that the token operators take: what their launches are, from their plans on the null device (tests/host_sanitize/reach.cpp), and, on a GPU, what comes
out behind the 2^32 threads that one launch holds along an axis."""
import os
import subprocess

import numpy as np
import pytest
import torch

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2102_13267_amd", "csrc")
HERE = os.path.join(ROOT, "tests", "host_sanitize")


def test_launches_of_the_largest_sizes(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    exe = str(tmp_path / "reach")
    srcs = [os.path.join(CSRC, f) for f in ("lt_api.cpp", "lt_barrier.cpp", "lt_lower.cpp", "lt_schedule.cpp")] + [os.path.join(HERE, f) for f in ("stubs.cpp", "reach.cpp")]
    build = subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", f"-I{rocm}/include", "-o", exe] + srcs + [f"-L{rocm}/lib", "-lamdhip64", f"-Wl,-rpath,{rocm}/lib"],
                           capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0 and "reach: ok" in run.stdout, (run.stdout + run.stderr)[-4000:]


@pytest.fixture
def room():
    """gives back what the large tensors of a test took"""
    yield
    torch.cuda.empty_cache()


def sampled(rg, tokens):
    """the first and last tokens, and some between"""
    return torch.tensor(np.unique(np.concatenate([np.arange(50), tokens - 1 - np.arange(50), rg.integers(0, tokens, 300)])), device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("dtype,tokens,vocab,dim,gigabytes", [("bf16", 2 ** 26 + 300, 200, 8, 110), ("f32", 2 ** 23, 2048, 128, 110)])
def test_a_cross_entropy_of_so_many_tokens(room, dtype, tokens, vocab, dim, gigabytes, each):
    """2^26 tokens: a wave each for packing and for dx; 2^23 whose logits are kept: a wave for 256 of them.  The first, the last and some other tokens are compared by
    themselves, with the bounds of test_gpu_token_operators; dw as the sum over all of them: p and lse are off by less than 10^-3 of p (logits of below 100 in
    all their terms), g and x dloss by a rounding, and a sum in fp32 takes 32 products a step in bf16, in fp32 chains of 256 and their sum."""
    from test_gpu_token_operators import E24, HALF, Eager, context, entropy_bounds, grads_bound, within
    rg = np.random.default_rng(1)
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    ctx, E = context(workspace_bytes=gigabytes << 30), Eager("f64")
    x = torch.empty((tokens, dim), dtype=kind, device="cuda")
    some = torch.randn((1 << 20, dim), device="cuda").to(kind)
    for at in range(0, tokens, 1 << 20):
        x[at:at + (1 << 20)] = some[:tokens - at]
    w = (torch.randn((vocab, dim), device="cuda") * (3.0 / dim ** 0.5)).to(kind)
    label = torch.randint(0, vocab, (tokens,), dtype=torch.int32, device="cuda")
    label[[3, tokens // 2, tokens - 2]] = -1
    weight = torch.rand(tokens, device="cuda") + 0.5
    if not each:
        weight[:] = 0.5
    X, W, L = ctx.tensor(x), ctx.tensor(w), ctx.tensor(label)
    loss, lse = ctx.linear_xent(X, W, L)
    dx, dw = ctx.linear_xent_grad(X, W, L, lse, ctx.tensor(weight) if each else 0.5)
    ctx.barrier()
    loss, lse, dx, dw = (_as_torch(ctx, v) for v in (loss, lse, dx, dw))
    rows = sampled(rg, tokens)
    xs, ws, ls, ds, got = x[rows].float().cpu().numpy(), w.float().cpu().numpy(), label[rows].cpu().numpy(), weight[rows].cpu().numpy(), [t[rows].float().cpu().numpy() for t in (loss, lse, dx)]
    ref = [t.data for t in E.linear_xent(E.tensor(xs, dtype), E.tensor(ws, dtype), E.tensor(ls))]
    there, dlse, dloss = entropy_bounds(xs, ws, ls, dtype)
    within(got[1][there], ref[1][there], dlse, "lse")
    within(got[0][there], ref[0][there], dloss, "loss")
    rx = E.linear_xent_grad(E.tensor(xs, dtype), E.tensor(ws, dtype), E.tensor(ls), E.tensor(got[1]), E.tensor(ds))[0].data
    within(got[2][there], rx[there], grads_bound(xs, ws, ls, got[1], ds, dtype)[1], "dx")
    assert (~there).any() and all((t[~there] == 0).all() for t in got)
    total, size = (torch.zeros((vocab, dim), dtype=torch.float64, device="cuda") for _ in range(2))
    for at in range(0, tokens, 1 << 18):
        xs, ls = x[at:at + (1 << 18)].double(), label[at:at + (1 << 18)]
        d = (weight[at:at + (1 << 18)] * (ls >= 0)).double()[:, None]
        l = xs @ w.double().t()
        p = torch.exp(l - torch.logsumexp(l, -1)[:, None]) * d
        hit = torch.zeros_like(p).scatter_(1, ls.clamp(min=0).long()[:, None], d)
        total += (p - hit).t() @ xs
        size += (p + hit).t() @ xs.abs()
    steps = tokens / 32 if dtype == "bf16" else 256 + tokens / 256
    bound = (2 * HALF[dtype] + 1e-3 + steps * E24) * size + HALF[dtype] * total.abs()
    assert ((dw.double() - total).abs() <= bound).all()
    ctx.close()


def _as_torch(ctx, t):
    """a result where it lies"""
    class Memory:
        __cuda_array_interface__ = {"shape": t.shape, "typestr": {"f32": "<f4", "bf16": "<i2"}[t.dtype], "data": (ctx.device_ptr(t), False), "version": 2, "strides": None}
    v = torch.as_tensor(Memory(), device="cuda")
    return v.view(torch.bfloat16) if t.dtype == "bf16" else v


@pytest.mark.gpu
def test_a_gradient_of_rows_so_long(room):
    """4096 tokens of 2^23 + 1 columns, read element by element: 2^26 waves and more, for the sums and for joining them; in place and beside its base"""
    from test_gpu_token_operators import context
    tokens, rows, dim = 4096, 8, 2 ** 23 + 1
    rg = np.random.default_rng(2)
    dy = torch.ones((tokens, dim), dtype=torch.bfloat16, device="cuda")
    dy[:, -1] = 2.0
    dy[:, dim // 2] = 0.5
    ids = rg.integers(0, rows, tokens).astype(np.int32)
    counts = torch.tensor(np.bincount(ids, minlength=rows), device="cuda").float()
    base = torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda")
    ctx = context(workspace_bytes=40 << 30)
    D, I, B = ctx.tensor(dy), ctx.tensor(ids), ctx.tensor(base, donatable=True)
    beside = ctx.embedding_grad(D, I, rows=rows)
    ctx.barrier()
    ctx.assign(B, ctx.embedding_grad(D, I, into=B))
    ctx.barrier()
    want = counts[:, None].to(torch.bfloat16).expand(rows, dim).clone()      # (whole numbers below 2^24, summed exactly and rounded once)
    want[:, -1] = (2 * counts).to(torch.bfloat16)
    want[:, dim // 2] = (counts / 2).to(torch.bfloat16)
    assert torch.equal(_as_torch(ctx, beside), want) and torch.equal(base, want)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [131072, 131073, 262145, 700001])
@pytest.mark.parametrize("kind", ["any", "one", "few", "padding"])
def test_gradients_of_so_many_tokens_that_a_piece_is_more_than_a_wave_reads(tokens, kind):
    """pieces of up to 256 sorted tokens, 64 at a time: whole numbers, whose sums are exact"""
    from test_gpu_token_operators import context
    torch.manual_seed(tokens)
    for rows, dim, into in ((1000, 9, "f32"), (300001, 16, "bf16"), (70, 33, None)):
        ids = {"any": torch.randint(-1, rows + 1, (tokens,), device="cuda"), "one": torch.full((tokens,), rows - 1, device="cuda"), "few": torch.randint(0, 3, (tokens,), device="cuda"),
               "padding": torch.where(torch.rand(tokens, device="cuda") < 0.9, -1, torch.randint(0, rows, (tokens,), device="cuda"))}[kind].int()
        dy = torch.randint(-2, 3, (tokens, dim), device="cuda").float()
        there = (ids >= 0) & (ids < rows)
        want = torch.zeros((rows, dim), dtype=torch.float64).index_add_(0, ids[there].long().cpu(), dy[there].double().cpu()).cuda()
        ctx = context(workspace_bytes=512 << 20)
        D, I = ctx.tensor(dy), ctx.tensor(ids)
        if into is None:
            got, want = ctx.embedding_grad(D, I, rows=rows), want.float()
        else:
            kind_of = torch.float32 if into == "f32" else torch.bfloat16
            base = torch.randint(-3, 4, (rows, dim), device="cuda").to(kind_of)
            want = (want + base.double()).float().to(kind_of)
            got = ctx.embedding_grad(D, I, into=ctx.tensor(base))
        ctx.barrier()
        assert torch.equal(_as_torch(ctx, got), want), (rows, dim, into)
        ctx.close()
