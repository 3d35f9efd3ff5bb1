"""The operators at the two ends of a language model's training step, as cases that can be timed and compared.

Families (`kind`):
  embed      rows of a table by token: a lookup, its gradient by token, or both; the gradient alone or added to another one
  dropout    forward, or forward with a residual and the backward pass, from a counter-based generator (no mask is stored)
  xent       cross entropy of x w^T against labels over a vocabulary, without keeping the logits: losses, or losses and gradients
  step       lookup -> dropout -> cross entropy with the same table, backward to the one gradient of that table

Formulas.  Lookup: y[n] = scale * table[id[n]], 0 where id[n] is no row.  Its gradient: base[v] + scale * the sum of dy[n] over
the n with id[n] = v.  Dropout: t = round(65536 * rate); element i in row-major order is kept where its 16 bits are at least t and
multiplied by 65536 / (65536 - t), otherwise 0; its bits are half-word i % 8 (low half of a word first) of the four words
that Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3) gives for the counter (i / 8, site,
step's low word, step's high word) and the seed's two words as key; the state is (seed, step).  Cross entropy: l = x w^T,
lse[n] = log sum_v exp l[n, v], loss[n] = lse[n] - l[n, label[n]], both 0 where the label is no row; the gradient
g[n, v] = (exp(l[n, v] - lse[n]) - (v == label[n])) * dloss[n], 0 for such rows, dx = g w, dw = g^T x.

A case whose `own` is set goes through a Context: record, a barrier that does not block, results left on the device.
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def listed():
    return [
        # the smallest call: the next tokens of eight requests
        {"name": "embed_8x4096", "kind": "embed", "tokens": 8, "vocab": 32768, "dim": 4096, "scale": 1.0, "pass": "forward", "pad": 0.0, "dtype": "bf16"},
        # a training batch, forward and backward, scaled as by the square root of the width
        {"name": "embed_train_16384x1024", "kind": "embed", "tokens": 16384, "vocab": 50000, "dim": 1024, "scale": 32.0, "pass": "train", "pad": 0.0, "dtype": "bf16"},
        # fp32, sizes that are no multiple of anything, a tenth of the tokens padding
        {"name": "embed_train_odd_5331x203", "kind": "embed", "tokens": 5331, "vocab": 30011, "dim": 203, "scale": 1.0, "pass": "train", "pad": 0.1, "dtype": "f32"},
        # a long batch's gradient joins the gradient that the table has already, in place
        {"name": "embed_join_32768x2048", "kind": "embed", "tokens": 32768, "vocab": 131072, "dim": 2048, "scale": 1.0, "pass": "join", "pad": 0.0, "dtype": "bf16"},
        # a layer's output, behind which the residual is added, and the backward pass
        {"name": "dropout_train_16384x4096", "kind": "dropout", "rows": 16384, "dim": 4096, "rate": 0.1, "site": 3, "residual": True, "grad": True, "dtype": "bf16"},
        # fp32, an odd number of elements in all
        {"name": "dropout_odd_1777x1001", "kind": "dropout", "rows": 1777, "dim": 1001, "rate": 0.25, "site": 0, "residual": False, "grad": True, "dtype": "f32"},
        # what one token's loss is, as in scoring an answer: the table is read once
        {"name": "xent_1x131072x4096", "kind": "xent", "tokens": 1, "vocab": 131072, "dim": 4096, "ignored": 0.0, "grad": False, "weights": False, "dtype": "bf16"},
        # a small model's training batch
        {"name": "xent_train_2048x32768x1024", "kind": "xent", "tokens": 2048, "vocab": 32768, "dim": 1024, "ignored": 0.0, "grad": True, "weights": False, "dtype": "bf16"},
        # sizes that are no multiple of anything, most tokens a prompt that is not trained on, a weight for each of the others
        {"name": "xent_train_odd_1501x10007x331", "kind": "xent", "tokens": 1501, "vocab": 10007, "dim": 331, "ignored": 0.6, "grad": True, "weights": True, "dtype": "bf16"},
        # fp32
        {"name": "xent_train_f32_1024x16000x768", "kind": "xent", "tokens": 1024, "vocab": 16000, "dim": 768, "ignored": 0.0, "grad": True, "weights": False, "dtype": "f32"},
        # a large vocabulary and a wide model: the logits alone would be 4.3 GB in fp32
        {"name": "xent_train_8192x131072x4096", "kind": "xent", "tokens": 8192, "vocab": 131072, "dim": 4096, "ignored": 0.1, "grad": True, "weights": False, "dtype": "bf16"},
        # both ends of a step with one table
        {"name": "step_4096x32768x1024", "kind": "step", "tokens": 4096, "vocab": 32768, "dim": 1024, "scale": 8.0, "rate": 0.1, "site": 1, "ignored": 0.05, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["embed", "dropout", "xent", "xent", "step"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    dim = rng.choice([64, 128, 256, 512, 768, 1024, 2048, 4096, _log(rng, 1, 4096), 8 * _log(rng, 1, 512)])
    if kind == "dropout":
        return {"kind": kind, "rows": _log(rng, 1, (1 << 26) // dim), "dim": dim, "rate": rng.choice([0.0, 0.1, 0.1, 0.25, 0.5, 0.9]), "site": rng.choice([0, 1, 77]),
                "residual": rng.random() < 0.5, "grad": rng.random() < 0.5, "dtype": dtype}
    vocab = rng.choice([_log(rng, 2, 131072), _log(rng, 4096, 131072), 32768, 50000, 131072])
    if kind == "embed":
        return {"kind": kind, "tokens": _log(rng, 1, min(131072, (1 << 27) // dim)), "vocab": vocab, "dim": dim, "scale": rng.choice([1.0, 1.0, 22.5]),
                "pass": rng.choice(["forward", "train", "train", "join"]), "pad": rng.choice([0.0, 0.1, 0.5]), "dtype": dtype}
    tokens = _log(rng, 1, min(16384, (1 << 41) // (vocab * dim)))
    if kind == "step":
        return {"kind": kind, "tokens": min(tokens, 8192), "vocab": vocab, "dim": dim, "scale": rng.choice([1.0, 8.0]), "rate": rng.choice([0.1, 0.25]), "site": 5, "ignored": rng.choice([0.0, 0.3]),
                "dtype": dtype}
    return {"kind": kind, "tokens": tokens, "vocab": vocab, "dim": dim, "ignored": rng.choice([0.0, 0.0, 0.1, 0.7]), "grad": rng.random() < 0.6, "weights": rng.random() < 0.4, "dtype": dtype}


# ---- inputs ----------------------------------------------------------------------------------
class _Make:
    """Tensors from a seed, on the device."""

    def __init__(self, seed):
        self.seed = int(seed) & 0x7FFFFFFF
        self.gen = torch.Generator(device="cuda").manual_seed(self.seed)

    def normal(self, *shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=self.gen) * scale).to(dtype)

    def uniform(self, *shape):
        return torch.rand(*shape, device="cuda", generator=self.gen)

    def tokens(self, count, vocab, nothing):
        """Tokens as a text has them: the k-th most frequent about 1 / k as often as the first, in any place of the vocabulary; a share
        `nothing` of them -1 (padding, labels that do not count)."""
        rank = torch.clamp((float(vocab) ** self.uniform(count)).floor().long() - 1, 0, vocab - 1)
        ids = torch.randperm(vocab, device="cuda", generator=self.gen)[rank]
        return torch.where(self.uniform(count) < nothing, torch.full_like(ids, -1), ids).to(torch.int32)

    def state(self):
        """A generator's (seed, step): both words of the seed in use, a step of a long run."""
        return torch.tensor([(self.seed * 2654435761 + 97) % 2**62, 100000 + self.seed % 1000], dtype=torch.int64, device="cuda")


def _inputs(case, seed):
    """name -> torch tensor.  Activations N(0, 1), as behind a norm; tables so that logits spread by about three."""
    mk, kind, dt, d = _Make(seed), case["kind"], _TORCH[case["dtype"]], case["dim"]
    if kind == "dropout":
        shape = (case["rows"], d)
        t = {"state": mk.state(), "x": mk.normal(*shape, dtype=dt)}
        if case["residual"]:
            t["residual"] = mk.normal(*shape, dtype=dt)
        if case["grad"]:
            t["dy"] = mk.normal(*shape, dtype=dt)
        return t
    n, v = case["tokens"], case["vocab"]
    if kind == "embed":
        t = {"ids": mk.tokens(n, v, case["pad"])}
        if case["pass"] != "join":
            t["table"] = mk.normal(v, d, dtype=dt)
        else:
            t["base"] = mk.normal(v, d, dtype=dt)
        if case["pass"] != "forward":
            t["dy"] = mk.normal(n, d, dtype=dt)
        return t
    t = {"labels": mk.tokens(n, v, case["ignored"]), "table": mk.normal(v, d, dtype=dt, scale=3.0 / math.sqrt(d))}
    if kind == "step":
        return {**t, "ids": mk.tokens(n, v, 0.0), "state": mk.state()}
    t["x"] = mk.normal(n, d, dtype=dt)
    if case["weights"]:
        t["dloss"] = (0.5 + mk.uniform(n)) / n
    return t


def _mean(case):
    """What a loss counts in the mean over all tokens."""
    return 1.0 / case["tokens"]


# ---- the plain forms ------------------------------------------------------------------------------
_LOW = 0xFFFFFFFF


def _half_words(count, state, site):
    """The 16 bits of each of `count` elements, int64: Philox4x32-10 on int64 tensors of 32-bit words."""
    block = torch.arange(-(-count // 8), device="cuda", dtype=torch.int64)
    seed, step = state[0], state[1]
    c0, c1, c2, c3 = block, torch.full_like(block, site), (step & _LOW).expand_as(block), ((step >> 32) & _LOW).expand_as(block)
    k0, k1 = seed & _LOW, (seed >> 32) & _LOW
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack((c0, c1, c2, c3), -1)
    return torch.stack((words & 0xFFFF, words >> 16), -1).reshape(-1)[:count]


def _drop(x, state, case, residual=None):
    level = round(case["rate"] * 65536)
    kept = (_half_words(x.numel(), state, case["site"]) >= level).reshape(x.shape)
    y = torch.where(kept, x.float() * (65536.0 / (65536 - level)), torch.zeros((), device="cuda"))
    return (y if residual is None else y + residual.float()).to(x.dtype)


def _lookup(table, ids, scale):
    there = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(there, ids, torch.zeros_like(ids)).long()].float() * scale
    return torch.where(there[:, None], rows, torch.zeros_like(rows)).to(table.dtype)


def _lookup_grad(dy, ids, base, rows, scale):
    there = (ids >= 0) & (ids < rows)
    total = torch.zeros((rows, dy.shape[1]), device="cuda") if base is None else base.float()
    total.index_add_(0, ids[there].long(), dy[there].float() * scale)
    return total.to(dy.dtype if base is None else base.dtype)


def _entropy(x, w, labels):
    """loss, lse, and the logits."""
    logits = x.float() @ w.float().t()
    top = logits.amax(-1, keepdim=True)
    lse = (torch.exp(logits - top).sum(-1, keepdim=True).log() + top)[:, 0]
    there = (labels >= 0) & (labels < w.shape[0])
    picked = logits.gather(1, torch.where(there, labels, torch.zeros_like(labels)).long()[:, None])[:, 0]
    nothing = torch.zeros_like(lse)
    return torch.where(there, lse - picked, nothing), torch.where(there, lse, nothing), logits


def _entropy_grad(x, w, labels, lse, logits, dloss):
    there = (labels >= 0) & (labels < w.shape[0])
    g = torch.exp(logits - lse[:, None])
    g -= (torch.arange(w.shape[0], device="cuda") == labels[:, None]).float()
    g = torch.where(there[:, None], g * dloss[:, None], torch.zeros((), device="cuda"))
    return (g @ w.float()).to(x.dtype), (g.t() @ x.float()).to(w.dtype)


def _plain(t, case):
    kind = case["kind"]
    if kind == "dropout":
        out = {"y": _drop(t["x"], t["state"], case, t.get("residual"))}
        if case["grad"]:
            out["dx"] = _drop(t["dy"], t["state"], case)
        return out
    if kind == "embed":
        out = {}
        if case["pass"] != "join":
            out["y"] = _lookup(t["table"], t["ids"], case["scale"])
        if case["pass"] == "train":
            out["dtable"] = _lookup_grad(t["dy"], t["ids"], None, case["vocab"], case["scale"])
        if case["pass"] == "join":
            t["base"].copy_(_lookup_grad(t["dy"], t["ids"], t["base"], case["vocab"], case["scale"]))
            out["base"] = t["base"]
        return out
    x = t["x"] if kind == "xent" else _drop(_lookup(t["table"], t["ids"], case["scale"]), t["state"], case)
    loss, lse, logits = _entropy(x, t["table"], t["labels"])
    out = {"loss": loss, "lse": lse}
    if kind == "xent" and not case["grad"]:
        return out
    dloss = t["dloss"] if "dloss" in t else torch.full_like(loss, _mean(case))
    dx, dw = _entropy_grad(x, t["table"], t["labels"], lse, logits, dloss)
    if kind == "xent":
        return {**out, "dx": dx, "dw": dw}
    return {**out, "dtable": _lookup_grad(_drop(dx, t["state"], case), t["ids"], dw, case["vocab"], case["scale"])}


# ---- the framework's operators --------------------------------------------------------------------
class _Memory:
    """A result's device memory, as torch can adopt it; holds the result."""

    def __init__(self, ctx, t):
        self.owner = t, ctx
        self.__cuda_array_interface__ = {"shape": t.shape, "typestr": {"f32": "<f4", "bf16": "<i2"}[t.dtype], "data": (ctx.device_ptr(t), False), "version": 2, "strides": None}


def _as_torch(ctx, t):
    v = torch.as_tensor(_Memory(ctx, t), device="cuda")
    return v.view(torch.bfloat16) if t.dtype == "bf16" else v


def _record(ctx, T, case):
    """Records a step's ops; what it leaves on the device, by name."""
    kind = case["kind"]
    if kind == "dropout":
        out = {"y": ctx.dropout(T["x"], T["state"], case["rate"], site=case["site"], residual=T.get("residual"))}
        if case["grad"]:
            out["dx"] = ctx.dropout_grad(T["dy"], T["state"], case["rate"], site=case["site"])
        return out
    if kind == "embed":
        out = {}
        if case["pass"] != "join":
            out["y"] = ctx.embedding(T["table"], T["ids"], scale=case["scale"])
        if case["pass"] == "train":
            out["dtable"] = ctx.embedding_grad(T["dy"], T["ids"], rows=case["vocab"], scale=case["scale"])
        if case["pass"] == "join":
            ctx.assign(T["base"], ctx.embedding_grad(T["dy"], T["ids"], into=T["base"], scale=case["scale"]))
        return out
    x = T["x"] if kind == "xent" else ctx.dropout(ctx.embedding(T["table"], T["ids"], scale=case["scale"]), T["state"], case["rate"], site=case["site"])
    loss, lse = ctx.linear_xent(x, T["table"], T["labels"])
    out = {"loss": loss, "lse": lse}
    if kind == "xent" and not case["grad"]:
        return out
    dx, dw = ctx.linear_xent_grad(x, T["table"], T["labels"], lse, T.get("dloss", _mean(case)))
    if kind == "xent":
        return {**out, "dx": dx, "dw": dw}
    back = ctx.dropout_grad(dx, T["state"], case["rate"], site=case["site"])
    return {**out, "dtable": ctx.embedding_grad(back, T["ids"], into=dw, scale=case["scale"])}


def _workspace(case):
    """Bytes for results (those of the step before too) and temporaries."""
    w = _BYTES[case["dtype"]]
    results = case["dim"] * (2 * case["rows"] if case["kind"] == "dropout" else 2 * case["tokens"] + 2 * case["vocab"]) * w
    return (1 << 30) + 3 * results


def prepare(case, seed):
    data = _inputs(case, seed)
    state = {"case": case, "data": data, "held": None}
    if own:
        from paper_2102_13267_amd import Context
        ctx = Context(device=torch.cuda.current_device(), workspace_bytes=_workspace(case))
        state.update(ctx=ctx, tensors={k: ctx.tensor(v, donatable=k == "base") for k, v in data.items()})
    return state


def run(state):
    case, data = state["case"], state["data"]
    if not own:
        return _plain(data, case)
    ctx = state["ctx"]
    results = _record(ctx, state["tensors"], case)
    ctx.barrier(False)
    state["held"] = results          # (the last step's results make room when the next step's replace them)
    out = {k: _as_torch(ctx, t) for k, t in results.items()}
    if "base" in data:
        out["base"] = data["base"]
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    w, kind, d = _BYTES[case["dtype"]], case["kind"], case["dim"]
    if kind == "dropout":
        n = case["rows"] * d
        passes = (3 if case["residual"] else 2) + (2 if case["grad"] else 0)
        return {"bytes": passes * n * w + 16, "flops": (2 if case["grad"] else 1) * n}
    n, v = case["tokens"], case["vocab"]
    if kind == "embed":
        used = round(n * (1.0 - case["pad"]))
        # (about so many different rows, each read once; their number is at most the tokens')
        rows = min(used, round(v * (1.0 - math.exp(-used / (v * max(1.0, math.log(v)) / 2)))) + 1)
        forward, backward, join = rows * d * w + n * d * w + 4 * n, used * d * w + 4 * n + v * d * w, used * d * w + 4 * n + 2 * rows * d * w
        moved = {"forward": forward, "train": forward + backward, "join": join}[case["pass"]]
        return {"bytes": moved, "flops": used * d * (2 if case["pass"] == "train" else 1)}
    used = round(n * (1.0 - case["ignored"]))
    product = 2 * used * v * d
    tables = (used + v) * d * w + 4 * n
    if kind == "xent":
        if not case["grad"]:
            return {"bytes": tables + 8 * n, "flops": product}
        # the logits are products once; dx and dw are the other two
        return {"bytes": tables + (n + v) * d * w + 8 * n + (4 * n if case["weights"] else 0), "flops": 3 * product}
    return {"bytes": v * d * w + 8 * n + 8 * n + v * d * w, "flops": 3 * product + 4 * n * d}


# ---- the same in 64 bits ------------------------------------------------------------------------
def _product_words(a, b):
    """High and low word of the product of 32-bit words a (tensor) and b (number), through 16-bit halves."""
    a0, a1, b0, b1 = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    low, mid, high = a0 * b0, a1 * b0 + a0 * b1, a1 * b1
    mid = mid + (low >> 16)
    return high + (mid >> 16), ((mid & 0xFFFF) << 16) | (low & 0xFFFF)


def _kept64(count, state, case):
    """Which of `count` elements are kept."""
    seed, step = (int(s) & 0xFFFFFFFFFFFFFFFF for s in state.tolist())
    ctr = [torch.arange((count + 7) // 8, device="cuda", dtype=torch.int64)]
    ctr += [torch.zeros_like(ctr[0]) + c for c in (case["site"], step % 2**32, step // 2**32)]
    for r in range(10):
        key = ((seed % 2**32 + r * 0x9E3779B9) % 2**32, (seed // 2**32 + r * 0xBB67AE85) % 2**32)
        h0, l0 = _product_words(ctr[0], 0xD2511F53)
        h2, l2 = _product_words(ctr[2], 0xCD9E8D57)
        ctr = [h2 ^ ctr[1] ^ key[0], l2, h0 ^ ctr[3] ^ key[1], l0]
    bits = torch.empty((ctr[0].numel(), 8), device="cuda", dtype=torch.int64)
    for i, word in enumerate(ctr):
        bits[:, 2 * i], bits[:, 2 * i + 1] = word % 65536, word // 65536
    return bits.flatten()[:count] >= round(65536 * case["rate"])


def _drop64(x, state, case):
    kept = _kept64(x.numel(), state, case).view(x.shape)
    return x.masked_fill(~kept, 0.0) / (1.0 - round(65536 * case["rate"]) / 65536)


def _lookup64(table, ids, scale):
    y = torch.zeros((ids.numel(), table.shape[1]), dtype=torch.float64, device="cuda")
    at = torch.nonzero((ids >= 0) & (ids < table.shape[0]))[:, 0]
    y[at] = table[ids[at].long()].double() * scale
    return y


def _lookup_grad64(dy, ids, total, scale):
    at = torch.nonzero((ids >= 0) & (ids < total.shape[0]))[:, 0]
    at = at[torch.argsort(ids[at], stable=True)]
    # sums of runs of equal tokens, as differences of running sums within pieces of columns
    keys, counts = torch.unique_consecutive(ids[at].long(), return_counts=True)
    ends = torch.cumsum(counts, 0)
    for c in range(0, dy.shape[1], 256):
        run = torch.cumsum(dy[at, c:c + 256].double(), 0)[ends - 1]
        total[keys, c:c + 256] += scale * torch.diff(run, dim=0, prepend=torch.zeros_like(run[:1]))
    return total


def _entropy64(x, w, labels, dloss):
    """x float64; dloss None: no gradients."""
    n, v = x.shape[0], w.shape[0]
    loss, lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    dx = dw = None
    wd = w.double()
    if dloss is not None:
        dx, dw = torch.zeros_like(x), torch.zeros_like(wd)
    at = torch.nonzero((labels >= 0) & (labels < v))[:, 0]
    for rows in torch.split(at, max(1, (1 << 27) // v)):
        l = x[rows] @ wd.t()
        lse[rows] = torch.logsumexp(l, -1)
        hit = labels[rows].long()[:, None]
        loss[rows] = lse[rows] - l.gather(1, hit)[:, 0]
        if dloss is not None:
            g = torch.exp(l - lse[rows][:, None])
            g.scatter_add_(1, hit, torch.full_like(g[:, :1], -1.0))
            g *= dloss[rows].double()[:, None]
            dx[rows] = g @ wd
            dw += g.t() @ x[rows]
    return loss, lse, dx, dw


def exact(case, seed):
    t, kind = _inputs(case, seed), case["kind"]
    if kind == "dropout":
        y = _drop64(t["x"].double(), t["state"], case)
        out = {"y": y + t["residual"].double() if case["residual"] else y}
        if case["grad"]:
            out["dx"] = _drop64(t["dy"].double(), t["state"], case)
        return out
    if kind == "embed":
        out = {}
        if case["pass"] != "join":
            out["y"] = _lookup64(t["table"], t["ids"], case["scale"])
        if case["pass"] == "train":
            out["dtable"] = _lookup_grad64(t["dy"], t["ids"], torch.zeros((case["vocab"], case["dim"]), dtype=torch.float64, device="cuda"), case["scale"])
        if case["pass"] == "join":
            out["base"] = _lookup_grad64(t["dy"], t["ids"], t["base"].double(), case["scale"])
        return out
    if kind == "xent":
        dloss = (t["dloss"] if case["weights"] else torch.full((case["tokens"],), _mean(case), device="cuda")) if case["grad"] else None
        loss, lse, dx, dw = _entropy64(t["x"].double(), t["table"], t["labels"], dloss)
        return {"loss": loss, "lse": lse, "dx": dx, "dw": dw} if case["grad"] else {"loss": loss, "lse": lse}
    # what goes on from one operator to the next is of the table's type: those roundings are the type's own
    dt = t["table"].dtype
    x = _drop64(_lookup64(t["table"], t["ids"], case["scale"]).to(dt).double(), t["state"], case).to(dt).double()
    loss, lse, dx, dw = _entropy64(x, t["table"], t["labels"], torch.full((case["tokens"],), _mean(case), device="cuda"))
    back = _drop64(dx.to(dt).double(), t["state"], case).to(dt)
    return {"loss": loss, "lse": lse, "dtable": _lookup_grad64(back, t["ids"], dw.to(dt).double(), case["scale"])}
