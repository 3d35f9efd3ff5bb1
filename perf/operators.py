"""The operators of decoding with a paged cache of keys and values, as cases that can be timed and compared.

Families (`kind`):
  rope       rotary positions on heads [..., heads, head]: a forward pass, or a training pass (forward and gradient)
  append     keys and values of new tokens, the keys rotated on the way, into a paged cache that is updated in place
  attention  one new token a sequence attends to everything its sequence has in the cache
  decode     the three in one step, as a model's layer makes them for every token that it answers with

The cache is [pages, 2, key heads, rows of a page, head]: keys at 0, values at 1.  Sequence s holds its position p in
row p % page of page table[s][p // page]; entries behind its last page are -1.  `lengths` counts the keys of each
sequence with the new tokens in, `offsets` says which rows of k and v are whose (without it, row s is sequence s's);
the tokens of a sequence are its last positions.

Formulas.  Rotation: pair i of dims / 2 turns by a = position * f_i, f_i = base^(-2i / dims); for long contexts
f_i * (g_i + (1 - g_i) / factor) with g_i = clamp((original * f_i / 2 pi - low) / (high - low), 0, 1), or g_i = 0 where
original is 0.  (x, y) -> amplitude * (x cos a - y sin a, y cos a + x sin a); pairs are (i, i + dims / 2), or
(2i, 2i + 1) interleaved; behind dims the head stays as it is.  The gradient turns back.  Attention:
softmax(scale * q K^T) V over the sequence's keys, 0 where it has none.

A case whose `own` is set goes through a Context: record, a barrier that does not block, results left on the device.
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
BASE, LOW, HIGH = 10000.0, 1.0, 32.0


def listed():
    return [
        # the smallest call: the queries of one token for each of a few requests, at far positions
        {"name": "rope_16x32x128", "kind": "rope", "batch": 1, "seq": 16, "heads": 32, "head": 128, "dims": 128, "interleaved": False,
         "factor": 1.0, "original": 0, "amplitude": 1.0, "grad": False, "start": 100000, "dtype": "bf16"},
        # a training step's batch, positions shared by its rows, forward and backward
        {"name": "rope_train_8x2048x16x64", "kind": "rope", "batch": 8, "seq": 2048, "heads": 16, "head": 64, "dims": 64, "interleaved": True,
         "factor": 1.0, "original": 0, "amplitude": 1.0, "grad": True, "start": 0, "dtype": "bf16"},
        # fp32, sizes that are no multiple of anything, half of the head rotated, positions interpolated
        {"name": "rope_train_3x1777x12x80", "kind": "rope", "batch": 3, "seq": 1777, "heads": 12, "head": 80, "dims": 40, "interleaved": False,
         "factor": 4.0, "original": 0, "amplitude": 1.0, "grad": True, "start": 0, "dtype": "f32"},
        # the queries of long prompts, scaled by frequency
        {"name": "rope_65536x32x128", "kind": "rope", "batch": 1, "seq": 65536, "heads": 32, "head": 128, "dims": 128, "interleaved": False,
         "factor": 8.0, "original": 8192, "amplitude": 1.2, "grad": False, "start": 0, "dtype": "bf16"},
        # one token for each of 64 requests
        {"name": "append_64", "kind": "append", "sequences": 64, "new": 1, "keys": 1024, "kv_heads": 8, "head": 128, "dims": 128, "interleaved": False,
         "factor": 1.0, "original": 0, "page": 16, "pad": 0, "dtype": "bf16"},
        # eight prompts of different lengths behind each other, the batch padded
        {"name": "append_8x2048", "kind": "append", "sequences": 8, "new": 2048, "keys": 4096, "kv_heads": 8, "head": 128, "dims": 128, "interleaved": False,
         "factor": 8.0, "original": 8192, "page": 64, "pad": 100, "dtype": "bf16"},
        # fp32, pages and heads that are no power of two, part of the head rotated
        {"name": "append_odd_5x267", "kind": "append", "sequences": 5, "new": 267, "keys": 1001, "kv_heads": 3, "head": 72, "dims": 36, "interleaved": True,
         "factor": 1.0, "original": 0, "page": 24, "pad": 3, "dtype": "f32"},
        # one request with little in the cache: latency
        {"name": "attention_1x300", "kind": "attention", "sequences": 1, "keys": 300, "heads": 32, "kv_heads": 8, "head": 128, "page": 16, "dtype": "bf16"},
        # 64 requests of all lengths, four of their places free
        {"name": "attention_64x4096", "kind": "attention", "sequences": 64, "idle": 4, "keys": 4096, "heads": 32, "kv_heads": 8, "head": 128, "page": 16, "dtype": "bf16"},
        # one request with a long document: the cache's length is all there is to share out
        {"name": "attention_1x131072", "kind": "attention", "sequences": 1, "keys": 131072, "heads": 32, "kv_heads": 8, "head": 128, "page": 64, "dtype": "bf16"},
        # fp32, pages that end inside a tile, a head of 80
        {"name": "attention_odd_7x3001", "kind": "attention", "sequences": 7, "keys": 3001, "heads": 12, "kv_heads": 4, "head": 80, "page": 24, "dtype": "f32"},
        # a layer's step for 32 requests
        {"name": "decode_32x2048", "kind": "decode", "sequences": 32, "keys": 2048, "heads": 32, "kv_heads": 8, "head": 128, "dims": 128, "interleaved": False,
         "factor": 1.0, "original": 0, "page": 16, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attention", "decode"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    head = rng.choice([32, 64, 72, 80, 96, 112, 128, 128, 160, 256, 20, 50])
    dims = head if rng.random() < 0.6 else max(2, head // 4 * 2)
    interleaved = rng.random() < 0.4
    factor, original = rng.choice([(1.0, 0), (4.0, 0), (8.0, 8192)])
    rotation = {"dims": dims, "interleaved": interleaved, "factor": factor, "original": original}
    if kind == "rope":
        heads = rng.choice([1, 4, 7, 8, 16, 32])
        tokens = _log(rng, 1, min(65536, (1 << 27) // (heads * head)))
        batch = rng.choice([b for b in (1, 2, 3, 8) if b <= tokens])
        return {"kind": kind, "batch": batch, "seq": tokens // batch, "heads": heads, "head": head, **rotation, "amplitude": rng.choice([1.0, 1.2]),
                "grad": rng.random() < 0.5, "start": rng.choice([0, 0, 100000]), "dtype": dtype}
    kv_heads = rng.choice([1, 2, 3, 4, 8, 16])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    sequences = _log(rng, 1, 256)
    most = min(131072, (1 << 27) // (kv_heads * head * sequences))
    keys = _log(rng, 1, most)
    if kind == "append":
        new = 1 if rng.random() < 0.4 else _log(rng, 1, max(1, keys // 2))
        return {"kind": kind, "sequences": sequences, "new": new, "keys": max(keys, new), "kv_heads": kv_heads, "head": head, **rotation, "page": page,
                "pad": rng.choice([0, 0, 5]) if new > 1 else 0, "dtype": dtype}
    case = {"kind": kind, "sequences": sequences, "keys": keys, "heads": kv_heads * rng.choice([1, 2, 4, 7, 8]), "kv_heads": kv_heads, "head": head, "page": page, "dtype": dtype}
    if kind == "attention":
        return {**case, "idle": rng.choice([0, 0, sequences // 4])}
    return {**case, **rotation}


# ---- inputs ----------------------------------------------------------------------------------
class _Make:
    """Tensors from a seed, on the device."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(int(seed) & 0x7FFFFFFF)

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(*shape, device="cuda", generator=self.gen).to(dtype)

    def order(self, n):
        return torch.randperm(n, device="cuda", generator=self.gen)


def _spread(most, count):
    """Lengths from about a sixteenth of `most` up to it: those of requests that have been running for different times."""
    return [max(1, round(most * 16.0 ** (-i / max(1, count - 1)))) for i in range(count)]


def _lengths(case):
    idle = case.get("idle", 0)
    return [0] * idle + _spread(case["keys"], case["sequences"] - idle)


def _news(case):
    """New tokens of each sequence, in the order of `_lengths`: no more than the sequence is long."""
    return [min(n, m) for n, m in zip(_spread(case["new"], case["sequences"]), _lengths(case))]


def _inputs(case, seed):
    """name -> torch tensor.  Activations N(0, 1), as behind a norm and a projection."""
    mk, kind, dt = _Make(seed), case["kind"], _TORCH[case["dtype"]]
    if kind == "rope":
        shape = (case["batch"], case["seq"], case["heads"], case["head"])
        t = {"x": mk.normal(*shape, dtype=dt), "positions": torch.arange(case["start"], case["start"] + case["seq"], device="cuda", dtype=torch.int32)}
        if case["start"]:    # tokens of different requests, each at a position of its own
            t["positions"] = t["positions"] + mk.order(case["seq"]).to(torch.int32)
        if case["grad"]:
            t["dy"] = mk.normal(*shape, dtype=dt)
        return t
    s, page, h, d = case["sequences"], case["page"], case["kv_heads"], case["head"]
    order = mk.order(s)
    lens = torch.tensor(_lengths(case), device="cuda")[order]
    per_seq = -(-case["keys"] // page)                        # pages a sequence may hold
    need = torch.div(lens + page - 1, page, rounding_mode="floor")
    total = sum(-(-n // page) for n in _lengths(case))
    pages = total + 4                                          # (a few pages that nobody holds)
    first = torch.cumsum(need, 0) - need
    slot = torch.arange(per_seq, device="cuda")
    ids = mk.order(pages)[torch.clamp(first[:, None] + slot[None, :], max=pages - 1)]
    t = {"lengths": lens.to(torch.int32), "table": torch.where(slot[None, :] < need[:, None], ids, torch.full_like(ids, -1)).to(torch.int32).contiguous(),
         "cache": mk.normal(pages, 2, h, page, d, dtype=dt)}
    if kind == "append" and case["new"] > 1:
        news = torch.tensor(_news(case), device="cuda")[order]
        t["offsets"] = torch.cat([torch.zeros_like(news[:1]), torch.cumsum(news, 0)]).to(torch.int32)
        tokens = sum(_news(case)) + case["pad"]
    else:
        tokens = s
    if kind != "attention":
        t["k"], t["v"] = mk.normal(tokens, h, d, dtype=dt), mk.normal(tokens, h, d, dtype=dt)
    if kind != "append":
        t["q"] = mk.normal(s, case["heads"], d, dtype=dt)
    if kind == "decode":
        t["positions"] = t["lengths"] - 1
    return t


# ---- the plain forms ------------------------------------------------------------------------------
def _frequencies(case):
    """f_i of the pairs, in 64 bits."""
    i = torch.arange(case["dims"] // 2, device="cuda", dtype=torch.float64)
    f = torch.pow(torch.tensor(BASE, device="cuda", dtype=torch.float64), -2.0 * i / case["dims"])
    if not case["original"]:
        return f / case["factor"]
    keep = torch.clamp((case["original"] * f / (2.0 * math.pi) - LOW) / (HIGH - LOW), 0.0, 1.0)
    return f * (keep + (1.0 - keep) / case["factor"])


def _rotate(x, positions, case, back=False):
    """x fp32 [..., heads, head], positions [...] or the last of these axes.  Angles in 64 bits: a far position times a frequency
    leaves 32 bits no digits behind the point."""
    angle = (positions.to(torch.float64)[..., None] * _frequencies(case))[..., None, :]
    amplitude = case.get("amplitude", 1.0)
    cos, sin = (torch.cos(angle) * amplitude).float(), (torch.sin(-angle if back else angle) * amplitude).float()
    n = case["dims"]
    if case["interleaved"]:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., : n // 2], x[..., n // 2:n]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., n:]), -1)


def _append(t, case):
    cache, k, v = t["cache"], t["k"].float(), t["v"].float()
    lengths, table, page = t["lengths"].long(), t["table"].long(), case["page"]
    token = torch.arange(k.shape[0], device="cuda")
    if "offsets" in t:
        offsets = t["offsets"].long()
        # rows behind the last sequence write what the first token writes, where it writes it
        token = torch.where(token < offsets[-1], token, torch.zeros_like(token))
        seq = torch.searchsorted(offsets, token, right=True) - 1
        pos = lengths[seq] - offsets[seq + 1] + token
    else:
        seq, pos = token, lengths - 1
    pid, row = table[seq, torch.div(pos, page, rounding_mode="floor")], pos % page
    cache[pid, 0, :, row] = _rotate(k[token], pos, case).to(cache.dtype)
    cache[pid, 1, :, row] = v[token].to(cache.dtype)


def _attend(q, t, case):
    cache, table, lengths = t["cache"], t["table"].long(), t["lengths"].long()
    s, h, d = case["sequences"], case["kv_heads"], case["head"]
    held = cache[torch.clamp(table, min=0)].float()                                # [s, slots, 2, h, page, d]
    n = held.shape[1] * held.shape[4]
    keys, values = (held[:, :, i].permute(0, 2, 1, 3, 4).reshape(s * h, n, d) for i in (0, 1))
    qs = q.float().reshape(s * h, case["heads"] // h, d) * (1.0 / math.sqrt(d))
    score = torch.matmul(qs, keys.transpose(1, 2).contiguous()).reshape(s, h, -1, n)
    there = torch.arange(n, device="cuda") < lengths[:, None]
    score = score.masked_fill(~there[:, None, None, :], -math.inf)
    top = torch.clamp(score.amax(-1, keepdim=True), min=-3.0e38)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    return torch.matmul(p.reshape(s * h, -1, n), values).reshape(s, case["heads"], d).to(q.dtype)


def _plain(t, case):
    kind = case["kind"]
    if kind == "rope":
        out = {"y": _rotate(t["x"].float(), t["positions"], case).to(t["x"].dtype)}
        if case["grad"]:
            out["dx"] = _rotate(t["dy"].float(), t["positions"], case, back=True).to(t["x"].dtype)
        return out
    if kind == "append":
        _append(t, case)
        return {"cache": t["cache"]}
    if kind == "attention":
        return {"o": _attend(t["q"], t, case)}
    _append(t, case)
    q = _rotate(t["q"].float(), t["positions"], case).to(t["q"].dtype)
    return {"o": _attend(q, t, case), "cache": t["cache"]}


# ---- the framework's operators --------------------------------------------------------------------
class _Memory:
    """A result's device memory, as torch can adopt it; holds the result."""

    def __init__(self, ctx, t):
        self.owner = t, ctx
        self.__cuda_array_interface__ = {"shape": t.shape, "typestr": {"f32": "<f4", "bf16": "<i2"}[t.dtype], "data": (ctx.device_ptr(t), False), "version": 2, "strides": None}


def _as_torch(ctx, t):
    v = torch.as_tensor(_Memory(ctx, t), device="cuda")
    return v.view(torch.bfloat16) if t.dtype == "bf16" else v


def _record(ctx, T, case, rotary):
    """Records a step's ops; what it leaves on the device, by name."""
    kind = case["kind"]
    if kind == "rope":
        out = {"y": ctx.rope(T["x"], T["positions"], rotary)}
        if case["grad"]:
            out["dx"] = ctx.rope_grad(T["dy"], T["positions"], rotary)
        return out
    if kind == "attention":
        return {"o": ctx.paged_attention(T["q"], T["cache"], T["lengths"], T["table"])}
    ctx.assign(T["cache"], ctx.cache_append(T["cache"], T["k"], T["v"], T["lengths"], T["table"], offsets=T.get("offsets"), rotary=rotary))
    if kind == "append":
        return {}
    return {"o": ctx.paged_attention(ctx.rope(T["q"], T["positions"], rotary), T["cache"], T["lengths"], T["table"])}


def prepare(case, seed):
    data = _inputs(case, seed)
    state = {"case": case, "data": data, "held": None}
    if own:
        from paper_2102_13267_amd import Context, Rotary
        # the workspace holds results and temporaries
        ctx = Context(device=torch.cuda.current_device(), workspace_bytes=(4 if case["kind"] == "rope" else 1) << 30)
        rotary = None
        if "dims" in case:
            rotary = Rotary(dims=case["dims"], base=BASE, interleaved=case["interleaved"], factor=case["factor"], original=case["original"], low=LOW, high=HIGH,
                            amplitude=case.get("amplitude", 1.0))
        state.update(ctx=ctx, rotary=rotary, tensors={k: ctx.tensor(v, donatable=k == "cache") for k, v in data.items()})
    return state


def run(state):
    case, data = state["case"], state["data"]
    if not own:
        return _plain(data, case)
    ctx = state["ctx"]
    results = _record(ctx, state["tensors"], case, state["rotary"])
    ctx.barrier(False)
    state["held"] = results          # (the last step's results make room when the next step's replace them)
    out = {k: _as_torch(ctx, t) for k, t in results.items()}
    if case["kind"] in ("append", "decode"):
        out["cache"] = data["cache"]
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    w, kind, d = _BYTES[case["dtype"]], case["kind"], case["head"]
    if kind == "rope":
        n, passes = case["batch"] * case["seq"] * case["heads"] * d, 2 if case["grad"] else 1
        return {"bytes": passes * 2 * w * n + 4 * case["seq"], "flops": passes * 3 * n}
    s, h = case["sequences"], case["kv_heads"]
    held = sum(_lengths(case)) * h * d                     # elements of all keys
    slots = 4 * sum(-(-n // case["page"]) for n in _lengths(case)) + 4 * s
    tokens = sum(_news(case)) if kind == "append" else s
    append = {"bytes": 4 * tokens * h * d * w, "flops": 3 * tokens * h * d}
    if kind == "append":
        return {"bytes": append["bytes"] + 8 * s + 4 * min(tokens, slots // 4), "flops": append["flops"]}
    attend = {"bytes": 2 * held * w + 2 * s * case["heads"] * d * w + slots, "flops": 4 * held * (case["heads"] // h)}
    if kind == "attention":
        return attend
    # the tokens' own rows are written once, and read as they are
    return {"bytes": attend["bytes"] + append["bytes"], "flops": attend["flops"] + append["flops"] + 3 * s * case["heads"] * d}


# ---- the same in 64 bits ------------------------------------------------------------------------
def _turn64(x, positions, case, back=False):
    """Rotation by complex factors."""
    half = case["dims"] // 2
    f = []
    for i in range(half):
        fi = BASE ** (-2.0 * i / case["dims"])
        g = 0.0 if not case["original"] else min(1.0, max(0.0, (case["original"] * fi / (2.0 * math.pi) - LOW) / (HIGH - LOW)))
        f.append(fi * (g + (1.0 - g) / case["factor"]))
    a = positions.double().unsqueeze(-1) * torch.tensor(f, dtype=torch.float64, device=x.device)
    turn = torch.polar(torch.full_like(a, case.get("amplitude", 1.0)), -a if back else a).unsqueeze(-2)
    y = x.clone()
    where = (slice(0, case["dims"], 2), slice(1, case["dims"], 2)) if case["interleaved"] else (slice(0, half), slice(half, case["dims"]))
    z = torch.complex(x[..., where[0]].contiguous(), x[..., where[1]].contiguous()) * turn
    y[..., where[0]], y[..., where[1]] = z.real, z.imag
    return y


def _append64(t, case, cache):
    lens, table, page = t["lengths"].tolist(), t["table"].long(), case["page"]
    offsets = t["offsets"].tolist() if "offsets" in t else list(range(len(lens) + 1))
    for s, n in enumerate(lens):
        rows = torch.arange(offsets[s], offsets[s + 1], device="cuda")
        pos = n - len(rows) + torch.arange(len(rows), device="cuda")
        at = table[s][pos // page]
        cache[at, 0, :, pos % page] = _turn64(t["k"][rows].double(), pos, case)
        cache[at, 1, :, pos % page] = t["v"][rows].double()


def _attend64(q, t, case, cache):
    out = torch.zeros_like(q)
    group = case["heads"] // case["kv_heads"]
    for s, n in enumerate(t["lengths"].tolist()):
        if not n:
            continue
        held = cache[t["table"][s, : -(-n // case["page"])].long()].double()               # [pages, 2, h, page, d]
        k, v = (x.transpose(0, 1).reshape(case["kv_heads"], -1, case["head"])[:, :n] for x in (held[:, 0], held[:, 1]))
        score = (q[s].reshape(case["kv_heads"], group, -1) @ k.transpose(1, 2).contiguous()) / math.sqrt(case["head"])
        out[s] = (torch.softmax(score, -1) @ v).reshape(case["heads"], -1)
    return out


def exact(case, seed):
    t, kind = _inputs(case, seed), case["kind"]
    if kind == "rope":
        out = {"y": _turn64(t["x"].double(), t["positions"], case)}
        if case["grad"]:
            out["dx"] = _turn64(t["dy"].double(), t["positions"], case, back=True)
        return out
    if kind == "attention":
        return {"o": _attend64(t["q"].double(), t, case, t["cache"])}
    cache = t["cache"].double()
    _append64(t, case, cache)
    if kind == "append":
        return {"cache": cache}
    # what is attended to is the keys as the cache holds them, and the query as it was rounded: those roundings are the type's own
    dt = t["cache"].dtype
    q = _turn64(t["q"].double(), t["positions"], case).to(dt).double()
    return {"o": _attend64(q, t, case, cache.to(dt)), "cache": cache}
