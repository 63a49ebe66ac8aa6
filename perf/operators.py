"""Appending to the paged KV cache and attention over it, as cases that can be timed and compared.

A case is a plain dict:

  op        "append"  kvh.append: keys (rotated) and values of new tokens go into the pages of the cache, queries are rotated on the way
            "attend"  kvh.attention: the queries of the new tokens over one layer of the cache
  store     "16" the cache holds the 16-bit type of the queries, "i8" int8 codes, "e4m3" 8-bit floats; the 8-bit caches have
            a scale per page and KV head, for K and V apart
  dt        "bf16" or "fp16": the type of queries, keys, values and outputs
  layers    append: layers written by one call; attend reads one layer of a cache of one
  heads, group, dim   KV heads, query heads per KV head, channels of a head
  page      tokens per page; pages are handed out in random order
  requests  requests of the batch
  ctx, new  tokens that a request has in the cache, and new tokens that the call brings
  mixed     the two are means of lognormal lengths (sigma 0.8, at most 8 times the mean) instead
  rot       append: channels of a head that are rotated, 0 for none; pairs: neighbours are rotated together, not halves
  sink, window   attend: a query sees the last `window` tokens and the first `sink` ones (0: all before it); causal or not
  lse       attend: the logarithms of the sums come back too

Heads of 128 channels, 8 KV heads, 32 layers, 256-token chunks, 16-token pages, contexts of 8192, 32768 and 131072 tokens and
lognormal lengths of mean 4096 are this repository's own configurations.
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
_TOP = {"i8": 127.0, "e4m3": 448.0}
_TEMPLATE = dict(op="", store="16", dt="bf16", layers=1, heads=8, group=4, dim=128, page=16, requests=1, ctx=0, new=1, mixed=False,
                 rot=0, pairs=False, sink=0, window=0, causal=True, lse=False)
WORKSPACE = 64 << 20  # bytes a serving program sets aside for the attention's partial results


def _case(**kw):
    return dict(_TEMPLATE, **kw)


def listed():
    return [
        # One request in the middle of its answer: the smallest calls there are, where latency counts.
        _case(name="append one token", op="append", ctx=299, rot=128),
        _case(name="attend one token, 300", op="attend", ctx=299),
        # A serving step of 64 requests, each with one new token, on a cache held in 8 bits.
        _case(name="append a step, int8", op="append", store="i8", requests=64, ctx=4096, mixed=True, rot=128),
        _case(name="attend a step, int8", op="attend", store="i8", requests=64, ctx=4096, mixed=True),
        # The same step on the 16-bit cache that stored entries are decoded into.
        _case(name="attend a step, bf16", op="attend", requests=64, ctx=4096, mixed=True),
        # One request with a very long context, and one that keeps its beginning and its end only.
        _case(name="attend one of 128K, e4m3", op="attend", store="e4m3", ctx=131072, lse=True),
        _case(name="attend kept tokens, fp16", op="attend", dt="fp16", requests=7, heads=5, group=7, dim=64, page=24, ctx=6001, new=5, mixed=True, sink=64, window=1000,
              lse=True),
        # A prompt of 8K tokens of the 8B-shaped model: its keys and values are stored, its queries see all before them.
        _case(name="append 8K prompt, e4m3", op="append", store="e4m3", new=8192, rot=128),
        _case(name="attend 8K prompt, bf16", op="attend", new=8192),
        # A cache hit of 32K tokens, and the 512 tokens of the question that follows it.
        _case(name="attend 512 after 32K, int8", op="attend", store="i8", ctx=32768, new=512),
        # All layers of a decoded 256-token chunk move into the 8-bit cache as they are.
        _case(name="append 32 layers, int8", op="append", store="i8", layers=32, new=256, group=0),
        # Prompts of mixed lengths of a model with narrow heads, half of each rotated in pairs, go into pages of odd size.
        _case(name="append prompts, fp16", op="append", dt="fp16", requests=16, heads=10, group=3, dim=64, page=20, ctx=100, new=1500, mixed=True, rot=32, pairs=True),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "attend", "attend"])
    store = rng.choice(["16", "i8", "e4m3"])
    dt = rng.choice(["bf16", "fp16"])
    dim = rng.choice([128, 128, 64])
    heads, group = rng.choice([(8, 4), (8, 4), (8, 8), (8, 1), (1, 8), (2, 4), (4, 7), (5, 3), (10, 2), (16, 1)])
    page = rng.choice([16, 16, 32, 64, 20, 24, 7])
    requests = spread(1, 64)
    mixed = rng.random() < 0.5
    case = _case(op=op, store=store, dt=dt, heads=heads, group=group, dim=dim, page=page, requests=requests, mixed=mixed)
    c = heads * dim
    if op == "append":
        case["rot"], case["pairs"] = rng.choice([0, dim, dim, dim // 2]), rng.random() < 0.3
        case["layers"] = rng.choice([1, 1, 1, spread(2, 32)])
        case["new"] = min(rng.choice([1, spread(1, 8192)]), max(1, (1 << 25) // (requests * case["layers"] * c * (1 + group))))
        case["ctx"] = min(spread(1, 4096) - 1, (1 << 28) // (requests * case["layers"] * c))
    else:
        case["new"] = rng.choice([1, 1, spread(1, 16), spread(16, 4096)])
        case["ctx"] = spread(1, 131072) - 1
        case["new"] = min(case["new"], max(1, 4096 // requests))
        pairs = (1 << (33 if mixed else 37)) // (requests * c * group)  # of new tokens and all tokens of a request
        case["new"] = min(case["new"], math.isqrt(pairs))
        case["ctx"] = min(case["ctx"], (1 << 28) // (requests * c), max(0, pairs // case["new"] - case["new"]))
        case["causal"] = rng.random() < 0.85
        if case["causal"] and rng.random() < 0.25:
            case["sink"], case["window"] = rng.choice([0, 4, 64]), spread(16, 8192)
        case["lse"] = rng.random() < 0.3
    return case


# ---- lengths: they are the case's, not the seed's ---------------------------------------------------------------
def _lengths(case):
    """(tokens in the cache with the new ones, new tokens) of each request."""
    b = case["requests"]
    g = np.random.default_rng([b, case["ctx"], case["new"]])

    def some(mean, least):
        if not case["mixed"] or mean <= least:
            return np.full(b, mean, dtype=np.int64)
        x = np.exp(g.normal(math.log(mean) - 0.32, 0.8, b))
        return np.clip(np.round(x).astype(np.int64), least, 8 * mean)

    new = some(case["new"], 1)
    return some(case["ctx"], 0) + new, new


def _seen(case, length, new):
    """Pairs of a query and a token that it sees, and tokens that some query sees, of one request."""
    p = np.arange(length - new, length, dtype=np.int64)
    end = p + 1 if case["causal"] else np.full(new, length, dtype=np.int64)
    if not case["window"]:
        return int(end.sum()), int(end.max())
    first = np.maximum(p - case["window"] + 1, 0)
    return int((end - first + np.minimum(first, case["sink"])).sum()), int(length - first[0] + min(first[0], case["sink"]))


def work(case):
    length, new = _lengths(case)
    c = case["heads"] * case["dim"]
    cq, width, t = c * case["group"], 2 if case["store"] == "16" else 1, int(new.sum())
    scales = 8 * case["heads"] if case["store"] != "16" else 0  # of K and V, a page
    if case["op"] == "append":
        pages = int(((length + case["page"] - 1) // case["page"] - (length - new) // case["page"]).sum())
        nbytes = case["layers"] * (t * 2 * c * (2 + width) + t * cq * 4 + pages * scales) + t * case["rot"] * 4
        turned = (c + cq) * case["rot"] // case["dim"]
        return {"bytes": nbytes, "flops": case["layers"] * t * (3 * turned + (4 * c if width == 1 else 0))}
    seen = [_seen(case, int(a), int(b)) for a, b in zip(length, new)]
    tokens = sum(s[1] for s in seen)
    nbytes = tokens * 2 * c * width + tokens * scales / case["page"] + t * cq * 4 + (t * cq // case["dim"] * 4 if case["lse"] else 0)
    return {"bytes": nbytes, "flops": 4.0 * sum(s[0] for s in seen) * cq}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _pool(g, shape, case):
    """Pages as they are after earlier steps: codes or values, and scales that differ from page to page and head to head."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float16 if case["store"] != "16" else _DT[case["dt"]])
    ch = torch.exp(0.5 * torch.randn(shape[-1], generator=g, device="cuda"))
    if case["store"] == "16":
        return x.mul_(ch), None
    scale = torch.exp(0.3 * torch.randn((shape[0], shape[1], case["heads"]), generator=g, device="cuda"))
    if case["store"] == "i8":
        return x.mul_(32 * ch.clamp(max=2.5)).round_().clamp_(-127, 127).to(torch.int8), scale / 32
    return x.mul_(100 * ch.clamp(max=2.5)).clamp_(-448, 448).to(torch.float8_e4m3fn), scale / 100


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    length, new = _lengths(case)
    b, c, t = case["requests"], case["heads"] * case["dim"], int(new.sum())
    cq, page, dt = c * case["group"], case["page"], _DT[case["dt"]]
    held = -(-length // page)
    order = torch.randperm(int(held.sum()) + 8, generator=g, device="cuda").to(torch.int32)
    table = torch.full((b, int(held.max())), -1, dtype=torch.int32, device="cuda")
    first = np.concatenate([[0], np.cumsum(held)])
    for i in range(b):
        table[i, :int(held[i])] = order[int(first[i]):int(first[i + 1])]
    shape = (case["layers"], len(order), page, c)
    k_cache, k_scale = _pool(g, shape, case)
    v_cache, v_scale = _pool(g, shape, case)
    s = dict(case=case, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale, page_table=table, max_new=int(new.max()),
             starts=torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda(),
             lens=torch.from_numpy(length.astype(np.int32)).cuda())
    if case["op"] == "append":
        def rows(channels):
            ch = torch.exp(0.5 * torch.randn(channels, generator=g, device="cuda"))
            return (torch.randn((case["layers"], t, channels), generator=g, device="cuda") * ch).to(dt)

        s["k"], s["v"] = rows(c), rows(c)
        s["q"] = rows(cq) if cq else None
        s["q_out"] = torch.empty_like(s["q"]) if cq else None
        s["rotation"] = None
        if case["rot"]:
            half = case["rot"] // 2
            at = torch.arange(int(length.max()), device="cuda", dtype=torch.float64)[:, None]
            at = at * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
            s["rotation"] = torch.cat([torch.cos(at), torch.sin(at)], 1).float()
    else:
        s["q"] = torch.randn((t, cq), generator=g, device="cuda").to(dt)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((t, cq // case["dim"]), dtype=torch.float32, device="cuda") if case["lse"] else None
        s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


def run(s):
    return (_append if s["case"]["op"] == "append" else _attend)(s)


# ---- the operators: the framework's calls, and their plain forms ----------------------------------------------------
def _tokens(s):
    """Request and index in it of each packed row."""
    row = torch.arange(s["k"].shape[1] if "k" in s else s["q"].shape[0], device="cuda")
    b = torch.searchsorted(s["starts"][1:].contiguous(), row, right=True)
    return b, row - s["starts"].long()[b]


def _append(s):
    case = s["case"]
    if own:
        import paper_2509_00105_amd as kvh

        kvh.append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["starts"], s["lens"], s["page_table"], s["max_new"], head_dim=case["dim"],
                   k_scale=s["k_scale"], v_scale=s["v_scale"], q=s["q"], q_out=s["q_out"], rotation=s["rotation"], pairs=case["pairs"])
    else:
        page, dim, heads = case["page"], case["dim"], case["heads"]
        b, i = _tokens(s)
        starts, lens, table = s["starts"].long(), s["lens"].long(), s["page_table"].long()
        before = lens - (starts[1:] - starts[:-1])
        slot = before[b] + i
        at, row = table[b, slot // page], slot % page

        def turned(x):
            x = x.float().unflatten(-1, (-1, dim))
            rot = case["rot"]
            if not rot:
                return x
            cos, sin = s["rotation"][slot][:, None].split(rot // 2, -1)
            y = x[..., :rot].unflatten(-1, (rot // 2, 2) if case["pairs"] else (2, rot // 2))
            x1, x2 = y.unbind(-1 if case["pairs"] else -2)
            y = torch.stack((x1 * cos - x2 * sin, x2 * cos + x1 * sin), -1 if case["pairs"] else -2).flatten(-2)
            return torch.cat((y, x[..., rot:]), -1)

        def put(x, cache, scale):
            if scale is None:
                cache[:, at, row] = x.flatten(-2).to(cache.dtype)
                return
            top, layers = _TOP[case["store"]], x.shape[0]
            most = torch.zeros_like(scale).index_reduce_(1, at, x.abs().amax(-1), "amax")
            now = torch.where(most < 2.0 ** -100, 0.0, most / top)
            old, held = table[torch.arange(len(before), device="cuda"), before // page], before % page  # the page that a request's tokens begin in
            had = torch.where(held[:, None] > 0, scale[:, old], 0.0)
            now[:, old] = torch.maximum(now[:, old], had)
            rate = torch.where((now[:, old] > had) & (had > 0), had / now[:, old], 1.0)
            codes = cache[:, old].float().unflatten(-1, (heads, dim)) * rate[:, :, None, :, None]
            codes = codes.round().to(torch.int8) if case["store"] == "i8" else codes.to(cache.dtype)
            kept = (torch.arange(page, device="cuda") < held[:, None])[None, :, :, None]
            raw = cache.view(torch.int8)
            raw[:, old] = torch.where(kept, codes.view(torch.int8).flatten(-2), raw[:, old])
            inv = torch.where(now > 0, 1.0 / now, 0.0)[:, at]
            codes = x * inv[..., None]
            codes = codes.round().to(torch.int8) if case["store"] == "i8" else codes.to(cache.dtype)
            raw[:, at, row] = codes.view(torch.int8).reshape(layers, -1, heads * dim)
            scale[:, at] = now[:, at]

        put(turned(s["k"]), s["k_cache"], s["k_scale"])
        put(s["v"].float().unflatten(-1, (-1, dim)), s["v_cache"], s["v_scale"])
        if s["q"] is not None:
            s["q_out"].copy_(turned(s["q"]).flatten(-2))
    return {n: s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale", "q_out") if s[n] is not None}


def _attend(s):
    case = s["case"]
    if own:
        import paper_2509_00105_amd as kvh

        kvh.attention(s["q"], s["k_cache"], s["v_cache"], 0, s["starts"], s["lens"], s["page_table"], s["max_new"], head_dim=case["dim"],
                      k_scale=s["k_scale"], v_scale=s["v_scale"], causal=case["causal"], sink=case["sink"], window=case["window"], out=s["out"],
                      lse=s["lse"], workspace=s["workspace"])
        return {"out": s["out"], "lse": s["lse"]} if case["lse"] else {"out": s["out"]}
    heads, group, dim, page, most = case["heads"], case["group"], case["dim"], case["page"], s["max_new"]
    starts, lens, table = s["starts"].long(), s["lens"].long(), s["page_table"].long()
    new = starts[1:] - starts[:-1]
    b, j = len(lens), torch.arange(table.shape[1] * page, device="cuda")

    def rows(cache, scale):  # [request][token][head][channel]
        x = cache[0][table].float().unflatten(-1, (heads, dim))
        return (x if scale is None else x * scale[0][table][:, :, None, :, None]).flatten(1, 2)

    i = torch.arange(most, device="cuda")
    q = s["q"][(starts[:-1, None] + i).clamp(max=len(s["q"]) - 1)].float().view(b, most, heads, group, dim)
    q = q.permute(0, 2, 1, 3, 4).reshape(b, heads, most * group, dim)
    w = torch.matmul(q, rows(s["k_cache"], s["k_scale"]).permute(0, 2, 3, 1).contiguous()).mul_(dim ** -0.5).view(b, heads, most, group, -1)
    p = (lens - new)[:, None, None] + i[:, None]
    see = (j < lens[:, None, None]).expand(b, most, len(j))
    if case["causal"]:
        see = see & (j <= p)
    if case["window"]:
        see = see & ((j > p - case["window"]) | (j < case["sink"]))
    see = see[:, None, :, None]
    top = w.masked_fill_(~see, -math.inf).amax(-1, keepdim=True)
    top = torch.where(see.any(-1, keepdim=True), top, 0.0)
    w = w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    v = rows(s["v_cache"], s["v_scale"]).masked_fill_((j >= lens[:, None])[:, :, None, None], 0.0)
    o = torch.matmul(w.view(b, heads, most * group, -1), v.transpose(1, 2).contiguous()).view(b, heads, most, group, dim) / total
    o = torch.where(see.any(-1, keepdim=True), o, 0.0)
    request, index = _tokens(s)
    out = {"out": o.permute(0, 2, 1, 3, 4)[request, index].reshape(len(s["q"]), -1).to(s["q"].dtype)}
    if case["lse"]:
        out["lse"] = (top + total.log())[..., 0].permute(0, 2, 1, 3)[request, index].reshape(len(s["q"]), -1)
    return out


# ---- the definition in 64 bits, request by request ----------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    length, new = _lengths(case)
    page, dim, heads, group = case["page"], case["dim"], case["heads"], case["group"]
    table, starts = s["page_table"].long(), np.concatenate([[0], np.cumsum(new)])
    if case["op"] == "append":
        got = {n: s[n].double() if s[n] is not None else None for n in ("k_scale", "v_scale")}
        got["k_cache"], got["v_cache"] = (s["k_cache"].double(), s["v_cache"].double()) if case["store"] == "16" else (None, None)
        got["q_out"] = s["q"].double() if s["q"] is not None else None
        if got["q_out"] is None:
            del got["q_out"]
        if case["store"] == "16":
            del got["k_scale"], got["v_scale"]

        def turn(x, p):
            x, half = x.double().reshape(x.shape[0], x.shape[1], -1, dim).clone(), case["rot"] // 2
            for d in range(half):
                lo, hi = (2 * d, 2 * d + 1) if case["pairs"] else (d, d + half)
                cos, sin = s["rotation"][p, d].double()[:, None], s["rotation"][p, d + half].double()[:, None]
                x[..., lo], x[..., hi] = x[..., lo] * cos - x[..., hi] * sin, x[..., hi] * cos + x[..., lo] * sin
            return x

        for r in range(case["requests"]):
            a, e = int(starts[r]), int(starts[r + 1])
            p = torch.arange(int(length[r] - new[r]), int(length[r]), device="cuda")
            at, row = table[r, p // page], p % page
            for x, n in ((turn(s["k"][:, a:e], p), "k"), (s["v"][:, a:e].double().unflatten(-1, (heads, dim)), "v")):
                if case["store"] == "16":
                    got[n + "_cache"][:, at, row] = x.flatten(-2)
                    continue
                for first in range(int(p[0]) // page, int(p[-1]) // page + 1):
                    mine = x[:, (p // page) == first].abs().amax((1, 3)) / _TOP[case["store"]]
                    where = int(table[r, first])
                    held = int(p[0]) > first * page
                    got[n + "_scale"][:, where] = torch.maximum(mine, got[n + "_scale"][:, where]) if held else mine
            if s["q"] is not None:
                got["q_out"][:, a:e] = turn(s["q"][:, a:e], p).flatten(-2)
        return got
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((len(s["q"]), heads * group), -math.inf, dtype=torch.float64, device="cuda")
    for r in range(case["requests"]):
        n, begin = int(length[r]), int(starts[r])
        j = torch.arange(n, device="cuda")
        for h in range(heads):
            def column(cache, scale):
                x = cache[0, :, :, h * dim:(h + 1) * dim][table[r, :-(-n // page)]].double()
                return (x if scale is None else x * scale[0, table[r, :-(-n // page)], h].double()[:, None, None]).flatten(0, 1)[:n]

            k, v = column(s["k_cache"], s["k_scale"]), column(s["v_cache"], s["v_scale"])
            for i0 in range(0, int(new[r]), 1024):
                i = torch.arange(i0, min(i0 + 1024, int(new[r])), device="cuda")
                p = (n - int(new[r]) + i)[:, None]
                hidden = (j > p) if case["causal"] else torch.zeros((len(i), n), dtype=torch.bool, device="cuda")
                if case["window"]:
                    hidden = hidden | ((j <= p - case["window"]) & (j >= case["sink"]))
                for u in range(h * group, (h + 1) * group):
                    x = (s["q"][begin + i, u * dim:(u + 1) * dim].double() @ k.T * dim ** -0.5).masked_fill(hidden, -math.inf)
                    lse[begin + i, u] = torch.logsumexp(x, -1)
                    out[begin + i, u * dim:(u + 1) * dim] = torch.softmax(x, -1) @ v
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
