"""Attention over selected pages of the paged KV cache, and copying, forking and compacting its pages, as cases that can be timed and compared.

A case is a plain dict:

  op        "bound"    kvh.bound_keys: lowest and highest key of each channel, page by page, of the pages that new tokens lie on
            "select"   kvh.select_pages: the pages that each new token and KV head shall read, by a score from those bounds
            "attend"   kvh.attention_pages: the queries of the new tokens over the pages chosen for them
            "copy"     kvh.copy_pages: pages of all layers to other pages
            "fork"     kvh.fork: rows of the page table become children of rows and grow; full pages are shared, an unfilled one is copied
            "compact"  kvh.compact: the pages in use move to the lowest numbers
  store     "16" the cache holds the 16-bit type of the queries, "i8" int8 codes, "e4m3" 8-bit floats; the 8-bit caches have
            a scale per page and KV head, for K and V apart
  dt        "bf16" or "fp16": the type of queries, keys, values and outputs
  layers    of the cache; select and attend work on one
  heads, group, dim   KV heads, query heads per KV head, channels of a head
  page      tokens per page; pages are handed out in random order
  requests  requests of the batch, rows of the page table
  ctx, new  tokens that a request has in the cache, and new tokens that the call brings (fork: by which a row grows)
  mixed     the two are means of lognormal lengths (sigma 0.8, at most 8 times the mean) instead
  count, first, last   pages that a token and head read, and how many of them are the request's first ones and its last ones
  lse       attend: the logarithms of the sums come back too
  beams     fork: groups of that many rows, which have `shared` tokens of their beginning in common, choose their parents among themselves
  ends      fork: every so many rows end, and a new request of `ctx` tokens takes their place (0: none does)
  pages     copy: pages copied by the call; compact: pages of the cache, of which the requests' are in use
  bounds    copy, fork, compact: the bounds of the keys go along

Heads of 128 channels, 8 KV heads, 32 layers, 256-token chunks, 16-token pages, contexts of 8192, 32768 and 131072 tokens and
lognormal lengths of mean 4096 are this repository's own configurations.
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
_TEMPLATE = dict(op="", store="16", dt="bf16", layers=1, heads=8, group=4, dim=128, page=16, requests=1, ctx=0, new=1, mixed=False,
                 count=64, first=1, last=2, lse=False, beams=1, shared=0, ends=0, pages=0, bounds=False)
WORKSPACE = 64 << 20  # bytes a serving program sets aside for partial results, scores and lists


def _case(**kw):
    return dict(_TEMPLATE, **kw)


def listed():
    return [
        # A serving step of 64 requests: each has one new key, whose page gets new bounds.
        _case(name="bound a step, bf16", op="bound", requests=64, ctx=4096, mixed=True),
        # A cache hit: all layers of a decoded 8K entry, moved into the 8-bit cache, get their bounds at once.
        _case(name="bound 32 layers of 8K, int8", op="bound", store="i8", layers=32, new=8192),
        # The pages that the next token of a request with a very long context reads: 4096 tokens of 131072.
        _case(name="select one of 128K", op="select", ctx=131072, count=256),
        # A step of 64 requests, each head with 1024 tokens of its own.
        _case(name="select a step", op="select", requests=64, ctx=4096, mixed=True),
        # The same step's attention on the 16-bit cache that stored entries are decoded into.
        _case(name="attend a step, bf16", op="attend", requests=64, ctx=4096, mixed=True),
        # A cache hit of 32K tokens, and the 512 tokens of the question that follows it.
        _case(name="attend 512 after 32K, int8", op="attend", store="i8", ctx=32768, new=512, lse=True),
        # One request's last pages go to three rows beside it: the smallest copy there is in a program with all layers in one cache.
        _case(name="copy 3 pages of 32 layers, int8", op="copy", store="i8", layers=32, pages=3, requests=4, ctx=500, bounds=True),
        # A cached prefix is duplicated, so that the copy can be changed: 8K tokens.
        _case(name="copy 8K tokens, bf16", op="copy", layers=8, pages=512, ctx=8192),
        # A step's growth: 64 rows, most of which need no page.
        _case(name="fork: a step grows, int8", op="fork", store="i8", heads=2, requests=64, ctx=4096, mixed=True, bounds=True),
        # 16 requests of 4 beams each reorder them; some requests end and others begin.  Pages and heads of other sizes.
        _case(name="fork: 16 of 4 beams, fp16", op="fork", dt="fp16", layers=8, heads=5, group=7, dim=64, page=24, requests=64, ctx=611, mixed=True, beams=4,
              shared=500, ends=9),
        # Half the requests have gone: the rest moves together, one layer of a tensor-parallel share.
        _case(name="compact a share, e4m3", op="compact", store="e4m3", heads=2, requests=8, ctx=1000, mixed=True, pages=1024),
        # The same with 8 layers and bounds.
        _case(name="compact 8 layers, bf16", op="compact", layers=8, requests=16, ctx=900, mixed=True, pages=1800, bounds=True),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["bound", "select", "attend", "attend", "copy", "fork", "compact"])
    store = rng.choice(["16", "i8", "e4m3"])
    dt = rng.choice(["bf16", "fp16"])
    dim = rng.choice([128, 128, 64])
    heads, group = rng.choice([(8, 4), (8, 4), (8, 8), (8, 1), (1, 8), (2, 4), (4, 7), (5, 3), (10, 2), (2, 20)])
    page = rng.choice([16, 16, 32, 64, 20, 24, 7])
    case = _case(op=op, store=store, dt=dt, heads=heads, group=group, dim=dim, page=page, mixed=rng.random() < 0.5)
    c = heads * dim
    if op in ("bound", "select", "attend"):
        case["requests"] = spread(1, 64)
        case["new"] = rng.choice([1, 1, spread(1, 16), spread(16, 512)])
        case["ctx"] = min(spread(1, 131072) - 1, (1 << 27) // (case["requests"] * c))
        case["first"], case["last"] = rng.choice([0, 1, 1, 4]), rng.choice([1, 2, 4, 8])
        case["count"] = case["first"] + case["last"] + spread(1, 256)
        if op == "bound":
            case["layers"] = rng.choice([1, 1, spread(2, 32)])
            case["new"] = rng.choice([1, spread(1, 8192)])
            room = (1 << 27) // (case["requests"] * case["layers"] * c)
            case["new"], case["ctx"] = min(case["new"], max(1, room // 2)), min(case["ctx"], room // 2)
            return case
        case["new"] = min(case["new"], max(1, 512 // case["requests"]))
        while _size(case)[0] > 1 << 25:  # scores
            case["ctx"], case["new"] = case["ctx"] // 2, -(-case["new"] // 2)
        if op == "attend":
            case["lse"] = rng.random() < 0.3
            while _size(case)[1] > 1 << 29 and case["count"] > case["first"] + case["last"]:  # channels that are read
                case["count"] -= 1
        return case
    case["bounds"] = rng.random() < 0.5
    case["requests"] = spread(1, 64)
    case["layers"] = rng.choice([1, 1, spread(2, 32)])
    room = (1 << 27) // (case["layers"] * c)  # tokens that the cache may hold
    case["requests"] = min(case["requests"], max(1, room // (8 * page)))
    if op == "fork":
        case["beams"] = rng.choice([1, 1, 2, 4, 8])
        case["ends"] = rng.choice([0, 0, 3, 8])
        case["new"] = rng.choice([1, 1, spread(1, 256)])
    case["ctx"] = min(spread(1, 4096), max(1, room // (6 * case["requests"]) - case["new"]))
    if op == "fork" and case["beams"] > 1:
        case["shared"] = rng.randrange(case["ctx"] + 1)
    if op == "copy":
        case["pages"] = max(1, min(spread(1, 512), room // (4 * page)))
    if op == "compact":
        case["pages"] = spread(1, 4) * case["requests"] * -(-case["ctx"] // page)
    return case


def _size(case):
    length, new = _lengths(case)
    rows = case["requests"] * int(new.max()) * case["heads"] * case["group"]
    return rows * -(-int(length.max()) // case["page"]), int(new.sum()) * case["count"] * case["page"] * case["heads"] * case["dim"]


# ---- lengths, tables and parents: they are the case's, not the seed's -----------------------------------------------
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


def _rows(case):
    """fork: (tokens of each row, its group's shared beginning, its parent, tokens it grows by)."""
    b, w = case["requests"], case["beams"]
    g = np.random.default_rng([b, w, case["ctx"]])
    total, new = _lengths(case)
    length = total - new
    group = np.arange(b) // w
    if w > 1:  # the beams of a request have the same length
        length = np.maximum(length[group * w], case["shared"])
    parent = np.minimum(group * w + g.integers(0, w, b), b - 1)
    if case["ends"]:
        over = np.arange(b) % case["ends"] == case["ends"] - 1
        parent, new = np.where(over, -1, parent), np.where(over, case["ctx"], new)
    return length, parent, new


def _held(case):
    """Pages of each request, and pages of the cache."""
    page = case["page"]
    if case["op"] == "fork":
        length, _, new = _rows(case)
        held = -(-length // page)
        spare = int((-(-new // page) + 1).sum())
        return held, int(held.sum()) + spare + 8
    length, _ = _lengths(case)
    held = -(-length // page)
    if case["op"] == "compact":
        return held, max(case["pages"], int(held.sum()))
    return held, int(held.sum()) + case["pages"] + 8


def _page_bytes(case):
    """Of one page: K and V of all layers, scales, bounds."""
    width = 2 if case["store"] == "16" else 1
    n = 2 * case["page"] * case["heads"] * case["dim"] * width + (8 * case["heads"] if width == 1 else 0)
    return case["layers"] * (n + (case["heads"] * (2 * case["dim"] + 4) if case["bounds"] else 0))


def _listed_pages(case):
    """select, attend: candidates of each new token, and tokens that it reads of those chosen."""
    length, new = _lengths(case)
    page = case["page"]
    p = np.concatenate([np.arange(a - n, a, dtype=np.int64) for a, n in zip(length, new)])
    candidates = p // page + 1
    return candidates, (np.minimum(candidates, case["count"]) - 1) * page + p % page + 1


def work(case):
    heads, dim, group, page = case["heads"], case["dim"], case["group"], case["page"]
    c, width = heads * dim, 2 if case["store"] == "16" else 1
    if case["op"] == "bound":
        length, new = _lengths(case)
        first = (length - new) // page
        pages = int((-(-length // page) - first).sum())
        tokens = int((length - first * page).sum())
        scales = 0 if width == 2 else 4 * heads
        return {"bytes": case["layers"] * (tokens * c * width + pages * (2 * c + 4 * heads + scales)), "flops": case["layers"] * (3 * tokens * c + 4 * pages * c)}
    if case["op"] == "select":
        length, new = _lengths(case)
        candidates, _ = _listed_pages(case)
        t = int(new.sum())
        return {"bytes": int((-(-length // page)).sum()) * heads * (2 * dim + 4) + t * heads * (2 * group * dim + 4 * case["count"]),
                "flops": 2.0 * dim * int(candidates.sum()) * heads * group}
    if case["op"] == "attend":
        length, new = _lengths(case)
        _, tokens = _listed_pages(case)
        t, read = int(new.sum()), int(tokens.sum())
        # a page that several tokens of a request read is wanted once
        once = sum(int(min(a, tokens[int(e) - int(n):int(e)].sum())) for a, n, e in zip(length, new, np.cumsum(new)))
        return {"bytes": once * c * 2 * width + t * heads * (4 * group * dim + 4 * case["count"] + (4 * group if case["lse"] else 0)),
                "flops": 4.0 * read * c * group}
    if case["op"] == "copy":
        return {"bytes": case["pages"] * (2 * _page_bytes(case) + 8), "flops": 0}
    held, pages = _held(case)
    if case["op"] == "fork":
        length, parent, new = _rows(case)
        old = np.where(parent < 0, 0, length[parent])
        first = np.array([parent[b] >= 0 and not (parent[:b] == parent[b]).any() for b in range(len(parent))])
        copies = int(((old % page != 0) & ~first).sum())
        after = int((-(-(old + new) // page)).sum())
        return {"bytes": 4 * (int(held.sum()) + after + 2 * pages + 5 * len(parent)) + copies * 2 * _page_bytes(case), "flops": 0}
    used = int(held.sum())
    moved = used * (pages - used) // pages  # of pages in random order
    return {"bytes": 4 * (2 * used + 3 * pages + len(held)) + moved * 2 * _page_bytes(case), "flops": 0}


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


def _some_bounds(g, case, pages):
    """Bounds of keys whose channels differ in their middle and in how far they reach."""
    shape = (case["layers"], pages, case["heads"], 1, case["dim"])
    middle = 24 * torch.randn(shape, generator=g, device="cuda")
    reach = 30 + 12 * torch.randn(shape, generator=g, device="cuda").abs()
    codes = torch.cat([(middle - reach).floor(), (middle + reach).ceil()], 3).clamp_(-127, 127).to(torch.int8)
    return codes, torch.exp(0.3 * torch.randn(shape[:3], generator=g, device="cuda")) / 32


def _some_pages(g, case, candidates):
    """[T][heads][count]: the first and last pages of each token and others of its request at random, ascending; -1 past the last."""
    n = torch.from_numpy(candidates).cuda()[:, None, None]
    most = int(candidates.max())
    j = torch.arange(most, device="cuda")
    key = torch.rand((len(candidates), case["heads"], most), generator=g, device="cuda")
    key = torch.where((j < case["first"]) | (j >= n - case["last"]), 2.0, key).masked_fill_(j >= n, -1.0)
    top = key.topk(min(case["count"], most), -1)
    at = torch.where(top.values >= 0, top.indices, most).sort(-1).values
    at = torch.where(at < most, at, -1).to(torch.int32)
    return torch.nn.functional.pad(at, (0, case["count"] - at.shape[-1]), value=-1).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, b, page, dt = case["op"], case["requests"], case["page"], _DT[case["dt"]]
    heads, dim = case["heads"], case["dim"]
    held, pages = _held(case)
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    length, new = _rows(case)[::2] if op == "fork" else _lengths(case)
    columns = int((held if op != "fork" else -(-(length.max() + new.max() + case["ctx"]) // page)).max())
    if op == "fork":  # a group's rows have their full shared pages in common
        table = np.full((b, columns), -1, dtype=np.int32)
        at, o = 0, order.cpu().numpy()
        for i in range(b):
            lead, mine = i - i % case["beams"], case["shared"] // page if i % case["beams"] else 0
            table[i, :mine] = table[lead, :mine]
            table[i, mine:held[i]] = o[at:at + held[i] - mine]
            at += int(held[i]) - mine
        table = torch.from_numpy(table).cuda()
    else:
        first = torch.from_numpy(np.concatenate([[0], np.cumsum(held)])).cuda()
        j = torch.arange(columns, device="cuda")
        table = torch.where(j < (first[1:] - first[:-1])[:, None], order[(first[:-1, None] + j).clamp_(max=pages - 1)], -1).to(torch.int32)
    s = dict(case=case, page_table=table, lens=torch.from_numpy(length.astype(np.int32)).cuda(), max_new=int(new.max()),
             starts=torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda(), workspace=torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda"))
    t, cq = int(new.sum()), heads * case["group"] * dim
    shape = (case["layers"], pages, page, heads * dim)
    s["k_scale"] = s["v_scale"] = s["bounds"] = s["bound_scale"] = None
    if op != "select":
        s["k_cache"], s["k_scale"] = _pool(g, shape, case)
        if op != "bound":
            s["v_cache"], s["v_scale"] = _pool(g, shape, case)
    if op == "bound":
        s["bounds"] = torch.zeros((case["layers"], pages, heads, 2, dim), dtype=torch.int8, device="cuda")
        s["bound_scale"] = torch.zeros((case["layers"], pages, heads), device="cuda")
    elif op == "select" or case["bounds"]:
        s["bounds"], s["bound_scale"] = _some_bounds(g, case, pages)
    if op in ("select", "attend"):
        s["q"] = torch.randn((t, cq), generator=g, device="cuda").to(dt)
        s["chosen"] = torch.empty((t, heads, case["count"]), dtype=torch.int32, device="cuda")
    if op == "attend":
        s["chosen"] = _some_pages(g, case, _listed_pages(case)[0])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((t, cq // dim), dtype=torch.float32, device="cuda") if case["lse"] else None
    if op == "copy":
        used = int(held.sum())
        n = case["pages"]
        s["src"] = order[torch.randperm(used, generator=g, device="cuda")[:n]].contiguous() if n <= used else order[torch.arange(n, device="cuda") % used].contiguous()
        s["dst"] = order[used:used + n].contiguous()
    if op in ("fork", "compact"):
        live = table[table >= 0].long()
        s["refs"] = torch.zeros(pages, dtype=torch.int32, device="cuda").index_add_(0, live, torch.ones_like(live, dtype=torch.int32))
        s["table_out"], s["refs_out"] = torch.empty_like(table), torch.empty_like(s["refs"])
    if op == "fork":
        length, parent, new = _rows(case)
        s["parents"], s["grow"] = (torch.from_numpy(x.astype(np.int32)).cuda() for x in (parent, new))
        s["lens_out"] = torch.empty_like(s["lens"])
    if op == "compact":
        s["moved"] = torch.empty_like(s["refs"])
    return s


def run(s):
    return {"bound": _bound, "select": _select, "attend": _attend, "copy": _copy, "fork": _fork, "compact": _compact}[s["case"]["op"]](s)


def _kept(s, *names):
    """Of the state's buffers, those there are."""
    return {n: s[n] for n in names if s.get(n) is not None}


# ---- the operators: the framework's calls, and their plain forms ----------------------------------------------------
def _bound(s):
    case = s["case"]
    if own:
        import paper_2509_00105_amd as kvh

        kvh.bound_keys(s["k_cache"], s["bounds"], s["bound_scale"], s["starts"], s["lens"], s["page_table"], s["max_new"], k_scale=s["k_scale"])
    else:
        page, heads, dim = case["page"], case["heads"], case["dim"]
        lens, starts, table = s["lens"].long(), s["starts"].long(), s["page_table"].long()
        new = starts[1:] - starts[:-1]
        j = ((lens - new) // page)[:, None] + torch.arange((s["max_new"] + page - 2) // page + 1, device="cuda")
        b, i = torch.nonzero(j * page < lens[:, None], as_tuple=True)
        at, here = table[b, j[b, i]], lens[b] - j[b, i] * page  # pages, and tokens on them
        x = s["k_cache"][:, at].float().unflatten(-1, (heads, dim))
        absent = (torch.arange(page, device="cuda") >= here[:, None])[None, :, :, None, None]
        lo, hi = x.masked_fill(absent, math.inf).amin(2), x.masked_fill(absent, -math.inf).amax(2)
        most = torch.maximum(lo.abs(), hi.abs()).amax(-1)
        none = most < 2.0 ** -100
        by = torch.where(none, 1.0, most)[..., None]
        codes = torch.stack([(127 * lo / by).floor(), (127 * hi / by).ceil()], -2)
        s["bounds"][:, at] = codes.masked_fill(none[..., None, None], 0.0).to(torch.int8)
        scale = torch.where(none, 0.0, most / 127)
        s["bound_scale"][:, at] = scale if s["k_scale"] is None else scale * s["k_scale"][:, at]
    return _kept(s, "bounds", "bound_scale")


def _tokens(s):
    """Request and logical position of each packed row."""
    row = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(s["starts"][1:].contiguous(), row, right=True)
    return b, s["lens"].long()[b] - s["starts"].long()[b + 1] + row


def _select(s):
    case = s["case"]
    if own:
        import paper_2509_00105_amd as kvh

        return {"chosen": kvh.select_pages(s["q"], s["bounds"], s["bound_scale"], 0, s["starts"], s["lens"], s["page_table"], s["max_new"], case["count"],
                                           block_tokens=case["page"], first=case["first"], last=case["last"], out=s["chosen"], workspace=s["workspace"])}
    heads, group, dim, page, most = case["heads"], case["group"], case["dim"], case["page"], s["max_new"]
    starts, lens, table = s["starts"].long(), s["lens"].long(), s["page_table"].long()
    n, columns = len(lens), table.shape[1]
    q = s["q"][(starts[:-1, None] + torch.arange(most, device="cuda")).clamp(max=len(s["q"]) - 1)].float().view(n, most, heads, group, dim)
    top = q.abs().amax(-1, keepdim=True)
    codes = torch.where(top > 0, 127 * q / torch.where(top > 0, top, 1.0), 0.0).round()
    both = torch.cat([codes.clamp(max=0), codes.clamp(min=0)], -1).permute(0, 2, 1, 3, 4).reshape(n, heads, most * group, 2 * dim).contiguous()
    bounds = s["bounds"][0][table.clamp(min=0)].float().flatten(3).permute(0, 2, 3, 1).contiguous()  # [request][head][lowest, highest][page]
    score = torch.matmul(both, bounds).view(n, heads, most, group, columns)  # whole numbers below 2^24: the same in any order
    score = (score * top.permute(0, 2, 1, 3, 4)).amax(3) * s["bound_scale"][0][table.clamp(min=0)].permute(0, 2, 1)[:, :, None]
    b, p = _tokens(s)
    score = score.permute(0, 2, 1, 3)[b, torch.arange(len(b), device="cuda") - starts[b]]
    j, end = torch.arange(columns, device="cuda"), (p // page + 1)[:, None, None]
    score = torch.where((j < case["first"]) | (j >= end - case["last"]), math.inf, score).masked_fill(j >= end, -math.inf)
    at = score.sort(dim=-1, descending=True, stable=True).indices[..., :case["count"]]
    at = torch.where(at < end, at, columns).sort(-1).values
    at = torch.where(at < columns, at, -1).to(torch.int32)
    return {"chosen": torch.nn.functional.pad(at, (0, case["count"] - at.shape[-1]), value=-1)}


def _attend(s):
    case = s["case"]
    if own:
        import paper_2509_00105_amd as kvh

        kvh.attention_pages(s["q"], s["k_cache"], s["v_cache"], 0, s["chosen"], s["starts"], s["lens"], s["page_table"], s["max_new"], head_dim=case["dim"],
                            k_scale=s["k_scale"], v_scale=s["v_scale"], out=s["out"], lse=s["lse"], workspace=s["workspace"])
        return _kept(s, "out", "lse")
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    b, p = _tokens(s)
    t, listed = len(b), s["chosen"].long()
    at = s["page_table"].long()[b[:, None, None], listed.clamp(min=0)]
    head = torch.arange(heads, device="cuda")[:, None]

    def rows(cache, scale):  # [token][head][listed token][channel]
        x = cache[0].unflatten(-1, (heads, dim)).transpose(1, 2)[at, head].float()
        return (x if scale is None else x * scale[0][at, head][..., None, None]).flatten(2, 3)

    seen = (listed >= 0)[..., None] & (listed[..., None] * page + torch.arange(page, device="cuda") <= p[:, None, None, None])
    seen = seen.flatten(2)[:, :, None]
    q = s["q"].float().view(t, heads, group, dim)
    w = torch.matmul(rows(s["k_cache"], s["k_scale"]), q.transpose(2, 3).contiguous()).transpose(2, 3) * dim ** -0.5
    w = w.masked_fill(~seen, -math.inf)
    top = w.amax(-1, keepdim=True)
    w = (w - top).exp()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.contiguous(), rows(s["v_cache"], s["v_scale"]).masked_fill(~seen.transpose(2, 3), 0.0)) / total
    out = {"out": o.reshape(t, -1).to(s["q"].dtype)}
    if case["lse"]:
        out["lse"] = (top + total.log())[..., 0].reshape(t, -1)
    return out


_CACHE = ("k_cache", "v_cache", "k_scale", "v_scale", "bounds", "bound_scale")


def _move(s, src, dst):
    for t in _kept(s, *_CACHE).values():
        raw = t.view(torch.int8) if t.dtype.itemsize == 1 else t
        raw[:, dst] = raw[:, src]


def _copy(s):
    if own:
        import paper_2509_00105_amd as kvh

        kvh.copy_pages(s["k_cache"], s["v_cache"], s["src"], s["dst"], head_dim=s["case"]["dim"], k_scale=s["k_scale"], v_scale=s["v_scale"], bounds=s["bounds"],
                       bound_scale=s["bound_scale"])
    else:
        _move(s, s["src"].long(), s["dst"].long())
    return _kept(s, *_CACHE)


def _fork(s):
    case = s["case"]
    if own:
        import paper_2509_00105_amd as kvh

        kvh.fork(s["k_cache"], s["v_cache"], s["page_table"], s["lens"], s["refs"], parents=s["parents"], grow=s["grow"], head_dim=case["dim"], k_scale=s["k_scale"],
                 v_scale=s["v_scale"], bounds=s["bounds"], bound_scale=s["bound_scale"], table_out=s["table_out"], lens_out=s["lens_out"], refs_out=s["refs_out"],
                 workspace=s["workspace"])
        return _kept(s, "table_out", "lens_out", "refs_out", *_CACHE)
    page, table, lens, parent = case["page"], s["page_table"].long(), s["lens"].long(), s["parents"].long()
    n, columns = table.shape
    j, row = torch.arange(columns, device="cuda"), torch.arange(n, device="cuda")
    old = torch.where(parent < 0, 0, lens[parent.clamp(min=0)])
    full, after = old // page, (old + s["grow"].long() + page - 1) // page
    first = torch.where(parent[:, None] == parent, row, n).amin(1) == row  # of its parent's children
    kept = torch.where((old % page != 0) & first, full + 1, full)
    src = table[parent.clamp(min=0)]

    def count(refs, pages, by):
        return refs.index_add(0, pages, torch.full_like(pages, by))

    refs = count(s["refs"].long(), table[j < ((lens + page - 1) // page)[:, None]], -1)
    refs = count(refs, src[j < kept[:, None]], 1)
    need = after - kept
    free, many = (refs != 0).to(torch.int8).sort(stable=True).indices, (refs == 0).sum()
    end = need.cumsum(0)
    fine = (need == 0) | (end <= many)
    at = free[((end - need - kept)[:, None] + j).clamp(0, len(refs) - 1)]
    out = torch.where(j < kept[:, None], src, torch.where(j < after[:, None], at, -1))
    refs = count(refs, src[(j < kept[:, None]) & ~fine[:, None]], -1)
    out = torch.where(fine[:, None], out, -1)
    refs = count(refs, out[(j >= kept[:, None]) & (out >= 0)], 1)
    b = torch.nonzero((old % page != 0) & ~first & fine)[:, 0]
    _move(s, src[b, full[b]], out[b, full[b]])
    return {"table_out": out.to(torch.int32), "lens_out": torch.where(fine, old + s["grow"].long(), 0).to(torch.int32), "refs_out": refs.to(torch.int32),
            **_kept(s, *_CACHE)}


def _compact(s):
    if own:
        import paper_2509_00105_amd as kvh

        kvh.compact(s["k_cache"], s["v_cache"], s["page_table"], s["lens"], s["refs"], head_dim=s["case"]["dim"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                    bounds=s["bounds"], bound_scale=s["bound_scale"], table_out=s["table_out"], refs_out=s["refs_out"], moved_out=s["moved"], workspace=s["workspace"])
        return _kept(s, "table_out", "refs_out", "moved", *_CACHE)
    page, table, refs = s["case"]["page"], s["page_table"].long(), s["refs"]
    at, used = torch.arange(len(refs), device="cuda"), refs > 0
    inside = at < used.sum()
    src, dst = at[used & ~inside], at[~used & inside]
    moved = torch.where(used, at, -1)
    moved[src] = dst
    held = torch.arange(table.shape[1], device="cuda") < ((s["lens"].long() + page - 1) // page)[:, None]
    out = torch.where(held, moved[table.clamp(min=0)], -1)
    _move(s, src, dst)
    return {"table_out": out.to(torch.int32), "refs_out": torch.zeros_like(refs).index_add_(0, moved[used], refs[used]), "moved": moved.to(torch.int32), **_kept(s, *_CACHE)}


# ---- the definitions in 64 bits, request by request and page by page ------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"bound": _exact_bound, "select": _exact_select, "attend": _exact_attend, "copy": _exact_copy, "fork": _exact_fork, "compact": _exact_compact}[case["op"]](s)


def _exact_bound(s):
    case, table = s["case"], s["page_table"].cpu().numpy()
    page, heads, dim = case["page"], case["heads"], case["dim"]
    length, new = _lengths(case)
    codes, scale = s["bounds"].clone(), s["bound_scale"].double()
    for r in range(case["requests"]):
        n, whole = int(length[r]), int(length[r]) // page
        begin = int(n - new[r]) // page
        for a, e, rows in ((begin, whole, page), (max(whole, begin), -(-n // page), n % page)):  # full pages, and one that is not
            if a >= e:
                continue
            at = torch.from_numpy(table[r, a:e].astype(np.int64)).cuda()
            for layer in range(case["layers"]):
                x = s["k_cache"][layer, at, :rows].double().view(e - a, rows, heads, dim)
                least, greatest = x.min(1).values, x.max(1).values
                a127 = x.abs().amax((1, 3))
                codes[layer, at, :, 0] = torch.floor(least * 127 / a127[..., None]).to(torch.int8)
                codes[layer, at, :, 1] = torch.ceil(greatest * 127 / a127[..., None]).to(torch.int8)
                scale[layer, at] = a127 / 127 * (1 if s["k_scale"] is None else s["k_scale"][layer, at].double())
    return {"bounds": codes, "bound_scale": scale}


def _exact_select(s):
    case = s["case"]
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    length, new = _lengths(case)
    out = torch.full((len(s["q"]), heads, case["count"]), -1, dtype=torch.int32, device="cuda")
    row = 0
    for r in range(case["requests"]):
        pages = s["page_table"][r, :-(-int(length[r]) // page)].long()
        lo, hi = s["bounds"][0, pages].double().unbind(2)
        for i in range(int(new[r])):
            p = int(length[r] - new[r]) + i
            n = p // page + 1
            q = s["q"][row].double().view(heads, group, dim)
            most = q.abs().amax(-1)
            whole = torch.round(q * 127 / most[..., None])
            for h in range(heads):
                dots = whole[h].clamp(min=0) @ hi[:n, h].T + whole[h].clamp(max=0) @ lo[:n, h].T
                # a score is a number of 32 bits by definition: each of its two products is rounded to one
                score = (dots * most[h, :, None]).float().amax(0).double() * s["bound_scale"][0, pages[:n], h].double()
                score = score.float().cpu().numpy()
                always = set(range(min(case["first"], n))) | set(range(max(0, n - case["last"]), n))
                rest = [int(x) for x in np.lexsort((np.arange(n), -score)) if int(x) not in always][:max(0, case["count"] - len(always))]
                chosen = sorted(always | set(rest))
                out[row, h, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
            row += 1
            if row > 256:  # host work of a second for each 100 rows
                return {"chosen": None}
    return {"chosen": out}


def _exact_attend(s):
    case = s["case"]
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    length, new = _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((len(s["q"]), heads * group), -math.inf, dtype=torch.float64, device="cuda")
    row = 0
    for r in range(case["requests"]):
        for i in range(int(new[r])):
            p = int(length[r] - new[r]) + i
            for h in range(heads):
                mine = s["chosen"][row, h]
                mine = mine[:int(min(case["count"], p // page + 1))].long()
                at = s["page_table"][r, mine].long()
                hidden = (mine[:, None] * page + torch.arange(page, device="cuda") > p).flatten()

                def column(cache, scale):
                    x = cache[0, at, :, h * dim:(h + 1) * dim].double()
                    return (x if scale is None else x * scale[0, at, h].double()[:, None, None]).flatten(0, 1)

                at0, at1 = h * group * dim, (h + 1) * group * dim
                x = (s["q"][row, at0:at1].double().view(group, dim) @ column(s["k_cache"], s["k_scale"]).T * dim ** -0.5).masked_fill(hidden, -math.inf)
                lse[row, h * group:(h + 1) * group] = torch.logsumexp(x, -1)
                out[row, at0:at1] = (torch.softmax(x, -1) @ column(s["v_cache"], s["v_scale"])).flatten()
            row += 1
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _after(s, pairs):
    """The cache's buffers after pages moved, one pair after the other."""
    got = {}
    for n, t in _kept(s, *_CACHE).items():
        t = t.clone()
        for a, b in pairs:
            t.view(torch.uint8)[:, b].copy_(t.view(torch.uint8)[:, a])
        got[n] = t
    return got


def _exact_copy(s):
    return _after(s, list(zip(s["src"].tolist(), s["dst"].tolist())))


def _exact_fork(s):
    page, table, lens, refs = s["case"]["page"], s["page_table"].tolist(), s["lens"].tolist(), s["refs"].tolist()
    parents, grow = s["parents"].tolist(), s["grow"].tolist()
    for row, n in zip(table, lens):
        for p in row[:-(-n // page)]:
            refs[p] -= 1
    rows, children, open_pages = [], set(), []
    for b, a in enumerate(parents):
        n = lens[a] if a >= 0 else 0
        mine = table[a][:n // page] if a >= 0 else []
        source = -1
        if n % page:
            if a in children:
                source = table[a][n // page]
            else:
                mine = mine + [table[a][n // page]]
        children.add(a)
        for p in mine:
            refs[p] += 1
        rows.append(mine)
        open_pages.append((n + grow[b], source))
    free = [p for p in range(len(refs)) if refs[p] == 0]
    pairs = []
    for b, (n, source) in enumerate(open_pages):
        need = -(-n // page) - len(rows[b])
        fresh, free = free[:need], free[need:]
        if source >= 0:
            pairs.append((source, fresh[0]))
        for p in fresh:
            refs[p] = 1
        rows[b] = rows[b] + fresh
    out = np.full((len(rows), len(table[0])), -1, dtype=np.int32)
    for b, r in enumerate(rows):
        out[b, :len(r)] = r
    to = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"table_out": torch.from_numpy(out).cuda(), "lens_out": to([n for n, _ in open_pages]), "refs_out": to(refs), **_after(s, pairs)}


def _exact_compact(s):
    page, table, lens, refs = s["case"]["page"], s["page_table"].tolist(), s["lens"].tolist(), s["refs"].tolist()
    used = [p for p in range(len(refs)) if refs[p] > 0]
    holes = [p for p in range(len(used)) if refs[p] <= 0]
    moved, pairs, after = [-1] * len(refs), [], [0] * len(refs)
    for p in used:
        moved[p] = p if p < len(used) else holes.pop(0)
        if moved[p] != p:
            pairs.append((p, moved[p]))
        after[moved[p]] = refs[p]
    out = [[moved[p] if j < -(-n // page) else -1 for j, p in enumerate(row)] for row, n in zip(table, lens)]
    to = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"table_out": to(out), "refs_out": to(after), "moved": to(moved), **_after(s, pairs)}
