"""A cache hit and the answer that follows it, end to end on the GPU: a stored entry is decoded, moves into an 8-bit serving cache, and
new tokens are appended to it and attend over it, one layer after the other.

  python examples/serve_step.py [--context 2000] [--question 40] [--answer 8] [--cache i8|e4m3|16] [--layers 4]

The "model" is random queries, keys and values of the right shapes: what runs is the path around the cache, as a serving program runs it.  Prints what the
cache holds and how far the attention is from one over the keys and values before they were compressed.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_00105_amd as kvh  # noqa: E402

HEADS, GROUP, DIM, PAGE = 8, 4, 128, 16  # KV heads, query heads per KV head, channels of a head, tokens of a page
C, CQ = HEADS * DIM, HEADS * GROUP * DIM


def rotation_table(positions: int) -> torch.Tensor:
    """[positions][DIM]: cosines, then sines, of the angles pos * 10000 ** (-2 i / DIM)."""
    at = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))
    return torch.cat([torch.cos(at), torch.sin(at)], 1).float().cuda()


class ServingCache:
    """Pages of one request, their scales if they hold codes, and the table that orders them."""

    def __init__(self, layers: int, tokens: int, kind: str):
        pages = -(-tokens // PAGE)
        dtype = {"16": torch.bfloat16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}[kind]
        self.k, self.v = (torch.zeros((layers, pages, PAGE, C), dtype=dtype, device="cuda") for _ in range(2))
        self.k_scale, self.v_scale = (None, None) if kind == "16" else \
            (torch.zeros((layers, pages, HEADS), device="cuda") for _ in range(2))
        self.table = torch.randperm(pages, device="cuda").to(torch.int32).view(1, pages)
        self.length = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def of(self, layer: int) -> dict:
        """The arguments of a call on one layer."""
        cut = lambda t: None if t is None else t[layer:layer + 1]  # noqa: E731
        return dict(k_cache=cut(self.k), v_cache=cut(self.v), k_scale=cut(self.k_scale), v_scale=cut(self.v_scale))


def run(context: int, question: int, answer: int, kind: str, layers: int, seed: int = 0) -> dict:
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = lambda n, ch: torch.randn((layers, n, ch), generator=g, device="cuda").bfloat16()  # noqa: E731
    table = rotation_table(context + question + answer)
    cache = ServingCache(layers, context + question + answer, kind)

    # An earlier request left its (rotated) keys and values in the store, at 8 bits.
    k0, v0 = rows(context, C), rows(context, C)
    blob = kvh.encode(k0, v0, 0)
    # The hit: decoded, and all layers into the serving cache at once, as they are.
    k, v = torch.empty_like(k0), torch.empty_like(v0)
    kvh.decode(blob, 0, context, k, v, status=cache.status)
    cache.length += context
    starts = torch.tensor([0, context], dtype=torch.int32, device="cuda")
    kvh.append(k, v, cache.k, cache.v, starts, cache.length, cache.table, context, k_scale=cache.k_scale, v_scale=cache.v_scale, status=cache.status)

    # The question's tokens at once, then the answer's one by one; a layer appends before it attends.
    workspace = torch.empty(max(kvh.attention_workspace(1, n, n, HEADS, HEADS * GROUP) for n in (question, 1)), dtype=torch.uint8, device="cuda")
    seen_k, seen_v, worst = k0, v0, 0.0
    for n in [question] + [1] * answer:
        q, k, v = rows(n, CQ), rows(n, C), rows(n, C)
        starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        cache.length += n
        out = []
        for layer in range(layers):
            at = cache.of(layer)
            one = slice(layer, layer + 1)
            turned = kvh.append(k[one], v[one], starts=starts, lens=cache.length, page_table=cache.table, max_new=n, q=q[one], q_out=torch.empty_like(q[one]),
                                rotation=table, status=cache.status, **at)
            out.append(kvh.attention(turned[0], layer=0, starts=starts, lens=cache.length, page_table=cache.table, max_new=n, out=torch.empty_like(turned[0]),
                                     workspace=workspace, status=cache.status, **at))
        # the same over what was never compressed
        past = seen_k.shape[1]
        seen_k, seen_v = torch.cat([seen_k, turn(k, table[past:past + n])], 1), torch.cat([seen_v, v], 1)
        want = plain(turn(q, table[past:past + n]), seen_k, seen_v)
        worst = max(worst, float((torch.stack(out).float() - want).norm() / want.norm()))
    assert not cache.status.any()
    return {"tokens": int(cache.length), "bytes": sum(t.numel() * t.element_size() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None),
            "error": worst}


def turn(x: torch.Tensor, table: torch.Tensor) -> torch.Tensor:
    a, b = x.float().unflatten(-1, (-1, 2, DIM // 2)).unbind(-2)
    cos, sin = (t[:, None] for t in table.split(DIM // 2, -1))
    return torch.stack((a * cos - b * sin, b * cos + a * sin), -2).flatten(-3)


def plain(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> torch.Tensor:
    l, n, past = q.shape[0], q.shape[1], k.shape[1] - q.shape[1]
    q = q.view(l, n, HEADS, GROUP, DIM).permute(0, 2, 3, 1, 4).reshape(l * HEADS, GROUP * n, DIM)
    k, v = (x.float().view(l, -1, HEADS, DIM).transpose(1, 2).reshape(l * HEADS, -1, DIM) for x in (k, v))
    s = torch.bmm(q, k.transpose(1, 2).contiguous()).view(l * HEADS, GROUP, n, -1) / math.sqrt(DIM)
    hidden = torch.arange(past + n, device="cuda") > past + torch.arange(n, device="cuda")[:, None]
    p = s.masked_fill(hidden, -math.inf).softmax(-1).view(l * HEADS, GROUP * n, -1)
    return torch.bmm(p, v.contiguous()).view(l, HEADS, GROUP, n, DIM).permute(0, 3, 1, 2, 4).reshape(l, n, CQ)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--context", type=int, default=2000)
    ap.add_argument("--question", type=int, default=40)
    ap.add_argument("--answer", type=int, default=8)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--cache", choices=("16", "i8", "e4m3"), default="i8")
    a = ap.parse_args()
    r = run(a.context, a.question, a.answer, a.cache, a.layers)
    print("%d tokens in %d layers of a %s cache: %.1f MB; attention %.4f off that over uncompressed keys and values"
          % (r["tokens"], a.layers, a.cache, r["bytes"] / 1e6, r["error"]))


if __name__ == "__main__":
    main()
