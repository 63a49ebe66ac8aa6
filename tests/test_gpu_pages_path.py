"""The calls on pages together, as a serving loop makes them: requests begin, fork, change places and end, tokens are appended, bounded, chosen and read, pages move together."""
import importlib.util
import os
import random

import numpy as np
import pytest

from oracle import pages_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS, HEADS, GROUP, DIM, BT, COLUMNS, PAGES = 6, 2, 3, 64, 8, 12, 60
C, CQ = HEADS * DIM, HEADS * GROUP * DIM


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind,bound", [("16", 0.02), ("i8", 0.025), ("e4m3", 0.06)])
def test_example(kvh, kind, bound):
    """With as many pages as there are the answer is the dense one, to the bounds that the example has without; with few it runs."""
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.run(context=1000, question=33, answer=3, kind=kind, layers=2, pages=65)["error"] < bound
    assert np.isfinite(m.run(context=1000, question=33, answer=2, kind=kind, layers=1, pages=9)["error"])


class Loop:
    def __init__(self, store, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dtype = {"16": torch.bfloat16, "i8": torch.int8}[store]
        self.g, self.store = g, store
        self.k, self.v = (torch.zeros((2, PAGES, BT, C), dtype=dtype, device="cuda") for _ in range(2))
        self.ks, self.vs = (None, None) if store == "16" else (torch.zeros((2, PAGES, HEADS), device="cuda") for _ in range(2))
        self.codes = torch.zeros((2, PAGES, HEADS, 2, DIM), dtype=torch.int8, device="cuda")
        self.scale = torch.zeros((2, PAGES, HEADS), device="cuda")
        self.table, self.lens, self.refs = ints([[-1] * COLUMNS] * ROWS), ints([0] * ROWS), ints([0] * PAGES)
        self.status = ints([0] * ROWS)

    def cache(self):
        return dict(k_cache=self.k, v_cache=self.v, head_dim=DIM, k_scale=self.ks, v_scale=self.vs)

    def step(self, kvh, parents, grow, k, v, q, max_new, count):
        """One step of all rows; q of layer 1.  -> lists and outputs."""
        box = dict(bounds=self.codes, bound_scale=self.scale)
        self.table, self.lens, self.refs = kvh.fork(page_table=self.table, lens=self.lens, refs=self.refs, parents=parents, grow=grow, status=self.status, **box, **self.cache())
        starts = torch.nn.functional.pad(grow.cumsum(0), (1, 0)).to(torch.int32)
        where = dict(starts=starts, lens=self.lens, page_table=self.table, max_new=max_new, status=self.status)
        kvh.append(k, v, **self.cache(), **where)
        kvh.bound_keys(self.k, self.codes, self.scale, k_scale=self.ks, **where)
        chosen = kvh.select_pages(q, self.codes, self.scale, 1, count=count, block_tokens=BT, **where)
        return chosen, kvh.attention_pages(q, layer=1, pages=chosen, **self.cache(), **where)

    def compact(self, kvh):
        self.table, self.refs, moved = kvh.compact(page_table=self.table, lens=self.lens, refs=self.refs, bounds=self.codes, bound_scale=self.scale, status=self.status,
                                                   **self.cache())
        return moved

    def values(self, which):
        x, s = (self.k, self.v)[which][1].double().cpu().unflatten(-1, (HEADS, DIM)), (self.ks, self.vs)[which]
        return (x if s is None else x * s[1].cpu().double()[:, None, :, None]).numpy()


@pytest.mark.parametrize("store", ["16", "i8"])
def test_loop(kvh, store):
    rng = random.Random(5)
    loop = Loop(store, 5)
    held = [[] for _ in range(ROWS)]  # of each row, its tokens' keys and values
    for step in range(12):
        if step == 0:
            parents, grow = [-1] * ROWS, [21, 40, 0, 0, 0, 0]
        elif step == 1:
            parents, grow = [0, 1, 0, 0, 1, 1], [1] * ROWS
        elif step % 4 == 0:  # one ends, another begins
            parents, grow = [0, -1, 2, 3, 4, 2], [1, rng.randint(1, 20), 1, 1, 1, 1]
        else:
            parents = [rng.choice([b, b, rng.randrange(ROWS)]) for b in range(ROWS)]
            grow = [1] * ROWS if step % 3 else [rng.randint(1, 3) for _ in range(ROWS)]
        T = sum(grow)
        k, v = (torch.randn((2, T, C), generator=loop.g, device="cuda").bfloat16() for _ in range(2))
        q = torch.randn((T, CQ), generator=loop.g, device="cuda").bfloat16()
        chosen, out = loop.step(kvh, ints(parents), ints(grow), k, v, q, max(grow), 4)
        assert not loop.status.any()
        starts = np.concatenate([[0], np.cumsum(grow)]).tolist()
        held = [(held[a] if a >= 0 else []) + [(k[:, t], v[:, t]) for t in range(starts[b], starts[b + 1])] for b, a in enumerate(parents)]
        table, lens = loop.table.tolist(), loop.lens.tolist()
        assert lens == [len(h) for h in held]
        # every row's tokens are where the table says: as they were (16 bits), or half a code and a rounding under each later scale off
        for b, tokens in enumerate(held):
            for which, cache, s in ((0, loop.k, loop.ks), (1, loop.v, loop.vs)):
                for p, pair in enumerate(tokens):
                    got = cache[:, table[b][p // BT], p % BT]
                    if store == "16":
                        assert torch.equal(got, pair[which])
                    else:
                        sc = s[:, table[b][p // BT]].repeat_interleave(DIM, -1)
                        assert ((got.float() * sc - pair[which].float()).abs() <= (0.5 * BT + 0.01) * sc).all()
        # bounds of all pages in use, the choice by them, and attention over it
        codes, scale = np.zeros(loop.codes.shape[1:]), np.zeros(loop.scale.shape[1:])
        x = loop.k[1].float().double().cpu().unflatten(-1, (HEADS, DIM)).numpy()
        whole = np.concatenate([[0], np.cumsum(lens)]).tolist()
        codes, scale = ref.bounds(x, None if loop.ks is None else loop.ks[1].cpu().numpy(), whole, lens, table, BT, codes, scale)
        used = sorted({p for row, n in zip(table, lens) for p in row[:-(-n // BT)]})
        assert np.array_equal(loop.codes[1].cpu().numpy()[used], codes[used])
        assert np.allclose(loop.scale[1].cpu().numpy()[used], scale[used], rtol=2.0 ** -22, atol=0)
        qh = q.double().cpu().unflatten(-1, (-1, DIM)).numpy()
        want = ref.select(qh, loop.codes[1].cpu().double().numpy(), loop.scale[1].cpu().numpy(), starts, lens, table, BT, 4, 1, 1, HEADS, np.zeros(chosen.shape))
        assert np.array_equal(chosen.cpu().numpy(), want)
        o, _, size, worth, _ = ref.attention(qh, loop.values(0), loop.values(1), starts, lens, table, BT, DIM ** -0.5, want.astype(int))
        bound = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2 * DIM * 2.0 ** -23 * worth[..., None] + 2.0 ** -16) * size + 2.0 ** -24
        assert (np.abs(out.double().cpu().unflatten(-1, (-1, DIM)).numpy() - o) <= bound).all()
        if step % 5 == 4:
            loop.compact(kvh)
            assert not loop.status.any() and all(r > 0 for r in loop.refs[:int((loop.refs > 0).sum())].tolist())


def test_loop_in_a_graph(kvh):
    """A step captured once and replayed: what the eager loop gives, step by step."""
    rng = random.Random(6)
    eager, caught = Loop("i8", 6), Loop("i8", 6)
    k, v = (torch.randn((2, 61, C), generator=eager.g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((61, CQ), generator=eager.g, device="cuda").bfloat16()
    for loop in (eager, caught):
        loop.step(kvh, ints([-1] * ROWS), ints([21, 40, 0, 0, 0, 0]), k, v, q, 40, 4)
        loop.step(kvh, ints([0, 1, 0, 0, 1, 1]), ints([1] * ROWS), k[:, :6].contiguous(), v[:, :6].contiguous(), q[:6].contiguous(), 1, 4)
    parents, grow = ints(list(range(ROWS))), ints([1] * ROWS)
    k, v = (torch.zeros((2, ROWS, C), device="cuda").bfloat16() for _ in range(2))
    q = torch.zeros((ROWS, CQ), device="cuda").bfloat16()
    state = [caught.table, caught.lens, caught.refs]
    kept = [t.clone() for t in (*state, caught.k, caught.v, caught.ks, caught.vs, caught.codes, caught.scale)]

    def step():
        chosen, out = caught.step(kvh, parents, grow, k, v, q, 1, 4)
        for t, new in zip(state, (caught.table, caught.lens, caught.refs)):
            t.copy_(new)
        caught.table, caught.lens, caught.refs = state
        return chosen, out

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for t, was in zip((*state, caught.k, caught.v, caught.ks, caught.vs, caught.codes, caught.scale), kept):
        t.copy_(was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chosen, out = step()
    for _ in range(5):
        order = [rng.choice([b, rng.randrange(ROWS)]) for b in range(ROWS)]
        parents.copy_(ints(order))
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=eager.g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = eager.step(kvh, parents, grow, k, v, q, 1, 4)
        assert torch.equal(want[0], chosen) and torch.equal(want[1], out)
        for a, b in ((eager.table, state[0]), (eager.lens, state[1]), (eager.refs, state[2]), (eager.scale, caught.scale), (eager.codes, caught.codes)):
            assert torch.equal(a, b)
    assert not caught.status.any() and not eager.status.any()


@pytest.mark.parametrize("store", ["16", "i8"])
def test_both_ways_into_a_call(kvh, store, monkeypatch):
    """With the call module and without it, with all outputs and workspaces given: the same results."""
    import paper_2509_00105_amd.binding as binding

    def run():
        loop = Loop(store, 9)
        T = 30
        k, v = (torch.randn((2, T, C), generator=loop.g, device="cuda").bfloat16() for _ in range(2))
        q = torch.randn((T, CQ), generator=loop.g, device="cuda").bfloat16()
        room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        box = dict(bounds=loop.codes, bound_scale=loop.scale, workspace=room, status=loop.status)
        table, lens, refs = torch.empty_like(loop.table), torch.empty_like(loop.lens), torch.empty_like(loop.refs)
        kvh.fork(page_table=loop.table, lens=loop.lens, refs=loop.refs, parents=ints([-1] * ROWS), grow=ints([5] * ROWS), table_out=table, lens_out=lens, refs_out=refs, **box,
                 **loop.cache())
        where = dict(starts=ints(list(range(0, 31, 5))), lens=lens, page_table=table, max_new=5, status=loop.status)
        kvh.append(k, v, **loop.cache(), **where)
        kvh.bound_keys(loop.k, loop.codes, loop.scale, k_scale=loop.ks, **where)
        chosen, out = torch.empty((T, HEADS, 3), dtype=torch.int32, device="cuda"), torch.empty_like(q)
        lse = torch.empty((T, HEADS * GROUP), device="cuda")
        kvh.select_pages(q, loop.codes, loop.scale, 1, count=3, block_tokens=BT, out=chosen, workspace=room, **where)
        kvh.attention_pages(q, layer=1, pages=chosen, out=out, lse=lse, workspace=room, scale=0.2, **loop.cache(), **where)
        kvh.copy_pages(src=ints([0, 1]), dst=ints([50, 51]), bounds=loop.codes, bound_scale=loop.scale, **loop.cache())
        ends = kvh.compact(page_table=table, lens=lens, refs=refs, table_out=torch.empty_like(table), refs_out=torch.empty_like(refs), moved_out=torch.empty_like(refs), **box,
                           **loop.cache())
        assert not loop.status.any()
        return [table, lens, refs, chosen, out, lse, *ends, loop.k, loop.v, loop.codes, loop.scale]

    one = run()
    monkeypatch.setattr(binding, "_fast", None)
    for x, y in zip(one, run()):
        assert torch.equal(x, y)


def test_the_call_module_takes_these_calls(kvh):
    """With everything given none of them goes the long way round, and what is on another device than the current one goes there, to be refused."""
    import paper_2509_00105_amd.binding as binding

    f = binding._fast
    assert f is not None
    loop = Loop("16", 10)
    loop.lens += 9
    loop.table[:, :2] = ints(list(range(12))).view(6, 2)
    loop.refs[:12] = 1
    starts, q = ints(list(range(7))), torch.zeros((ROWS, CQ), device="cuda").bfloat16()
    room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    chosen, out = torch.zeros((ROWS, HEADS, 2), dtype=torch.int32, device="cuda"), torch.empty_like(q)
    spare = [torch.empty_like(t) for t in (loop.table, loop.lens, loop.refs, loop.refs)]
    where, cache, box = (starts, loop.lens, loop.table, 1), (DIM, None, None), (loop.codes, loop.scale)

    def calls(f):
        return [f.bound_keys(loop.k, *box, *where, None, None, None), f.select_pages(q, *box, 0, *where, 2, BT, 1, 1, chosen, room, None, None),
                f.attention_pages(q, loop.k, loop.v, 0, chosen, *where, DIM, None, None, None, out, None, room, None, None),
                f.copy_pages(loop.k, loop.v, ints([1]), ints([20]), *cache, *box, None, None),
                f.fork(loop.k, loop.v, loop.table, loop.lens, loop.refs, None, None, *cache, *box, spare[0], spare[1], spare[2], room, None, None),
                f.compact(loop.k, loop.v, loop.table, loop.lens, loop.refs, *cache, *box, spare[0], spare[2], spare[3], room, None, None)]

    assert calls(f) == [0] * 6
    torch.cuda.synchronize()
    elsewhere = type(f)(lambda: 1, binding._raw_stream, *[0] * 8, *[1] * 6)  # no call gets as far as its function
    assert calls(elsewhere) == [None] * 6


def test_launch_events(kvh):
    """kvh_time_next_launch times each of them."""
    loop = Loop("i8", 11)
    loop.lens += 9
    loop.table[:, :2] = ints(list(range(12))).view(6, 2)
    loop.refs[:12] = 1
    starts, q = ints(list(range(7))), torch.zeros((ROWS, CQ), device="cuda").bfloat16()
    chosen = torch.zeros((ROWS, HEADS, 2), dtype=torch.int32, device="cuda")
    where = (starts, loop.lens, loop.table, 1)
    rows = dict(page_table=loop.table, lens=loop.lens, refs=loop.refs)
    for call in (lambda: kvh.bound_keys(loop.k, loop.codes, loop.scale, *where, k_scale=loop.ks), lambda: kvh.select_pages(q, loop.codes, loop.scale, 0, *where, 2, block_tokens=BT),
                 lambda: kvh.attention_pages(q, loop.k, loop.v, 0, chosen, *where, head_dim=DIM, k_scale=loop.ks, v_scale=loop.vs),
                 lambda: kvh.copy_pages(src=ints([1]), dst=ints([20]), **loop.cache()), lambda: kvh.fork(**rows, **loop.cache()), lambda: kvh.compact(**rows, **loop.cache())):
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record(), stop.record()
        kvh.time_next_launch(start, stop)
        call()
        torch.cuda.synchronize()
        assert 0 < start.elapsed_time(stop) < 100
