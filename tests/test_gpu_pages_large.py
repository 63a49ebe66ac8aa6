"""The forms that the calls on pages take at larger sizes, as the tests at small ones compare them: picks of many tokens and heads over wide tables, bounds and copies past the
caches, forks whose counts or tables one block does not plan, and pages that run out in each of them."""
import random

import numpy as np
import pytest

from oracle import pages_ref as ref
from test_gpu_pages_attention import Listed
from test_gpu_pages_hold import BAD, NO_PAGES, Held, Pool, fork, ints
from test_gpu_pages_select import Batch, Keys

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


# ---- selection: from 1024 picks on, over tables of more than 1024 pages, through memory -----------------------------------------------------------------
@pytest.mark.parametrize("news,heads,group,dim,count,ties", [([260, 253], 2, 4, 64, 40, 0), ([517], 2, 7, 64, 9, 0), ([130, 1, 135], 4, 3, 64, 260, 0), ([520], 2, 2, 128, 33, 3)])
def test_many_picks(kvh, news, heads, group, dim, count, ties):
    b = Batch(news, [1201, 1100, 640][:len(news)], heads=heads, group=group, dim=dim, bt=1, seed=70, layers=1, ties=ties, behind=5)
    assert sum(news) * heads >= 1024 and b.table.shape[1] > 1024
    b.check(kvh, count, 1, 2)
    assert not b.status.any()


# ---- bounds: from 8 MiB of keys on, counted as 512 or 1024 channels at a time -----------------------------------------------------------------------------
@pytest.mark.parametrize("kind,dt", [("16", "bf16"), ("16", "fp16"), ("i8", "bf16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("shape", [dict(news=[2050], lens=[2063], heads=8, dim=128, layers=4), dict(news=[4301, 0], lens=[4310, 30], heads=5, dim=64, bt=24, layers=4)])
def test_bounds_past_the_caches(kvh, shape, kind, dt):
    b = Keys(kind=kind, dt=dt, seed=71, **shape)
    per = 512 if kind == "16" else 1024
    assert (sum(b.news) // b.bt) * -(-b.heads * b.dim // per) * per * b.bt * shape["layers"] >= 8 << 20
    b.run(kvh)
    b.check()
    assert not b.status.any()


# ---- copies: from 16 MiB of K and V on ----------------------------------------------------------------------------------------------------------------------
POOLS = [dict(pages=110, store="fp16", heads=5, dim=128, bt=64, pad=8), dict(pages=4400, store="i8", layers=3, heads=3, bt=7), dict(pages=420, store="e4m3", heads=8, dim=128, bt=24, pad=16),
         dict(pages=1100, store="bf16", heads=2, dim=64, bt=33, layers=3, bounds=False)]


def copied(p):
    """Bytes of K and V of a page, all layers."""
    return 2 * p.k.shape[0] * p.bt * p.heads * p.dim * p.k.element_size()


@pytest.mark.parametrize("pool", range(len(POOLS)))
def test_copy_past_the_caches(kvh, pool):
    p = Pool(seed=pool, **POOLS[pool])
    n = p.pages // 2 - 1
    at = random.Random(pool).sample(range(p.pages), 2 * n)
    src, dst = at[:n], at[n:]
    src[1], dst[5] = src[0], -1  # twice the same page, and a pair that is refused
    assert (n - 1) * copied(p) >= 16 << 20
    before, status = p.words(), ints([0] * n)
    kvh.copy_pages(src=ints(src), dst=ints(dst), status=status, **p.args())
    p.check(before, [(s, d) for s, d in zip(src, dst) if d >= 0])
    assert status.tolist() == [BAD if i == 5 else 0 for i in range(n)]


@pytest.mark.parametrize("store,n,bt,columns,spare,heads,dim,pad", [("i8", 40, 16, 30, 2400, 2, 128, 16), ("fp16", 20, 33, 40, 900, 3, 64, 0), ("bf16", 9, 5, 300, 7000, 2, 64, 8)])
def test_compact_past_the_caches(kvh, store, n, bt, columns, spare, heads, dim, pad):
    held = Held(random.Random(n), n, columns * bt, bt, columns, spare, 3, extra=3)
    pool = Pool(held.pages, store=store, bt=bt, heads=heads, dim=dim, layers=2, pad=pad, seed=n)
    assert pool.pages // 2 * copied(pool) >= 16 << 20
    status, before = torch.zeros(n, dtype=torch.int32, device="cuda"), pool.words()
    got = kvh.compact(status=status, **held.arrays(), **pool.args())
    table, refs, moved, said, pairs = ref.compact(held.table, held.lens, held.refs, bt)
    assert got[0].tolist() == table and got[1].tolist() == refs and got[2].tolist() == moved and status.tolist() == said == [0] * n
    assert len(pairs) > 50
    pool.check(before, pairs)


# ---- forks that run out of pages, planned by one block and in three launches ------------------------------------------------------------------------------------
FORKS = [dict(n=12, bt=4, columns=40, spare=6, share=4, most=60, more=60), dict(n=300, bt=16, columns=5, spare=40, share=3), dict(n=1024, bt=2, columns=6, spare=100, share=2),  # one block
         dict(n=1025, bt=2, columns=6, spare=100, share=2), dict(n=1400, bt=3, columns=5, spare=60, share=7),  # more than 1024 rows
         dict(n=40, bt=1, columns=900, spare=30, share=1, lens=[400 + b for b in range(40)], more=80, same=1),  # more than 16128 pages
         dict(n=66, bt=16, columns=8000, spare=9, share=3, most=300, more=50, same=0.8)]  # more than 512K entries of the table


@pytest.mark.parametrize("case", range(len(FORKS)))
def test_fork_until_pages_run_out(kvh, case):
    """Rows that grow, are copied, end and begin, with fewer pages than they want: those in front are served, what the others kept is given back, and the next step finds it."""
    f = FORKS[case]
    n, bt, columns = f["n"], f["bt"], f["columns"]
    rng = random.Random(80 + case)
    held = Held(rng, n, f.get("most", columns * bt // 2), bt, columns, f["spare"], f["share"], extra=2)
    if "lens" in f:
        held.lens = f["lens"]
        at = np.concatenate([[0], np.cumsum(held.lens)]).tolist()
        held.pages = at[-1] + f["spare"]
        place = rng.sample(range(held.pages), held.pages)
        held.table = [place[at[b]:at[b + 1]] + [-1] * (columns - held.lens[b]) for b in range(n)]
        held.refs = [0] * held.pages
        for p in place[:at[-1]]:
            held.refs[p] = 1
    pool = Pool(held.pages, store="i8", bt=bt, heads=1, layers=1, seed=case)
    seen, copies = set(), 0
    for step in range(5):
        parents = [b if rng.random() < f.get("same", 0.7) else rng.choice([b - b % f["share"] + rng.randrange(f["share"]), -1]) for b in range(n)]
        parents = [min(p, n - 1) for p in parents]
        grow = [rng.choice([0, 1, 1, bt, rng.randint(0, 3 * bt + f.get("more", 0))]) for _ in range(n)]
        if step == 4:
            grow[rng.randrange(n)] = -1
        said, pairs = fork(kvh, pool, held, parents if step != 1 else None, grow)
        seen |= set(said)
        copies += len(pairs)
    assert seen == {0, BAD, NO_PAGES} and (copies > 0 or bt == 1)


# ---- attention --------------------------------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind,news,lens,count", [("16", [1] * 64, [1024] * 64, 64), ("i8", [512], [4096], 64), ("e4m3", [3, 1], [9000, 2000], 500)])
def test_attention_repeats_itself(kvh, kind, news, lens, count):
    """Blocks that share a list, or not, in whatever order they run: the same bits."""
    b = Listed(news, lens, heads=8, group=4, kind=kind, dt="bf16", seed=72, layers=1).choose(count, 1)
    want, lse = b.run(kvh), b.lse
    for _ in range(5):
        assert torch.equal(b.run(kvh), want) and torch.equal(b.lse, lse)
    if len(news) > 2:
        b.check(want)
