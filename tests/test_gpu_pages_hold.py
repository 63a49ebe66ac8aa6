"""kvh_copy_pages, kvh_fork and kvh_compact against plain lists: everything is copied or counted, so everything has to be equal."""
import random

import pytest

from oracle import pages_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BAD, NO_PAGES = 2, 3  # KVH_DEV_BAD_REQUEST, KVH_DEV_NO_PAGES
STORES = {"fp16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    """A cache of random bytes, NaN among them, and bounds."""

    def __init__(self, pages, store="fp16", layers=2, heads=2, dim=64, bt=16, pad=0, bounds=True, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.pages, self.heads, self.dim, self.bt, dt = pages, heads, dim, bt, STORES[store]

        def some(shape, raw, dtype):
            top = torch.iinfo(raw).max
            return torch.randint(-top, top, shape, generator=g, device="cuda", dtype=torch.int64).to(raw).view(dtype)

        raw = torch.int16 if dt.itemsize == 2 else torch.int8
        self.k, self.v = (some((layers, pages, bt, heads * dim + pad), raw, dt)[..., :heads * dim] for _ in range(2))
        self.ks = self.vs = self.codes = self.scale = None
        if dt.itemsize == 1:
            self.ks, self.vs = (torch.rand((layers, pages, heads), generator=g, device="cuda") for _ in range(2))
        if bounds:
            self.codes = some((layers, pages, heads, 2, dim), torch.int8, torch.int8)
            self.scale = torch.rand((layers, pages, heads), generator=g, device="cuda")

    def args(self):
        return dict(k_cache=self.k, v_cache=self.v, head_dim=self.dim, k_scale=self.ks, v_scale=self.vs, bounds=self.codes, bound_scale=self.scale)

    def words(self):
        """Every buffer as it lies in memory, padding included."""
        got = []
        for t in (self.k, self.v, self.ks, self.vs, self.codes, self.scale):
            if t is not None:
                whole = t if t._base is None else t._base
                got.append(whole.view(torch.int16 if t.element_size() == 2 else torch.int8 if t.element_size() == 1 else torch.int32).clone())
        return got

    def after(self, before, pairs):
        c = self.heads * self.dim
        for t in before:
            old = t.clone()
            for src, dst in pairs:
                if t.dim() == 4 and t.shape[2] == self.bt:  # the cache: what lies between its rows is not touched
                    t[:, dst, :, :c] = old[:, src, :, :c]
                else:
                    t[:, dst] = old[:, src]
        return before

    def check(self, before, pairs):
        for want, got in zip(self.after(before, pairs), self.words()):
            assert torch.equal(want, got)


POOLS = [dict(pages=9), dict(pages=40, store="i8", layers=3, heads=3, bt=7), dict(pages=12, store="bf16", heads=1, dim=128, bt=1, bounds=False),
         dict(pages=20, store="e4m3", heads=8, dim=128, bt=24, pad=16), dict(pages=6, store="fp16", heads=5, dim=128, bt=64, pad=8, layers=1),
         dict(pages=300, store="i8", heads=1, bt=16, bounds=False, layers=1)]


@pytest.mark.parametrize("pool", range(len(POOLS)))
def test_copy(kvh, pool):
    p = Pool(seed=pool, **POOLS[pool])
    rng = random.Random(pool)
    for n in (1, 2, p.pages // 2):
        at = rng.sample(range(p.pages), 2 * n)
        src, dst = at[:n], at[n:]
        if n > 1:
            src[1] = src[0]  # a page may be copied twice
        before, status = p.words(), ints([0] * n)
        kvh.copy_pages(src=ints(src), dst=ints(dst), status=status, **p.args())
        p.check(before, list(zip(src, dst)))
        assert not status.any()


def test_copy_refusals(kvh):
    p = Pool(8, seed=7)
    src, dst = [-1, 8, 2, 3, 1 << 30, 5, -5], [4, 6, 2, -1, 0, 8, -3]
    before, status = p.words(), ints([0] * 7)
    kvh.copy_pages(src=ints(src), dst=ints(dst), status=status, **p.args())
    p.check(before, [])
    assert status.tolist() == [0, BAD, 0, BAD, BAD, BAD, 0]
    kvh.copy_pages(src=ints(src + [0]), dst=ints(dst + [7]), **p.args())
    p.check(before, [(0, 7)])
    kvh.copy_pages(src=ints([]), dst=ints([]), **p.args())
    p.check(before, [])


def test_copy_past_32_bits(kvh):
    """Pages past 4 GiB of a cache, and many pairs."""
    pages = 1_100_000
    k = torch.zeros((1, pages, 16, 256), dtype=torch.int8, device="cuda")
    v = torch.zeros_like(k)
    s = torch.zeros((1, pages, 2), device="cuda")
    src = torch.arange(500, dtype=torch.int32, device="cuda")
    dst = pages - 1 - src
    for t in (k, v):
        t[0, :500] = torch.randint(-127, 127, (500, 16, 256), device="cuda").to(torch.int8)
    s[0, :500] = torch.rand((500, 2), device="cuda")
    kvh.copy_pages(k, v, src, dst, k_scale=s, v_scale=s.clone())
    for t in (k, v, s):
        assert torch.equal(t[0, :500], t[0, pages - 500:].flip(0)) and not t[0, 500:pages - 500].any()
    kvh.copy_pages(k, v, dst, src + 600, k_scale=s, v_scale=s.clone())
    assert torch.equal(k[0, :500], k[0, 600:1100])


class Held:
    """Rows with random lengths; groups of `share` rows have the full pages of their shortest row in common."""

    def __init__(self, rng, n, most, bt, columns, spare, share=1, extra=0):
        self.bt, self.columns = bt, columns
        self.lens = [rng.randint(0, min(most, columns * bt)) for _ in range(n)]
        rows, at = [], 0
        for b in range(n):
            lead = b - b % share
            common = 0 if b == lead else min(self.lens[lead:lead + share]) // bt
            need = -(-self.lens[b] // bt) - common
            rows.append((rows[lead][:common] if common else []) + list(range(at, at + need)))
            at += need
        self.pages = max(1, at + spare)
        place = rng.sample(range(self.pages), self.pages)
        self.table = [[place[p] for p in r] + [rng.choice([-1, 1 << 30, 0])] * (columns - len(r)) for r in rows]
        self.refs = [0] * self.pages
        for row, length in zip(self.table, self.lens):
            for p in row[:-(-length // bt)]:
                self.refs[p] += 1
        for p in rng.sample(range(self.pages), min(extra, self.pages)):
            self.refs[p] += 1  # held by something else too

    def arrays(self):
        return dict(page_table=ints(self.table), lens=ints(self.lens), refs=ints(self.refs))


def fork(kvh, pool, held, parents=None, grow=None, **kw):
    status = torch.zeros(len(held.lens), dtype=torch.int32, device="cuda")
    before = pool.words()
    arrays = held.arrays()
    got = kvh.fork(**arrays, parents=None if parents is None else ints(parents), grow=None if grow is None else ints(grow), status=status, **pool.args(), **kw)
    table, lens, refs, said, pairs = ref.fork(held.table, held.lens, held.refs, held.bt, parents, grow)
    assert got[0].tolist() == table and got[1].tolist() == lens and got[2].tolist() == refs and status.tolist() == said
    pool.check(before, pairs)
    assert arrays["page_table"].tolist() == held.table and arrays["lens"].tolist() == held.lens and arrays["refs"].tolist() == held.refs
    held.table, held.lens, held.refs = table, lens, refs
    return said, pairs


@pytest.mark.parametrize("store", ["fp16", "i8"])
@pytest.mark.parametrize("n,bt,columns,share", [(1, 16, 4, 1), (8, 4, 40, 4), (5, 1, 30, 1), (70, 7, 12, 2), (300, 16, 5, 3), (3, 24, 700, 3), (1100, 2, 6, 2), (4, 1, 9000, 1)])
def test_fork_step_after_step(kvh, n, bt, columns, share, store):
    """Growth, beams that change places, rows that end, rows that begin, again and again; sooner or later the pages run out."""
    rng = random.Random(n * bt + columns)
    held = Held(rng, n, columns * bt // 2, bt, columns, n * 3 + 4, share, extra=2)
    pool = Pool(held.pages, store=store, bt=bt, heads=1, layers=2, seed=n)
    seen = set()
    for step in range(9):
        parents = [rng.choice([b, b, b - b % share + rng.randrange(share), -1 if rng.random() < 0.3 else b]) for b in range(n)]
        parents = [min(p, n - 1) for p in parents]
        grow = [rng.choice([0, 1, 1, 1, bt, rng.randint(0, 3 * bt)]) for _ in range(n)]
        said, _ = fork(kvh, pool, held, parents if step % 3 else None, grow if step % 4 != 3 else None)
        seen |= set(said)
    assert seen <= {0, BAD, NO_PAGES}


def test_fork_one_prompt_into_many(kvh):
    rng = random.Random(1)
    held = Held(rng, 40, 0, 16, 10, 60)
    pool = Pool(held.pages, bt=16, seed=1)
    fork(kvh, pool, held, None, [101] + [0] * 39)
    said, pairs = fork(kvh, pool, held, [0] * 40, [1] * 40)
    assert not any(said) and len(pairs) == 39 and max(held.refs) == 40 and held.lens == [102] * 40
    fork(kvh, pool, held, [-1] * 40, None)
    assert not any(held.refs) and held.lens == [0] * 40 and all(x == -1 for row in held.table for x in row)


def test_fork_refusals(kvh):
    rng = random.Random(2)
    held = Held(rng, 8, 60, 16, 4, 20)
    held.lens = [17, 33, 64, 5, 16, 40, 1, 20]
    held.table = [[3 * b + j if j < -(-held.lens[b] // 16) else -1 for j in range(4)] for b in range(8)]
    held.refs = [0] * 40
    for row, n in zip(held.table, held.lens):
        for p in row[:-(-n // 16)]:
            held.refs[p] += 1
    held.refs[39] = -3  # no count at all: neither free nor held
    held.table[2][1], held.table[5][2] = 40, -1
    held.lens[3], held.lens[7] = -1, 65
    pool = Pool(40, bt=16, seed=2)
    said, _ = fork(kvh, pool, held, [0, 8, 2, 3, 1 << 30, 5, 6, 7], [0, 0, 0, 0, 0, 1, -1, 0])
    assert said == [0, BAD, BAD, BAD, BAD, BAD, BAD, BAD]


def test_fork_with_no_page_to_spare(kvh):
    """The rows in order, as far as the pages go; who needs none is served."""
    held = Held(random.Random(3), 4, 0, 16, 4, 0)
    held.pages, held.lens, held.refs = 5, [30, 32, 10, 0], [1, 1, 1, 1, 1]
    held.table = [[4, 0, -1, -1], [2, 1, -1, -1], [3, -1, -1, -1], [-1, -1, -1, -1]]
    pool = Pool(5, bt=16, seed=3)
    said, _ = fork(kvh, pool, held, None, [2, 1, 3, 0])
    assert said == [0, NO_PAGES, 0, 0]
    said, _ = fork(kvh, pool, held, [0, 2, 2, -1], [0, 20, 0, 0])  # two pages are free again, which 33 tokens on page 3 and two more take; the copy for row 2 has none
    assert said == [0, 0, NO_PAGES, 0]


def test_fork_first_child_refused(kvh):
    """The first child grows past the table: the second one keeps the page, which nobody else is handed, the third one gets a copy."""
    held = Held(random.Random(4), 4, 0, 16, 3, 0)
    held.pages, held.lens, held.refs = 5, [20, 0, 0, 0], [1, 1, 0, 0, 0]
    held.table = [[1, 0, -1], [-1] * 3, [-1] * 3, [-1] * 3]
    pool = Pool(5, bt=16, seed=4)
    said, pairs = fork(kvh, pool, held, [0, -1, 0, 0], [29, 20, 1, 2])
    assert said == [BAD, 0, 0, 0] and held.table == [[-1] * 3, [2, 3, -1], [1, 0, -1], [1, 4, -1]] and pairs == [(0, 4)]


@pytest.mark.parametrize("store", ["fp16", "e4m3"])
@pytest.mark.parametrize("n,bt,columns,spare,share", [(1, 16, 4, 0, 1), (6, 7, 20, 50, 2), (30, 16, 40, 3000, 3), (2, 1, 3, 1, 1), (90, 4, 30, 700, 1), (5, 1, 3000, 40000, 1)])
def test_compact(kvh, n, bt, columns, spare, share, store):
    rng = random.Random(n + spare)
    held = Held(rng, n, columns * bt, bt, columns, spare, share, extra=3)
    pool = Pool(held.pages, store=store, bt=bt, heads=1, layers=2, seed=n)
    status, before, arrays = torch.zeros(n, dtype=torch.int32, device="cuda"), pool.words(), held.arrays()
    got = kvh.compact(status=status, **arrays, **pool.args())
    table, refs, moved, said, pairs = ref.compact(held.table, held.lens, held.refs, bt)
    assert got[0].tolist() == table and got[1].tolist() == refs and got[2].tolist() == moved and status.tolist() == said == [0] * n
    pool.check(before, pairs)
    assert all(refs[p] > 0 for p in range(sum(x > 0 for x in refs)))
    again = kvh.compact(**pool.args(), page_table=got[0], lens=arrays["lens"], refs=got[1])
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    pool.check(before, [])


def test_compact_refusals(kvh):
    held = Held(random.Random(5), 4, 0, 16, 3, 0)
    held.pages, held.refs = 7, [0, 2, -1, 1, 0, 1, 0]
    held.table, held.lens = [[5, 1, 9], [2, 3, 1], [7, -1, 3], [3, 5, 1]], [32, 48, 47, 49]
    pool = Pool(7, bt=16, seed=5)
    status, before = torch.zeros(4, dtype=torch.int32, device="cuda"), pool.words()
    got = kvh.compact(status=status, **held.arrays(), **pool.args())
    table, refs, moved, said, pairs = ref.compact(held.table, held.lens, held.refs, 16)
    assert got[0].tolist() == table and got[1].tolist() == refs and got[2].tolist() == moved and status.tolist() == said == [0, BAD, BAD, BAD]
    pool.check(before, pairs)


def test_given_outputs_strides_streams_and_graphs(kvh):
    """Wide tables, outputs that hold anything, a captured step that is replayed with its results as the next inputs."""
    rng = random.Random(6)
    held = Held(rng, 12, 100, 16, 9, 60, 4)
    pool = Pool(held.pages, store="i8", bt=16, seed=6)
    wide = [torch.full((12, 20), 12345, dtype=torch.int32, device="cuda") for _ in range(2)]
    table = [w[:, 3:12] for w in wide]
    lens, refs = [ints(held.lens), ints([9] * 12)], [ints(held.refs), ints([9] * held.pages)]
    table[0].copy_(ints(held.table))
    parents, grow = ints(list(range(12))), ints([1] * 12)
    room = torch.full((kvh.fork_workspace(12, held.pages),), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(12, dtype=torch.int32, device="cuda")

    def step(i):
        kvh.fork(page_table=table[i], lens=lens[i], refs=refs[i], parents=parents, grow=grow, table_out=table[1 - i], lens_out=lens[1 - i], refs_out=refs[1 - i],
                 workspace=room, status=status, **pool.args())

    start = [t.clone() for t in (*wide, *lens, *refs, pool.k, pool.v, pool.ks, pool.vs, pool.codes, pool.scale)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(0), step(1)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0), step(1)
    for t, was in zip((*wide, *lens, *refs, pool.k, pool.v, pool.ks, pool.vs, pool.codes, pool.scale), start):
        t.copy_(was)
    for turn in range(4):
        order = [rng.choice([b, b - b % 4 + rng.randrange(4)]) for b in range(12)]
        parents.copy_(ints(order))
        before, pairs = pool.words(), []
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for _ in range(2):
            held.table, held.lens, held.refs, said, moved = ref.fork(held.table, held.lens, held.refs, 16, order, [1] * 12)
            before = pool.after(before, moved)
            assert not any(said)
        pool.check(before, pairs)
        assert table[0].tolist() == held.table and lens[0].tolist() == held.lens and refs[0].tolist() == held.refs, turn
        assert (wide[0][:, :3] == 12345).all() and (wide[1][:, 12:] == 12345).all()


def test_binding_refuses(kvh):
    pool, i = Pool(4, bt=16), ints([0, 1])
    table, refs = ints([[0, -1], [1, -1]]), ints([1, 1, 0, 0])
    bad = [dict(refs=refs[:3]), dict(page_table=table[:1]), dict(lens=i[:1]), dict(lens=i.long()), dict(parents=i[:1]), dict(table_out=table[:, :1].contiguous()),
           dict(refs_out=refs[:2].clone()), dict(workspace=i)]
    for kw in bad:
        with pytest.raises(ValueError):
            kvh.fork(**dict(dict(page_table=table, lens=i, refs=refs), **kw), **pool.args())
    for kw in (dict(table_out=table), dict(refs_out=refs), dict(lens_out=i)):
        with pytest.raises(kvh.KVHError):
            kvh.fork(**dict(dict(page_table=table, lens=i, refs=refs), **kw), **pool.args())
    with pytest.raises(ValueError):
        kvh.copy_pages(src=i, dst=i[:1], **pool.args())
    with pytest.raises(ValueError):
        kvh.copy_pages(src=i, dst=i, **dict(pool.args(), bound_scale=None))
