"""kvh_bound_keys and kvh_select_pages against their definitions in 64 bits.

Codes of bounds and chosen pages are whole numbers and have to be equal: the quotients behind the codes lie on whole numbers or 2^-19 of their size away from
them, further than their one rounding of 2^-24, and scores are defined with their two roundings to 32 bits.  A scale is a quotient and, over 8 bits, a product, each off by
2^-24 of its value at most (2^-149 where that is subnormal)."""
import math

import numpy as np
import pytest

from oracle import pages_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BAD = 2  # KVH_DEV_BAD_REQUEST
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Keys:
    """A random K cache with what no request holds as NaN (int8: full scale), and bounds of 77 and 7.0 where none were made."""

    def __init__(self, news, lens, heads=2, dim=128, bt=16, kind="16", dt="bf16", seed=0, layers=2, wide=0):
        g = torch.Generator().manual_seed(seed)
        self.news, self.lens_h, self.bt, self.heads, self.dim, self.kind = news, list(lens), bt, heads, dim, kind
        self.starts_h = np.concatenate([[0], np.cumsum(news)]).tolist()
        held = [-(-n // bt) for n in lens]
        self.pages, c = sum(held) + 2, heads * dim
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table_h = [[order.pop() for _ in range(h)] + [-7] * (max(1, max(held)) + wide - h) for h in held]
        shape = (layers, self.pages, bt, c)
        x = torch.randn(shape, generator=g) * torch.exp(0.5 * torch.randn(c, generator=g))
        mine = torch.zeros((self.pages, bt), dtype=torch.bool)
        for b, n in enumerate(lens):
            for p in range(n):
                mine[self.table_h[b][p // bt], p % bt] = True
        self.ks = None
        if kind == "16":
            x = x.to(DT[dt])
            x.view(torch.int16)[:, ~mine] = 0x7fff
        elif kind == "i8":
            x = (30 * x).round().clamp(-127, 127).to(torch.int8)
            x[:, ~mine] = 127
        else:
            x = (90 * x).clamp(-448, 448).to(torch.float8_e4m3fn)
            x.view(torch.int8)[:, ~mine] = 0x7f
        self.k = x.cuda()
        if kind != "16":
            self.ks = (torch.exp(0.5 * torch.randn((layers, self.pages, heads), generator=g)) / 30).cuda()
        self.codes = torch.full((layers, self.pages, heads, 2, dim), 77, dtype=torch.int8, device="cuda")
        self.scale = torch.full((layers, self.pages, heads), 7.0, device="cuda")
        self.starts, self.lens, self.table = ints(self.starts_h), ints(self.lens_h), ints(self.table_h)
        self.status = torch.zeros(len(news), dtype=torch.int32, device="cuda")

    def run(self, kvh, **kw):
        kvh.bound_keys(self.k, self.codes, self.scale, self.starts, self.lens, self.table, kw.pop("max_new", max(1, max(self.news))), k_scale=self.ks, status=self.status, **kw)

    def check(self):
        for layer in range(self.k.shape[0]):
            x = self.k[layer].float().double().cpu().unflatten(-1, (self.heads, self.dim)).numpy()
            ks = None if self.ks is None else self.ks[layer].cpu().numpy()
            codes, scale = ref.bounds(x, ks, self.starts_h, self.lens_h, self.table_h, self.bt, np.full(self.codes.shape[1:], 77), np.full(self.scale.shape[1:], 7.0))
            assert np.array_equal(self.codes[layer].cpu().numpy(), codes)
            got = self.scale[layer].double().cpu().numpy()
            assert ((np.abs(got - scale) <= 2.0 ** -23 * scale + 2.0 ** -149) | (np.isnan(got) & np.isnan(scale))).all()


SHAPES = [
    dict(news=[1], lens=[1]),
    dict(news=[1, 1, 1], lens=[16, 17, 300], heads=8),
    dict(news=[5, 0, 40], lens=[20, 9, 40], heads=3, dim=64, bt=24),
    dict(news=[33, 2], lens=[33, 700], heads=5, dim=64, bt=7),
    dict(news=[20], lens=[21], heads=9, dim=128, bt=1),
    dict(news=[100, 0], lens=[400, 0], heads=1, dim=64, bt=256),
    dict(news=[300], lens=[300], heads=17, dim=64, bt=20, wide=3),
]


@pytest.mark.parametrize("kind,dt", [("16", "bf16"), ("16", "fp16"), ("i8", "bf16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_bounds(kvh, shape, kind, dt):
    b = Keys(kind=kind, dt=dt, seed=shape, **SHAPES[shape])
    b.run(kvh)
    b.check()
    assert not b.status.any()
    b.run(kvh)  # again: the same
    b.check()


@pytest.mark.parametrize("kind,dt", [("16", "bf16"), ("16", "fp16"), ("e4m3", "bf16")])
def test_bounds_of_odd_pages(kvh, kind, dt):
    """Zeros, one value alone, tiny and huge ones, infinities and NaN in sight, on pages of their own."""
    b = Keys([160], [160], heads=2, kind=kind, dt=dt, seed=20, layers=1)
    page = [int(p) for p in b.table_h[0]]
    x = b.k.view(1, b.pages, 16, 2, 128)
    low = b.k.view(torch.int16 if kind == "16" else torch.int8).view(x.shape)
    low[0, page[0]] = 0
    low[0, page[1], :, 0] = 0
    low[0, page[1], 3, 0, 5] = 1  # the smallest number there is
    nan = 0x7fff if kind == "16" else 0x7f
    low[0, page[2], 15, 1, 127] = nan
    if kind == "16":
        big = torch.finfo(DT[dt]).max
        x[0, page[3], 2, 0, 0], x[0, page[3], 2, 1, 0] = math.inf, -math.inf
        x[0, page[4], :, :, 7] = -big
        x[0, page[4], 1, :, 8] = big
    if kind == "16" and dt == "bf16":
        x[0, page[5]] = (x[0, page[5]].float() * 2.0 ** -110).to(x.dtype)  # all below 2^-100
        x[0, page[6]] = (x[0, page[6]].float().clamp(1, 2) * 2.0 ** -100).to(x.dtype)
        x[0, page[6], :, :, 3] = 2.0 ** -126
    if kind == "e4m3":
        b.ks[0, page[3], 0], b.ks[0, page[3], 1] = math.inf, math.nan
        b.ks[0, page[0], 0] = math.inf  # zeros under it
        b.ks[0, page[4], 0] = 0.0
        b.ks[0, page[5], 0] = torch.finfo(torch.float32).max
        b.ks[0, page[6], 0] = 2.0 ** -149
    b.run(kvh)
    b.check()
    assert b.scale[0, page[2]].isnan().tolist() == [False, True] and b.scale[0, page[3]].isnan().all()


def test_bounds_refusals(kvh):
    b = Keys([1, 6, 2], [40, 50, 17], dim=64, heads=1, kind="i8", seed=21)
    b.run(kvh, max_new=2)
    assert b.status.tolist() == [0, BAD, 0]
    b.news[1], keep, b.starts_h = 0, b.starts_h, [0, 1, 1, 3]
    b.check()
    b = Keys([1, 6, 2], [40, 50, 17], dim=64, heads=1, kind="i8", seed=21)
    b.table[0, 2], b.table[2, 1] = -1, b.pages
    b.lens[1] = 5  # fewer than the new ones
    b.run(kvh)
    assert b.status.tolist() == [BAD, BAD, BAD]
    first = b.table_h[2][0]  # of the third request the page before is bounded all the same
    assert (b.scale[:, [p for p in range(b.pages) if p != first]] == 7).all() and (b.scale[:, first] != 7).all()


def test_bounds_strided_and_past_32_bits(kvh):
    """Rows wider than the channels, layers and pages apart, pages past 4 GiB."""
    b = Keys([20], [50], heads=2, dim=64, kind="i8", seed=22, layers=1)
    pages = 8_500_000
    far = Keys([20], [50], heads=1, dim=64, bt=8, kind="i8", seed=23, layers=1)
    cache = torch.zeros((1, pages, 8, 64), dtype=torch.int8, device="cuda")  # 4.05 GiB
    ks = torch.zeros((1, pages, 1), device="cuda")
    base = pages - far.pages
    cache[:, base:], ks[:, base:] = far.k, far.ks
    codes = torch.full((1, pages, 1, 2, 64), 77, dtype=torch.int8, device="cuda")
    scale = torch.full((1, pages, 1), 7.0, device="cuda")
    table = torch.where(far.table >= 0, far.table + base, far.table)
    kvh.bound_keys(cache, codes, scale, far.starts, far.lens, table, 20, k_scale=ks)
    far.run(kvh)
    far.check()
    assert torch.equal(codes[:, base:], far.codes) and torch.equal(scale[:, base:], far.scale) and (scale[:, :base] == 7).all()
    room = torch.full((3, b.pages, 16, 256), 99, dtype=torch.int8, device="cuda")
    room[1:2, :, :, 64:192] = b.k
    box = torch.full((2, b.pages, 5, 2, 64), 77, dtype=torch.int8, device="cuda")
    sc = torch.full((2, b.pages, 6), 7.0, device="cuda")
    kvh.bound_keys(room[1:2, :, :, 64:192], box[:1, :, 1:3], sc[1:, :, 2:4], b.starts, b.lens, b.table, 20, k_scale=b.ks)
    b.run(kvh)
    b.check()
    assert torch.equal(box[:1, :, 1:3], b.codes) and torch.equal(sc[1:, :, 2:4], b.scale)
    assert (box[1] == 77).all() and (box[0, :, [0, 3, 4]] == 77).all() and (sc[0] == 7).all() and (sc[1, :, [0, 1, 4, 5]] == 7).all()


# ---- selection ----------------------------------------------------------------------------------------------------
class Batch:
    """Random queries and bounds; the pages of no request have bounds that would always be chosen."""

    def __init__(self, news, lens, heads=2, group=2, dim=128, bt=16, dt="bf16", seed=0, layers=2, pad=0, behind=0, ties=0):
        g = torch.Generator().manual_seed(seed)
        self.news, self.lens_h, self.bt, self.heads, self.dim, self.group, self.layer = news, list(lens), bt, heads, dim, group, layers - 1
        self.starts_h = np.concatenate([[0], np.cumsum(news)]).tolist()
        held = [-(-n // bt) for n in lens]
        self.pages, self.T = sum(held) + 2, self.starts_h[-1] + behind
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table_h = [[order.pop() for _ in range(h)] + [1 << 30] * (max(1, max(held)) - h) for h in held]
        shape = (layers, self.pages, heads, 1, dim)
        middle, reach = 40 * torch.randn(shape, generator=g), 30 * torch.randn(shape, generator=g).abs()
        self.codes = torch.cat([(middle - reach).floor(), (middle + reach).ceil()], 3).clamp(-127, 127).to(torch.int8).cuda()
        self.scale = (torch.exp(0.4 * torch.randn(shape[:3], generator=g)) / 30).cuda()
        if ties:  # few kinds of pages
            kinds = torch.arange(self.pages, device="cuda") % ties
            self.codes, self.scale = self.codes[:, kinds].contiguous(), self.scale[:, kinds].contiguous()
        for p in order:
            self.codes[:, p], self.scale[:, p] = 127, 1e30
        self.q = torch.randn((self.T, heads * group * dim + pad), generator=g).to(DT[dt]).cuda()[:, :heads * group * dim]
        self.starts, self.lens, self.table = ints(self.starts_h), ints(self.lens_h), ints(self.table_h)
        self.status = torch.zeros(len(news), dtype=torch.int32, device="cuda")

    def run(self, kvh, count, first=1, last=1, **kw):
        out = torch.full((self.T, self.heads, count), -9, dtype=torch.int32, device="cuda")
        got = kvh.select_pages(self.q, self.codes, self.scale, self.layer, self.starts, self.lens, self.table, kw.pop("max_new", max(1, max(self.news))), count,
                               block_tokens=self.bt, first=first, last=last, out=out, status=self.status, **kw)
        assert got is out
        return out

    def want(self, count, first=1, last=1):
        q = self.q.double().cpu().unflatten(-1, (-1, self.dim)).numpy()
        out = np.full((self.T, self.heads, count), -9)
        return ref.select(q, self.codes[self.layer].cpu().double().numpy(), self.scale[self.layer].cpu().numpy(), self.starts_h, self.lens_h, self.table_h, self.bt, count,
                          first, last, self.heads, out)

    def check(self, kvh, count, first=1, last=1, **kw):
        assert np.array_equal(self.run(kvh, count, first, last, **kw).cpu().numpy(), self.want(count, first, last))


CHOICES = [
    dict(news=[1], lens=[1]),
    dict(news=[1, 1, 1], lens=[33, 700, 16], heads=8, group=4),
    dict(news=[1, 0, 1, 1], lens=[257, 9, 1, 1300], heads=1, group=8, dim=64),
    dict(news=[5, 2], lens=[41, 900], heads=2, group=7, dim=64, bt=24, behind=3),
    dict(news=[3, 1], lens=[100, 64], heads=2, group=20, bt=32, pad=16),
    dict(news=[40], lens=[40], heads=1, group=3, bt=7),
    dict(news=[37, 1, 17], lens=[130, 77, 400], heads=2, group=1, dim=64, bt=3),
    dict(news=[9, 2], lens=[4, 300], heads=2, group=16),  # more queries than tokens: the first ones see nothing
    dict(news=[6, 1], lens=[1200, 3000], heads=1, group=5, dim=64, bt=1),
]


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("count,first,last", [(1, 0, 1), (8, 1, 2), (9, 8, 1), (64, 0, 5), (300, 3, 200)])
@pytest.mark.parametrize("shape", range(len(CHOICES)))
def test_selection(kvh, shape, count, first, last, dt):
    b = Batch(dt=dt, seed=shape, **CHOICES[shape])
    b.check(kvh, count, first, last)
    assert not b.status.any()


@pytest.mark.parametrize("ties", [1, 2, 5])
@pytest.mark.parametrize("count", [2, 7, 40, 130])
def test_equal_scores_go_to_the_first(kvh, count, ties):
    b = Batch([1, 3], [2100, 700], heads=2, group=4, seed=30, ties=ties)
    b.check(kvh, count)
    b.codes.zero_()  # all scores are zero, of either sign
    b.scale *= torch.where(torch.arange(b.pages, device="cuda")[:, None] % 3 == 0, 0.0, 1.0)
    b.check(kvh, count)


@pytest.mark.parametrize("lens", [[20000], [9000, 70], [33000]])
def test_long_requests(kvh, lens):
    """Thousands of pages: page tables of 8 tokens."""
    b = Batch([2] * len(lens), lens, heads=2, group=4, dim=64, bt=8, seed=31, layers=1)
    b.check(kvh, 257, 1, 4)
    b.check(kvh, 2048, 0, 1)


def test_pages_of_many_tokens_and_many_requests(kvh):
    g = np.random.default_rng(3)
    news = [int(x) for x in g.integers(0, 4, 150)]
    lens = [n + int(x) for n, x in zip(news, g.integers(0, 200, 150))]
    Batch(news, lens, heads=1, group=2, dim=64, bt=4, seed=32, layers=1, behind=5).check(kvh, 11, 1, 2)


def test_odd_scores(kvh):
    """Scales that are no finite numbers (their pages come first), scores past fp32, queries of zeros, infinities and NaN (they count as zeros)."""
    b = Batch([1, 1, 1, 1, 1], [640] * 5, heads=1, group=3, dim=64, dt="bf16", seed=33, layers=1)
    s = b.scale[0, :, 0]
    for r in range(5):
        row = b.table_h[r]
        s[row[3]], s[row[30]], s[row[17]] = math.nan, math.inf, 0.0
    q = b.q.view(5, 3, 64)
    q[0, 0, 5], q[0, 1, 6], q[0, 2, 7] = math.nan, math.inf, -math.inf
    q[1, 0] = 0
    q[1, 1] *= 2.0 ** -105
    q[2] *= 2.0 ** 120
    b.scale[0, b.table_h[2][9], 0] = 1e30
    q[3, 1, 9] = math.inf
    b.check(kvh, 12)
    b.check(kvh, 3)


def test_workspace_in_turns(kvh):
    """Too many pages for a block to keep their scores: through memory, all tokens at once and in turns."""
    b = Batch([3, 1, 9], [100, 18001, 90], heads=2, group=4, dim=64, bt=1, seed=34, layers=1)
    want = b.run(kvh, 20)
    assert np.array_equal(want.cpu().numpy(), b.want(20))
    pitch = -(-len(b.table_h[0]) // 4) * 4
    for tokens in (1, 2, 5):
        room = torch.full((2 * pitch * 4 * tokens + 8,), 255, dtype=torch.uint8, device="cuda")
        assert torch.equal(want, b.run(kvh, 20, workspace=room))
    with pytest.raises(kvh.KVHError) as e:
        b.run(kvh, 20, workspace=room[:2 * pitch * 4 - 1])
    assert e.value.status == -4


@pytest.mark.parametrize("group", [1, 4, 6, 17])
def test_with_and_without_a_workspace(kvh, group):
    """Scores through memory or not, tokens together or each by itself: the same pages."""
    b = Batch([2, 5], [9000, 40], heads=1, group=group, dim=64, bt=2, seed=37, layers=1)
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    one, two = b.run(kvh, 50), b.run(kvh, 50, workspace=none)
    assert torch.equal(one, two) and np.array_equal(one.cpu().numpy(), b.want(50))


@pytest.mark.parametrize("group", [1, 3, 4, 6, 8])
@pytest.mark.parametrize("count", [20, 400])
def test_many_new_tokens_share_products(kvh, group, count):
    """Tiles of 8 and 16 tokens that begin and end inside requests, a request without tokens, rows behind the last one; in turns too, and without a workspace."""
    b = Batch([45, 0, 21, 70], [1300, 5, 30, 72], heads=2, group=group, dim=64, bt=1, seed=38, layers=1, behind=3)
    want = b.want(count, 2, 3)
    assert np.array_equal(b.run(kvh, count, 2, 3).cpu().numpy(), want)
    token = 2 * 1300 * 4
    for size in (0, 16 * token, 37 * token, 3 * token):
        room = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        assert np.array_equal(b.run(kvh, count, 2, 3, workspace=room).cpu().numpy(), want), size
    assert not b.status.any()


def test_many_new_tokens_refused(kvh):
    b = Batch([45, 33, 21, 70], [1300, 900, 30, 72], heads=1, group=4, dim=128, bt=1, seed=39, layers=1)
    b.lens[1] = -1
    b.table_h[0][700], b.table_h[3][9] = -1, b.pages
    b.table = ints(b.table_h)
    out = b.run(kvh, 40).cpu().numpy()
    want = b.want(40)
    assert b.status.tolist() == [BAD, BAD, 0, BAD] and (out[45:78] == -9).all()
    assert np.array_equal(out[:45], want[:45]) and np.array_equal(out[78:], want[78:])


def test_selection_refusals(kvh):
    shape = dict(news=[1, 6, 2], lens=[400, 500, 170], heads=1, dim=64, seed=35)
    b = Batch(**shape)
    out = b.run(kvh, 5, max_new=2)
    assert b.status.tolist() == [0, BAD, 0] and (out[1:7] == -9).all() and (out[0] >= 0).all() and (out[7:] >= 0).all()
    b = Batch(**shape)
    b.lens[0], b.lens[1] = -1, 16 * b.table.shape[1] + 1
    out = b.run(kvh, 5)
    assert b.status.tolist() == [BAD, BAD, 0] and (out[:7] == -9).all()
    b = Batch(**shape)
    b.starts[3] = 10
    assert (b.run(kvh, 5)[7:] == -9).all() and b.status.tolist() == [0, 0, BAD]
    b = Batch(**shape)
    for r, j, bad in ((0, 0, -1), (0, 7, b.pages), (1, 31, 1 << 30), (2, 3, -2 ** 31)):  # among them pages that are always chosen
        b.table_h[r][j] = bad
    b.table = ints(b.table_h)
    b.check(kvh, 9, 2, 2)
    assert b.status.tolist() == [BAD, BAD, BAD]
    b.check(kvh, 60, 1, 1)


def test_selection_on_other_streams_and_in_graphs(kvh):
    b = Batch([1, 2], [3000, 41], heads=2, group=4, seed=36, layers=1)
    want = b.run(kvh, 33)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out, room = torch.empty_like(want), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    call = lambda: kvh.select_pages(b.q, b.codes, b.scale, 0, b.starts, b.lens, b.table, 2, 33, out=out, workspace=room)  # noqa: E731
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        b.q.copy_(torch.randn(b.q.shape).to(b.q.dtype))
        b.lens -= 7
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        b.lens_h = [n - 7 for n in b.lens_h]
        assert np.array_equal(out.cpu().numpy(), b.want(33)), i
