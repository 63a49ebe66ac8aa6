"""kvh_attention_pages against a plain 64-bit implementation, with the bounds of test_gpu_serving_attention (the arithmetic is the same)."""
import math

import numpy as np
import pytest

from oracle import pages_ref as ref
from test_gpu_serving_attention import BAD, U, Batch

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


class Listed(Batch):
    """A batch with a random list of pages for each token and head: some empty, some without the token's own page, some all pages."""

    def choose(self, count, seed=0, full=False):
        g = np.random.default_rng(seed)
        self.lists = np.full((self.q.shape[0], self.heads, count), -1, dtype=np.int32)
        for b, n in enumerate(self.news):
            for i in range(n):
                p = self.lens_h[b] - n + i
                for h in range(self.heads):
                    have = p // self.bt + 1 if p >= 0 else 0
                    k = min(have, count) if full else int(g.integers(0, min(have, count) + 1))
                    self.lists[self.starts_h[b] + i, h, :k] = np.sort(g.permutation(have)[:k])
        self.chosen = torch.from_numpy(self.lists).cuda()
        return self

    def run(self, kvh, **kw):
        kw = dict(dict(head_dim=self.dim, k_scale=self.ks, v_scale=self.vs, status=self.status), **kw)
        self.lse = torch.full((self.q.shape[0], self.heads * self.group), 7.0, device="cuda")
        return kvh.attention_pages(self.q, self.kc, self.vc, self.layer, self.chosen, self.starts, self.lens, self.table, kw.pop("max_new", max(1, max(self.news))),
                                   lse=self.lse, **kw)

    def check(self, out, scale=None):
        q = self.q.double().cpu().unflatten(-1, (-1, self.dim)).numpy()
        scale = self.dim ** -0.5 if scale is None else scale
        want, lse, size, worth, total = ref.attention(q, self.values(0), self.values(1), self.starts_h, self.lens_h, self.table_h.tolist(), self.bt, scale, self.lists)
        e = (self.dim * 2.0 ** -23 * worth)[..., None]
        p = U[self.dt] if self.kind == "16" else 2.0 ** -11
        got = out.double().cpu().unflatten(-1, (-1, self.dim)).numpy()
        with np.errstate(invalid="ignore"):
            bound = U[self.dt] * np.abs(want) + (p + 2 * e + 2.0 ** -16) * size + 2.0 ** -24 * total + (2.0 ** -24 if self.dt == "fp16" else 2.0 ** -130)
            off = np.abs(got - want)
            fine = (off <= bound) | (np.isnan(want) & np.isnan(got)) | (want == got)
            assert fine.all(), (off[~fine].max(), bound[~fine].min(), np.argwhere(~fine)[:5])
            of = self.lse.double().cpu().numpy()
            close = (np.abs(of - lse) <= e[..., 0] + 2.0 ** -20 * (1 + np.abs(lse))) | (np.isneginf(of) & np.isneginf(lse)) | (np.isnan(of) & np.isnan(lse))
            assert close.all(), (np.abs(of - lse)[~close].max(), np.argwhere(~close)[:5])


SHAPES = [
    dict(news=[1], lens=[1]),
    dict(news=[1], lens=[16], heads=8, group=4),
    dict(news=[1, 1, 1], lens=[33, 700, 15], heads=2, group=1),
    dict(news=[1, 0, 1, 1], lens=[257, 9, 1, 1300], heads=1, group=8, dim=64),
    dict(news=[5, 2], lens=[41, 900], heads=2, group=7, dim=64, bt=24),
    dict(news=[3, 1], lens=[100, 64], heads=2, group=20, dim=128, bt=32, pad=16),
    dict(news=[40], lens=[40], heads=1, group=3, dim=128, bt=7),
    dict(news=[70, 1, 17], lens=[130, 77, 400], heads=2, group=4, dim=128),
    dict(news=[9], lens=[4], heads=2, group=2, dim=128),  # more queries than tokens: the first ones see nothing
    dict(news=[2, 2], lens=[0, 3], heads=2, group=2, dim=64),
    dict(news=[11], lens=[70], heads=1, group=40, dim=64, bt=1),
    dict(news=[2], lens=[700], heads=2, group=3, dim=128, bt=256),
]


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_lists(kvh, shape, kind, dt):
    b = Listed(kind=kind, dt=dt, seed=shape, **SHAPES[shape]).choose(9, shape)
    b.check(b.run(kvh))
    b.choose(70, shape)
    b.check(b.run(kvh, scale=0.31), scale=0.31)
    assert not b.status.any()


@pytest.mark.parametrize("kind,dt", [("16", "bf16"), ("16", "fp16"), ("i8", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("workspace", [0, 1 << 17, None])
def test_long_lists_split(kvh, kind, dt, workspace):
    """All the room for parts, some of it, and none."""
    b = Listed([1, 1, 2, 1], [9001, 5, 4099, 6000], heads=2, group=4, kind=kind, dt=dt, seed=7, layers=1).choose(600, 1)
    room = None if workspace is None else torch.full((workspace,), 255, dtype=torch.uint8, device="cuda")
    b.check(b.run(kvh, workspace=room))
    assert not b.status.any()


@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
def test_all_pages_are_the_dense_attention(kvh, kind):
    b = Listed([1, 7], [600, 300], heads=2, group=4, kind=kind, dt="bf16", seed=8).choose(64, full=True)
    Batch.check(b, b.run(kvh))  # the bound of attention over the whole request


def test_many_requests(kvh):
    g = np.random.default_rng(3)
    news = [int(x) for x in g.integers(0, 3, 150)]
    lens = [n + int(x) for n, x in zip(news, g.integers(0, 90, 150))]
    b = Listed(news, lens, heads=1, group=2, dim=64, kind="i8", dt="fp16", seed=4, layers=1).choose(4, 2)
    b.check(b.run(kvh))


@pytest.mark.parametrize("kind", ["16", "e4m3"])
def test_odd_values_stay_where_they_are_listed(kvh, kind):
    """NaN and infinities on a page that some tokens list and others do not, and behind a token on its own page."""
    for bad in ([math.nan, math.inf, -math.inf] if kind == "16" else [math.nan]):
        for which in (0, 1):
            ever = False
            for p in (199, 195, 90):
                b = Listed([20], [200], heads=2, group=2, dim=64, kind=kind, dt="fp16", seed=6, layers=1).choose(13, 5)
                cache = (b.kc, b.vc)[which]
                raw = torch.tensor([bad]).to(cache.dtype).view(torch.int16 if kind == "16" else torch.int8)
                clean = b.run(kvh).view(20, 2, 2, 64).clone()
                cache.view(raw.dtype)[0, int(b.table_h[0, p // 16]), p % 16, 3] = raw.item()  # of head 0
                got = b.run(kvh).view(20, 2, 2, 64)
                sees = torch.tensor([[h == 0 and p // 16 in b.lists[t, h] and p <= 180 + t for h in range(2)] for t in range(20)], device="cuda")
                same = (got == clean) | (got.isnan() & clean.isnan())
                assert same[~sees].all()
                ever |= bool(sees.any())
                assert not got[sees][..., 3].isfinite().any() if which == 1 else (not math.isnan(bad) or got[sees].isnan().all())
            assert ever


def test_scales_that_are_no_numbers(kvh):
    b = Listed([6], [200], heads=1, group=2, dim=64, kind="i8", dt="bf16", seed=9, layers=1).choose(13, 3)
    page = int(b.table_h[0, 4])
    sees = torch.tensor([4 in b.lists[t, 0] for t in range(6)], device="cuda")
    assert sees.any() and not sees.all()
    for z in (math.nan, math.inf):
        for s in (b.ks, b.vs):
            keep = s.clone()
            want = b.run(kvh)
            s[0, page] = z
            got = b.run(kvh)
            assert torch.equal(got[~sees], want[~sees]) and got[sees].isnan().all()
            s.copy_(keep)


def test_lists_that_break_the_rules(kvh):
    """A list ends at an entry that is not larger than the one before or lies past the token's own page, and says so."""
    b = Listed([2, 1, 1, 1], [100, 200, 50, 60], heads=1, group=2, dim=64, kind="16", dt="fp16", seed=10, layers=1).choose(6, full=True)
    lists = np.array([[0, 3, 3, 5, -1, -1], [1, 2, 6, -1, 4, -1], [5, 2, 7, 8, 9, 10], [1, 4, 2, -1, -1, -1], [0, 2 ** 31 - 1, 3, -1, -1, -1]])
    b.chosen = torch.from_numpy(lists.astype(np.int32)).cuda().view(5, 1, 6)
    kept = [[0, 3], [1, 2, 6], [5], [1], [0]]  # request 2 has pages 0 .. 3 only
    b.lists = np.array([k + [-1] * (6 - len(k)) for k in kept]).reshape(5, 1, 6)
    b.check(b.run(kvh))
    assert b.status.tolist() == [BAD, BAD, BAD, BAD]
    b = Listed([1], [100], heads=1, group=2, dim=64, kind="16", dt="fp16", seed=10, layers=1).choose(4)
    b.chosen[0, 0] = torch.tensor([7, 1, 2, 3])  # nothing is left: as a token that sees nothing
    out = b.run(kvh)
    assert not out.any() and torch.isneginf(b.lse).all() and b.status.tolist() == [BAD]


def test_device_refusals(kvh):
    def fresh():
        return Listed([1, 6, 2], [40, 50, 17], heads=1, group=2, dim=64, kind="i8", dt="bf16", seed=16, layers=1).choose(3, full=True)

    b = fresh()
    out = torch.full(b.q.shape, 5.0, dtype=b.q.dtype, device="cuda")
    b.run(kvh, max_new=2, out=out)
    assert b.status.tolist() == [0, BAD, 0] and (out[1:7] == 5).all() and (b.lse[1:7] == 7).all() and not (out[0] == 5).any() and not (out[7:] == 5).any()
    b = fresh()
    b.lens[0], b.lens[1] = -1, 16 * b.table.shape[1] + 1
    b.run(kvh, out=out.fill_(5.0))
    assert b.status.tolist() == [BAD, BAD, 0] and (out[:7] == 5).all() and not (out[7:] == 5).any()
    b = fresh()
    b.starts[3] = 8  # a row behind the last sequence
    b.run(kvh, out=out.fill_(5.0))
    assert not b.status.any() and (out[8] == 5).all() and not (out[7] == 5).any()
    b = fresh()
    b.table[0, 1], b.table[1, 3] = -1, b.pages  # tokens on them are not seen
    out = b.run(kvh)
    assert b.status[0] == BAD and out.isfinite().all()
    b = fresh()
    b.table[2, :] = b.pages  # nothing else to see
    assert b.run(kvh)[7:].isnan().all() and b.status.tolist() == [0, 0, BAD]


def test_other_stream_and_graph(kvh):
    b = Listed([1, 1], [3000, 41], heads=2, group=4, kind="e4m3", dt="bf16", seed=17, layers=1).choose(128, full=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = b.run(kvh)
    torch.cuda.synchronize()
    got = b.run(kvh, stream=side)
    side.synchronize()
    assert torch.equal(want, got)
    out, room, chosen = torch.empty_like(b.q), torch.empty(1 << 22, dtype=torch.uint8, device="cuda"), b.chosen
    call = lambda: kvh.attention_pages(b.q, b.kc, b.vc, 0, chosen, b.starts, b.lens, b.table, 1, k_scale=b.ks, v_scale=b.vs, out=out, workspace=room)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        b.q.copy_(torch.randn(b.q.shape).to(b.q.dtype))
        b.lens -= 7
        b.lens_h = [n - 7 for n in b.lens_h]
        chosen.copy_(b.choose(128, 60 + i).chosen)
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, b.run(kvh)), i
        b.check(out)


def test_two_streams_at_once(kvh):
    """Two calls under way together, each with a workspace of its own."""
    many = [Listed([1], [5000 + i], heads=2, group=4, kind="16", dt="bf16", seed=20 + i, layers=1).choose(200, full=True) for i in range(2)]
    want = [b.run(kvh) for b in many]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in many]
    got = [[], []]
    for _ in range(5):
        for b, side, to in zip(many, sides, got):
            to.append(b.run(kvh, stream=side))
    torch.cuda.synchronize()
    for w, to in zip(want, got):
        assert all(torch.equal(w, x) for x in to)
