"""kvh_attention against a plain 64-bit implementation of its formula.

The bound of an output element o = sum w v / sum w, with u the rounding of the output's type, p that of the weights (fp16: 2^-11; bf16
caches: 2^-8) and e what the fp32 exponents may be off (a dot product of d terms in fp32, scaled: d 2^-23 of sum |q||k|):
  u |o| + (p + 2 e + 2^-16) (sum w |v| / sum w) + 2^-24 sum |v| (weights that fp16 holds as subnormals) + the type's smallest step
The logarithm of the sum: e + 2^-20 (1 + |lse|)."""
import math

import numpy as np
import pytest

from oracle import serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BAD = 2  # KVH_DEV_BAD_REQUEST
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


class Batch:
    """Random queries over a random cache; what no request holds is NaN (16 bits, e4m3) or full scale, and its table entries are none."""

    def __init__(self, news, lens, heads=2, group=2, dim=128, bt=16, kind="16", dt="bf16", seed=0, pad=0, layers=2, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.dt, self.bt, self.heads, self.dim, self.group, self.layer = kind, dt, bt, heads, dim, group, layers - 1
        self.news, self.lens_h = list(news), list(lens)
        self.starts_h = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        held = [-(-n // bt) for n in lens]
        self.pages = sum(held) + 2
        order = torch.randperm(self.pages, generator=g).to(torch.int32)
        self.table_h = torch.full((len(news), max(1, max(held)) + 1), 1 << 30, dtype=torch.int32)
        T, c = int(self.starts_h[-1]), heads * dim
        mine, at = torch.zeros((self.pages, bt), dtype=torch.bool), 0
        for b, h in enumerate(held):
            self.table_h[b, :h] = order[at:at + h]
            at += h
            for p in range(lens[b]):
                mine[int(self.table_h[b, p // bt]), p % bt] = True
        shape = (layers, self.pages, bt, c)
        self.q = (torch.randn((T, c * group + pad), generator=g) * spread).to(DT[dt]).cuda()[:, :c * group]
        self.ks = self.vs = None
        made = []
        for _ in range(2):
            x = torch.randn(shape, generator=g) * torch.exp(0.5 * torch.randn(c, generator=g))
            if kind == "16":
                x = x.to(DT[dt])
            elif kind == "i8":
                x = (x * 30).round().clamp(-127, 127).to(torch.int8)
            else:
                x = (x * 90).clamp(-448, 448).to(torch.float8_e4m3fn)
            if kind == "i8":
                x[:, ~mine] = 127
            else:
                raw = x.view(torch.int16 if kind == "16" else torch.int8)
                raw[:, ~mine] = 0x7fff if kind == "16" else 0x7f
            if pad:
                wide = torch.zeros(shape[:3] + (c + 2 * pad,), dtype=torch.int16 if kind == "16" else torch.int8).view(x.dtype).cuda()
                wide.view(torch.int16 if kind == "16" else torch.int8)[..., :c] = x.view(torch.int16 if kind == "16" else torch.int8).cuda()
                made.append(wide[..., :c])
            else:
                made.append(x.cuda())
        self.kc, self.vc = made
        if kind != "16":
            self.ks, self.vs = ((torch.exp(0.7 * torch.randn((layers, self.pages, heads), generator=g)) / (30 if kind == "i8" else 90)).cuda() for _ in range(2))
        self.starts = torch.from_numpy(self.starts_h).cuda()
        self.lens = torch.tensor(self.lens_h, dtype=torch.int32).cuda()
        self.table = self.table_h.cuda()
        self.status = torch.zeros(len(news), dtype=torch.int32, device="cuda")

    def values(self, which):
        x = (self.kc, self.vc)[which][self.layer].float().cpu().double().unflatten(-1, (self.heads, self.dim))
        s = (self.ks, self.vs)[which]
        return (x if s is None else x * s[self.layer].cpu().double()[:, None, :, None]).numpy()

    def run(self, kvh, **kw):
        kw = dict(dict(head_dim=self.dim, k_scale=self.ks, v_scale=self.vs, status=self.status), **kw)
        self.lse = torch.full((self.q.shape[0], self.heads * self.group), 7.0, device="cuda")
        return kvh.attention(self.q, self.kc, self.vc, self.layer, self.starts, self.lens, self.table, kw.pop("max_new", max(1, max(self.news))), lse=self.lse, **kw)

    def check(self, out, scale=None, **mask):
        q = self.q.double().cpu().unflatten(-1, (-1, self.dim)).numpy()
        scale = self.dim ** -0.5 if scale is None else scale
        want, lse, size, worth, total = ref.attention(q, self.values(0), self.values(1), self.starts_h, self.lens_h, self.table_h.tolist(), self.bt, scale, **mask)
        e = (self.dim * 2.0 ** -23 * worth)[..., None]
        p = U[self.dt] if self.kind == "16" else 2.0 ** -11
        with np.errstate(invalid="ignore"):
            bound = U[self.dt] * np.abs(want) + (p + 2 * e + 2.0 ** -16) * size + 2.0 ** -24 * total + (2.0 ** -24 if self.dt == "fp16" else 2.0 ** -130)
            off = np.abs(out.double().cpu().unflatten(-1, (-1, self.dim)).numpy() - want)
            blind = np.isneginf(lse)
            fine = (off <= bound) | (np.isnan(want) & np.isnan(out.float().cpu().unflatten(-1, (-1, self.dim)).numpy())) | (want == out.double().cpu().unflatten(-1, (-1, self.dim)).numpy())
            assert fine.all(), (off[~fine].max(), bound[~fine].min(), np.argwhere(~fine)[:5])
            got = self.lse.double().cpu().numpy()
            close = (np.abs(got - lse) <= e[..., 0] + 2.0 ** -20 * (1 + np.abs(lse))) | (np.isneginf(got) & blind) | (np.isnan(got) & np.isnan(lse))
            assert close.all(), (np.abs(got - lse)[~close].max(), np.argwhere(~close)[:5])


SHAPES = [
    dict(news=[1], lens=[1]),
    dict(news=[1], lens=[16], heads=8, group=4),
    dict(news=[1, 1, 1], lens=[33, 700, 15], heads=2, group=1),
    dict(news=[1, 0, 1, 1], lens=[257, 9, 0 + 1, 1300], heads=1, group=8, dim=64),
    dict(news=[5, 2], lens=[41, 900], heads=2, group=7, dim=64, bt=24),
    dict(news=[3, 1], lens=[100, 64], heads=2, group=20, dim=128, bt=32, pad=16),
    dict(news=[40], lens=[40], heads=1, group=3, dim=128, bt=7),
    dict(news=[130, 1, 17], lens=[130, 77, 400], heads=2, group=4, dim=128),
    dict(news=[65], lens=[500], heads=3, group=2, dim=64, bt=256),
    dict(news=[9], lens=[4], heads=2, group=2, dim=128),  # more queries than tokens: the first ones see nothing
    dict(news=[2, 2], lens=[0, 3], heads=2, group=2, dim=64),
    dict(news=[33], lens=[70], heads=1, group=1, dim=64, bt=1),
]


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_causal(kvh, shape, kind, dt):
    b = Batch(kind=kind, dt=dt, seed=shape, **SHAPES[shape])
    b.check(b.run(kvh))
    assert not b.status.any()


@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("shape", [2, 4, 7, 8, 9, 10])
def test_all_tokens_seen(kvh, shape, kind):
    b = Batch(kind=kind, dt="fp16", seed=50 + shape, **SHAPES[shape])
    b.check(b.run(kvh, causal=False, scale=0.31), causal=False, scale=0.31)


@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("sink,window", [(0, 1), (4, 16), (64, 100), (40, 33), (0, 5000)])
@pytest.mark.parametrize("shape", [2, 3, 4, 7, 8])
def test_window(kvh, shape, sink, window, kind):
    b = Batch(kind=kind, dt="bf16", seed=80 + shape, **SHAPES[shape])
    b.check(b.run(kvh, sink=sink, window=window), sink=sink, window=window)
    assert not b.status.any()


@pytest.mark.parametrize("kind,dt", [("16", "bf16"), ("16", "fp16"), ("i8", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("workspace", [0, 1 << 16, None])
def test_long_and_split(kvh, kind, dt, workspace):
    """Long requests beside short ones, with all the room for parts, some of it, and none: the same results."""
    b = Batch([1, 1, 2, 1], [9001, 5, 4099, 12345], heads=2, group=4, kind=kind, dt=dt, seed=7, layers=1)
    room = None if workspace is None else torch.empty(workspace, dtype=torch.uint8, device="cuda")
    b.check(b.run(kvh, workspace=room))


@pytest.mark.parametrize("kind", ["16", "i8"])
def test_many_requests(kvh, kind):
    """More requests than a wave has lanes, some without tokens."""
    g = np.random.default_rng(3)
    news = [int(x) for x in g.integers(0, 3, 150)]
    lens = [n + int(x) for n, x in zip(news, g.integers(0, 90, 150))]
    b = Batch(news, lens, heads=1, group=2, dim=64, kind=kind, dt="fp16", seed=4, layers=1)
    b.check(b.run(kvh))


@pytest.mark.parametrize("kind", ["16", "e4m3"])
@pytest.mark.parametrize("news,lens", [([6], [40]), ([70], [200]), ([1], [64])])
def test_odd_values_stay_where_they_are_seen(kvh, kind, news, lens):
    """NaN and infinities among the values: rows that do not see them give what they give without, rows that do give what the
    formula gives; the same for keys."""
    for bad in ([math.nan, math.inf, -math.inf] if kind == "16" else [math.nan]):
        for which in (0, 1):
            for p in (lens[0] - 1, lens[0] - 3, max(0, lens[0] - 40)):
                b = Batch(news, lens, heads=1, group=2, dim=64, kind=kind, dt="fp16", seed=6, layers=1)
                cache = (b.kc, b.vc)[which]
                raw = torch.tensor([bad]).to(cache.dtype).view(torch.int16 if kind == "16" else torch.int8)
                cache.view(raw.dtype)[0, int(b.table_h[0, p // 16]), p % 16, 3] = raw.item()
                out = b.run(kvh)
                first = max(0, p - (lens[0] - news[0]))  # the first row that sees it
                plain = Batch(news, lens, heads=1, group=2, dim=64, kind=kind, dt="fp16", seed=6, layers=1)
                clean = plain.run(kvh)
                got, was = out.float().unflatten(-1, (2, 64)), clean.float().unflatten(-1, (2, 64))
                assert torch.allclose(got[:first], was[:first], rtol=2.0 ** -9, atol=2.0 ** -9) and not got[:first].isnan().any()
                if which == 1:
                    assert torch.allclose(got[first:, :, :3], was[first:, :, :3], rtol=2.0 ** -9, atol=2.0 ** -9)
                    assert not got[first:, :, 3].isfinite().any()
                elif math.isnan(bad):
                    assert got[first:].isnan().all()


def test_scales_far_apart(kvh):
    """Pages whose values are all zero, tiny and large next to each other: the weights keep their precision."""
    b = Batch([1, 4], [200, 90], heads=2, group=2, dim=128, kind="i8", dt="bf16", seed=13, layers=1)
    g = torch.Generator().manual_seed(1)
    b.vs.copy_(torch.exp2(torch.randint(-50, 12, b.vs.shape, generator=g).float()).cuda())
    b.vs[0, int(b.table_h[0, 2])] = 0.0
    b.check(b.run(kvh))
    b.vs[0, :] = 0.0
    out = b.run(kvh)
    b.check(out)
    assert not out.any()


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 30])
def test_queries_of_any_size(kvh, size):
    """bf16 queries beyond fp16's range, over codes whose scales make up for them."""
    b = Batch([3], [77], heads=2, group=2, dim=128, kind="e4m3", dt="bf16", seed=14, layers=1, spread=size)
    b.ks /= size
    b.check(b.run(kvh))


def test_rows_that_see_equal_scores_and_large_ones(kvh):
    """Scores of +-3000 (the softmax is one token) and all equal (the mean)."""
    b = Batch([2], [300], heads=1, group=1, dim=64, kind="16", dt="fp16", seed=15, layers=1, spread=100.0)
    b.check(b.run(kvh, scale=3.0), scale=3.0)
    b.check(b.run(kvh, scale=0.0), scale=0.0)


def test_device_refusals(kvh):
    def fresh():
        return Batch([1, 6, 2], [40, 50, 17], heads=1, group=2, dim=64, kind="i8", dt="bf16", seed=16, layers=1)

    b = fresh()
    out = torch.full(b.q.shape, 5.0, dtype=b.q.dtype, device="cuda")
    b.run(kvh, max_new=2, out=out)
    assert b.status.tolist() == [0, BAD, 0] and (out[1:7] == 5).all() and (b.lse[1:7] == 7).all() and not (out[0] == 5).any() and not (out[7:] == 5).any()
    b = fresh()
    b.lens[0], b.lens[1] = -1, 16 * b.table.shape[1] + 1
    b.run(kvh, out=out.fill_(5.0))
    assert b.status.tolist() == [BAD, BAD, 0] and (out[:7] == 5).all() and not (out[7:] == 5).any()
    b = fresh()
    b.starts[3] = 10
    b.run(kvh, out=out.fill_(5.0))
    assert b.status.tolist() == [0, 0, BAD] and (out[7:] == 5).all()
    b = fresh()
    b.table[0, 1], b.table[1, 3] = -1, b.pages  # tokens on them are not seen
    keep = b.table_h.clone()
    out = b.run(kvh)
    assert b.status.tolist() == [BAD, BAD, 0]
    b.status.zero_()
    assert out.isfinite().all()
    b = fresh()
    b.table[0, 0] = -1  # a page that the window does not reach is none of the call's business
    mask = dict(window=8)
    out = b.run(kvh, **mask)
    assert not b.status.any()
    b.table_h = keep
    b.check(out, **mask)


def test_other_stream_and_graph(kvh):
    """On a stream of its own, then captured and replayed after changes of the inputs: every replay is what an eager call gives."""
    b = Batch([1, 1], [3000, 41], heads=2, group=4, kind="e4m3", dt="bf16", seed=17, layers=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = b.run(kvh)
    torch.cuda.synchronize()
    got = b.run(kvh, stream=side)
    side.synchronize()
    assert torch.equal(want, got)
    out, room = torch.empty_like(b.q), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    call = lambda: kvh.attention(b.q, b.kc, b.vc, 0, b.starts, b.lens, b.table, 1, k_scale=b.ks, v_scale=b.vs, out=out, workspace=room)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        b.q.copy_(torch.randn(b.q.shape).to(b.q.dtype))
        b.lens -= 7
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, b.run(kvh)), i
        b.lens_h = [n - 7 for n in b.lens_h]
        b.check(out) if i == 3 else None


def test_pages_beyond_32_bits(kvh):
    """A cache of more than 4 GiB whose pages in use lie past that."""
    pages, bt, c = 600_000, 16, 512
    kc = torch.zeros((1, pages, bt, c), dtype=torch.int8, device="cuda")
    vc = torch.zeros_like(kc)
    ks = torch.ones((1, pages, 4), device="cuda")
    b = Batch([1], [100], heads=4, group=2, dim=128, kind="i8", dt="bf16", seed=18, layers=1)
    far = torch.arange(pages - b.pages, pages, dtype=torch.int32)
    kc[:, far.long().cuda()], vc[:, far.long().cuda()] = b.kc, b.vc
    ks[:, far.long().cuda()] = b.ks
    vs = ks.clone()
    vs[:, far.long().cuda()] = b.vs
    table = torch.where(b.table < b.pages, b.table + (pages - b.pages), b.table)
    want = b.run(kvh)
    got = kvh.attention(b.q, kc, vc, 0, b.starts, b.lens, table, 1, k_scale=ks, v_scale=vs)
    assert torch.equal(want, got)
    x = torch.randn((1, 1, c)).bfloat16().cuda()
    kvh.append(x, x, kc, vc, b.starts, torch.tensor([1], dtype=torch.int32, device="cuda"), far[-1:].view(1, 1).cuda(), 1, k_scale=ks, v_scale=vs)
    assert (kc[0, -1, 0].float().abs().view(4, 128).amax(-1) == 127).all() and not kc[0, 0].any()
