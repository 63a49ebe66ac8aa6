"""kvh_append against its definition: 16-bit caches within the rounding of the type of a 64-bit rotation, 8-bit caches bit for bit
against the fp32 steps that include/kvh.h spells out and within half a code of the 64-bit values."""
import numpy as np
import pytest

from oracle import serving_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BAD = 2  # KVH_DEV_BAD_REQUEST
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
CODE = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}  # rounding to nearest, relative


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


def rotation(n, rot):
    at = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
    return torch.from_numpy(np.concatenate([np.cos(at), np.sin(at)], 1).astype(np.float32))


class Batch:
    """Random requests with pages in random order; caches full of what earlier steps left there."""

    def __init__(self, news, befores, heads=2, dim=128, bt=16, layers=1, kind="16", dt="bf16", group=2, seed=0, pad=0):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.dt, self.bt, self.heads, self.dim, self.layers = kind, dt, bt, heads, dim, layers
        self.news, self.lens_h = list(news), [a + b for a, b in zip(news, befores)]
        self.starts_h = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        held = [-(-n // bt) for n in self.lens_h]
        self.pages = sum(held) + 3
        order = torch.randperm(self.pages, generator=g).to(torch.int32)
        self.table_h = torch.full((len(news), max(1, max(held)) + 2), -7, dtype=torch.int32)
        at = 0
        for b, h in enumerate(held):
            self.table_h[b, :h] = order[at:at + h]
            at += h
        T, c = int(self.starts_h[-1]), heads * dim

        def rows(ch):
            return (torch.randn((layers, T, ch + pad), generator=g) * torch.exp(torch.randn(ch + pad, generator=g))).to(DT[dt]).cuda()[..., :ch]

        self.k, self.v, self.q = rows(c), rows(c), rows(c * group)
        shape = (layers, self.pages, bt, c)
        self.ks = self.vs = None
        if kind == "16":
            self.kc, self.vc = (torch.randn(shape, generator=g).to(DT[dt]).cuda() for _ in range(2))
        else:
            make = (lambda: torch.randint(-127, 128, shape, generator=g).to(torch.int8)) if kind == "i8" else \
                (lambda: (torch.randn(shape, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn))
            self.kc, self.vc = make().cuda(), make().cuda()
            self.ks, self.vs = ((torch.rand((layers, self.pages, heads), generator=g) * 0.05).cuda() for _ in range(2))
        self.starts = torch.from_numpy(self.starts_h).cuda()
        self.lens = torch.tensor(self.lens_h, dtype=torch.int32).cuda()
        self.table = self.table_h.cuda()
        self.status = torch.zeros(len(news), dtype=torch.int32, device="cuda")

    def append(self, kvh, **kw):
        kw = dict(dict(head_dim=self.dim, k_scale=self.ks, v_scale=self.vs, status=self.status), **kw)
        return kvh.append(self.k, self.v, self.kc, self.vc, self.starts, self.lens, self.table, kw.pop("max_new", max(1, max(self.news))), **kw)


def turned32(x, pos, table, pairs):
    """[l][T][heads][d] fp32, every product and sum rounded: what the kernel computes, bit for bit."""
    x, half = x.clone(), table.shape[1] // 2
    c, s = table[pos, :half][:, None], table[pos, half:][:, None]
    rot = 2 * half
    y = x[..., :rot].unflatten(-1, (half, 2) if pairs else (2, half))
    a, b = y.unbind(-1 if pairs else -2)
    x[..., :rot] = torch.stack((a * c - b * s, b * c + a * s), -1 if pairs else -2).flatten(-2)
    return x


def coded32(x, old_codes, old_scale, batch, kind):
    """The 8-bit pages after x [l][T][heads][d] fp32 was appended: (codes as fp32, scales), by the steps of the definition."""
    codes, scale = old_codes.float().cpu().clone(), old_scale.cpu().clone()
    l, P, bt, _ = codes.shape
    codes = codes.unflatten(-1, (batch.heads, batch.dim))
    to_code = (lambda y: torch.round(y)) if kind == "i8" else (lambda y: y.to(torch.float8_e4m3fn).float())
    pages = {}
    for b, t, p, page, row in ref.slots(batch.starts_h, batch.lens_h, batch.table_h.tolist(), bt):
        pages.setdefault(page, []).append((t, row))
    for page, new in pages.items():
        ts, rows = [t for t, _ in new], [r for _, r in new]
        most = x[:, ts].abs().amax((1, 3))
        t = torch.where(most < 2.0 ** -100, torch.zeros(()), most * (1 / torch.tensor(ref.TOP[kind], dtype=torch.float32)))
        old = scale[:, page] if rows[0] > 0 else torch.zeros_like(t)
        now = torch.maximum(old, t)
        grew = (now > old) & (old > 0)
        rate = torch.where(grew, old / now, torch.ones(()))
        codes[:, page, :rows[0]] = torch.where(grew[:, None, :, None], to_code(codes[:, page, :rows[0]] * rate[:, None, :, None]), codes[:, page, :rows[0]])
        inv = torch.where(now > 0, 1.0 / now, torch.zeros(()))
        codes[:, page, rows] = to_code(x[:, ts] * inv[:, None, :, None])
        scale[:, page] = now
    return codes.flatten(-2), scale


def positions_of(batch):
    return torch.tensor([p for _, _, p in ref.tokens(batch.starts_h, batch.lens_h)], dtype=torch.long)


SHAPES = [
    dict(news=[1], befores=[0]),
    dict(news=[1], befores=[31], heads=8, group=4),
    dict(news=[1, 0, 1, 1], befores=[16, 5, 17, 0], heads=3, bt=16, group=1),
    dict(news=[37, 1, 130], befores=[3, 15, 0], heads=2, bt=16, dim=64),
    dict(news=[50, 9], befores=[20, 61], heads=1, bt=7, dim=128, layers=3),
    dict(news=[129], befores=[63], heads=5, bt=64, dim=64, pad=24),
    dict(news=[300, 2], befores=[100, 254], heads=2, bt=256, dim=128, pad=8),
    dict(news=[40], befores=[2], heads=2, bt=1, dim=128),
]


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_append(kvh, shape, kind, dt):
    s = SHAPES[shape]
    rot, pairs = [(128, False), (64, False), (64, True), (32, False), (16, True), (48, False), (0, False), (64, False)][shape]
    rot = min(rot, s.get("dim", 128))
    b = Batch(kind=kind, dt=dt, seed=shape, **s)
    old = [t.clone() if t is not None else None for t in (b.kc, b.vc, b.ks, b.vs)]
    table = rotation(max(b.lens_h) + 1, rot) if rot else None
    q_out = b.append(kvh, rotation=table.cuda() if rot else None, pairs=pairs, q=b.q)
    torch.cuda.synchronize()
    assert not b.status.any()
    pos = positions_of(b)
    split = lambda x: x.float().cpu().unflatten(-1, (-1, b.dim))  # noqa: E731
    k32 = turned32(split(b.k), pos, table, pairs) if rot else split(b.k)
    if not rot:
        assert torch.equal(q_out, b.q)
    else:
        want = turned32(split(b.q), pos, table, pairs).to(DT[dt])
        assert torch.equal(q_out.cpu(), want.flatten(-2))
        for layer in range(b.layers):  # and in 64 bits
            x = split(b.q)[layer].double().numpy()
            exact = np.stack([ref.rotate(x[t], int(pos[t]), table.numpy(), pairs) for t in range(len(pos))])
            bound = U[dt] * np.abs(exact) + 2.0 ** -22 * (np.abs(x).max(-1, keepdims=True) * 2) + 2.0 ** -25
            assert (np.abs(split(q_out)[layer].double().numpy() - exact) <= bound).all()
    for x, before, after, scale0, scale1 in ((k32, old[0], b.kc, old[2], b.ks), (split(b.v), old[1], b.vc, old[3], b.vs)):
        if kind == "16":
            want = before.cpu().clone()
            for r, t, p, page, row in ref.slots(b.starts_h, b.lens_h, b.table_h.tolist(), b.bt):
                want[:, page, row] = x[:, t].to(DT[dt]).flatten(-2)
            assert torch.equal(after.cpu().view(torch.int16), want.view(torch.int16))
            continue
        codes, scales = coded32(x, before, scale0, b, kind)
        assert torch.equal(scale1.cpu(), scales)
        assert torch.equal(after.cpu().float(), codes)
        for layer in range(b.layers):  # and in 64 bits
            exact = ref.page_scales(x[layer].double().numpy(), b.starts_h, b.lens_h, b.table_h.tolist(), b.bt, kind, scale0[layer].cpu().double().numpy())
            np.testing.assert_allclose(scale1[layer].cpu().double().numpy(), exact, rtol=2.0 ** -23 + 2.0 ** -40)  # two roundings
            value = after[layer].cpu().double().unflatten(-1, (b.heads, b.dim)).numpy() * scale1[layer].cpu().double().numpy()[:, None, :, None]
            for r, t, p, page, row in ref.slots(b.starts_h, b.lens_h, b.table_h.tolist(), b.bt):
                y, step = x[layer, t].double().numpy(), scale1[layer, page].cpu().double().numpy()[:, None]
                bound = step * (0.5 + 2.0 ** -14) if kind == "i8" else np.maximum(np.abs(y) * (2.0 ** -4 + 2.0 ** -20), step * (2.0 ** -10 + 2.0 ** -20))
                assert (np.abs(value[page, row] - y) <= bound).all()


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_page_grown_token_by_token(kvh, kind):
    """40 tokens of growing size, one call each, on pages of 16: every value stays within what its roundings allow - half a step of the
    scale of the call that stored it and of each scale that the page grew to since."""
    heads, dim, bt = 2, 128, 16
    g = torch.Generator().manual_seed(5)
    x = (torch.randn((40, heads * dim), generator=g) * torch.linspace(0.5, 4, 40)[:, None]).half().cuda()
    kc = torch.zeros((1, 4, bt, heads * dim), dtype=CODE[kind], device="cuda")
    vc, ks = torch.zeros_like(kc), torch.full((1, 4, heads), 9.0, device="cuda")  # stale scales: a page's first token replaces them
    vs = ks.clone()
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    loss = torch.zeros((40, heads), dtype=torch.float64)
    last = torch.zeros((4, heads), dtype=torch.float64)
    for i in range(40):
        row = x[i].view(1, 1, -1)
        kvh.append(row, row, kc, vc, starts, torch.tensor([i + 1], dtype=torch.int32, device="cuda"), table, 1, head_dim=dim, k_scale=ks, v_scale=vs)
        page, now = [2, 0, 3][i // bt], ks[0].cpu().double()
        top = now[page] * ref.TOP[kind]
        step = now[page] * (0.5 + 2.0 ** -14) if kind == "i8" else top * (2.0 ** -4 + 2.0 ** -20)
        grew = (now[page] != last[page])[None]
        loss[i - i % bt:i + 1] += torch.where(grew | (torch.arange(i - i % bt, i + 1) == i)[:, None], step, 0.0)
        last = now
    torch.cuda.synchronize()
    assert torch.equal(kc.view(torch.int8), vc.view(torch.int8)) and torch.equal(ks[0, [2, 0, 3]], vs[0, [2, 0, 3]])
    value = torch.stack([kc[0, [2, 0, 3][i // bt], i % bt].double().view(heads, dim) * ks[0, [2, 0, 3][i // bt]].double()[:, None] for i in range(40)]).cpu()
    assert ((value - x.double().cpu().view(40, heads, dim)).abs() <= loss[..., None]).all()
    assert (ks[0, 1] == 9.0).all()  # a page that no one appended to


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_zeros_and_tiny_values(kvh, kind):
    """Nothing but zeros, values below 2^-100, and a real token after them on the same page."""
    kc = torch.zeros((1, 1, 16, 64), dtype=CODE[kind], device="cuda")
    vc = torch.zeros_like(kc)
    ks, vs = torch.full((1, 1, 1), 3.0, device="cuda"), torch.full((1, 1, 1), 3.0, device="cuda")
    table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 1] = 2.0 ** -101
    kvh.append(x, x, kc, vc, starts, torch.tensor([2], dtype=torch.int32, device="cuda"), table, 2, head_dim=64, k_scale=ks, v_scale=vs)
    assert ks.item() == 0 and vs.item() == 0 and not kc.float().any()
    x.fill_(2.0)
    kvh.append(x[:, :1], x[:, :1], kc, vc, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"), table, 1,
               head_dim=64, k_scale=ks, v_scale=vs)
    assert ks.item() == np.float32(2.0) * (np.float32(1.0) / np.float32(ref.TOP[kind])) and (kc[0, 0, 2].float() == ref.TOP[kind]).all() and not kc[0, 0, :2].float().any()


def test_sixteen_bits_keep_every_pattern(kvh):
    """V and unrotated K are stored as they are, NaN and infinities included; rotated NaN stay NaN."""
    b = Batch([20], [5], heads=1, dim=64, kind="16", dt="fp16", seed=9)
    bits = torch.randint(-32768, 32768, b.k.shape, dtype=torch.int16).cuda()
    b.k = b.v = bits.view(torch.float16)
    b.append(kvh)
    got = torch.stack([b.kc[0, page, row] for _, _, _, page, row in ref.slots(b.starts_h, b.lens_h, b.table_h.tolist(), 16)])
    assert torch.equal(got.view(torch.int16), bits[0])
    table = rotation(64, 32).cuda()
    b.append(kvh, rotation=table)
    got = torch.stack([b.kc[0, page, row] for _, _, _, page, row in ref.slots(b.starts_h, b.lens_h, b.table_h.tolist(), 16)])
    want = turned32(b.k.float().cpu().unflatten(-1, (1, 64)), positions_of(b), table.cpu(), False).half().flatten(-2)[0]
    assert torch.equal(got.cpu().isnan(), want.isnan()) and torch.equal(got.cpu().nan_to_num(), want.nan_to_num())


def test_positions_in_place_and_other_stream(kvh):
    """Positions of the caller's (tokens of a cache whose middle was dropped keep their angles), q rotated in place, on a stream of its own."""
    b = Batch([6, 70], [10, 40], heads=2, dim=128, kind="16", dt="bf16", seed=11)
    table = rotation(5000, 128)
    pos = torch.randint(0, 5000, (76,), dtype=torch.int32)
    q0 = b.q.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert b.append(kvh, rotation=table.cuda(), positions=pos.cuda(), q=b.q, q_out=b.q, stream=side) is b.q
    side.synchronize()
    want = turned32(q0.float().cpu().unflatten(-1, (-1, 128)), pos.long(), table, False).bfloat16().flatten(-2)
    assert torch.equal(b.q.cpu(), want)
    k = turned32(b.k.float().cpu().unflatten(-1, (-1, 128)), pos.long(), table, False).bfloat16().flatten(-2)
    for _, t, _, page, row in ref.slots(b.starts_h, b.lens_h, b.table_h.tolist(), 16):
        assert torch.equal(b.kc[0, page, row].cpu(), k[0, t])


@pytest.mark.parametrize("kind", ["16", "i8"])
def test_what_the_device_refuses(kvh, kind):
    """Requests that break the call's limits are refused as a whole, tokens without a page or a position alone; the rest is served."""
    def fresh():
        b = Batch([3, 4, 20, 2], [0, 14, 8, 30], heads=1, dim=64, kind=kind, dt="bf16", seed=3)
        return b, [t.clone() for t in (b.kc, b.vc)]

    def unchanged(b, old, r):
        pages = b.table_h[r, :-(-b.lens_h[r] // 16)].long().cuda()
        return all(torch.equal(x[:, pages].view(torch.int8), y[:, pages].view(torch.int8)) for x, y in zip((b.kc, b.vc), old))

    b, old = fresh()
    b.append(kvh, max_new=4)  # request 2 brings 20
    assert b.status.tolist() == [0, 0, BAD, 0] and unchanged(b, old, 2) and not unchanged(b, old, 1) and not unchanged(b, old, 3)
    b, old = fresh()
    b.lens[0] = 2  # fewer tokens than new ones
    b.lens[3] = 16 * b.table.shape[1] + 1  # more than its row of the table has pages for
    b.append(kvh)
    assert b.status.tolist() == [BAD, 0, 0, BAD] and unchanged(b, old, 0) and unchanged(b, old, 3) and not unchanged(b, old, 2)
    b, old = fresh()
    b.starts[4] = 30  # past the packed rows
    b.starts[0] = -1
    b.append(kvh, max_new=50)
    assert b.status.tolist() == [BAD, 0, 0, BAD] and unchanged(b, old, 3)
    b, old = fresh()
    page = int(b.table[2, 1])
    b.table[2, 1] = b.pages  # no page of the cache
    b.table[1, 1] = -1
    b.append(kvh)
    assert b.status.tolist() == [0, BAD, BAD, 0]
    assert torch.equal(b.kc[:, page].view(torch.int8), old[0][:, page].view(torch.int8)) and not unchanged(b, old, 0)
    b, old = fresh()
    b.append(kvh, rotation=rotation(20, 16).cuda())  # positions 20 and on of requests 2 and 3 have no angles
    assert b.status.tolist() == [0, 0, BAD, BAD] and not unchanged(b, old, 1)
    page = int(b.table_h[3, 1])
    assert torch.equal(b.kc[:, page, 14:].view(torch.int8), old[0][:, page, 14:].view(torch.int8))  # their keys are not stored


def test_replayed_graph(kvh):
    """Captured once, replayed with the program's own work in between: every replay is what an eager call gives."""
    b = Batch([1, 1, 1], [17, 40, 3], heads=2, dim=128, kind="i8", dt="bf16", seed=21)
    table = rotation(64, 128).cuda()
    out = torch.empty_like(b.q)
    b.append(kvh, rotation=table, q=b.q, q_out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.append(kvh, rotation=table, q=b.q, q_out=out)
    mine = [t.clone() for t in (b.kc, b.vc, b.ks, b.vs)]
    for i in range(4):
        b.k.copy_(torch.randn(b.k.shape).to(b.k.dtype) * (i + 1))
        b.q.copy_(torch.randn(b.q.shape).to(b.q.dtype))
        b.lens += 1
        graph.replay()
        torch.cuda.synchronize()
        want = kvh.append(b.k, b.v, mine[0], mine[1], b.starts, b.lens, b.table, 1, head_dim=128, k_scale=mine[2], v_scale=mine[3], q=b.q, rotation=table)
        for x, y in zip((b.kc, b.vc, b.ks, b.vs, out), (*mine, want)):
            assert torch.equal(x.view(torch.int8), y.view(torch.int8)), i
