"""The serving cache's calls at the ends of what they take.  Tolerances are those of test_gpu_serving_attention.py."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import test_gpu_serving_append as appending  # noqa: E402
from test_gpu_serving_attention import Batch  # noqa: E402

BAD = 2  # KVH_DEV_BAD_REQUEST
TOP = 2 ** 31 - 1


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


# ---- scales that are no finite numbers: their pages hold NaN -------------------------------------------------------
# new tokens, whole pages before the last token's, for few rows of a KV head, pairs of row tiles, and many rows
ROWS = [([2], 4), ([10], 5), ([40], 9), ([150], 21)]
ODD = [math.nan, math.inf]


def scaled(rows, kind, bt, dim=64, dt="bf16", seed=71):
    news, pages = ROWS[rows]
    return Batch(news, [pages * bt + 1], heads=2, group=2, dim=dim, bt=bt, kind=kind, dt=dt, seed=seed, layers=1)  # the last token has a page of its own


def spoil(b, which, page, value):
    """Of one head of the first request."""
    (b.ks, b.vs)[which][0, int(b.table_h[0, page]), 0] = value


def check(b, out, **mask):
    for s in (b.ks, b.vs):
        s.masked_fill_(s.isinf(), math.nan)
    b.check(out, **mask)


def some_rows_see(kvh, kind, bt, rows, value, which):
    """The last token's page, or one in the middle of the new tokens: the rows before are as exact as ever, the others NaN (from a V scale the outputs, and
    not the logarithm of the sum)."""
    for dim in (64, 128):
        for back in (0, 1):
            b = scaled(rows, kind, bt, dim)
            spoil(b, which, ROWS[rows][1] - back, value)
            check(b, b.run(kvh))
            assert not b.status.any()


def no_row_sees(kvh, kind, bt, rows, value, which):
    """Pages between sink and window share steps with pages that are seen."""
    for mask in (dict(window=9), dict(window=9, sink=3)):
        b = scaled(rows, kind, bt)
        for page in range(1 if "sink" in mask else 0, (b.lens_h[0] - b.news[0] - 9) // bt):
            spoil(b, which, page, value)
        check(b, b.run(kvh, **mask), **mask)


def another_owns(kvh, kind, bt, rows, value, which):
    """Tokens on no page of the cache: what page 0, which is none of the request's, holds does not matter."""
    seed = next(s for s in range(100, 200) if 0 not in scaled(rows, kind, bt, seed=s).table_h[0, :ROWS[rows][1] + 1].tolist())
    outs = []
    for scale in (1.0, value):
        b = scaled(rows, kind, bt, seed=seed)
        b.table[0, 1] = -1
        (b.ks, b.vs)[which][0, 0] = scale
        outs.append((b.run(kvh), b.lse))
        assert b.status.tolist() == [BAD] and outs[-1][0].isfinite().all()
        assert torch.equal(outs[-1][0], outs[0][0]) and torch.equal(outs[-1][1], outs[0][1])


def scales_of_zero_beside(kvh, kind, bt, rows, value, which):
    """Zero, next to zero and no number in neighbouring pages."""
    b = scaled(rows, kind, bt)
    last = ROWS[rows][1]
    spoil(b, which, last - 2, 0.0)
    spoil(b, which, last - 1, 2.0 ** -70)
    spoil(b, which, last, value)
    check(b, b.run(kvh))


WAYS = [some_rows_see, no_row_sees, another_owns, scales_of_zero_beside]


@pytest.mark.parametrize("value", ODD)
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("bt", [16, 24])
@pytest.mark.parametrize("rows", range(len(ROWS)))
@pytest.mark.parametrize("way", WAYS)
def test_v_scale(kvh, way, rows, bt, kind, value):
    way(kvh, kind, bt, rows, value, 1)


@pytest.mark.parametrize("value", ODD)
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("news", [[1], [90]])
def test_v_scale_where_the_batch_is_cut(kvh, kind, news, value):
    b = Batch(news, [4001], heads=2, group=2, dim=64, kind=kind, dt="fp16", seed=73, layers=1)
    spoil(b, 1, 2000 // 16, value)
    check(b, b.run(kvh, window=200), window=200)
    spoil(b, 1, 4000 // 16, value)
    check(b, b.run(kvh))


@pytest.mark.parametrize("value", ODD)
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("bt", [16, 24])
@pytest.mark.parametrize("rows", range(len(ROWS)))
@pytest.mark.parametrize("way", WAYS)
def test_k_scale(kvh, way, rows, bt, kind, value):
    way(kvh, kind, bt, rows, value, 0)


@pytest.mark.parametrize("value", ODD)
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("news", [[1], [90]])
def test_k_scale_where_the_batch_is_cut(kvh, kind, news, value):
    b = Batch(news, [4001], heads=2, group=2, dim=64, kind=kind, dt="fp16", seed=75, layers=1)
    spoil(b, 0, 2000 // 16, value)
    check(b, b.run(kvh, window=200), window=200)
    spoil(b, 0, 4000 // 16, value)
    check(b, b.run(kvh))


# ---- workspace ------------------------------------------------------------------------------------------------------
def test_a_long_prompt_takes_no_memory_for_parts(kvh):
    b = Batch([8192], [8192], heads=2, group=4, dim=64, kind="i8", dt="bf16", seed=77, layers=1)
    q = b.q.repeat(1, 4)  # 8 heads of 64 channels, 32 query heads
    kc, vc = b.kc.repeat(1, 1, 1, 4), b.vc.repeat(1, 1, 1, 4)
    ks, vs = b.ks.repeat(1, 1, 4), b.vs.repeat(1, 1, 4)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out = kvh.attention(q, kc, vc, 0, b.starts, b.lens, b.table, 8192, head_dim=64, k_scale=ks, v_scale=vs)
    assert torch.cuda.max_memory_allocated() - before <= out.numel() * 2 + (1 << 20)
    want = kvh.attention(b.q, b.kc, b.vc, 0, b.starts, b.lens, b.table, 8192, head_dim=64, k_scale=b.ks, v_scale=b.vs,
                         workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))  # whole tiles too
    assert torch.equal(out[:, :512], want) and torch.equal(out[:, -512:], want)


# ---- limits at the top of int32 -------------------------------------------------------------------------------------
@pytest.mark.parametrize("news", [1, 40])
def test_lengths_at_the_top_are_refused(kvh, news):
    """A table that has room for 2^31 tokens (one page, again and again), and a request that says it holds them."""
    bt, c = 1 << 16, 64
    kc = torch.zeros((1, 1, bt, c), dtype=torch.int8, device="cuda")
    vc = torch.zeros_like(kc)
    ks, vs = torch.ones((1, 1, 1), device="cuda"), torch.ones((1, 1, 1), device="cuda")
    table = torch.zeros((1, 1 << 15), dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, news], dtype=torch.int32, device="cuda")
    q = torch.ones((news, c), dtype=torch.float16, device="cuda")
    for length in (TOP, TOP - 126):
        lens = torch.tensor([length], dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 5.0)
        kvh.attention(q, kc, vc, 0, starts, lens, table, news, head_dim=64, k_scale=ks, v_scale=vs, out=out, status=status)
        assert status.tolist() == [BAD] and (out == 5).all()
        status.zero_()
        kvh.append(q[None], q[None], kc, vc, starts, lens, table, news, head_dim=64, k_scale=ks, v_scale=vs, status=status)
        assert status.tolist() == [BAD] and not kc.any() and not vc.any()


@pytest.mark.parametrize("kind", ["16", "i8"])
@pytest.mark.parametrize("news,lens", [([2], [70]), ([60], [300]), ([1], [5000]), ([90], [2100])])
def test_sink_of_any_size(kvh, kind, news, lens):
    """A sink that holds every token there can be: a causal attention."""
    b = Batch(news, lens, heads=2, group=2, dim=64, kind=kind, dt="fp16", seed=79, layers=1)
    for sink in (TOP, TOP - 31, 1 << 30):
        b.check(b.run(kvh, sink=sink, window=5), sink=sink, window=5)


@pytest.mark.parametrize("group", [1, 2, 8])
def test_window_of_any_size_and_rows_before_the_first_token(kvh, group):
    """More queries than tokens, and a window that reaches past every position."""
    b = Batch([13], [4], heads=2, group=group, dim=64, kind="16", dt="fp16", seed=83, layers=1)
    for window in (TOP, TOP - 5, 1 << 30):
        b.check(b.run(kvh, window=window), window=window)
        b.check(b.run(kvh, window=window, sink=2), window=window, sink=2)


# ---- steps without tokens -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["16", "i8"])
def test_a_step_without_tokens(kvh, kind):
    """No row at all, as a step of requests that all wait gives it: nothing is done, and nothing is raised."""
    b = Batch([0, 0], [40, 0], heads=2, group=2, dim=64, kind=kind, dt="fp16", seed=89, layers=1)
    before = [t.clone() for t in (b.kc, b.vc)]
    out = b.run(kvh)
    assert out.shape == (0, 256)
    assert kvh.attention(b.q, b.kc, b.vc, 0, b.starts, b.lens, b.table, 1, head_dim=64, k_scale=b.ks, v_scale=b.vs, out=out, lse=b.lse,
                         workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")) is out
    x = torch.empty((1, 0, 128), dtype=torch.float16, device="cuda")
    q = torch.empty((1, 0, 256), dtype=torch.float16, device="cuda")
    assert kvh.append(x, x, b.kc, b.vc, b.starts, b.lens, b.table, 1, head_dim=64, k_scale=b.ks, v_scale=b.vs, q=q,
                      rotation=appending.rotation(50, 64).cuda()).shape == q.shape
    assert not b.status.any() and all(torch.equal(x.view(torch.int8), y.view(torch.int8)) for x, y in zip((b.kc, b.vc), before))


# ---- tokens without a position --------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("bt", [16, 40])
def test_tokens_without_a_position(kvh, kind, bt):
    """Neither their keys nor their values nor their queries are stored, nor do they count for a page's scales; the others' are."""
    b = appending.Batch([30, 1, 6], [3, 20, 0], heads=2, dim=64, kind=kind, bt=bt, seed=91)
    table = appending.rotation(64, 64)
    pos = torch.randint(0, 64, (37,), dtype=torch.int32)
    lost = [2, 3, 17, 30]
    pos[lost] = torch.tensor([64, -1, 1 << 30, -(1 << 31)], dtype=torch.int32)
    b.v[:, lost] *= 100  # would show in a scale
    old = [t.clone() if t is not None else None for t in (b.kc, b.vc, b.ks, b.vs)]
    q_out = torch.full_like(b.q, 5.0)
    b.append(kvh, rotation=table.cuda(), positions=pos.cuda(), q=b.q, q_out=q_out)
    assert b.status.tolist() == [BAD, BAD, 0]
    keep = [t for t in range(37) if t not in lost]
    split = lambda x: x.float().cpu().unflatten(-1, (-1, 64))  # noqa: E731
    at = pos.clamp(0, 63).long()
    k32 = appending.turned32(split(b.k), at, table, False)
    assert (q_out[:, lost] == 5).all()
    assert torch.equal(q_out[:, keep].cpu(), appending.turned32(split(b.q), at, table, False).to(b.q.dtype).flatten(-2)[:, keep])
    slots = [(t, page, row) for _, t, _, page, row in appending.ref.slots(b.starts_h, b.lens_h, b.table_h.tolist(), bt)]
    for x, before, after, scale0, scale1 in ((k32, old[0], b.kc, old[2], b.ks), (split(b.v), old[1], b.vc, old[3], b.vs)):
        if kind == "16":
            want = before.cpu().clone()
            for t, page, row in slots:
                if t not in lost:
                    want[:, page, row] = x[:, t].to(b.k.dtype).flatten(-2)
            assert torch.equal(after.cpu().view(torch.int16), want.view(torch.int16))
            continue
        # the values of the tokens that are not stored count as zeros for the scale; what stands in their rows is of no account
        x = x.clone()
        x[:, lost] = 0.0
        codes, scales = appending.coded32(x, before, scale0, b, kind)
        got = after.cpu().float()
        for t, page, row in slots:
            if t in lost:
                assert torch.equal(got[:, page, row], before.cpu().float()[:, page, row])
                got[:, page, row] = codes[:, page, row]
        assert torch.equal(scale1.cpu(), scales) and torch.equal(got, codes)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("pairs", [False, True])
def test_channels_past_the_rotation_keep_every_pattern(kvh, dt, pairs):
    """What is not rotated is stored as it is, in rows whose first channels are."""
    b = appending.Batch([20], [5], heads=2, dim=64, kind="16", dt=dt, seed=97)
    g = torch.Generator().manual_seed(1)
    for name in ("k", "q"):
        x = getattr(b, name)
        setattr(b, name, torch.randint(-32768, 32768, x.shape, generator=g, dtype=torch.int16).cuda().view(x.dtype))
    q_out = b.append(kvh, rotation=appending.rotation(64, 32).cuda(), pairs=pairs, q=b.q)
    got = torch.stack([b.kc[0, page, row] for _, _, _, page, row in appending.ref.slots(b.starts_h, b.lens_h, b.table_h.tolist(), 16)])
    for x, y in ((got, b.k[0]), (q_out[0], b.q[0])):
        assert torch.equal(x.view(torch.int16).unflatten(-1, (-1, 64))[..., 32:], y.view(torch.int16).unflatten(-1, (-1, 64))[..., 32:])


# ---- strides of one entry -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["16", "i8"])
@pytest.mark.parametrize("by_ctypes", [False, True])
def test_a_stride_of_one_entry_is_of_no_account(kvh, kind, by_ctypes, monkeypatch):
    """One token, one layer: keys beside values of another tensor, whatever the strides of those dimensions are, by either way into the calls."""
    import paper_2509_00105_amd.binding as binding

    if by_ctypes:
        monkeypatch.setattr(binding, "_fast", None)
    b = Batch([1], [33], heads=2, group=2, dim=64, kind=kind, dt="fp16", seed=93, layers=1)
    g = torch.Generator().manual_seed(2)
    row = torch.randn((1, 516), generator=g).half().cuda()  # queries, keys and values of a token; 516 is no multiple of 8
    q, k, v = row[None, :, :256], row[None, :, 256:384], row[:, 384:512].clone()[None]
    k, q = k.as_strided(k.shape, (3, 5, 1)), q.as_strided(q.shape, (7, 516, 1))
    table = appending.rotation(64, 64).cuda()
    want = [t.clone() if t is not None else None for t in (b.kc, b.vc, b.ks, b.vs)]
    out = kvh.append(k.contiguous(), v, *want[:2], b.starts, b.lens, b.table, 1, head_dim=64, k_scale=want[2], v_scale=want[3], q=q.contiguous(), rotation=table)
    odd = lambda t: None if t is None else t.as_strided(t.shape, (5, *t.stride()[1:]))  # noqa: E731
    for q_out in (None, torch.empty((1, 1, 256), dtype=torch.float16, device="cuda")):
        got = [t.clone() if t is not None else None for t in (b.kc, b.vc, b.ks, b.vs)]
        assert torch.equal(out, kvh.append(k, v, odd(got[0]), got[1], b.starts, b.lens, b.table, 1, head_dim=64, k_scale=got[2], v_scale=odd(got[3]), q=q, q_out=q_out,
                                           rotation=table))
        assert all(x is None or torch.equal(x.view(torch.int8), y.view(torch.int8)) for x, y in zip(got, want))
    plain = kvh.attention(out[0], *want[:2], 0, b.starts, b.lens, b.table, 1, head_dim=64, k_scale=want[2], v_scale=want[3])
    room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for o, ws in ((None, None), (torch.empty_like(plain), room)):
        assert torch.equal(plain, kvh.attention(out[0].as_strided((1, 256), (3, 1)), odd(want[0]), want[1], 0, b.starts, b.lens, b.table, 1, head_dim=64,
                                                k_scale=want[2], v_scale=odd(want[3]), out=o, workspace=ws))
