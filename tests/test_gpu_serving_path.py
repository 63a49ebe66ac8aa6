"""The serving cache's calls together: the example's path, the two ways into a call, and what the attention's two kernels and its cuts have to agree on."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_serving_attention import Batch  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


@pytest.mark.parametrize("kind,bound", [("16", 0.02), ("i8", 0.025), ("e4m3", 0.06)])
def test_example(kvh, kind, bound):
    """Keys and values of unit size through 8-bit blobs (steps of 1/32 at most), bf16 and the cache (int8: steps of 1/30; e4m3: 1/16 of a value at most):
    relative errors of 1 % and less, 1 % and 3 % of the values, and as much again from the weights that follow the keys."""
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.run(context=1000, question=33, answer=3, kind=kind, layers=2)
    assert r["tokens"] == 1036 and r["error"] < bound, r
    assert r["bytes"] == 2 * 2 * 65 * (16 * 1024 * (2 if kind == "16" else 1) + (0 if kind == "16" else 32))


@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
def test_both_ways_into_a_call(kvh, kind, monkeypatch):
    """With the call module and without it: the same results, for views with strides of their own too."""
    import paper_2509_00105_amd.binding as binding

    b = Batch([3, 1], [70, 33], heads=2, group=2, dim=64, kind=kind, dt="fp16", seed=31, pad=16)
    room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    one = b.run(kvh, workspace=room, out=torch.empty((4, 256), dtype=torch.float16, device="cuda")[:, :256]), b.lse.clone()
    x = torch.randn((2, 4, 128), device="cuda").half()
    kc, vc = b.kc.clone(), b.vc.clone()
    table = torch.rand((80, 32), device="cuda")
    args = dict(head_dim=64, q=x, rotation=table, pairs=True)
    scales = [None, None] if kind == "16" else [b.ks.clone(), b.vs.clone()]
    out1 = kvh.append(x, x, kc, vc, b.starts, b.lens, b.table, 3, k_scale=scales[0], v_scale=scales[1], q_out=torch.empty_like(x), **args)
    monkeypatch.setattr(binding, "_fast", None)
    two = b.run(kvh, workspace=room, out=torch.empty_like(b.q)), b.lse
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    again = [None, None] if kind == "16" else [b.ks.clone(), b.vs.clone()]
    k2, v2 = b.kc.clone(), b.vc.clone()
    out2 = kvh.append(x, x, k2, v2, b.starts, b.lens, b.table, 3, k_scale=again[0], v_scale=again[1], q_out=torch.empty_like(x), **args)
    assert torch.equal(out1, out2)
    for p, q in ((kc, k2), (vc, v2), *([] if kind == "16" else zip(scales, again))):
        assert torch.equal(p.view(torch.int8) if p.element_size() == 1 else p.nan_to_num(), q.view(torch.int8) if q.element_size() == 1 else q.nan_to_num())


@pytest.mark.parametrize("kind", ["16", "i8"])
@pytest.mark.parametrize("most", [2, 30])
def test_more_requests_than_lanes_cut(kvh, kind, most):
    """130 requests, few rows and many rows each, some without tokens, long enough to be cut."""
    g = torch.Generator().manual_seed(most)
    news = torch.randint(0, most + 1, (130,), generator=g).tolist()
    lens = [n + int(x) for n, x in zip(news, torch.randint(0, 900, (130,), generator=g))]
    b = Batch(news, lens, heads=1, group=2, dim=64, kind=kind, dt="fp16", seed=41, layers=1)
    b.check(b.run(kvh))


@pytest.mark.parametrize("kind,dt,dim,bt", [("16", "bf16", 128, 16), ("i8", "bf16", 128, 24), ("e4m3", "fp16", 64, 32), ("16", "fp16", 64, 7)])
@pytest.mark.parametrize("mask", [dict(), dict(causal=False), dict(sink=70, window=400)])
def test_many_rows_cut(kvh, kind, dt, dim, bt, mask):
    """More rows than a tile, over tokens that are cut between and inside tiles."""
    b = Batch([90, 3, 33], [2100, 700, 90], heads=2, group=3, dim=dim, bt=bt, kind=kind, dt=dt, seed=43, layers=1)
    b.check(b.run(kvh, **mask), **mask)
    assert not b.status.any()


@pytest.mark.parametrize("heads", [1, 2, 3, 4, 8])
def test_heads_of_a_block(kvh, heads):
    """Blocks that take one, two and four heads of a cut batch."""
    b = Batch([1, 2], [2500, 600], heads=heads, group=2, kind="i8", dt="bf16", seed=47, layers=1)
    b.check(b.run(kvh))


def test_scale_of_either_sign(kvh):
    """A negative factor of the scores, few rows and many."""
    for news in ([2], [50]):
        b = Batch(news, [120], heads=1, group=2, dim=64, kind="e4m3", dt="bf16", seed=53, layers=1)
        b.check(b.run(kvh, scale=-0.2), scale=-0.2)


def test_launch_events(kvh):
    """kvh_time_next_launch times either call."""
    b = Batch([1], [300], heads=2, group=2, kind="16", dt="bf16", seed=59, layers=1)
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record(), stop.record()
    kvh.time_next_launch(start, stop)
    b.run(kvh)
    torch.cuda.synchronize()
    assert 0 < start.elapsed_time(stop) < 100


@pytest.mark.parametrize("heads,kind,dt,dim,bt", [(2, "i8", "bf16", 128, 16), (4, "16", "fp16", 64, 16), (8, "e4m3", "bf16", 64, 24), (12, "i8", "fp16", 64, 16)])
@pytest.mark.parametrize("mask", [dict(), dict(sink=40, window=7900)])
def test_blocks_of_neighbouring_heads(kvh, heads, kind, dt, dim, bt, mask):
    """So many steps that a block's waves take heads of their own: one long request among short ones."""
    n = 80 // heads + 1
    b = Batch([1] * n, [8300] + [1 + 37 * i % 400 for i in range(1, n)], heads=heads, group=2, dim=dim, bt=bt, kind=kind, dt=dt, seed=61, layers=1)
    b.check(b.run(kvh, **mask), **mask)
    assert not b.status.any()


@pytest.mark.parametrize("kind", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("new,length,mask", [(1, 640, {}), (1, 4001, {}), (8, 3000, {}), (16, 3000, {}), (100, 2500, dict(sink=70, window=1200)), (300, 1500, {})])
def test_one_request_cut(kvh, kind, new, length, mask):
    """A request alone, in a few rows, in pairs of row tiles and in many."""
    b = Batch([new], [length], heads=2, group=2, dim=128, kind=kind, dt="bf16", seed=67, layers=1)
    b.check(b.run(kvh, **mask), **mask)
    assert not b.status.any()
