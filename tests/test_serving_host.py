"""CPU-only checks of kvh_append and kvh_attention: argument errors are found on the host, before anything is launched."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def b():
    from paper_2509_00105_amd import build

    if not os.path.exists(build.LIB):
        build.build()
    import paper_2509_00105_amd.binding as m

    m.lib()
    return m


def cache(b, **kw):
    f = dict(k=4096, v=8192, k_scale=None, v_scale=None, layer_stride=0, token_stride=1024, scale_layer_stride=0, scale_page_stride=8, layers=2, pages=10,
             block_tokens=16, heads=8, head_dim=128, kind=b.CACHE_16)
    return b._Cache(**dict(f, **kw))


def coded(b, **kw):
    return cache(b, **dict(dict(k_scale=64, v_scale=64, kind=b.CACHE_I8), **kw))


def requests(b, **kw):
    return b._Requests(**dict(dict(starts=64, lens=64, page_table=64, table_stride=4, table_pages=4, n_requests=1, max_new=1, n_tokens=1), **kw))


def rows(b, p=4096, ls=0, ts=4096):
    return b._Rows(p, ls, ts)


ARG, SHAPE, ALIGN = -1, -3, -5
BAD_CACHES = [
    (dict(k=None), ARG), (dict(v=None), ARG), (dict(kind=3), ARG), (dict(kind=-1), ARG), (dict(k_scale=64), ARG), (dict(kind=1), ARG),
    (dict(kind=1, k_scale=64), ARG), (dict(kind=2, k_scale=64, v_scale=64, scale_page_stride=7), ARG), (dict(kind=2, k_scale=64, v_scale=66), ALIGN),
    (dict(head_dim=96), SHAPE), (dict(head_dim=0), SHAPE), (dict(heads=0), SHAPE), (dict(heads=5000), SHAPE), (dict(layers=0), SHAPE), (dict(pages=0), SHAPE),
    (dict(block_tokens=0), ARG), (dict(token_stride=1016), ARG), (dict(token_stride=1 << 20), ARG), (dict(layer_stride=-8), ARG),
    (dict(k=4100), ALIGN), (dict(token_stride=1028), ALIGN), (dict(layer_stride=4), ALIGN), (dict(kind=1, k_scale=64, v_scale=64, token_stride=1032), ALIGN),
]
BAD_REQUESTS = [dict(starts=None), dict(lens=None), dict(page_table=None), dict(n_requests=0), dict(n_requests=65536), dict(max_new=0), dict(n_tokens=-1),
                dict(table_pages=0), dict(table_stride=-1)]


def append(b, c=None, r=None, dt=1, kv=(4096, 4096, 0, 1024), q=None, out=None, q_heads=32, rot=None):
    ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    view = None if kv is None else b._KVView(*kv)
    return b.lib().kvh_append(ref(c or cache(b)), ref(r or requests(b)), dt, ref(view), ref(q), ref(out), q_heads, ref(rot), None, None)


def attend(b, c=None, r=None, dt=1, layer=0, q=0, out=0, q_heads=32, lse=None, scale=1.0, causal=1, sink=0, window=0, ws=None):
    ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    q, out = (rows(b) if x == 0 else x for x in (q, out))
    return b.lib().kvh_attention(ref(c or cache(b)), layer, ref(r or requests(b)), dt, ref(q), ref(out), q_heads, lse, scale, causal, sink, window, ws, 0, None, None)


@pytest.mark.parametrize("call", [append, attend])
def test_bad_caches_and_requests(b, call):
    for kw, want in BAD_CACHES:
        assert call(b, c=cache(b, **kw)) == want, kw
    for kw in BAD_REQUESTS:
        assert call(b, r=requests(b, **kw)) == ARG, kw
    assert call(b, dt=2) == ARG


@pytest.mark.parametrize("call", [append, attend])
def test_nothing_to_do(b, call):
    assert call(b, r=requests(b, n_tokens=0)) == 0
    assert call(b, c=coded(b), r=requests(b, n_tokens=0)) == 0


def test_append_arguments(b):
    assert append(b, kv=None) == ARG and append(b, kv=(None, 4096, 0, 1024)) == ARG and append(b, kv=(4096, None, 0, 1024)) == ARG
    assert append(b, kv=(4096, 4096, 0, 1016)) == ARG and append(b, kv=(4096, 4096, -8, 1024)) == ARG
    assert append(b, kv=(4104, 4096, 0, 1024)) == ALIGN and append(b, kv=(4096, 4096, 4, 1024)) == ALIGN and append(b, kv=(4096, 4096, 0, 1028)) == ALIGN
    assert append(b, q=rows(b)) == ARG  # nowhere to put it
    assert append(b, q=rows(b), out=rows(b, ts=4088)) == ARG and append(b, q=rows(b, p=8), out=rows(b)) == ALIGN
    assert append(b, q=rows(b), out=rows(b), q_heads=0) == SHAPE
    rot = lambda **kw: b._Rotation(**dict(dict(table=64, positions=None, table_stride=128, n_positions=9, rot=128, pairs=0), **kw))  # noqa: E731
    for kw, want in ((dict(table=None), ARG), (dict(n_positions=0), ARG), (dict(table_stride=-4), ARG), (dict(rot=0), SHAPE), (dict(rot=24), SHAPE),
                     (dict(rot=144), SHAPE), (dict(table=72), ALIGN), (dict(table_stride=130), ALIGN)):
        assert append(b, rot=rot(**kw)) == want, kw


def test_attention_arguments(b):
    assert attend(b, q=None) == ARG and attend(b, out=None) == ARG
    assert attend(b, layer=-1) == SHAPE and attend(b, layer=2) == SHAPE
    assert attend(b, q_heads=0) == SHAPE and attend(b, q_heads=12) == SHAPE and attend(b, q_heads=4) == SHAPE
    assert attend(b, q=rows(b, ts=4088)) == ARG and attend(b, out=rows(b, p=None)) == ARG
    assert attend(b, q=rows(b, p=8)) == ALIGN and attend(b, out=rows(b, ts=4100)) == ALIGN
    assert attend(b, scale=float("nan")) == ARG and attend(b, scale=float("inf")) == ARG
    assert attend(b, sink=-1) == ARG and attend(b, window=-1) == ARG and attend(b, window=4, causal=0) == ARG and attend(b, sink=4) == ARG
    assert attend(b, ws=8) == ALIGN and attend(b, lse=2) == ALIGN


def test_workspace(b):
    size = b.lib().kvh_attention_workspace
    assert size(0, 1, 1, 8, 32, 128) == 0 and size(1, 0, 1, 8, 32, 128) == 0 and size(1, 1, 0, 8, 32, 128) == 0
    assert size(1, 1, 1, 8, 12, 128) == 0 and size(1, 1, 1, 8, 32, 96) == 0 and size(70000, 1, 1, 8, 32, 128) == 0
    assert 0 < size(1, 1, 1, 8, 32, 64) < size(1, 1, 1, 8, 32, 128) <= size(64, 1, 64, 8, 32, 128)


def test_binding_refuses(b):
    """What the tensors themselves show is refused by the binding, host tensors before anything else."""
    import paper_2509_00105_amd as kvh

    x = torch.zeros((1, 1, 128), dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    pages = torch.zeros((1, 1, 16, 128), dtype=torch.float16)
    with pytest.raises(ValueError):
        kvh.append(x, x, pages, pages, i, i[:1], i.view(1, 2), 1)
    with pytest.raises(ValueError):
        kvh.attention(x[0], pages, pages, 0, i, i[:1], i.view(1, 2), 1)
