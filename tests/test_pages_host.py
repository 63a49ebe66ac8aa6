"""CPU-only checks of the calls that select, read, copy, fork and compact pages: argument errors are found on the host, before anything is launched."""
import ctypes

import pytest
from test_serving_host import ALIGN, ARG, BAD_CACHES, BAD_REQUESTS, SHAPE, b, cache, coded, requests, rows  # noqa: F401

torch = pytest.importorskip("torch")
SIZE = -4


def ref(x):
    return None if x is None else ctypes.byref(x)


def bounds(b, **kw):
    return b._Bounds(**dict(dict(codes=4096, scale=64, layer_stride=0, page_stride=2048, scale_layer_stride=0, scale_page_stride=8, layers=2, pages=10,
                                 block_tokens=16, heads=8, head_dim=128, reserved=0), **kw))


def held(b, **kw):
    return b._RowsOfPages(**dict(dict(table=64, table_out=128, table_stride=4, table_out_stride=4, lens=64, refs=64, refs_out=128, table_pages=4, n_requests=2), **kw))


BAD_BOUNDS = [(dict(codes=None), ARG), (dict(scale=None), ARG), (dict(head_dim=96), SHAPE), (dict(layers=0), SHAPE), (dict(pages=0), SHAPE), (dict(heads=0), SHAPE),
              (dict(block_tokens=0), ARG), (dict(layer_stride=-16), ARG), (dict(page_stride=2032), ARG), (dict(scale_page_stride=7), ARG),
              (dict(scale_layer_stride=-1), ARG), (dict(codes=4104), ALIGN), (dict(page_stride=2056), ALIGN), (dict(layer_stride=8), ALIGN), (dict(scale=66), ALIGN)]
OTHER_BOUNDS = [dict(layers=1), dict(pages=11), dict(block_tokens=32), dict(heads=4), dict(head_dim=64)]  # not those of the cache


def bound(b, c=None, r=None, dt=1, box=0):
    return b.lib().kvh_bound_keys(ref(c or cache(b)), ref(r or requests(b)), dt, ref(bounds(b) if box == 0 else box), None, None)


def select(b, box=0, r=None, dt=1, layer=0, q=0, q_heads=32, first=1, last=1, count=4, out=64, ws=64, size=1 << 20):
    return b.lib().kvh_select_pages(ref(bounds(b) if box == 0 else box), layer, ref(r or requests(b)), dt, ref(rows(b) if q == 0 else q), q_heads, first, last, count, out,
                                    ws, size, None, None)


def attend(b, c=None, r=None, dt=1, layer=0, q=0, out=0, q_heads=32, pages=64, count=4, lse=None, scale=1.0, ws=None):
    q, out = (rows(b) if x == 0 else x for x in (q, out))
    return b.lib().kvh_attention_pages(ref(c or cache(b)), layer, ref(r or requests(b)), dt, ref(q), ref(out), q_heads, pages, count, lse, scale, ws, 0, None, None)


def copy(b, c=None, box=None, src=64, dst=64, n=1):
    return b.lib().kvh_copy_pages(ref(c or cache(b)), ref(box), src, dst, n, None, None)


def fork(b, c=None, box=None, h=0, parents=None, grow=None, lens_out=128, ws=64, size=1 << 20):
    return b.lib().kvh_fork(ref(c or cache(b)), ref(box), ref(held(b) if h == 0 else h), parents, grow, lens_out, ws, size, None, None)


def compact(b, c=None, box=None, h=0, moved=64, ws=64, size=1 << 20):
    return b.lib().kvh_compact(ref(c or cache(b)), ref(box), ref(held(b) if h == 0 else h), moved, ws, size, None, None)


@pytest.mark.parametrize("call", [bound, attend, copy, fork, compact])
def test_bad_caches(b, call):
    for kw, want in BAD_CACHES:
        assert call(b, c=cache(b, **kw)) == want, kw


@pytest.mark.parametrize("call", [bound, select, attend])
def test_bad_requests(b, call):
    for kw in BAD_REQUESTS:
        assert call(b, r=requests(b, **kw)) == ARG, kw
    assert call(b, dt=2) == ARG
    assert call(b, r=requests(b, n_tokens=0)) == 0


@pytest.mark.parametrize("call", [bound, select, copy, fork, compact])
def test_bad_bounds(b, call):
    for kw, want in BAD_BOUNDS:
        assert call(b, box=bounds(b, **kw)) == want, kw
    if call is not select:
        for kw in OTHER_BOUNDS:
            assert call(b, box=bounds(b, **dict(kw, page_stride=4096))) == SHAPE, kw
    if call in (bound, select):
        assert call(b, box=None) == ARG


def test_select_arguments(b):
    assert select(b, q=None) == ARG and select(b, out=None) == ARG
    assert select(b, layer=-1) == SHAPE and select(b, layer=2) == SHAPE and select(b, q_heads=12) == SHAPE and select(b, q_heads=0) == SHAPE
    assert select(b, q=rows(b, ts=4088)) == ARG and select(b, q=rows(b, p=8)) == ALIGN
    for kw in (dict(first=-1), dict(last=0), dict(first=3, last=2), dict(count=0), dict(count=4097), dict(first=2 ** 31 - 1), dict(last=2 ** 31 - 1)):
        assert select(b, **kw) == ARG, kw
    assert select(b, ws=72) == ALIGN and select(b, out=66) == ALIGN
    wide = requests(b, table_pages=20001, table_stride=20001)
    assert select(b, r=wide, ws=None) == SIZE and select(b, r=wide, size=8 * 20004 * 4 - 1) == SIZE


def test_attention_arguments(b):
    assert attend(b, q=None) == ARG and attend(b, out=None) == ARG and attend(b, pages=None) == ARG
    assert attend(b, layer=-1) == SHAPE and attend(b, layer=2) == SHAPE and attend(b, q_heads=12) == SHAPE
    assert attend(b, q=rows(b, ts=4088)) == ARG and attend(b, out=rows(b, p=8)) == ALIGN
    assert attend(b, scale=float("nan")) == ARG and attend(b, count=0) == ARG and attend(b, count=4097) == ARG
    assert attend(b, c=cache(b, block_tokens=1 << 20), count=2048) == SHAPE
    assert attend(b, ws=8) == ALIGN and attend(b, lse=2) == ALIGN and attend(b, pages=66) == ALIGN


def test_copy_arguments(b):
    assert copy(b, n=-1) == ARG and copy(b, n=(1 << 24) + 1) == ARG and copy(b, src=None) == ARG and copy(b, dst=None) == ARG
    assert copy(b, src=66) == ALIGN and copy(b, dst=65) == ALIGN
    assert copy(b, n=0) == 0 and copy(b, src=None, dst=None, n=0) == 0 and copy(b, c=coded(b), box=bounds(b), n=0) == 0


@pytest.mark.parametrize("call", [fork, compact])
def test_bad_rows(b, call):
    for kw in (dict(table=None), dict(table_out=None), dict(lens=None), dict(refs=None), dict(refs_out=None), dict(n_requests=0), dict(n_requests=65536),
               dict(table_pages=0), dict(table_stride=3), dict(table_out_stride=-1), dict(table_out=64), dict(refs_out=64)):
        assert call(b, h=held(b, **kw)) == ARG, kw
    for kw in (dict(table=66), dict(table_out=129), dict(lens=66), dict(refs=66), dict(refs_out=130)):
        assert call(b, h=held(b, **kw)) == ALIGN, kw
    assert call(b, h=None) == ARG and call(b, ws=None) == ARG and call(b, ws=66) == ALIGN


def test_fork_and_compact_arguments(b):
    lib = b.lib()
    assert fork(b, lens_out=None) == ARG and fork(b, lens_out=64) == ARG and fork(b, lens_out=130) == ALIGN
    assert fork(b, parents=66) == ALIGN and fork(b, grow=66) == ALIGN and fork(b, size=lib.kvh_fork_workspace(2, 10) - 1) == SIZE
    assert compact(b, moved=None) == ARG and compact(b, moved=66) == ALIGN and compact(b, size=lib.kvh_compact_workspace(10) - 1) == SIZE


def test_workspaces(b):
    lib = b.lib()
    assert lib.kvh_select_workspace(0, 1, 8, 4) == 0 and lib.kvh_select_workspace(1, 0, 8, 4) == 0 and lib.kvh_select_workspace(1, 1, 0, 4) == 0
    assert lib.kvh_select_workspace(1, 1, 8, 20001) >= 8 * 20001 * 4 and lib.kvh_select_workspace(1, 1 << 20, 8, 20001) <= 64 << 20
    assert lib.kvh_select_workspace(64, 64, 8, 256) == 0
    size = lib.kvh_attention_pages_workspace
    assert size(0, 8, 32, 128, 16, 64) == 0 and size(1, 8, 12, 128, 16, 64) == 0 and size(1, 8, 32, 96, 16, 64) == 0 and size(1, 8, 32, 128, 0, 64) == 0
    assert size(1, 8, 32, 128, 16, 0) == 0 and size(1, 8, 32, 128, 16, 4097) == 0 and size(1, 8, 32, 128, 16, 256) > 0 and size(512, 8, 32, 128, 16, 256) == 0
    assert lib.kvh_fork_workspace(0, 1) == 0 and lib.kvh_fork_workspace(1, 0) == 0 and lib.kvh_fork_workspace(65536, 1) == 0 and lib.kvh_compact_workspace(0) == 0


def test_binding_refuses(b):
    """Host tensors, before anything else."""
    import paper_2509_00105_amd as kvh

    i = torch.zeros(2, dtype=torch.int32)
    table, q = i.view(1, 2), torch.zeros((1, 128), dtype=torch.float16)
    pages = torch.zeros((1, 1, 16, 128), dtype=torch.float16)
    codes, scale = torch.zeros((1, 1, 1, 2, 128), dtype=torch.int8), torch.zeros((1, 1, 1))
    for call in (lambda: kvh.bound_keys(pages, codes, scale, i, i[:1], table, 1), lambda: kvh.select_pages(q, codes, scale, 0, i, i[:1], table, 1, 2),
                 lambda: kvh.attention_pages(q, pages, pages, 0, torch.zeros((1, 1, 2), dtype=torch.int32), i, i[:1], table, 1), lambda: kvh.copy_pages(pages, pages, i, i),
                 lambda: kvh.fork(pages, pages, table, i[:1], i[:1]), lambda: kvh.compact(pages, pages, table, i[:1], i[:1])):
        with pytest.raises(ValueError):
            call()


def test_oracle_of_forking_by_hand():
    """Two samples of one prompt of 5 tokens on pages of 4, a row that ends, one that begins, and too few pages."""
    from oracle import pages_ref as r

    table, lens = [[3, 1, -1], [2, -1, -1], [-1, -1, -1]], [5, 4, 0]
    out = r.fork(table, lens, [0, 1, 1, 1, 0, 0], 4, [0, 0, -1], [1, 3, 1])
    assert out == ([[3, 1, -1], [3, 0, -1], [2, -1, -1]], [6, 8, 1], [1, 1, 1, 2, 0, 0], [0, 0, 0], [(1, 0)])
    out = r.fork(table, lens, [0, 1, 1, 1, 0, 0], 4, [0, 1, -1], [7, 8, 5])
    assert out == ([[3, 1, 0], [2, 4, 5], [-1, -1, -1]], [12, 12, 0], [1, 1, 1, 1, 1, 1], [0, 0, r.NO_PAGES], [])
    # pages 1, 3 and 5 are in use: 3 and 5 move to 0 and 2
    assert r.compact([[5, 1], [3, 5]], [5, 4], [0, 1, 0, 1, 0, 2], 4) == ([[2, 1], [0, -1]], [1, 1, 2, 0, 0, 0], [-1, 1, -1, 0, -1, 2], [0, 0], [(3, 0), (5, 2)])
