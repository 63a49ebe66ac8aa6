"""CPU-only checks of kvh_append and kvh_attention at the ends of what they take."""
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


@pytest.mark.parametrize("n_requests,max_new,n_tokens,heads,q_heads", [(1, 8192, 8192, 8, 32), (1, 131072, 131072, 8, 32), (1, 32768, 32768, 64, 64),
                                                                      (64, 2048, 60000, 8, 32), (600, 1, 600, 8, 32)])
def test_no_workspace_for_what_is_never_split(b, n_requests, max_new, n_tokens, heads, q_heads):
    assert b.attention_workspace(n_requests, max_new, n_tokens, heads, q_heads) == 0


def test_workspace_has_a_bound(b):
    for heads in (1, 2, 3, 8, 40, 100, 511, 512, 700, 1023, 1024, 4096):
        for group in (1, 4, 7, 16):
            for dim in (64, 128):
                for n in (1, 2, 17, 100, 1000, 10 ** 4, 10 ** 6, 2 ** 31 - 1):
                    for requests in (1, 64, 65535):
                        assert b.attention_workspace(requests, n, n, heads, heads * group, dim) <= 256 << 20


def test_rows_of_no_length_need_no_address(b):
    """n_tokens 0: nothing is done, with the null pointers of empty tensors; what describes cache and requests is checked all the same."""
    import ctypes

    cache = b._Cache(4096, 8192, None, None, 0, 1024, 0, 8, 2, 10, 16, 8, 128, b.CACHE_16)
    req = b._Requests(64, 64, 64, 4, 4, 1, 1, 0)
    kv, rows = b._KVView(None, None, 0, 1024), b._Rows(None, 0, 4096)
    rot = b._Rotation(64, None, 128, 9, 128, 0)
    ref = ctypes.byref
    assert b.lib().kvh_append(ref(cache), ref(req), 1, ref(kv), ref(rows), ref(rows), 32, ref(rot), None, None) == 0
    assert b.lib().kvh_append(ref(cache), ref(req), 1, ref(kv), None, None, 0, None, None, None) == 0
    attend = lambda layer=0, q_heads=32, scale=1.0: b.lib().kvh_attention(ref(cache), layer, ref(req), 1, ref(rows), ref(rows), q_heads, None, scale, 1, 0, 0, None, 0, None, None)  # noqa: E731
    assert attend() == 0 and attend(layer=2) == -3 and attend(q_heads=12) == -3 and attend(scale=float("nan")) == -1
    rot.rot = 24
    assert b.lib().kvh_append(ref(cache), ref(req), 1, ref(kv), None, None, 0, ref(rot), None, None) == -3
