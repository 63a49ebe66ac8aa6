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
