"""The calls on selected pages at inputs that are malformed, or of which little is left: what the header says of them, and nothing else touched."""
import numpy as np
import pytest

from test_gpu_pages_attention import Listed
from test_gpu_serving_attention import BAD

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvh():
    import paper_2509_00105_amd as m

    m.lib()
    return m


# Lists of a request of 4 pages, and what is left of them.  Past its end a list may hold anything: entries of memory that was never set.
ENDED = [([0, 2, -100, -1, 3, 1], [0, 2], 0), ([1, 3, -1, 2, 3, -1], [1, 3], 0), ([-2 ** 31, -5, -1, 0, 1, 2], [], 0), ([-7, 0, -9, -1, -3, -2], [], 0),
         ([2, 2, -50, -2, -1, 3], [2], BAD), ([3, 4, -2 ** 31, -1, 0, 1], [3], BAD), ([0, 1, 2, 3, -3, -1], [0, 1, 2, 3], 0), ([0, -2 ** 31, 2 ** 31 - 1, -1, 1, 2], [0], 0)]


@pytest.mark.parametrize("kind", ["16", "i8"])
def test_lists_past_their_end(kvh, kind):
    """Negative entries that rise again after the end.  The table is a view far inside of a larger tensor."""
    n = len(ENDED)
    b = Listed([1] * n, [60] * n, heads=1, group=2, dim=64, kind=kind, dt="fp16", seed=40, layers=1).choose(6)
    wide = torch.full((3 * n, 300), 1 << 29, dtype=torch.int32, device="cuda")
    columns = b.table.shape[1]
    wide[n:2 * n, 200:200 + columns] = b.table
    b.table = wide[n:2 * n, 200:200 + columns]
    b.chosen = torch.tensor([e for e, _, _ in ENDED], device="cuda").to(torch.int32).view(n, 1, 6)
    b.lists = np.array([left + [-1] * (6 - len(left)) for _, left, _ in ENDED]).reshape(n, 1, 6)
    b.check(b.run(kvh))
    assert b.status.tolist() == [said for _, _, said in ENDED]


def test_long_lists_past_their_end(kvh):
    """The same where a list is shared by blocks and joined."""
    b = Listed([1, 1], [9001, 4000], heads=2, group=4, kind="16", dt="bf16", seed=41, layers=1).choose(500, 1)
    held = np.array([[(x >= 0).sum() for x in row] for row in b.lists])
    junk = np.random.default_rng(4).integers(-2 ** 31, 0, b.lists.shape)
    behind = np.arange(500) > held[..., None]  # one -1 stays
    b.chosen = torch.from_numpy(np.where(behind, junk, b.lists).astype(np.int32)).cuda()
    b.chosen[1, 1] = torch.from_numpy(junk[1, 1].astype(np.int32)).cuda()  # nothing is listed
    b.lists[1, 1] = -1
    b.check(b.run(kvh))
    assert not b.status.any()
