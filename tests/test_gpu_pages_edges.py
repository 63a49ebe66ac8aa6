"""The calls on selected pages at inputs that are malformed, or of which little is left: what the header says of them, and nothing else touched."""
import numpy as np
import pytest

from test_gpu_pages_attention import Listed
from test_gpu_pages_select import Batch as Choice
from test_gpu_pages_select import ints
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


# How the scores are laid out: in LDS, tokens by themselves, in pairs and in fours, and through memory, with picks of 8 and of 16 waves and of 4 that are many.
LAYOUTS = [dict(news=[1, 1], lens=[300, 3300]), dict(news=[2, 3], lens=[400, 90], group=6), dict(news=[5, 8], lens=[900, 400], group=4),
           dict(news=[1, 1], lens=[500, 90], bt=1), dict(news=[1, 2], lens=[9000, 500], bt=2, dim=64), dict(news=[1], lens=[9000], bt=1, dim=64, heads=1),
           dict(news=[20, 5], lens=[1300, 700], group=3, bt=1, dim=64), dict(news=[260, 253], lens=[1100, 1201], group=4, bt=1, dim=64)]


def spoil(b, keep):
    """Table entries that are no pages, but for the places that keep(n) gives of a request with n pages."""
    bad = [-1, b.pages, 1 << 30, -2 ** 31]
    for r, n in enumerate(b.lens_h):
        held = -(-n // b.bt)
        stay = {j % held for j in keep(held)}
        for j in range(held):
            if j not in stay:
                b.table_h[r][j] = bad[j % 4]
    b.table = ints(b.table_h)


@pytest.mark.parametrize("layout", range(len(LAYOUTS)))
@pytest.mark.parametrize("keep", [(), (0, -1), (0,), (0, -1, 3), (5,), (2, 3, 4, -2)])
def test_pages_that_are_none_are_not_chosen(kvh, layout, keep):
    """All of a request's pages lie outside of the cache, or all but those that are chosen in any case, or a few others: what is left is listed, and -1."""
    b = Choice(seed=50 + layout, layers=1, **LAYOUTS[layout])
    spoil(b, lambda n: keep)
    for count, first, last in ((2, 0, 1), (5, 1, 1), (4, 2, 2)) if len(b.q) < 100 else ((5, 1, 1),):
        b.status.zero_()
        b.check(kvh, count, first, last)
        assert (b.status == BAD).all()


# starts that fall, how many of the first rows belong to requests ahead of that, max_new
FALLS = [([0, 3, -5, 5, 9], 3, 9), ([0, 2, 6, 0, 9], 6, 4), ([0, 3, 6, -2 ** 31, 9], 6, 9), ([0, 1, 2 ** 31 - 1, 2, 9], 1, 9)]


def refused(starts, max_new, rows=9):
    return [BAD if not 0 <= s <= e <= rows or e - s > max_new else 0 for s, e in zip(starts, starts[1:])]


@pytest.mark.parametrize("more", [0, 100])
@pytest.mark.parametrize("starts,rows,max_new", FALLS)
@pytest.mark.parametrize("lens,bt", [([400, 310, 290, 333], 16), ([400, 310, 290, 333], 1), ([1100, 310, 290, 333], 1)])
def test_selection_ahead_of_falling_starts(kvh, lens, bt, starts, rows, max_new, more):
    """Requests that share no rows with others and lie ahead are what they are without those behind them."""
    b = Choice([3, 3, 2, 1] + [0] * more, lens + [20] * more, heads=2, group=2, dim=64, bt=bt, seed=60, layers=1)
    b.starts = ints(starts + [9] * more)
    out = b.run(kvh, 7, max_new=max_new).cpu().numpy()
    assert b.status.tolist() == refused(starts, max_new) + [0] * more
    ahead = starts.index(rows)
    b.starts_h, b.lens_h = starts[:ahead + 1], lens[:ahead]
    assert np.array_equal(out[:rows], b.want(7)[:rows])


@pytest.mark.parametrize("more", [0, 100])
@pytest.mark.parametrize("starts,rows,max_new", FALLS)
@pytest.mark.parametrize("most,count", [(5000, 300), (60, 4)])
def test_attention_ahead_of_falling_starts(kvh, most, count, starts, rows, max_new, more):
    """The same, lists shared by blocks and joined among them."""
    ahead = starts.index(rows)
    news = [e - s for s, e in zip(starts[:ahead], starts[1:])] + [9 - rows] + [0] * (3 - ahead + more)
    b = Listed(news, [most, 40, 50, 60] + [20] * more, heads=2, group=4, dim=64, kind="16", dt="fp16", seed=61, layers=1).choose(count, 1)
    want, lse = b.run(kvh, max_new=9), b.lse
    assert not b.status.any()
    b.starts = ints(starts + [9] * more)
    out = b.run(kvh, max_new=max_new)
    assert torch.equal(out[:rows], want[:rows]) and torch.equal(b.lse[:rows], lse[:rows])
    assert b.status.tolist() == refused(starts, max_new) + [0] * more


@pytest.mark.parametrize("longest,bt", [(300, 16), (1100, 1)])
@pytest.mark.parametrize("group", [2, 7])
def test_gaps_among_many_requests(kvh, group, longest, bt):
    """Refused requests, one after the other and alone, among more than 64, where neighbouring tokens share products; rows behind the last one."""
    n = 300
    lens = [int(x) for x in np.random.default_rng(8).integers(3, 90, n)]
    lens[200] = longest
    b = Choice([3] * n, lens, heads=1, group=group, dim=64, bt=bt, seed=62, layers=1, behind=40)
    gone = [0, 1, 2, 70, 71, 90, 150, *range(220, 260), 299]
    b.lens[gone] = -1
    out = b.run(kvh, 5).cpu().numpy()
    assert b.status.tolist() == [BAD if r in gone else 0 for r in range(n)]
    want = b.want(5)
    for r in gone:
        want[3 * r:3 * r + 3] = -9
    assert np.array_equal(out, want)


def test_widest_table_without_a_workspace(kvh):
    """14220 pages are the most whose scores a block keeps by itself; a table for one more needs the workspace."""
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    b = Choice([1], [14220], heads=1, group=4, dim=64, bt=1, seed=63, layers=1)
    b.check(kvh, 30, workspace=none)
    b = Choice([1], [14221], heads=1, group=4, dim=64, bt=1, seed=64, layers=1)
    with pytest.raises(kvh.KVHError) as e:
        b.run(kvh, 30, workspace=none)
    assert e.value.status == -4
    b.check(kvh, 30)
