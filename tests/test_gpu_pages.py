"""The page map's calls against its rules as a sequential program: random programs with repeated,
foreign and impossible list entries, pools too small, and the records that move."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import MapModel

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def _ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Both:
    """A map on the device and its model, with two pools of different page sizes."""

    def __init__(self, n_pages, page, rows, row_pages, words=(128, 4160), seed=0):
        self.m = MapModel(n_pages, page, rows, row_pages)
        self.c = S.PagedCache(n_pages, page, rows, row_pages)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.pools = [torch.randint(-2 ** 31, 2 ** 31 - 1, (n_pages, w), generator=g, device="cuda", dtype=torch.int32) for w in words]
        self.want = [p.clone() for p in self.pools]

    def _copies(self, copies):
        if copies:
            src, dst = map(list, zip(*copies))
            for w in self.want:
                w[dst] = w[src]

    def extend(self, rows, counts):
        ends, copies = self.m.extend(rows, counts)
        self._copies(copies)
        got = S.spectra_pages_extend(self.c, _ints(rows), _ints(counts), self.pools)
        assert got.tolist() == ends
        self.check()
        return ends

    def fork(self, parents, children):
        ends = self.m.fork(parents, children)
        assert S.spectra_pages_fork(self.c, _ints(parents), _ints(children)).tolist() == ends
        self.check()

    def truncate(self, rows, keep=None):
        self.m.truncate(rows, keep)
        S.spectra_pages_truncate(self.c, _ints(rows), None if keep is None else _ints(keep))
        self.check()

    def compact(self):
        moved, copies = self.m.compact()
        self._copies(copies)
        assert S.spectra_pages_compact(self.c, self.pools).tolist() == moved.tolist()
        self.check()

    def check(self):
        self.m.check(self.c)
        for p, w in zip(self.pools, self.want):
            assert torch.equal(p, w)


def test_growth_of_one_row():
    b = Both(20, 64, 2, 12)
    for n in (0, 1, 63, 1, 63, 128, 500):
        b.extend([0], [n])
    b.extend([0], [1000])   # more than the row's slots
    b.truncate([0], [65])
    b.truncate([0], [65])
    b.truncate([0], [64])
    b.extend([0, 1], [1, 1])
    b.truncate([0, 1])


def test_copies_before_a_shared_page_is_written():
    b = Both(40, 64, 9, 8)
    b.extend([0], [100])
    b.fork([0, 0, 0], [1, 2, 3])
    b.extend([1], [1])          # a copy
    b.extend([2, 0], [1, 1])    # a copy each but the last owner's
    b.extend([3, 1], [70, 63])
    b.fork([3, 1], [4, 5])
    b.truncate([3], [101])      # row 4 still has the pages
    b.extend([3, 4], [1, 1])
    b.fork([4], [6])
    b.extend([6], [0])          # nothing to write: no copy
    b.truncate([6], [128])      # whole pages: shared ones stay shared
    b.extend([6], [1])


def test_two_owners_in_one_list():
    b = Both(40, 64, 4, 8)
    b.extend([0], [10])
    b.fork([0, 0], [1, 2])
    b.extend([0, 1, 2], [5, 60, 1])


def test_refused_entries_change_nothing():
    b = Both(30, 64, 6, 8)
    b.extend([0, 1], [100, 64])
    b.extend([0, 0, -1, 6, 2, 3], [3, 4, 5, 6, -1, 513])
    b.fork([0, 0, 1, 2, 7, 1, 0, 3], [2, 2, 0, 3, 4, -1, 1, 5])
    b.fork([0], [0])
    b.truncate([9, -3, 0], [1, 2, 90])
    b.truncate([0, 0, 0], [95, 70, 80])  # the fewest


def test_too_few_pages():
    b = Both(10, 64, 8, 8)
    b.extend([0, 1, 2], [300, 100, 10])       # 5 + 2 + 1
    b.fork([2, 2], [3, 4])
    b.extend([5, 6, 7], [64, 128, 64])        # one, then too few for the rest
    b.truncate([5])
    b.extend([1, 0, 3, 4, 2], [1, 200, 1, 1, 1])  # 0 needs three of two; sharers behind it are refused
    b.extend([1, 3, 4, 2], [1, 1, 1, 1])
    b.extend([1], [1])


def test_compaction():
    b = Both(50, 64, 6, 10)
    b.compact()
    b.extend([0, 1, 2, 3], [200, 300, 400, 640])
    b.fork([1], [4])
    b.truncate([0, 2], [0, 100])
    b.compact()
    b.compact()
    b.extend([0, 2, 4], [60, 60, 60])
    b.truncate([3])
    b.truncate([1])
    b.compact()
    b.truncate([0, 1, 2, 3, 4, 5])
    b.compact()


@pytest.mark.parametrize("seed", range(6))
def test_random_programs(seed):
    rng = np.random.default_rng(seed)
    rows = int(rng.integers(3, 60))
    b = Both(int(rng.integers(20, 300)), 64 * int(rng.integers(1, 4)), rows, int(rng.integers(2, 20)), seed=seed)
    for _ in range(25):
        n = int(rng.integers(1, 2 * rows))
        pick = lambda: rng.integers(-1, rows + 1, n)  # noqa: E731
        op = rng.integers(5)
        if op <= 1:
            b.extend(pick(), rng.integers(-1, 200, n))
        elif op == 2:
            b.fork(pick(), pick())
        elif op == 3:
            b.truncate(pick()[: n // 2 + 1], None if rng.random() < 0.3 else rng.integers(-1, 600, n // 2 + 1))
        else:
            b.compact()


def test_large_pool_and_long_lists():
    # several rounds of the page scan; 1024 entries
    b = Both(70001, 64, 1100, 70, words=(64,))
    rng = np.random.default_rng(3)
    b.extend(np.arange(1024), rng.integers(1, 4000, 1024))
    b.truncate(rng.permutation(1100)[:700], rng.integers(0, 2000, 700))
    b.extend(rng.permutation(1024), rng.integers(0, 3000, 1024))
    b.fork(rng.permutation(1024)[:60], 1024 + np.arange(60))
    b.extend(1024 + np.arange(60), rng.integers(1, 100, 60))
    b.truncate(rng.permutation(1100)[:500])
    b.compact()


def test_more_pools_than_one_launch_takes():
    b = Both(12, 64, 3, 4, words=(64,) * 70)
    b.extend([0], [100])
    b.fork([0], [1])
    b.extend([1], [5])
    b.truncate([0])
    b.compact()


def test_inconsistent_maps_stay_in_bounds():
    # lengths and table entries that no call would have left: refused or passed over
    c = S.PagedCache(8, 64, 4, 3)
    c.lens.copy_(torch.tensor([500, -2, 70, 64]))
    c.table.copy_(torch.tensor([[0, 1, 2], [3, 4, 5], [6, 99, -1], [-7, -1, -1]]))
    c.refs.copy_(torch.tensor([1, 1, 1, 1, 1, 1, 1, 0]))
    pool = torch.arange(8 * 64, device="cuda", dtype=torch.int32).view(8, 64)
    rows = _ints([0, 1, 2, 3])
    assert S.spectra_pages_extend(c, rows, _ints([1, 1, 1, 1]), pool).tolist() == [-1, -1, -1, 65]
    assert c.table[3].tolist() == [-7, 7, -1] and c.refs.tolist() == [1] * 8
    S.spectra_pages_truncate(c, rows)
    assert c.lens.tolist() == [500, -2, 0, 0] and c.refs.tolist() == [1, 1, 1, 1, 1, 1, 0, 0]
    S.spectra_pages_compact(c, pool)
    assert pool.view(-1).tolist() == list(range(512))
