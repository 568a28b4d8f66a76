"""Room for new tokens where pages run out in the middle of a list: who is refused, as the header says."""
import pytest

import paper_2608_07915_amd as S

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def _ints(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _map():
    """Rows 0 and 1 share their only, partly filled page; row 2 has a full one; one page is free."""
    m = S.PagedCache(3, 64, 4, 4)
    assert S.spectra_pages_extend(m, _ints(0, 2), _ints(10, 64), []).tolist() == [10, 64]
    assert S.spectra_pages_fork(m, _ints(0), _ints(1)).tolist() == [10]
    return m


def test_without_a_shortage_the_last_owner_keeps_the_page():
    m = _map()
    assert S.spectra_pages_extend(m, _ints(0, 1), _ints(1, 1), []).tolist() == [11, 11]
    assert m.table[0, 0] == 2 and m.table[1, 0] == 0 and m.refs.tolist() == [1, 1, 1]


def test_behind_a_shortage_an_entry_that_shared_its_page_with_one_before_is_refused():
    m = _map()
    assert S.spectra_pages_extend(m, _ints(0, 2, 1, 3), _ints(1, 1, 1, 0), []).tolist() == [11, -1, -1, 0]
    assert m.lens.tolist() == [11, 10, 64, 0] and m.refs.tolist() == [1, 1, 1]
    # it is served by the next call: the page is its own by then
    assert S.spectra_pages_extend(m, _ints(1), _ints(54), []).tolist() == [64]
    assert m.table[1, 0] == 0 and m.refs.tolist() == [1, 1, 1]


def test_the_shared_page_of_a_refused_entry_stays_shared():
    m = _map()
    S.spectra_pages_extend(m, _ints(2), _ints(1), [])  # the last free page
    before = [t.clone() for t in (m.table, m.lens, m.refs)]
    assert S.spectra_pages_extend(m, _ints(0, 1, 2), _ints(1, 1, 1), []).tolist() == [-1, -1, 66]
    assert torch.equal(m.table, before[0]) and torch.equal(m.refs, before[2]) and m.lens.tolist() == [10, 10, 66, 0]
