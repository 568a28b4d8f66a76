"""Accepted paths refuse a pool that is listed twice: two workgroups would move its records at once, each reading what the
other has moved. No GPU is needed (pointers are never followed)."""
import ctypes

from paper_2608_07915_amd import _lib
from paper_2608_07915_amd._lib import spectra_pool
from test_paged_refusals import EINVAL, P, _map


def accept(*pools, n=4):
    made = (spectra_pool * max(len(pools), 1))(*pools)
    return _lib.get().spectra_pages_accept(ctypes.byref(_map()), P, P, P, 8, P, n, made, len(pools), 3, P, None)


def test_a_pool_listed_twice():
    words = 64 * 3 * 8
    a, b, none = spectra_pool(P, words), spectra_pool(P + 4096, words), spectra_pool(P, 0)
    for pools in ((a, a), (a, b, a), (b, a, spectra_pool(P, 64 * 3 * 5)), (none, a, none, a)):
        assert accept(*pools) == EINVAL and b"listed before" in _lib.get().spectra_last_error()
    many = [spectra_pool(P + 64 * i, words) for i in range(300)]
    assert accept(*many, many[7]) == EINVAL and b"pool 300 is listed before, as pool 7" in _lib.get().spectra_last_error()
    assert accept(a, a, n=0) == 0  # nothing to do
