"""Paged attention and append at the ends of their ranges: many sequences, pools past 2^31 words,
many heads beside wide records, query rows that are not finite."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D
from test_gpu_paged_attention import ALL, B8, Case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_many_short_sequences(f32):
    # more sequences than a workgroup looks at together; chunks, single tokens and empty ones in turn
    rng = np.random.default_rng(0)
    new = [int(x) for x in rng.choice([0, 1, 2, 4, 9, 70], 1100, p=[0.2, 0.5, 0.1, 0.1, 0.07, 0.03])]
    lens = [n + int(x) for n, x in zip(new, rng.integers(0, 100, 1100))]
    c = Case(lens, new, 4, B8, B8, 8, f32=f32, seed=20)
    c.check(c.run())


def test_the_most_sequences():
    # all rows of one table row: they share their pages
    c = Case([200], [1], 4, B8, B8, 8, seed=21, f32=True)
    one = c.run()
    n = 16384
    cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    out = S.spectra_paged_attention(c.cache, c.ck, c.cv, *c.pools, c.q.expand(n, -1, -1), cu, 1, 200,
                                    rows=torch.zeros(n, dtype=torch.int32, device="cuda"))
    # both cut and sum the same tokens in fp32, in another order
    assert (out - one).abs().max() <= 2.0 ** -16 * one.abs().max()
    assert (out == out[:1]).all()


@pytest.mark.parametrize("n_qh", [12, 13, 16])
@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_many_heads_beside_wide_records(n_qh, f32):
    for words in (36, 40):
        c = Case([150, 300], [1, 1], n_qh, [[8, 8, 8, 8], [8, 0, 8, 8]], [[8, 8, 8, 8]] * 2, words, f32=f32, seed=22)
        c.check(c.run())


@pytest.mark.parametrize("n_qh,new", [(4, 3), (4, 40), (16, 1), (7, 2)])
@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_rows_that_are_not_finite_reach_no_other(n_qh, new, f32):
    c = Case([200, 120], [new, new], n_qh, ALL, ALL, 30, f32=f32, seed=23)
    want = c.run()
    c.check(want)
    bad = torch.zeros(c.q.shape[:2], dtype=torch.bool, device="cuda")
    for t, h, x in ((0, 0, float("inf")), (2 * new - 1, 2 * n_qh - 1, float("nan")), (new - 1, 1, -float("inf")), (new, n_qh, float("nan"))):
        c.q[t, h, 5 + h] = x
        bad[t, h] = True
    out = c.run()
    assert torch.isnan(out[bad]).any(-1).all()
    # rows of a KV head share a power of two that scales their two fp16 parts: 2^-20 of the score
    off = (out.float() - want.float()).abs()[~bad]
    assert (off <= (2.0 ** -15 if f32 else 2.0 ** -7) * want.float().abs().max()).all()


def test_pools_past_two_to_the_31_words():
    c = Case([700, 130, 65], [1, 40, 1], 4, ALL, ALL, 30, seed=24, f32=True)
    want = c.run()
    n, small, words = 600_000, c.cache.n_pages, c.pools[0].shape[1]
    assert n * words > 2 ** 31
    far = S.PagedCache(n, c.page, c.cache.rows, c.cache.row_pages)
    pools = [torch.zeros((n, words), dtype=torch.int32, device="cuda") for _ in range(2)]
    for p, s in zip(pools, c.pools):
        p[n - small:] = s
    far.table.copy_(torch.where(c.cache.table >= 0, c.cache.table + (n - small), c.cache.table))
    far.lens.copy_(c.cache.lens)
    far.refs[n - small:] = c.cache.refs
    near, near_pools = c.cache, c.pools
    c.cache, c.pools = far, pools
    assert torch.equal(c.run(), want)
    x = torch.randn((42, 2, D), device="cuda")
    for cache, ps in ((near, near_pools), (far, pools)):
        S.spectra_paged_encode(cache, c.ck, c.cv, *ps, x, x, c.cu)
    for p, s in zip(pools, near_pools):
        assert torch.equal(p[n - small:], s) and not p[:n - small].any()
    want = c.run()
    moved = S.spectra_pages_compact(far, pools)  # over the whole distance
    used = int((near.refs > 0).sum())
    assert int(moved[-1]) == used and (far.table[0, :11] < used).all() and int((far.refs > 0).sum()) == used
    assert torch.equal(c.run(), want)


@pytest.mark.parametrize("n_qh,new", [(4, [1, 1, 1]), (1, [4, 2, 1]), (2, [2, 0, 2]), (5, [1, 1, 1])])
@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_few_rows_whatever_the_longest_that_the_call_allows(n_qh, new, f32):
    # short sequences under bounds of their own length and far above
    c = Case([300, 65, 1], new, n_qh, ALL, ALL[::-1], 30, f32=f32, seed=25)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    for bound in (300, 2049, 1_000_000):
        c.check(c.run(max_tokens=bound, lse=lse), lse)
