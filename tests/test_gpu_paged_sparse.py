"""Boxes of blocks, the selection by them, and attention over listed blocks, against the definitions in 64 bits; and the
calls of a serving step together."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D, MapModel, codec, from_pool, records, to_pool
from paged_sparse_ref import ALL, B8, BLOCK, NONE, block_values, box_of, boxes, cache, check, list_sees, tree, tree_sees

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def whole(c, **kw):
    """Boxes of all blocks of cache c."""
    box = c.cache.empty_bounds(c.ck)
    S.spectra_paged_bounds(c.cache, c.ck, c.pools[0], box, ints(np.concatenate([[0], np.cumsum(c.lens)])), sum(c.lens), **kw)
    return box


# ---------------------------------------------------------------------------
# Boxes
# ---------------------------------------------------------------------------
def check_boxes(c, box, bits, page, first, ends=None, start=-7):
    """Blocks from first[b] on hold their slots' least and largest values, all other words `start`."""
    got = box.cpu().numpy()
    untouched = np.full(got.shape, start, np.int32)
    table = c.cache.table.cpu().numpy()
    tpp = page // 64
    raw = untouched.reshape(got.shape[0], c.H, tpp, 4, 32)
    for b, L in enumerate(c.lens if ends is None else ends):
        for h in range(c.H):
            want = boxes(c.coef[b][h][0], max(L, 0))
            for i in range(first[b], len(want)):
                mine, _ = box_of(got, table[b], i, page, h, c.H, bits[h])
                live = np.repeat(np.asarray(bits[h]) > 0, 32)
                # one rounding to fp16, and the coefficient's own before it: half a step each, of 2^-11, and of subnormals
                tol = 2 * 2.0 ** -11 * np.abs(want[i]) + 2.0 ** -24
                assert (np.abs(mine - want[i])[:, live] <= tol[:, live]).all(), (b, h, i)
                kept = int((np.asarray(bits[h]) > 0).sum())
                raw[table[b, i // tpp], h, i % tpp, :kept] = got.reshape(raw.shape)[table[b, i // tpp], h, i % tpp, :kept]
    assert np.array_equal(got, untouched)


@pytest.mark.parametrize("page", [64, 128, 192])
@pytest.mark.parametrize("bits,words", [(B8, 8), (ALL, 30), (NONE, 30), ([[8, 8, 8, 8]], 36), ([[1, 0, 0, 0]], 5), ([[0, 0, 0, 0]], 5),
                                        ([[3, 0, 7, 0], [0, 6, 0, 0], [2, 2, 2, 0]], 16)])
def test_boxes(bits, words, page):
    lens = [300, 1, 64, 65, 0, 127, 700]
    c = cache(lens, [1] * 7, 1, bits, bits, words, page=page, seed=words)
    rng = np.random.default_rng(words)
    for new in (lens, [min(1, n) for n in lens], [int(rng.integers(0, n + 1)) for n in lens]):
        box = c.cache.empty_bounds(c.ck).fill_(-7)
        S.spectra_paged_bounds(c.cache, c.ck, c.pools[0], box, ints(np.concatenate([[0], np.cumsum(new)])), sum(new))
        check_boxes(c, box, bits, page, [(n - m) // 64 if m else 99 for n, m in zip(lens, new)])


def test_boxes_of_ends_rows_and_missing_pages():
    lens = [300, 90, 200, 64]
    c = cache(lens, [1] * 4, 1, seed=1)
    ends = [130, -1, 200, 3]
    new = [100, 5, 40, 9]  # of the last, six lie before slot 0
    box = c.cache.empty_bounds(c.ck).fill_(-7)
    cu = ints(np.concatenate([[0], np.cumsum(new)]))
    S.spectra_paged_bounds(c.cache, c.ck, c.pools[0], box, cu, sum(new), ends=ints(ends))
    check_boxes(c, box, B8, 64, [0, 99, 2, 0], ends)
    # fewer tokens than the starts say: cut
    box2 = c.cache.empty_bounds(c.ck).fill_(-7)
    S.spectra_paged_bounds(c.cache, c.ck, c.pools[0], box2, cu, 100, ends=ints(ends))
    check_boxes(c, box2, B8, 64, [0, 99, 99, 99], ends)
    # rows in another order, one of them out of range; a page out of range is passed over
    c.cache.table[2, 3] = c.cache.n_pages
    box3 = c.cache.empty_bounds(c.ck).fill_(-7)
    S.spectra_paged_bounds(c.cache, c.ck, c.pools[0], box3, ints([0, 200, 264, 300]), 300, rows=ints([2, 3, 9]))
    c.cache.table[2, 3] = 0
    c.lens = [0, 0, 192, 64]
    check_boxes(c, box3, B8, 64, [9, 9, 0, 0])


def test_boxes_of_metadata_that_is_not_finite():
    """It counts as 0 and reaches no other coefficient; scales too large for fp16 are lowered."""
    c = cache([64], [1], 1, [[4, 4, 0, 0]], [[4, 4, 0, 0]], 10, seed=2)
    page = int(c.cache.table[0, 0])
    words = c.pools[0][page].view(1, 10, 64)
    words[0, 0, 5] = 0x7C00  # infinite scale of group 0, slot 5
    words[0, 1, 9] = 0x7E00 << 16  # NaN zero point of group 1, slot 9
    words[0, 0, 11] = 0x7BFF  # a scale of 65504
    words[0, 2:6, 11] = 0x11111111  # codes 1, so 65504 each; lowered to 65472 / 15
    box = whole(c)
    got, _ = box_of(box.cpu().numpy(), c.cache.table[0].cpu().numpy(), 0, 64, 0, 1, [4, 4, 0, 0])
    coef = c.coef[0][0][0].copy()
    coef[5, :32], coef[9, 32:64], coef[11, :32] = 0.0, 0.0, float(np.float16(65472.0 / 15))
    want = boxes(coef, 64)[0]
    assert np.isfinite(got).all() and (np.abs(got - want) <= 2 * 2.0 ** -11 * np.abs(want) + 2.0 ** -24).all()


# ---------------------------------------------------------------------------
# Selection
# ---------------------------------------------------------------------------
def select(c, box, n_blocks, **kw):
    kw.setdefault("max_tokens", max(c.lens + [1]))
    return S.spectra_paged_select(c.cache, c.ck, box, kw.pop("q", c.q), c.cu, n_blocks, **kw)


def check_selection(c, got, box, bits, page, n_blocks, first=1, last=1, ends=None):
    """Every list: ascending, as many as there are up to n_blocks, the first and last among them, and no block left out
    whose value passes a chosen one's by more than the products' errors (2^-20 of sum |q' box|, twice, for the
    values and the best of their heads)."""
    got, raw = got.cpu().numpy(), box.cpu().numpy()
    q = c.q.float().cpu().numpy().astype(np.float64)
    table = c.cache.table.cpu().numpy()
    at = 0
    for b, n in enumerate(c.new):
        L = c.lens[b] if ends is None else ends[b]
        for h in range(c.H):
            basis = c.state(h)[0]
            boxed = np.stack([box_of(raw, table[b], i, page, h, c.H, bits[h])[0] for i in range(-(-max(L, 0) // 64))] or [np.zeros((2, D))])
            boxed = boxed * np.repeat(np.asarray(bits[h]) > 0, 32)
            for i in range(n):
                lim = max(0, L - n + i + 1) if L >= 0 else 0
                have = -(-lim // 64)
                mine = got[at + i, h]
                k = min(have, n_blocks)
                assert (mine[k:] == -1).all() and (np.diff(mine[:k]) > 0).all(), (b, h, i, mine)
                if k == 0:
                    continue
                assert mine[0] >= 0 and mine[k - 1] < have
                forced = {j for j in range(have) if j < first or j >= have - last}
                assert have <= n_blocks or forced <= set(mine.tolist())
                v, size = block_values(q[at + i, h * c.n_qh:(h + 1) * c.n_qh], boxed, basis, np.arange(len(boxed)) < have)
                taken = [j for j in mine[:k] if j not in forced]
                left = np.setdiff1d(np.arange(have), mine[:k])
                if taken and len(left):
                    assert v[taken].min() >= v[left].max() - 4 * 2.0 ** -20 * size, (b, h, i)
        at += n


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([64 * 40], [1]), ([64 * 40 + 1], [1]), ([5000], [70]), ([3000, 0, 64, 65, 4000], [3, 0, 1, 2, 21]),
                                      ([700, 2000, 1500], [1, 1, 1]), ([900], [900])])
def test_selection(lens, new, f32):
    c = cache(lens, new, f32=f32, seed=sum(lens))
    box = whole(c)
    for n_blocks, first, last in ((8, 1, 1), (3, 1, 2), (1, 0, 0), (30, 4, 5), (100, 0, 0)):
        check_selection(c, select(c, box, n_blocks, first=first, last=last), box, B8, 64, n_blocks, first, last)


@pytest.mark.parametrize("n_qh", [1, 2, 3, 7, 9, 16])
def test_selection_heads(n_qh):
    for new in ([1, 1], [5, 40]):
        c = cache([3000, 2000], new, n_qh, seed=n_qh)
        box = whole(c)
        check_selection(c, select(c, box, 9), box, B8, 64, 9)


@pytest.mark.parametrize("bits,words,page", [(ALL, 30, 128), (NONE, 30, 64), ([[8, 8, 8, 8]], 36, 192), ([[0, 0, 0, 0]], 5, 64), ([[1, 0, 0, 0]], 5, 64)])
def test_selection_widths(bits, words, page):
    c = cache([2000, 1000], [3, 2], 3, bits, bits, words, page=page, seed=words)
    box = whole(c)
    check_selection(c, select(c, box, 9), box, bits, page, 9)


def test_selection_long():
    """More blocks than LDS holds keys for, one sequence; and a call of many tokens."""
    lens = [64 * 20000 + 7]
    rng = np.random.default_rng(0)
    ck, _ = codec([[4, 4, 0, 0]], 10, 1)
    n_pages = -(-lens[0] // 1024)
    cache_ = S.PagedCache(n_pages, 1024, 1, n_pages)
    cache_.table[0] = ints(rng.permutation(n_pages))
    cache_.lens[0] = lens[0]
    box = torch.randn((n_pages, 1, 16, 4, 2, 32), device="cuda").sort(-2).values.half().contiguous()
    q = torch.randn((2, 4, D), device="cuda")
    cu = ints([0, 2])
    got = S.spectra_paged_select(cache_, ck, box.view(torch.int32).view(n_pages, -1), q, cu, 200, lens[0]).cpu().numpy()
    flat = box[cache_.table[0].long()].reshape(-1, 4, 2, 32)[:20001].double()
    qp = q.double() @ ck.basis[0].double()
    for t in range(2):
        x = flat[:, :2].permute(0, 2, 1, 3).reshape(-1, 2, 64)  # [blocks, side, 64]
        s = qp[t, :, :64].clamp(min=0) @ x[:, 1].T + qp[t, :, :64].clamp(max=0) @ x[:, 0].T
        v = (s - s.amax(1, keepdim=True)).amax(0).cpu().numpy()
        mine = got[t, 0]
        assert (np.diff(mine) > 0).all() and mine[0] == 0 and mine[-1] == 20000
        left = np.setdiff1d(np.arange(20001), mine)
        size = float((qp[t].abs()[:, :64] @ x.abs().amax(1).T).max())
        assert v[mine[1:-1]].min() >= v[left].max() - 4 * 2.0 ** -20 * size


@pytest.mark.parametrize("n", [40, 500, 1500, 3000, 10000, 17000])
def test_selection_of_equal_values(n):
    """Boxes of small whole numbers and an identity basis: values are exact, ties go to the lowest index, however many
    there are."""
    ck, _ = codec([[4, 0, 0, 0]], 10, 1)
    ck.basis[0] = torch.eye(D)
    m = S.PagedCache(n, 64, 1, n)
    m.table[0] = ints(np.arange(n)[::-1].copy())
    m.lens[0] = n * 64
    box = torch.zeros((n, 1, 1, 4, 2, 32), dtype=torch.float16, device="cuda")
    pool = box.view(torch.int32).view(n, -1)
    rng = np.random.default_rng(n)
    ks = [1, 2, 5, 15, 16, 20, 25, 39] + [k for k in (n // 3, n // 2, n - 1) if k <= 4096]
    # a few values again and again; one block far below, beside which the others are nearly alike; two values; all alike
    for vals in (np.array([3, 7, 7, 1, 7, 2, 5, 5] * n)[:n], np.where(np.arange(n) == 11, -60000, rng.integers(0, 5, n)),
                 rng.integers(0, 2, n), np.zeros(n, np.int64)):
        box[m.table[0].long(), 0, 0, 0, 1, 0] = torch.tensor(vals, dtype=torch.float16, device="cuda")
        for heads in (1, 4):
            q = torch.zeros((1, heads, D), device="cuda")
            q[:, :, 0] = 2.0
            for k in ks:
                got = S.spectra_paged_select(m, ck, pool, q, ints([0, 1]), k, n * 64, first=0, last=0).cpu().numpy()[0, 0]
                assert np.array_equal(got, np.sort(np.argsort(-vals, kind="stable")[:k])), (heads, k)
            got = S.spectra_paged_select(m, ck, pool, q, ints([0, 1]), 6, n * 64, first=1, last=2).cpu().numpy()[0, 0]
            rest = 1 + np.argsort(-vals[1:n - 2], kind="stable")[:3]
            assert got.tolist() == sorted([0, n - 2, n - 1, *rest.tolist()])
    # many tokens: another way through the scores
    vals = np.where(np.arange(n) == 11, -60000, rng.integers(0, 5, n))
    box[m.table[0].long(), 0, 0, 0, 1, 0] = torch.tensor(vals, dtype=torch.float16, device="cuda")
    for heads in (1, 3, 7, 16):
        q = torch.zeros((300, heads, D), device="cuda")
        q[:, :, 0] = 1.0 + torch.arange(300, device="cuda")[:, None] % 3
        got = S.spectra_paged_select(m, ck, pool, q, ints([0, 300]), 20, n * 64, first=0, last=0).cpu().numpy()[:, 0]
        for t in (0, 36, 100, 299):
            have = -(-(n * 64 - 300 + t + 1) // 64)
            assert np.array_equal(got[t], np.sort(np.argsort(-vals[:have], kind="stable")[:20])), (heads, t)


def test_selection_of_what_is_not_finite():
    c = cache([2000], [4], 4, f32=True, seed=3)
    box = whole(c)
    want = select(c, box, 8)
    q = c.q.clone()
    q[1, 0, 3] = float("nan")  # one head of four: the others decide
    q[2, :4] = float("nan")    # all heads of a KV head: the lowest indices
    q[3, 5, 0] = float("inf")
    got = select(c, box, 8, q=q)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1, 1], want[1, 1]) and torch.equal(got[2, 1], want[2, 1])
    assert torch.equal(got[3, 0], want[3, 0])
    assert got[2, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 31]
    for t in got.reshape(-1, 8).tolist():
        assert t == sorted(set(t)) and t[0] == 0 and t[-1] == 31 and min(t) >= 0


def test_selection_rows_left_and_ends():
    lens, new = [2000, 900, 1500, 70], [3, 2, 4, 5]
    c = cache(lens, new, seed=4)
    box = whole(c)
    ends = [2000, -1, 700, 3]
    out = torch.full((14 + 2, 2, 6), 77, dtype=torch.int32, device="cuda")
    q = torch.cat([c.q, c.q[:2]])
    S.spectra_paged_select(c.cache, c.ck, box, q, c.cu, 6, 2000, ends=ints(ends), out=out)
    assert (out[14:] == 77).all() and (out[3:5] == -1).all() and (out[9:11] == -1).all()
    check_selection(c, out[:14], box, B8, 64, 6, ends=ends)
    out.fill_(77)
    S.spectra_paged_select(c.cache, c.ck, box, q, c.cu, 6, 1999, out=out)
    assert (out[:3] == 77).all() and not (out[3:14] == 77).any()


# ---------------------------------------------------------------------------
# Attention over lists
# ---------------------------------------------------------------------------
def attend(c, blocks, **kw):
    return S.spectra_paged_sparse_attention(c.cache, c.ck, c.cv, *c.pools, kw.pop("q", c.q), c.cu, ints(blocks), **kw)


def lists(c, most, seed=0, ends=None):
    rng = np.random.default_rng([seed, 3])
    out = np.full((sum(c.new), c.H, most), -1)
    at = 0
    for b, n in enumerate(c.new):
        L = c.lens[b] if ends is None else ends[b]
        for i in range(n):
            have = -(-max(0, L - n + i + 1) // 64)
            for h in range(c.H):
                k = int(rng.integers(0, min(have, most) + 1))
                out[at + i, h, :k] = np.sort(rng.permutation(have)[:k])
        at += n
    return out


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new,most", [([1], [1], 1), ([64], [1], 3), ([65], [1], 2), ([2000], [1], 7), ([2000], [1], 32), ([500], [500], 5),
                                           ([1000, 1, 63, 0, 65, 700], [1, 1, 1, 0, 1, 1], 9), ([900, 2500], [33, 70], 12), ([30000], [2], 400),
                                           ([700], [200], 11)])
def test_lists(lens, new, most, f32):
    c = cache(lens, new, f32=f32, seed=sum(lens) + most)
    blocks = lists(c, most, seed=most)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    check(c, list_sees(lens, new, blocks), attend(c, blocks, lse=lse), lse)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_qh", [1, 3, 7, 8, 16])
def test_list_heads(n_qh, f32):
    c = cache([900, 700], [1, 30], n_qh, f32=f32, seed=n_qh)
    blocks = lists(c, 8, seed=n_qh)
    check(c, list_sees(c.lens, c.new, blocks), attend(c, blocks))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("bits_k,bits_v,words,page", [(ALL, ALL[::-1], 30, 128), (NONE, ALL, 30, 64), (ALL, NONE, 30, 192),
                                                      ([[8, 8, 8, 8]], [[8, 8, 8, 8]], 36, 64), ([[0, 0, 0, 0]], [[0, 0, 0, 0]], 5, 64)])
def test_list_widths_and_pages(bits_k, bits_v, words, page, f32):
    c = cache([900, 300], [2, 9], 3, bits_k, bits_v, words, page=page, f32=f32, seed=words)
    blocks = lists(c, 6, seed=words)
    check(c, list_sees(c.lens, c.new, blocks), attend(c, blocks))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_lists_that_do_not_ascend(f32):
    """Entries not above all before them, out of range or unseen are passed over, in every chunk of a list."""
    rng = np.random.default_rng(5)
    c = cache([3000, 1000], [3, 2], f32=f32, seed=5)
    blocks = rng.integers(-3, 60, (5, 2, 700))
    blocks[0, 0, :] = np.repeat(np.arange(350), 2)  # every block twice
    blocks[1, 0, :] = 2 ** 31 - 1
    blocks[1, 1, :] = np.arange(700)[::-1]
    blocks[2, 0, :5] = [7, 2 ** 31 - 1, 8, 9, 10]   # nothing is above that
    blocks[2, 1, :] = -1
    blocks[2, 1, 699] = 11
    lse = torch.empty(c.q.shape[:2], device="cuda")
    check(c, list_sees(c.lens, c.new, blocks), attend(c, blocks, lse=lse), lse)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_all_blocks_are_causal_attention(f32):
    c = cache([900, 300, 2000], [5, 90, 1], f32=f32, seed=6)
    blocks = np.tile(np.arange(32), (96, 2, 1))
    got = attend(c, blocks).float()
    want = S.spectra_paged_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, 90, 2000).float()
    assert (got - want).norm() <= (1e-5 if f32 else 8e-3) * want.norm()
    check(c, list_sees(c.lens, c.new, blocks), got.to(c.q.dtype))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_sparse_rows_that_see_nothing_strides_and_nan(f32):
    lens, new = [500, 200, 100, 300], [3, 4, 5, 6]
    c = cache(lens, new, f32=f32, seed=7)
    ends = [500, -1, 2, 300]
    blocks = lists(c, 5, seed=7, ends=ends)
    blocks[-1] = -1
    lse = torch.empty(c.q.shape[:2], device="cuda")
    out = attend(c, blocks, ends=ints(ends), lse=lse)
    check(c, list_sees(ends, new, blocks), out, lse)
    assert (out[3:10] == 0).all() and (out[-1] == 0).all() and torch.isneginf(lse[-1]).all()
    # strides; a type of its own for the output; rows that no sequence holds
    n, H = c.q.shape[:2]
    wide = torch.full((H, n + 2, D + 8), float("nan"), dtype=c.q.dtype, device="cuda")
    wide[:, :n, :D] = c.q.transpose(0, 1)
    q = torch.cat([c.q, c.q[:2]])
    more = np.concatenate([blocks, blocks[:2]])
    buf = torch.full_like(q, 7.0)
    assert torch.equal(out, attend(c, blocks, q=wide.transpose(0, 1)[:n, :, :D], ends=ints(ends)))
    attend(c, more, q=q, ends=ints(ends), out=buf)
    assert (buf[-2:] == 7).all() and torch.equal(buf[:-2], out)
    other = torch.empty(c.q.shape, dtype=torch.bfloat16 if f32 else torch.float32, device="cuda")
    check(c, list_sees(ends, new, blocks), attend(c, blocks, ends=ints(ends), out=other))
    # not finite
    q = c.q.clone()
    q[1, 2, 5] = float("nan")
    bad = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    bad[1, 2] = True
    got = attend(c, blocks, q=q, ends=ints(ends))
    assert torch.equal(got[~bad], out[~bad])
    assert torch.isnan(got[1, 2]).all() or (blocks[1, 0] < 0).all()


def test_sparse_starts_that_fall_and_pages_out_of_range_stay_inside():
    c = cache([900, 300, 2000], [5, 20, 7], seed=8)
    box = whole(c)
    blocks = lists(c, 6, seed=8)
    c.cache.table[0, 1] = 2 ** 31 - 1
    c.cache.table[2, 3] = -5
    for cu in ([0, 20, 10, 30], [-5, 90, 2, 200], [30, 3, 2, 1]):
        out = torch.zeros((32 + 64, *c.q.shape[1:]), dtype=c.q.dtype, device="cuda")
        S.spectra_paged_sparse_attention(c.cache, c.ck, c.cv, *c.pools, c.q, ints(cu), ints(blocks), out=out[32:-32])
        assert (out[:32] == 0).all() and (out[-32:] == 0).all() and torch.isfinite(out.float()).all()
        sel = torch.full((32 + 64, 2, 6), 77, dtype=torch.int32, device="cuda")
        S.spectra_paged_select(c.cache, c.ck, box, c.q, ints(cu), 6, 2000, out=sel[32:-32])
        assert (sel[:32] == 77).all() and (sel[-32:] == 77).all()
        b2 = torch.zeros((box.shape[0] + 2, box.shape[1]), dtype=torch.int32, device="cuda")
        S.spectra_paged_bounds(c.cache, c.ck, c.pools[0], b2[1:-1], ints(cu), 30)
        assert (b2[0] == 0).all() and (b2[-1] == 0).all()


def test_pools_past_32_bits():
    """Pages whose records lie past 2^31 words."""
    rng = np.random.default_rng(9)
    bits = [[5, 1, 0, 0]] * 8
    (ck, pk), (cv, pv) = codec(bits, 8, 1), codec(bits, 8, 2)
    page, n_pages, L, new = 256, 140000, 700, 3
    m = S.PagedCache(n_pages, page, 1, 4)
    ids = [n_pages - 1, n_pages - 7, n_pages - 3]
    m.table[0, :3] = ints(ids)
    m.lens[0] = L
    pools = [m.empty_pool(x) for x in (ck, cv)]
    assert pools[0].numel() > 2 ** 31
    small = [np.zeros((3, page * 8 * 8), np.int32) for _ in range(2)]
    coef = []
    for h in range(8):
        got = [records(bits[h], p, L, rng) for p in (pk, pv)]
        for t in (0, 1):
            to_pool(small[t], got[t][0], np.arange(3), page, h, 8)
        coef.append((got[0][1], got[1][1]))
    for t in (0, 1):
        pools[t][ids] = torch.from_numpy(small[t]).cuda()

    class C:
        lens, H, n_qh, cache = [L], 8, 4, m
    c = C()
    c.new, c.ck, c.cv, c.pools, c.coef = [new], ck, cv, pools, [coef]
    c.state = lambda h: [t.cpu().numpy().astype(np.float64) for t in (ck.basis[h], ck.mean[h], cv.basis[h], cv.mean[h])]
    c.q = torch.from_numpy((2 * rng.standard_normal((new, 32, D))).astype(np.float32)).cuda().bfloat16()
    c.cu = ints([0, new])
    p = tree("star", [new])
    check(c, tree_sees([L], [new], p), S.spectra_paged_tree_attention(m, ck, cv, *pools, c.q, c.cu, ints(p), new, L))
    box = whole(c)
    sel = S.spectra_paged_select(m, ck, box, c.q, c.cu, 5, L)
    check_selection(c, sel, box, bits, page, 5)
    check(c, list_sees([L], [new], sel.cpu().numpy()), S.spectra_paged_sparse_attention(m, ck, cv, *pools, c.q, c.cu, sel))
    before = pools[0][ids].clone()
    ends = S.spectra_pages_accept(_with_refs(m, ids), ints([0]), ints([3]), ints([[1, 2, 0]]), ints([2]), pools, 8)
    assert ends.tolist() == [L - 1]
    got, was = (from_pool(x.cpu().numpy(), np.arange(3), L, page, 3, 8, 8) for x in (pools[0][ids], before))
    was[L - 3:L - 1] = was[L - 2:L]
    assert np.array_equal(got, was)


def _with_refs(m, ids):
    m.refs[ids] = 1
    return m


# ---------------------------------------------------------------------------
# Graphs, streams, and the calls together
# ---------------------------------------------------------------------------
def test_captured_and_on_other_streams():
    c = cache([3000, 900], [2, 30], seed=10)
    box = whole(c)
    ws = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (
        S.spectra_paged_select_workspace_bytes(32, 8, 2, 3000), S.spectra_paged_sparse_attention_workspace_bytes(32, 8, 2, 9))]
    q, sel, out = c.q.clone(), torch.empty((32, 2, 9), dtype=torch.int32, device="cuda"), torch.empty_like(c.q)
    boxes_ = torch.zeros_like(box)
    cu_all = ints([0, 3000, 3900])

    def step(stream=None):
        S.spectra_paged_bounds(c.cache, c.ck, c.pools[0], boxes_, cu_all, 3900, stream=stream)
        S.spectra_paged_select(c.cache, c.ck, boxes_, q, c.cu, 9, 3000, out=sel, workspace=ws[0], stream=stream)
        S.spectra_paged_sparse_attention(c.cache, c.ck, c.cv, *c.pools, q, c.cu, sel, out=out, workspace=ws[1], stream=stream)
    q2 = (c.q.float() * 0.7 + 0.1).bfloat16()
    want = []
    for x in (c.q, q2):
        q.copy_(x)
        step()
        want.append((sel.clone(), out.clone()))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for i in range(6):
        q.copy_(c.q if i % 2 == 0 else q2)
        sel.fill_(0)
        boxes_.zero_()
        graphs[i // 2 % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(boxes_, box)
        assert torch.equal(sel, want[i % 2][0]) and torch.equal(out, want[i % 2][1])
    side = torch.cuda.Stream()
    q.copy_(c.q)
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want[0][1])


def test_speculative_steps_over_selected_blocks():
    """A serving loop: prompts, then steps that draft a tree, attend with it, keep a path and attend over selected
    blocks. The cache ends as if the kept tokens alone had been appended, byte for byte, and the boxes likewise."""
    rng = np.random.default_rng(12)
    H, qh, words, page, B = 2, 4, 8, 64, 3
    bits = [[5, 1, 0, 0], [4, 2, 0, 0]]
    (ck, _), (cv, _) = codec(bits, words, 1), codec(bits[::-1], words, 2)
    maps = [S.PagedCache(80, page, B, 20) for _ in range(2)]  # with drafts, and without
    pools = [[m.empty_pool(x) for x in (ck, cv)] for m in maps]
    box = [m.empty_bounds(ck) for m in maps]
    rows = ints(range(B))

    def append(i, n, k, v):
        cu = ints(np.concatenate([[0], np.cumsum(n)]))
        ends = S.spectra_pages_extend(maps[i], rows, ints(n), pools[i])
        S.spectra_paged_encode(maps[i], ck, cv, *pools[i], k, v, cu, rows=rows, ends=ends)
        S.spectra_paged_bounds(maps[i], ck, pools[i][0], box[i], cu, int(sum(n)), rows=rows, ends=ends)
        return cu

    def new(n):
        return [torch.from_numpy(rng.standard_normal((int(sum(n)), H, D)).astype(np.float32)).cuda().bfloat16() for _ in range(2)]
    n = [700, 64, 333]
    k, v = new(n)
    for i in range(2):
        append(i, n, k, v)
    lens = np.array(n)
    for _ in range(4):
        n = rng.integers(1, 30, B)
        k, v = new(n)
        cu = append(0, n, k, v)
        at = np.concatenate([[0], np.cumsum(n)])
        p = tree("random", list(n), seed=int(sum(n)))
        q = torch.from_numpy(rng.standard_normal((int(sum(n)), H * qh, D)).astype(np.float32)).cuda().bfloat16()
        out = S.spectra_paged_tree_attention(maps[0], ck, cv, *pools[0], q, cu, ints(p), 30, 1000, rows=rows)
        # a path from a random leaf to the history
        path, counts, kept = np.full((B, 30), -1), [], []
        for b in range(B):
            leaf, up = int(rng.integers(0, n[b])), []
            while leaf >= 0:
                up.append(leaf)
                leaf = int(p[at[b] + leaf])
            path[b, :len(up)] = up[::-1]
            counts.append(len(up))
            kept.append(at[b] + np.array(up[::-1]))
        ends = S.spectra_pages_accept(maps[0], rows, ints(n), ints(path), ints(counts), pools[0], H)
        lens = lens + np.array(counts)
        assert ends.tolist() == lens.tolist()
        S.spectra_paged_bounds(maps[0], ck, pools[0][0], box[0], ints(np.concatenate([[0], np.cumsum(counts)])), int(sum(counts)), rows=rows, ends=ends)
        pick = torch.from_numpy(np.concatenate(kept)).cuda()
        cu1 = append(1, counts, k[pick], v[pick])
        # the kept tokens' causal attention is their attention in the tree
        causal = S.spectra_paged_attention(maps[1], ck, cv, *pools[1], q[pick], cu1, 30, 1000, rows=rows)
        assert (causal.float() - out[pick].float()).norm() <= 8e-3 * causal.float().norm()
        # what the two maps hold
        tables = [m.table.cpu().numpy() for m in maps]
        for b in range(B):
            for t, w in enumerate((words, words)):
                for h in range(H):
                    a, c = (from_pool(pools[i][t].cpu().numpy(), tables[i][b], lens[b], page, h, H, w) for i in range(2))
                    assert np.array_equal(a, c), (b, t, h)
            nb = -(-int(lens[b]) // page)
            assert torch.equal(box[0][tables[0][b, :nb]], box[1][tables[1][b, :nb]])
        one = q[pick][torch.tensor(np.cumsum(counts) - 1, device="cuda")].contiguous()
        cub = ints(range(B + 1))
        got = []
        for i in range(2):
            sel = S.spectra_paged_select(maps[i], ck, box[i], one, cub, 5, 1000, rows=rows)
            got.append((sel, S.spectra_paged_sparse_attention(maps[i], ck, cv, *pools[i], one, cub, sel, rows=rows)))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        # every block listed: causal attention of the single tokens
        full = S.spectra_paged_sparse_attention(maps[0], ck, cv, *pools[0], one, cub, ints(np.tile(np.arange(16), (B, H, 1))), rows=rows)
        dense = S.spectra_paged_attention(maps[0], ck, cv, *pools[0], one, cub, 1, 1000, rows=rows)
        assert (full.float() - dense.float()).norm() <= 8e-3 * dense.float().norm()


def test_boxes_follow_their_pages():
    """Forked, copied on write and compacted together with the records."""
    c = cache([300, 100], [1, 1], seed=13)
    m, rng = MapModel(30, 64, 6, 8), np.random.default_rng(1)
    for b, n in enumerate(c.lens):
        k = -(-n // 64)
        m.table[b, :k] = c.cache.table[b, :k].cpu().numpy()
        m.lens[b] = n
        m.refs[m.table[b, :k]] = 1
    mc = m.cache()
    pools = [torch.zeros((30, p.shape[1]), dtype=torch.int32, device="cuda") for p in c.pools]
    for p, o in zip(pools, c.pools):
        p[:o.shape[0]] = o
    box = mc.empty_bounds(c.ck)
    S.spectra_paged_bounds(mc, c.ck, pools[0], box, ints([0, 300, 400]), 400)
    S.spectra_pages_fork(mc, ints([0, 1]), ints([2, 3]))
    S.spectra_pages_extend(mc, ints([2, 3]), ints([10, 3]), [*pools, box])
    S.spectra_pages_truncate(mc, ints([2, 3, 0]), ints([300, 100, 70]))
    S.spectra_pages_compact(mc, [*pools, box])
    q = torch.from_numpy(rng.standard_normal((2, 8, D)).astype(np.float32)).cuda()
    table = mc.table.cpu().numpy()
    for row, L in ((2, 300), (3, 100), (0, 70)):
        for h in range(2):
            src = c.coef[{2: 0, 3: 1, 0: 0}[row]][h][0]
            want = boxes(src, {2: 300, 3: 100, 0: 128}[row])  # a cut block's box still holds its slots
            for i in range(-(-L // 64)):
                got, _ = box_of(box.cpu().numpy(), table[row], i, 64, h, 2, B8[h])
                live = np.repeat(np.asarray(B8[h]) > 0, 32)
                assert (np.abs(got - want[i])[:, live] <= (2 * 2.0 ** -11 * np.abs(want[i]) + 2.0 ** -24)[:, live]).all()
    sel = S.spectra_paged_select(mc, c.ck, box, q, ints([0, 1, 2]), 3, 300, rows=ints([2, 3]))
    assert sel.shape == (2, 2, 3) and sel.min() >= -1


@pytest.mark.parametrize("n", [160, 600, 1100])
def test_selection_of_many_tokens_that_are_not_finite(n):
    """Heads that have no number are passed over, and no token reaches another's, whichever way the best heads are found."""
    c = cache([2600], [n], 4, f32=True, seed=9)
    box = whole(c)
    want = select(c, box, 8)
    check_selection(c, want, box, B8, 64, 8)
    q, copy = c.q.clone(), c.q.clone()
    q[1, 0, 3], copy[1, 0] = float("nan"), c.q[1, 1]  # as if the head were another's twin
    q[n // 2, :4] = float("nan")
    q[n - 1, 5, 0] = float("inf")
    got, twin = select(c, box, 8, q=q), select(c, box, 8, q=copy)
    same = torch.ones(n, dtype=torch.bool, device="cuda")
    same[[1, n // 2, n - 1]] = False
    assert torch.equal(got[same], want[same]) and torch.equal(got[1], twin[1])
    have = -(-(2600 - n + n // 2 + 1) // 64)
    assert got[n // 2, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, have - 1] and torch.equal(got[n // 2, 1], want[n // 2, 1])
    assert torch.equal(got[n - 1, 0], want[n - 1, 0])


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3, 40, 150])
def test_lists_over_metadata_that_is_not_finite(new, f32):
    c = cache([300], [new], f32=f32, seed=10)
    page = int(c.cache.table[0, 1])
    k, v = (c.pools[i][page].view(2, 8, 64) for i in (0, 1))
    k[0, 0, 5] = 0x7C00
    k[1, 1, 9] = 0x7E00 << 16
    v[0, 1, 7] = 0xFC00
    v[0, 0, 11] = 0x7BFF
    v[0, 2:6, 11] = 0x11111111
    c.coef[0][0][0][69, :32] = c.coef[0][1][0][73, 32:64] = c.coef[0][0][1][71, 32:64] = 0.0
    c.coef[0][0][1][75, :32] = float(np.float16(65472.0 / 15))
    blocks = np.broadcast_to(np.array([0, 1, 3]), (new, 2, 3)).copy()
    lse = torch.empty(c.q.shape[:2], device="cuda")
    check(c, list_sees([300], [new], blocks), attend(c, blocks, lse=lse), lse)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_more_sequences_than_threads(f32):
    """Boxes, selection and lists of 300 short sequences over three KV heads, some with nothing new."""
    rng = np.random.default_rng(18)
    lens = rng.integers(6, 200, 300)
    new = rng.integers(1, 6, 300) * (rng.random(300) > 0.1)
    bits = [[5, 1, 0, 0], [4, 2, 0, 0], [1, 1, 1, 3]]
    c = cache(lens.tolist(), new.tolist(), 4, bits, bits[::-1], 10, f32=f32, seed=18)
    box = whole(c)
    check_boxes(c, box, bits, 64, [0] * 300, start=0)
    got = select(c, box, 3)
    check_selection(c, got, box, bits, 64, 3)
    blocks = got.cpu().numpy()
    lse = torch.empty(c.q.shape[:2], device="cuda")
    check(c, list_sees(lens, new, blocks), attend(c, blocks, lse=lse), lse)


@pytest.mark.parametrize("tokens", [1030, 2100])
@pytest.mark.parametrize("n", [200, 1500, 3000, 10000, 17000])
def test_equal_values_of_many_tokens(n, tokens):
    """As above, where a KV head's values are kept instead of its heads' scores."""
    ck, _ = codec([[4, 0, 0, 0]], 10, 1)
    ck.basis[0] = torch.eye(D)
    m = S.PagedCache(n, 64, 1, n)
    m.table[0] = ints(np.arange(n)[::-1].copy())
    m.lens[0] = n * 64
    box = torch.zeros((n, 1, 1, 4, 2, 32), dtype=torch.float16, device="cuda")
    vals = np.where(np.arange(n) == 11, -60000, np.random.default_rng(n).integers(0, 5, n))
    box[m.table[0].long(), 0, 0, 0, 1, 0] = torch.tensor(vals, dtype=torch.float16, device="cuda")
    for heads in (1, 3, 7, 16):
        q = torch.zeros((tokens, heads, D), device="cuda")
        q[:, :, 0] = 1.0 + torch.arange(tokens, device="cuda")[:, None] % 3
        got = S.spectra_paged_select(m, ck, box.view(torch.int32).view(n, -1), q, ints([0, tokens]), 20, n * 64, first=0, last=0)
        got = got.cpu().numpy()[:, 0]
        for t in (0, 36, 100, 299, tokens - 1):
            have = -(-(n * 64 - tokens + t + 1) // 64)
            assert np.array_equal(got[t], np.sort(np.argsort(-vals[:have], kind="stable")[:20])), (heads, t)


@pytest.mark.parametrize("n_qh", [1, 3, 7, 16])
@pytest.mark.parametrize("new", [[300, 0, 260], [1000, 7, 193]])
def test_selection_heads_of_many_tokens(new, n_qh):
    lens = [2600, 130, 700]
    c = cache(lens, new, n_qh, seed=n_qh + len(new))
    box = whole(c)
    check_selection(c, select(c, box, 9, first=2, last=1), box, B8, 64, 9, first=2)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_qh", [1, 3, 4, 7, 8])
def test_lists_of_neighbouring_tokens(n_qh, f32):
    """Tokens enough that neighbours' lists are read together: sequences of odd lengths, lists that fall, repeat, are
    empty or name blocks that a token does not see."""
    lens, new = [900, 2500, 64, 0, 333], [61, 83, 3, 0, 50]
    c = cache(lens, new, n_qh, f32=f32, seed=n_qh + 30)
    rng = np.random.default_rng(n_qh)
    blocks = lists(c, 12, seed=n_qh)
    blocks[5] = rng.integers(-3, 20, (2, 12))
    blocks[6, 0] = blocks[6, 0][::-1].copy()
    blocks[100:104, 1] = rng.integers(0, 60, (4, 12))
    blocks[70:75] = -1
    blocks[8, 1], blocks[9, 1] = 3, 2 ** 31 - 1
    lse = torch.empty(c.q.shape[:2], device="cuda")
    out = attend(c, blocks, lse=lse)
    check(c, list_sees(lens, new, blocks), out, lse)
    # a page out of range counts as nothing there, for its own sequence alone
    table = c.cache.table.clone()
    c.cache.table[1, 0] = -5
    got = attend(c, blocks)
    assert torch.isfinite(got.float()).all() and torch.equal(got[:61], out[:61]) and torch.equal(got[144:], out[144:])
    c.cache.table.copy_(table)


def test_lists_of_neighbouring_tokens_captured_and_not_finite():
    c = cache([3000], [140], f32=True, seed=31)
    blocks = ints(lists(c, 9, seed=31))
    want = S.spectra_paged_sparse_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, blocks)
    q, out = c.q.clone(), torch.empty_like(c.q)
    q[17, 3, 5], q[90, 0, 0] = float("nan"), float("inf")
    ws = torch.empty(S.spectra_paged_sparse_attention_workspace_bytes(140, 8, 2, 9), dtype=torch.uint8, device="cuda")
    call = lambda: S.spectra_paged_sparse_attention(c.cache, c.ck, c.cv, *c.pools, q, c.cu, blocks, out=out, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    same = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
    same[17, 3] = same[90, 0] = False
    for _ in range(3):
        out.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[same], want[same])
        assert torch.isnan(out[17, 3]).all() or (blocks[17, 0] < 0).all()
        assert torch.equal(S.spectra_paged_sparse_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, blocks), want)
