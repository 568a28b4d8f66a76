"""Drafted trees over pages: attention against the definition in 64 bits, and the accepted path against a list model."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D, MapModel
from paged_sparse_ref import ALL, B8, NONE, cache, check, tree, tree_sees

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def attend(c, parents, **kw):
    kw.setdefault("max_new", max(c.new + [1]))
    kw.setdefault("max_tokens", max(c.lens + [1]))
    return S.spectra_paged_tree_attention(c.cache, c.ck, c.cv, *c.pools, kw.pop("q", c.q), c.cu, ints(parents), **kw)


LENS = [([1], [1]), ([5], [5]), ([64], [64]), ([64], [1]), ([65], [2]), ([300], [8]), ([130], [64]), ([127], [63]), ([700], [4]),
        ([1000, 1, 63, 64, 65, 700], [3, 1, 20, 64, 2, 33]), ([90, 0, 200], [7, 0, 0]), ([333, 500, 5], [33, 16, 5])]


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new", LENS)
def test_lengths(lens, new, f32):
    c = cache(lens, new, f32=f32, seed=sum(lens) + sum(new))
    lse = torch.empty(c.q.shape[:2], device="cuda")
    for kind in ("random", "star"):
        p = tree(kind, new, seed=sum(new))
        check(c, tree_sees(lens, new, p), attend(c, p, lse=lse), lse)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", ["chain", "star", "pairs", "comb", "random"])
def test_shapes(kind, f32):
    lens, new = [500, 40, 64 * 9 + 20], [40, 40, 64]
    c = cache(lens, new, f32=f32, seed=3)
    p = tree(kind, new)
    check(c, tree_sees(lens, new, p), attend(c, p))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_qh", [1, 2, 3, 5, 7, 8, 12, 16])
def test_heads(n_qh, f32):
    for lens, new in (([200, 77], [1, 1]), ([210, 97], [3, 5]), ([300, 150], [21, 64])):
        c = cache(lens, new, n_qh=n_qh, f32=f32, seed=n_qh)
        p = tree("random", new)
        check(c, tree_sees(lens, new, p), attend(c, p))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("bits_k,bits_v,words", [(ALL, ALL[::-1], 30), (NONE, ALL, 30), (ALL, NONE, 30), (B8, NONE, 8),
                                                 ([[8, 8, 8, 8]], [[8, 8, 8, 8]], 36), ([[1, 0, 0, 0]], [[0, 0, 0, 1]], 5),
                                                 ([[3, 0, 7, 0]], [[0, 6, 0, 0]], 16), ([[0, 0, 0, 0]], [[0, 0, 0, 0]], 5)])
def test_widths(bits_k, bits_v, words, f32):
    for lens, new in (([257, 100], [2, 1]), ([257, 140], [9, 50])):
        c = cache(lens, new, 3, bits_k, bits_v, words, f32=f32, seed=words)
        p = tree("random", new)
        check(c, tree_sees(lens, new, p), attend(c, p))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("page", [128, 192, 1024])
def test_pages(page, f32):
    lens, new = [1200, 100, 191, 193], [10, 64, 30, 40]
    c = cache(lens, new, page=page, f32=f32, seed=page)
    p = tree("random", new)
    check(c, tree_sees(lens, new, p), attend(c, p))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_long_history(f32):
    for new in ([40], [3], [1]):
        lens = [20011]
        c = cache(lens, new, f32=f32, seed=9)
        p = tree("random", new)
        lse = torch.empty(c.q.shape[:2], device="cuda")
        check(c, tree_sees(lens, new, p), attend(c, p, lse=lse), lse)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_parents_that_are_no_earlier_token_count_as_none(f32):
    lens, new = [100, 70, 65], [20, 64, 7]
    c = cache(lens, new, f32=f32, seed=4)
    p = tree("random", new)
    rng = np.random.default_rng(0)
    bad = rng.permutation(len(p))[:40]
    at = np.concatenate([np.arange(n) for n in new])
    p[bad] = np.where(np.arange(40) % 4 == 0, at[bad], np.where(np.arange(40) % 4 == 1, at[bad] + 1, np.where(
        np.arange(40) % 4 == 2, 2 ** 31 - 1, -2 ** 31)))
    check(c, tree_sees(lens, new, p), attend(c, p))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_tokens_that_see_nothing_and_sequences_left_out(f32):
    lens, new = [200, 90, 150, 30], [20, 9, 64, 12]
    c = cache(lens, new, f32=f32, seed=5)
    p = tree("random", new)
    # sequence 0 got no room, 1 has four slots for nine tokens
    ends = [-1, 4, 150, 30]
    lse = torch.empty(c.q.shape[:2], device="cuda")
    out = attend(c, p, ends=ints(ends), lse=lse)
    check(c, tree_sees(ends, new, p), out, lse)
    assert (out[:25] == 0).all() and torch.isneginf(lse[:25]).all()
    # past the call's bounds: rows as they were
    full = attend(c, p)
    for kw, left in ((dict(max_new=20), 2), (dict(max_tokens=199), 0)):
        out, lse = torch.full_like(c.q, 7.0), torch.full(c.q.shape[:2], 7.0, device="cuda")
        attend(c, p, out=out, lse=lse, **kw)
        at = np.concatenate([[0], np.cumsum(new)])
        for b in range(4):
            r = slice(int(at[b]), int(at[b + 1]))
            assert (out[r] == 7).all() == (b == left) and (lse[r] == 7).all() == (b == left)
            if b != left:
                assert (out[r].float() - full[r].float()).abs().max() <= 2.0 ** -6 * full.float().abs().max()
    # rows that no sequence holds
    q = torch.cat([c.q, c.q[:3]])
    out = torch.full_like(q, 7.0)
    more = torch.cat([ints(p), ints([0, 0, 0])])
    S.spectra_paged_tree_attention(c.cache, c.ck, c.cv, *c.pools, q, c.cu, more, 64, 200, out=out)
    assert (out[-3:] == 7).all() and not (out[:-3] == 7).all()


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_chain_is_causal_attention(f32):
    lens, new = [700, 70, 5000], [30, 64, 2]
    c = cache(lens, new, f32=f32, seed=6)
    p = tree("chain", new)
    got = attend(c, p).float()
    want = S.spectra_paged_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, 64, 5000).float()
    check(c, tree_sees(lens, new, p), got.to(c.q.dtype))
    # both within the formats' errors of the definition
    assert (got - want).norm() <= (1e-5 if f32 else 8e-3) * want.norm()


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_strides_rows_scale_types(f32):
    lens, new = [300, 100, 420], [11, 33, 2]
    c = cache(lens, new, f32=f32, seed=7)
    p = tree("random", new)
    n, H = c.q.shape[:2]
    wide = torch.full((H, n + 3, D + 8), float("nan"), dtype=c.q.dtype, device="cuda")
    wide[:, :n, :D] = c.q.transpose(0, 1)
    q = wide.transpose(0, 1)[:n, :, :D]
    a, b = attend(c, p), attend(c, p, q=q)
    assert torch.equal(a, b)
    out = attend(c, p, softmax_scale=0.2)
    check(c, tree_sees(lens, new, p), out, scale=float(np.float32(0.2)))
    # the other output type
    other = torch.empty(c.q.shape, dtype=torch.bfloat16 if f32 else torch.float32, device="cuda")
    check(c, tree_sees(lens, new, p), attend(c, p, out=other))
    # map rows in another order
    perm = [2, 0, 1]
    c2 = cache(lens, new, f32=f32, seed=7)
    table, ln = c2.cache.table.clone(), c2.cache.lens.clone()
    c2.cache.table[perm], c2.cache.lens[perm] = table, ln
    assert torch.equal(a, attend(c2, p, rows=ints(perm)))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_queries_that_are_not_finite_reach_no_other_row(f32):
    lens, new = [300, 100], [11, 33]
    c = cache(lens, new, f32=f32, seed=8)
    p = tree("random", new)
    want = attend(c, p)
    q = c.q.clone()
    q[3, 1, 5], q[20, 7, 0] = float("nan"), float("inf")
    lse = torch.empty(q.shape[:2], device="cuda")
    out = attend(c, p, q=q, lse=lse)
    bad = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    bad[3, 1] = bad[20, 7] = True
    assert torch.equal(out[~bad], want[~bad]) and torch.isnan(out[3, 1]).all() and torch.isnan(lse[3, 1])
    assert torch.isfinite(lse[~bad]).all()


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_qh", [1, 4])
def test_rows_that_see_their_own_slot_alone(n_qh, f32):
    """No history, no parents: a token's weight lies on its own slot, however low its score."""
    lens, new = [64, 40, 33], [64, 40, 33]
    for q_scale in (2.0, 12.0):
        c = cache(lens, new, n_qh=n_qh, f32=f32, seed=14, q_scale=q_scale)
        p = tree("star", new)
        lse = torch.empty(c.q.shape[:2], device="cuda")
        check(c, tree_sees(lens, new, p), attend(c, p, lse=lse), lse)


def test_pages_out_of_range_and_many_sequences():
    lens, new = [300, 64, 130], [20, 8, 64]
    c = cache(lens, new, seed=10)
    p = tree("random", new)
    ok = attend(c, p)
    table = c.cache.table.clone()
    c.cache.table[1, 0] = 2 ** 31 - 1
    out = attend(c, p)
    assert torch.equal(out[:20], ok[:20]) and torch.equal(out[28:], ok[28:]) and torch.isfinite(out.float()).all()
    c.cache.table.copy_(table)
    # more sequences than a workgroup has threads, most with nothing to do
    B = 600
    rows, n = np.arange(B) % 3, np.zeros(B, np.int64)
    n[[0, 301, 599]] = [20, 8, 64]
    rows[[0, 301, 599]] = [0, 1, 2]
    cu = ints(np.concatenate([[0], np.cumsum(n)]))
    out = S.spectra_paged_tree_attention(c.cache, c.ck, c.cv, *c.pools, c.q, cu, ints(p), 64, 300, rows=ints(rows))
    c.cu = cu
    check(c, tree_sees(lens, new, p), out)
    assert (out.float() - ok.float()).norm() <= 8e-3 * ok.float().norm()


def test_starts_that_fall_stay_inside():
    """Lists of sequences that overlap: nothing is touched outside the outputs."""
    lens, new = [300, 64, 130], [20, 8, 64]
    c = cache(lens, new, seed=10)
    p = ints(tree("random", new))
    for cu in ([0, 64, 10, 70], [-5, 90, 2, 200], [80, 3, 2, 1], [0, 60, 0, 64]):
        out = torch.zeros((c.q.shape[0] + 64, *c.q.shape[1:]), dtype=c.q.dtype, device="cuda")
        S.spectra_paged_tree_attention(c.cache, c.ck, c.cv, *c.pools, c.q, ints(cu), p, 64, 300, out=out[32:-32])
        assert (out[:32] == 0).all() and (out[-32:] == 0).all()


def test_captured_calls_and_workspaces():
    lens, new = [900, 64, 130], [20, 8, 64]
    c = cache(lens, new, seed=11)
    p, q2 = ints(tree("random", new)), (c.q.float() * 0.5).bfloat16()
    need = S.spectra_paged_tree_attention_workspace_bytes(3, sum(new), 8, 2, 64, 900)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    call = lambda q, **kw: S.spectra_paged_tree_attention(c.cache, c.ck, c.cv, *c.pools, q, c.cu, p, 64, 900, **kw)  # noqa: E731
    want, want2 = call(c.q, workspace=ws), call(q2)
    q, out, lse = c.q.clone(), torch.empty_like(c.q), torch.empty(c.q.shape[:2], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(q, out=out, lse=lse, workspace=ws)
    torch.cuda.current_stream().wait_stream(s)
    graphs = []
    for _ in range(2):  # two graphs on one workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(q, out=out, lse=lse, workspace=ws)
        graphs.append(g)
    for i in range(6):
        q.copy_(c.q if i % 2 == 0 else q2)
        out.fill_(5.0)
        graphs[i % 2 if i < 4 else 0].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want if i % 2 == 0 else want2)
    # a given stream, while the current one is busy
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(c.q, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


# ---------------------------------------------------------------------------
# The accepted path
# ---------------------------------------------------------------------------
class Accept:
    """Rows with drafted slots, pools of random words, and the rules as a sequential program."""

    def __init__(self, lens, page=64, heads=(3, 2), words=(8, 5), seed=0, shared=()):
        self.rng = np.random.default_rng(seed)
        m = self.model = MapModel(sum(-(-n // page) for n in lens) + 4, page, len(lens) + 1, max(-(-n // page) for n in lens) + 2)
        self.page, self.H = page, 2
        m.extend(np.arange(len(lens)), lens)
        for r in shared:
            m.refs[m.table[r, (lens[r] - 1) // page]] += 1
        self.pools = [torch.randint(-2 ** 31, 2 ** 31 - 1, (m.n_pages, page * self.H * w), dtype=torch.int32, device="cuda") for w in words]
        self.words = words

    def run(self, rows, drafted, path, counts, **kw):
        m, page = self.model, self.page
        c = m.cache()
        pools = [p.clone() for p in self.pools]
        ends = S.spectra_pages_accept(c, ints(rows), ints(drafted), ints(path), ints(counts), pools, self.H, **kw)
        want = [p.cpu().numpy().reshape(m.n_pages, self.H, page // 64, w, 64) for p, w in zip(self.pools, self.words)]
        got_ends, seen, before = [], set(), m.refs.copy()
        for i, r in enumerate(map(int, rows)):
            n, k = int(drafted[i]), int(counts[i])
            ok = 0 <= r < m.rows and r not in seen
            seen.add(r)
            L = int(m.lens[r]) if 0 <= r < m.rows else -1
            ok = ok and 0 <= n <= min(L, 64) and 0 <= k <= min(n, path.shape[1])
            p = [int(x) for x in path[i][:max(k, 0)]]
            ok = ok and all(0 <= x < n for x in p) and all(a < b for a, b in zip(p, p[1:]))
            if ok and n:
                pages = [m.table[r, t // page] for t in range(L - n, L)]
                ok = all(0 <= q < m.n_pages and before[q] == 1 for q in pages)
            if not ok:
                got_ends.append(-1)
                continue
            f = L - n
            at = lambda t: (m.table[r, t // page], slice(None), t % page // 64, slice(None), t % 64)  # noqa: E731
            for w in want:
                kept = [w[at(f + x)].copy() for x in p]
                for j, x in enumerate(kept):
                    w[at(f + j)] = x
            m.truncate([r], [f + k])
            got_ends.append(f + k)
        assert ends.cpu().tolist() == got_ends
        m.check(c)
        t = c.table.cpu().numpy()
        for i, r in enumerate(map(int, rows)):
            if got_ends[i] >= 0:
                assert (t[r, m.pages(m.lens[r]):] == -1).all()
        for p, w in zip(pools, want):
            assert np.array_equal(p.cpu().numpy(), w.reshape(p.shape))
        return got_ends


def paths(rng, drafted, counts, most):
    p = np.full((len(drafted), most), 99)
    for i, (n, k) in enumerate(zip(drafted, counts)):
        p[i, :k] = np.sort(rng.permutation(n)[:k])
    return p


@pytest.mark.parametrize("page", [64, 128, 192])
@pytest.mark.parametrize("seed", range(4))
def test_accept(page, seed):
    rng = np.random.default_rng([page, seed])
    lens = rng.integers(1, 400, 9).tolist()
    lens[:4] = [1, 64, 65, 128]
    a = Accept(lens, page, seed=seed)
    rows = rng.permutation(9)
    drafted = [int(rng.integers(0, min(64, lens[r]) + 1)) for r in rows]
    drafted[0] = min(64, lens[rows[0]])
    counts = [int(rng.integers(0, n + 1)) for n in drafted]
    counts[1] = drafted[1]
    ends = a.run(rows, drafted, paths(rng, drafted, counts, 64), counts)
    assert min(ends) >= 0


def test_accept_refusals():
    lens = [100, 200, 70, 130, 64, 90]
    a = Accept(lens, seed=1, shared=[3])
    good = np.tile(np.arange(8), (1, 1))
    for rows, drafted, path, counts in (
            ([7], [3], good, [1]), ([-1], [3], good, [1]), ([0], [101], good, [1]), ([0], [65], good, [1]), ([0], [-1], good, [0]),
            ([0], [5], good, [6]), ([0], [5], good, [-1]), ([0], [20], good, [9]), ([0], [5], np.array([[0, 0]]), [2]),
            ([0], [5], np.array([[2, 1]]), [2]), ([0], [5], np.array([[0, 5]]), [2]), ([0], [5], np.array([[-1, 5]]), [1]),
            ([3], [5], good, [2]), ([6], [1], good, [0]), ([6], [1], good, [1])):
        assert a.run(rows, drafted, path, counts) == [-1], (rows, drafted, counts)
    # a row listed again is refused the second time; others of the list are served; an empty row may keep none of none
    got = a.run([0, 1, 0, 2, 6, 1], [10, 64, 5, 1, 0, 2], np.tile(np.arange(8), (6, 1)), [3, 8, 2, 1, 0, 1])
    assert got == [93, 144, -1, 70, 0, -1]
    a.model.table[4, 0] = -1
    assert a.run([4], [3], good, [1]) == [-1]
    # no path at all
    assert a.run([5], [90 - 30], np.zeros((1, 0), np.int64), [0]) == [30]


def test_accept_of_many_pools_and_captured():
    lens = [150] * 40
    a = Accept(lens, words=(8,) * 70, seed=2)
    rng = np.random.default_rng(3)
    drafted = rng.integers(1, 65, 40)
    counts = [int(rng.integers(0, n + 1)) for n in drafted]
    path = paths(rng, drafted, counts, 64)
    a.run(np.arange(40), drafted, path, counts)
    a = Accept(lens[:5], seed=4)
    c, pools = a.model.cache(), [p.clone() for p in a.pools]
    before = [c.table.clone(), c.lens.clone(), c.refs.clone()]
    rows, d, pth, cnt = ints(np.arange(5)), ints(drafted[:5]), ints(path[:5]), ints(counts[:5])
    ends = torch.empty(5, dtype=torch.int32, device="cuda")
    call = lambda: S.spectra_pages_accept(c, rows, d, pth, cnt, pools, 2, ends=ends)  # noqa: E731
    call()
    want, maps = [p.clone() for p in pools], [c.table.clone(), c.lens.clone(), c.refs.clone()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(3):
        for p, o in zip(pools, a.pools):
            p.copy_(o)
        for t, b in zip((c.table, c.lens, c.refs), before):
            t.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(pools, want))
        assert all(torch.equal(x, y) for x, y in zip((c.table, c.lens, c.refs), maps))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [4, 8, 20, 40])
def test_metadata_that_is_not_finite(new, f32):
    """It counts as 0 and reaches no other slot; a scale too large for fp16 is lowered."""
    c = cache([150], [new], f32=f32, seed=16)
    page = int(c.cache.table[0, 0])
    k, v = (c.pools[i][page].view(2, 8, 64) for i in (0, 1))
    k[0, 0, 5] = 0x7C00           # an infinite scale
    k[1, 1, 9] = 0x7E00 << 16     # NaN as zero point
    v[0, 1, 7] = 0xFC00           # minus infinity
    v[0, 0, 11] = 0x7BFF          # 65504 as scale: codes 1, lowered to 65472 / 15
    v[0, 2:6, 11] = 0x11111111
    c.coef[0][0][0][5, :32] = c.coef[0][1][0][9, 32:64] = c.coef[0][0][1][7, 32:64] = 0.0
    c.coef[0][0][1][11, :32] = float(np.float16(65472.0 / 15))
    p = tree("random", [new])
    lse = torch.empty(c.q.shape[:2], device="cuda")
    check(c, tree_sees([150], [new], p), attend(c, p, lse=lse), lse)


def test_few_and_many_rows_together_captured():
    """Sequences on both sides of 128 rows a KV head in one call, in graphs replayed between eager calls."""
    lens, new = [5000, 300, 700, 90, 2000], [64, 20, 40, 1, 33]
    c = cache(lens, new, seed=17)
    p = tree("random", new)
    lse, out = torch.empty(c.q.shape[:2], device="cuda"), torch.empty_like(c.q)
    want = attend(c, p, lse=lse)
    check(c, tree_sees(lens, new, p), want, lse)
    first, up = lse.clone(), ints(p)
    ws = torch.empty(S.spectra_paged_tree_attention_workspace_bytes(5, sum(new), 8, 2, 64, 5000) + 4096, dtype=torch.uint8, device="cuda")
    call = lambda: S.spectra_paged_tree_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, up, 64, 5000, out=out, lse=lse, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(4):
        out.fill_(3.0)
        lse.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, first)
        assert torch.equal(attend(c, p), want)
