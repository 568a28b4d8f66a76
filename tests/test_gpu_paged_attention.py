"""Attention of new tokens over pages against the definition in 64 bits: single tokens and chunks,
ragged batches, every width, head counts, page sizes, tokens that see nothing, garbage behind a
sequence's end, strides, and the log-sum-exp."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D, MapModel, allowed, attention64, codec, default_scale, from_pool, records, to_pool

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

B8 = [[5, 1, 0, 0], [4, 2, 0, 0]]           # 8-word records
ALL = [[8, 7, 6, 5], [1, 2, 3, 4]]          # every width
NONE = [[0, 0, 0, 0], [0, 3, 0, 2]]         # nothing kept; a dropped first group


class Case:
    """A paged cache of sequences of the given lengths, new tokens included, with its inputs."""

    def __init__(self, lens, new, n_qh, bits_k, bits_v, words, page=64, f32=False, seed=0, scale=1.0, q_scale=2.0,
                 junk=True):
        rng = np.random.default_rng([seed, 17])
        self.lens, self.new, self.n_qh, self.page, self.f32 = lens, new, n_qh, page, f32
        self.H = H = len(bits_k)
        (self.ck, pk), (self.cv, pv) = codec(bits_k, words, seed + 1), codec(bits_v, words, seed + 2)
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + 5
        ids = rng.permutation(n_pages)
        self.model = m = MapModel(n_pages, page, len(lens), max(need + [1]) + 2)
        pools = [np.full((n_pages, page * H * words), -1 if junk else 0, np.int32) for _ in range(2)]  # NaN metadata
        self.coef = []
        for b, n in enumerate(lens):
            m.table[b, :need[b]] = ids[sum(need[:b]):sum(need[:b + 1])]
            m.refs[m.table[b, :need[b]]] = 1
            m.lens[b] = n
            per = []
            for h in range(H):
                rk, ck = records(bits_k[h], pk, n, rng, scale)
                rv, cv = records(bits_v[h], pv, n, rng, scale)
                to_pool(pools[0], rk, m.table[b], page, h, H)
                to_pool(pools[1], rv, m.table[b], page, h, H)
                per.append((ck, cv))
            self.coef.append(per)
        self.pools = [torch.from_numpy(p).cuda() for p in pools]
        N = sum(new)
        q = (q_scale * rng.standard_normal((N, H * n_qh, D))).astype(np.float32)
        self.q = torch.from_numpy(q).cuda() if f32 else torch.from_numpy(q).cuda().bfloat16()
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        self.cache = m.cache()

    def run(self, **kw):
        kw.setdefault("max_new", max(self.new + [1]))
        kw.setdefault("max_tokens", max(self.lens + [1]))
        return S.spectra_paged_attention(self.cache, self.ck, self.cv, *self.pools, kw.pop("q", self.q), self.cu, **kw)

    def check(self, out, lse=None, softmax_scale=None, ends=None):
        """Every row within the bound of the formats."""
        assert torch.isfinite(out.float()).all()
        got, q = out.float().cpu().numpy().astype(np.float64), self.q.float().cpu().numpy().astype(np.float64)
        at = 0
        worst = 0.0
        for b, (L, n) in enumerate(zip(self.lens, self.new)):
            if ends is not None:
                L = ends[b]
            for h in range(self.H):
                hs = slice(h * self.n_qh, (h + 1) * self.n_qh)
                st = [t.cpu().numpy().astype(np.float64) for t in (self.ck.basis[h], self.ck.mean[h], self.cv.basis[h],
                                                                   self.cv.mean[h])]
                ck, cv = self.coef[b][h]
                want, wlse, swing, most = attention64(q[at:at + n, hs], ck[:max(L, 0)], cv[:max(L, 0)], *st, n,
                                                      softmax_scale or default_scale())
                bf16 = out.dtype == torch.bfloat16
                tol = allowed(want, swing, most, max(L, 1), bf16, not bf16)
                if n * self.n_qh <= 16:
                    tol = tol + 2.0 ** -16 * swing  # few rows: softmax weights are two bf16 parts (2^-17)
                off = np.abs(got[at:at + n, hs] - want)
                assert (off <= tol).all(), (b, h, float((off / np.maximum(tol, 1e-300)).max()))
                worst = max(worst, float((off / np.maximum(tol, 1e-300)).max(initial=0.0)))
                if lse is not None:
                    g = lse[at:at + n, hs].cpu().numpy().astype(np.float64)
                    assert np.array_equal(np.isinf(g), np.isinf(wlse)) and (g[np.isinf(g)] < 0).all()
                    ok = np.isfinite(wlse)
                    f = 40 * 2.0 ** -24 + (2 * 2.0 ** -11 if bf16 else 3 * 2.0 ** -22)
                    lim = f * most + 2.0 ** -18 + (L / 16 + 200) * 2.0 ** -24 + 2.0 ** -21 * np.abs(np.where(ok, wlse, 0.0))
                    assert (np.abs(g[ok] - wlse[ok]) <= lim[ok]).all()
            at += n
        return worst


LENS = [([1], [1]), ([64], [1]), ([65], [1]), ([2], [2]), ([300], [1]), ([1000, 1, 63, 64, 65, 700], [1] * 6),
        ([130], [130]), ([333, 500, 5], [33, 70, 5]), ([700], [5]), ([90, 0, 200], [7, 0, 0]), ([1300], [700])]


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new", LENS)
def test_lengths(lens, new, f32):
    c = Case(lens, new, 4, B8, B8[::-1], 8, f32=f32, seed=len(lens) + sum(new))
    lse = torch.empty(c.q.shape[:2], device="cuda")
    c.check(c.run(lse=lse), lse)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_qh", [1, 2, 5, 7, 8, 12, 16])
def test_heads(n_qh, f32):
    for lens, new in (([200, 77], [1, 1]), ([210, 97], [40, 3])):
        c = Case(lens, new, n_qh, B8, B8, 8, f32=f32, seed=n_qh)
        c.check(c.run())


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("bits_k,bits_v,words", [(ALL, ALL[::-1], 30), (NONE, ALL, 30), (ALL, NONE, 30), (B8, NONE, 8),
                                                 ([[8, 8, 8, 8]], [[8, 8, 8, 8]], 36), ([[1, 0, 0, 0]], [[0, 0, 0, 1]], 5),
                                                 ([[3, 0, 7, 0]], [[0, 6, 0, 0]], 16)])
def test_widths(bits_k, bits_v, words, f32):
    for lens, new in (([257, 100], [1, 1]), ([257, 140], [50, 30])):
        c = Case(lens, new, 3, bits_k, bits_v, words, f32=f32, seed=words)
        c.check(c.run())


def test_no_records_at_all():
    # records of no words: every token's weight is alike and the output the rotated mean
    ck, _ = codec([[0] * 4], 1, 3)
    cv, _ = codec([[0] * 4], 1, 4)
    cache = S.PagedCache(4, 64, 1, 4)
    cache.table[0, :2] = torch.tensor([2, 0], dtype=torch.int32)
    cache.lens[0] = 100
    pools = [cache.empty_pool(c) for c in (ck, cv)]
    q = torch.randn((1, 4, D), device="cuda")
    lse = torch.empty((1, 4), device="cuda")
    out = S.spectra_paged_attention(cache, ck, cv, *pools, q, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), 1,
                                    100, lse=lse)
    want = (cv.mean[0].double() @ cv.basis[0].double().T).expand(4, D)
    assert ((out[0].double() - want).abs() <= 2.0 ** -20 * (cv.mean[0].double().abs() @ cv.basis[0].double().abs().T)).all()
    k = ck.basis[0].double() @ ck.mean[0].double() / np.sqrt(D)
    assert (lse[0].double() - np.log(100) - q[0].double() @ k).abs().max() < 1e-4


@pytest.mark.parametrize("page", [64, 128, 448])
def test_pages(page):
    for lens, new in (([900, 449], [1, 1]), ([900, 448], [200, 448])):
        c = Case(lens, new, 4, B8, B8, 8, page=page, seed=page)
        c.check(c.run())


def test_rows_that_see_nothing():
    # more new tokens than slots: the first see none; a sequence that got no room; one of no slots
    c = Case([40, 300, 100, 1], [100, 20, 1, 3], 4, B8, B8, 8, f32=True, seed=5)
    ends = [40, -1, 0, 1]
    lse = torch.empty(c.q.shape[:2], device="cuda")
    out = c.run(ends=torch.tensor(ends, dtype=torch.int32, device="cuda"), lse=lse)
    c.check(out, lse, ends=ends)
    assert (out[:60] == 0).all() and (out[100:121] == 0).all()


def test_rows_behind_and_bounds_are_left_alone():
    c = Case([200, 300, 90], [10, 60, 10], 4, B8, B8, 8, seed=6)
    c.cu = torch.tensor([0, 10, 70, 75], dtype=torch.int32, device="cuda")  # five rows behind the last sequence
    out = torch.full_like(c.q, 7.0)
    lse = torch.full(c.q.shape[:2], 7.0, device="cuda")
    c.run(out=out, lse=lse, max_new=20, max_tokens=250)                       # the second has more than the bounds
    assert (out[10:70] == 7).all() and (out[75:] == 7).all() and (lse[10:70] == 7).all() and (lse[75:] == 7).all()
    assert not (out[:10] == 7).all(-1).any() and not (out[70:75] == 7).all(-1).any()
    full = c.run(max_new=60, max_tokens=300)
    assert torch.equal(full[:10], out[:10]) or (full[:10].float() - out[:10].float()).abs().max() < 0.05


def test_strides_rows_and_scale():
    # query rows inside a wider projection, map rows in another order, lens from the map
    c = Case([200, 130, 77], [9, 1, 77], 4, B8, B8, 8, seed=8)
    H = c.H * 4
    wide = torch.zeros((c.q.shape[0], 3 * H, D), dtype=c.q.dtype, device="cuda")
    wide[:, H:2 * H] = c.q
    out = c.run(q=wide[:, H:2 * H], softmax_scale=0.3)
    c.check(out, softmax_scale=np.float32(0.3).astype(np.float64))
    heads_first = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(c.run(q=heads_first, softmax_scale=0.3), out)
    rows = torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda")
    order = [1, 2, 0]  # sequence of each map row
    back = S.PagedCache(c.cache.n_pages, c.page, 3, c.cache.row_pages)
    for r, b in enumerate(order):
        back.table[r], back.lens[r] = c.cache.table[b], c.cache.lens[b]
    c.cache = back
    assert torch.equal(c.run(q=heads_first, softmax_scale=0.3, rows=rows), out)


def test_mixed_output_types():
    c = Case([300], [40], 4, B8, B8, 8, seed=9)
    out = torch.empty(c.q.shape, dtype=torch.float32, device="cuda")
    c.check(c.run(out=out))
    c = Case([300], [40], 4, B8, B8, 8, seed=9, f32=True)
    out = torch.empty(c.q.shape, dtype=torch.bfloat16, device="cuda")
    c.check(c.run(out=out))


@pytest.mark.parametrize("new", [[1, 1], [50, 30]])
def test_page_out_of_range_is_a_page_of_zeros(new):
    c = Case([200, 150], new, 4, B8, B8, 8, f32=True, seed=10)
    for b, i, bad in ((0, 1, -5), (1, 0, c.cache.n_pages), (1, 2, 2 ** 31 - 1)):
        c.cache.table[b, i] = bad
        for ck, cv in c.coef[b]:
            ck[64 * i:64 * i + 64] = 0.0
            cv[64 * i:64 * i + 64] = 0.0
    c.check(c.run())


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_later_tokens_with_infinite_metadata_do_not_reach_earlier_ones(f32):
    c = Case([100], [40], 4, B8, B8, 8, f32=f32, seed=11)
    want = c.run()
    page = int(c.model.table[0, 1])
    for p in c.pools:  # token 99's metadata: infinite scales, NaN zero points
        t = p.view(c.cache.n_pages, c.H, 1, 8, 64)
        t[page, :, 0, :2, 99 - 64] = 0x7E007C00
    out = c.run()
    assert torch.isfinite(out.float()).all()
    assert torch.equal(out[:39], want[:39])


@pytest.mark.parametrize("new", [1, 60])
def test_large_and_small_magnitudes(new):
    # coefficients of 2^-8 and of 2^12 of the usual size
    for scale in (2.0 ** -8, 2.0 ** 12):
        c = Case([300], [new], 4, B8, B8, 8, f32=True, seed=12, scale=scale, q_scale=2.0 / max(scale, 1.0))
        c.ck.mean.zero_()
        c.cv.mean.zero_()
        c.check(c.run())


def test_empty_calls():
    c = Case([100], [1], 4, B8, B8, 8, seed=13)
    none = torch.empty((0, 8, D), dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert S.spectra_paged_attention(c.cache, c.ck, c.cv, *c.pools, none, zero, 1, 100).shape == (0, 8, D)
    S.spectra_paged_encode(c.cache, c.ck, c.cv, *c.pools, none[:, :2], none[:, :2], zero)


def test_reading_back_what_encode_wrote():
    # the tests' own page layout is the library's: records through spectra_paged_encode
    c = Case([100], [100], 4, B8, B8, 8, seed=14, junk=False)
    x = torch.randn((100, 2, D), device="cuda").bfloat16()
    S.spectra_paged_encode(c.cache, c.ck, c.cv, *c.pools, x, x, c.cu)
    flat = c.ck.empty_packed(128)
    S.spectra_encode(c.ck, x.transpose(0, 1), 0, flat, 128)
    got = from_pool(c.pools[0].cpu().numpy(), c.model.table[0], 100, 64, 1, 2, 8)
    want = flat.cpu().numpy().view(np.uint32).reshape(2, 2, 8, 64)[1].transpose(0, 2, 1).reshape(128, 8)[:100]
    assert np.array_equal(got, want)
