"""Chunks whose slots are split into parts and joined: against attention in 64 bits, by element, in
the mean square, and in the log-sum-exp."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_cases import SPLIT, Built, check_split, records_of
from paged_ref import D, G, default_scale, records

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

B8 = [[5, 1, 0, 0], [4, 2, 0, 0]]
ALL = [[8, 7, 6, 5], [1, 2, 3, 4]]


def _run(c, **kw):
    lse = torch.empty(c.q.shape[:2], device="cuda")
    out = S.spectra_paged_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, max(c.new), max(c.lens), lse=lse, **kw)
    return out, lse


def _random(lens, new, n_qh, bits_k, bits_v, words, seed, **kw):
    rng = np.random.default_rng([seed, 29])
    return Built(lens, new, n_qh, bits_k, bits_v, words, lambda b, h, t, bits, p, n: records(bits, p, n, rng),
                 lambda c: 2.0 * rng.standard_normal((sum(new), c.H * n_qh, D)), seed=seed, **kw)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("name", SPLIT)
def test_split_chunks(name, f32):
    lens, new, n_qh = SPLIT[name]
    c = _random(lens, new, n_qh, B8, B8[::-1], 8, len(name), f32=f32)
    check_split(c, *_run(c))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
def test_split_chunks_of_all_widths(f32):
    for page in (64, 448):
        c = _random([2900, 64], [50, 20], 3, ALL, ALL[::-1], 30, 7, page=page, f32=f32)
        check_split(c, *_run(c))


def _far_below(level, f32):
    """One sequence of 2600 slots whose scores without the key mean's part all lie near `level`
    (log2), those of the first 1500 a little higher, with values of opposite signs."""
    rng = np.random.default_rng(31)
    lens, new, n_qh = [2600], [40], 4

    def coefs(b, h, t, bits, p, n):
        codes = np.stack([rng.integers(0, 2 ** int(w), (n, G)) for w in bits], 1).reshape(n, D)
        early = (np.arange(n) < 1500)[:, None]
        step = np.full((n, len(bits)), 0.5) / np.maximum(1, 2.0 ** np.asarray(bits) - 1)
        z = 0.1 * rng.standard_normal((n, len(bits)))
        z = z + (np.where(early, 5.9, 6.0) if t == 0 else np.where(early, 2.0, -2.0))
        return records_of(codes, z, step, bits, p)

    def query(c):
        q = np.zeros((sum(new), c.H * n_qh, D))
        for h in range(c.H):
            vk = c.state(h)[0]
            live = np.repeat(np.asarray(B8[h]) > 0, G)
            qp = -np.where(live, 1.0 + 0.2 * rng.standard_normal((sum(new), n_qh, D)), 0.0)
            s = qp @ c.coef[0][h][0].mean(0)                             # [n, heads], negative
            qp = qp * (level * np.log(2.0) / s)[..., None]
            q[:, h * n_qh:(h + 1) * n_qh] = qp @ vk.T / default_scale()
        return q
    return Built(lens, new, n_qh, B8, B8[::-1], 8, coefs, query, mean_k=0.0, mean_v=0.1, seed=3, f32=f32)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("level", [-100, -150, -300, 300])
def test_scores_far_from_zero_in_every_part(level, f32):
    c = _far_below(level, f32)
    out, lse = _run(c)
    check_split(c, out, lse)
    # the same rows in a call with too many units to split: no other result than by the order of sums
    n = 130
    cu = torch.arange(n + 1, dtype=torch.int32, device="cuda") * 40
    whole = S.spectra_paged_attention(c.cache, c.ck, c.cv, *c.pools, c.q.repeat(n, 1, 1), cu, 40, 2600,
                                      rows=torch.zeros(n, dtype=torch.int32, device="cuda"))
    check_split(c, whole[:40])
    # The scores are the same numbers. bf16: an output a step apart (2^-7), and weights rounded at another
    # reference (2^-11 on either side); fp32: exponents of up to 2^9 rounded (2^-15, two on either side);
    # of values whose absolute sum is at most 4 times the largest output.
    step = 2.0 ** -11 if f32 else 2.0 ** -6
    assert (whole[:40].float() - out.float()).abs().max() <= step * out.float().abs().max()
