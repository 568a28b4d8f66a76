"""Paged attention over records and codec states at the ends of what they can hold."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_cases import Built, check_split, records_of
from paged_ref import D, G, default_scale, records

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

B8 = [[5, 1, 0, 0], [4, 2, 0, 0]]
FORMS = [([200, 90], [1, 1], 4), ([200, 90], [40, 7], 4)]   # few rows, chunks


def _run(c, bound=None):
    lse = torch.empty(c.q.shape[:2], device="cuda")
    return S.spectra_paged_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, max(c.new), bound or max(c.lens), lse=lse), lse


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new,n_qh", FORMS)
@pytest.mark.parametrize("tensor", [0, 1])
@pytest.mark.parametrize("table", [[8, 8, 8, 8], [9, 0, 0, 0], [255, 1, 1, 1]])
def test_width_tables_that_do_not_fit_keep_nothing(table, tensor, lens, new, n_qh, f32):
    rng = np.random.default_rng([37, tensor])
    c = Built(lens, new, n_qh, B8, B8, 8, lambda b, h, t, bits, p, n: records(bits, p, n, rng),
              lambda c: rng.standard_normal((sum(new), c.H * n_qh, D)), f32=f32)
    (c.ck, c.cv)[tensor].bits[1] = torch.tensor(table, dtype=torch.uint8)
    for b, n in enumerate(lens):  # head 1's coefficients of that tensor are gone
        gone = list(c.coef[b][1])
        gone[tensor] = np.zeros((n, D))
        c.coef[b][1] = tuple(gone)
    check_split(c, *_run(c))


def _large(tensor, lens, new, n_qh, f32):
    """Every third token's groups of one tensor reach past fp16's largest number, by either sign."""
    rng = np.random.default_rng([41, tensor])

    def coefs(b, h, t, bits, p, n):
        if t != tensor:
            return records(bits, p, n, rng)
        codes = np.stack([rng.integers(0, 2 ** int(w), (n, G)) for w in bits], 1)
        top = np.maximum(1, 2.0 ** np.asarray(bits) - 1)
        codes[..., 0], codes[..., 1] = 0, top
        codes = codes.reshape(n, D)
        far = (np.arange(n) % 3 == 0)[:, None]
        sign = rng.choice([-1.0, 1.0], (n, 1))
        z = np.where(far, sign * 3e4, rng.standard_normal((n, len(bits))))
        step = np.where(far, sign * rng.uniform(1e4, 6e4, (n, len(bits))), 1.0) / top
        return records_of(codes, z, step, bits, p)
    return Built(lens, new, n_qh, B8, B8, 8, coefs,
                 lambda c: (2.0 ** -14 if tensor == 0 else 1.0) * rng.standard_normal((sum(new), c.H * n_qh, D)), f32=f32,
                 mean_k=0.0, mean_v=0.0)


def _lowered(c, tensor):
    """The scale of a token's group with a coefficient past 65504 lowered until there is none, to fp16."""
    changed = 0
    for b, per in enumerate(c.coef):
        for h, pair in enumerate(per):
            x = pair[tensor].reshape(-1, D // G, G)
            # every group holds codes 0 (the zero point) and 2^b - 1
            bits = np.asarray(B8[h])
            for g in np.flatnonzero(bits):
                top = 2 ** int(bits[g]) - 1
                z = np.where(x[:, g].mean(1) > 0, x[:, g].min(1), x[:, g].max(1))
                end = np.where(x[:, g].mean(1) > 0, x[:, g].max(1), x[:, g].min(1))
                far = np.abs(end) > 65504
                code = (x[:, g] - z[:, None]) / np.where(end != z, (end - z) / top, 1.0)[:, None]
                step = ((np.sign(end) * 65472 - z) / top).astype(np.float16).astype(np.float64)
                low = z[:, None] + step[:, None] * np.rint(code)
                x[far, g] = low[far]
                changed += int(far.sum())
    return changed


# (keys beside 16-bit outputs would need queries below what fp16 holds in full)
@pytest.mark.parametrize("tensor,f32", [(0, True), (1, True), (1, False)], ids=["keys-f32", "values-f32", "values-bf16"])
@pytest.mark.parametrize("lens,new,n_qh", FORMS)
def test_coefficients_past_the_largest_fp16_number(tensor, lens, new, n_qh, f32):
    c = _large(tensor, lens, new, n_qh, f32)
    out, lse = _run(c)
    few_rows_in_fp32 = f32 and max(new) * n_qh <= 16
    if not few_rows_in_fp32:
        assert _lowered(c, tensor) > 50
    check_split(c, out, lse)


@pytest.mark.parametrize("new,n_qh", [([1, 1, 1], 4), ([4, 1, 2], 1), ([2, 0, 1], 2)])
@pytest.mark.parametrize("bound", [2600, 2 ** 22])
def test_few_rows_by_either_kernel(bound, new, n_qh):
    # records of 8 words and one quad of rows: a call that may hold many long sequences takes the latent scan
    rng = np.random.default_rng(43)
    lens = [2600, 70, 5]
    c = Built(lens, new, n_qh, B8, B8[::-1], 8, lambda b, h, t, bits, p, n: records(bits, p, n, rng),
              lambda c: 2.0 * rng.standard_normal((sum(new), c.H * n_qh, D)))
    check_split(c, *_run(c, bound))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new,n_qh,bound", [([2600, 300], [1, 1], 4, None), ([2600, 300], [1, 1], 4, 2 ** 22),
                                                 ([300, 50], [30, 9], 4, None), ([2600], [40], 4, None)],
                         ids=["few", "scan", "chunk", "parts"])
@pytest.mark.parametrize("spread", [1.0, 10.0, 30.0])
def test_scores_of_a_spread(spread, lens, new, n_qh, bound, f32):
    # the standard deviation of a row's scores over its slots, in nats
    rng = np.random.default_rng(47)

    def query(c):
        q = rng.standard_normal((sum(new), c.H * n_qh, D))
        for h in range(c.H):
            hs = slice(h * n_qh, (h + 1) * n_qh)
            s = default_scale() * (q[:, hs] @ c.state(h)[0]) @ c.coef[0][h][0].T
            q[:, hs] *= (spread / s.std(-1))[..., None]
        return q
    c = Built(lens, new, n_qh, B8, B8[::-1], 8, lambda b, h, t, bits, p, n: records(bits, p, n, rng), query, f32=f32)
    check_split(c, *_run(c, bound))


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new,n_qh", FORMS)
@pytest.mark.parametrize("of_keys,of_values", [(2.0 ** -6, 2.0 ** 8), (2.0 ** 8, 2.0 ** -6)])
def test_magnitudes(of_keys, of_values, lens, new, n_qh, f32):
    # coefficients and q' of both stay where fp16 holds all its bits but for a few
    rng = np.random.default_rng(53)
    c = Built(lens, new, n_qh, B8, B8[::-1], 8, lambda b, h, t, bits, p, n: records(bits, p, n, rng, (of_keys, of_values)[t]),
              lambda c: 2.0 / of_keys * rng.standard_normal((sum(new), c.H * n_qh, D)), mean_k=of_keys, mean_v=of_values, f32=f32)
    check_split(c, *_run(c))
