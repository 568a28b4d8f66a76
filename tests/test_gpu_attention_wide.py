"""Decode-step attention over records of large budgets: what is staged fits the LDS, and the
shapes that do not are refused."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D, allowed, attention64, codec, default_scale, records

torch = pytest.importorskip("torch")


def test_sixteen_heads_beside_the_widest_records_are_refused():
    # on the host, before anything is launched
    ck, cv = codec([[8] * 4], 36, 1, device="cpu")[0], codec([[8] * 4], 36, 2, device="cpu")[0]
    import ctypes
    from paper_2608_07915_amd import _lib
    P = 1 << 20

    def call(heads, a, b):
        for c in (a, b):
            c.struct.basis = c.struct.mean = c.struct.var = c.struct.bits = P
        return _lib.get().spectra_decode_attention(ctypes.byref(a.struct), ctypes.byref(b.struct), P, P, 64, 64, P, 0, 1, heads, 1,
                                                   0.0, P, P, 0, None)
    assert call(13, ck, cv) == call(16, ck, cv) == -2
    assert call(12, ck, cv) == -4          # as far as the (missing) workspace
    small = codec([[8, 8, 8, 0]], 31, 3, device="cpu")[0]
    assert call(16, ck, small) == -4


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")
@pytest.mark.parametrize("words,n_qh", [(64, 5), (64, 12), (36, 12), (40, 1), (33, 16)])
def test_wide_records(words, n_qh):
    rng = np.random.default_rng(words + n_qh)
    bits = [[8, 8, 8, 8]] if words >= 36 else [[8, 8, 8, 5]]
    (ck, pk), (cv, pv) = codec(bits, words, 5), codec(bits, words, 6)
    T, cap = 300, 320
    packed, coef = [], []
    for c, p in ((ck, pk), (cv, pv)):
        rec, co = records(bits[0], p, T, rng)
        full = np.zeros((cap, words), np.uint32)
        full[:T] = rec
        packed.append(torch.from_numpy(full.reshape(cap // 64, 64, words).transpose(0, 2, 1).copy().view(np.int32).reshape(-1)).cuda())
        coef.append(co)
    q = torch.randn((1, n_qh, D), device="cuda")
    out = S.spectra_decode_attention(ck, cv, *packed, cap, T, q, 1)
    st = [t.cpu().numpy().astype(np.float64) for t in (ck.basis[0], ck.mean[0], cv.basis[0], cv.mean[0])]
    want, _, swing, most = attention64(q.cpu().numpy().astype(np.float64), *coef, *st, 1, default_scale())
    # the scan's weights are two bf16 parts (2^-17): more than the pairs of fp16 parts leave
    tol = allowed(want, swing, most, T, False, True) + 2.0 ** -16 * swing
    assert (np.abs(out.cpu().numpy() - want) <= tol).all()
