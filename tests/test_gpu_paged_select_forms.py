"""Block selection where its forms meet: one query head to a KV head, and scores that are infinite."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D, codec

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("n_qh", [1, 2])
@pytest.mark.parametrize("tokens", [3, 400, 1023, 1025, 1300])
@pytest.mark.parametrize("n", [100, 5000, 17000])
def test_an_infinite_score_counts_as_no_number(n, tokens, n_qh):
    """A block whose bound is infinite has the value inf - inf, no number, and takes every other block's value to minus
    infinity: all are least, so the lowest indices are chosen. On both sides of 1024 tokens times KV heads."""
    ck, _ = codec([[4, 0, 0, 0]], 10, 1)
    ck.basis[0] = torch.eye(D)
    m = S.PagedCache(n, 64, 1, n)
    m.table[0] = ints(np.arange(n))
    m.lens[0] = n * 64
    box = torch.zeros((n, 1, 1, 4, 2, 32), dtype=torch.float16, device="cuda")
    box[:, 0, 0, 0, 1, 1] = torch.arange(n, device="cuda").remainder(50).half()
    far = n // 2
    box[far, 0, 0, 0, 0, 0] = float("-inf")
    q = torch.zeros((tokens, n_qh, D), device="cuda")
    q[:, :, 0] = -(1 + 2.0 ** -13)  # both fp16 parts negative
    q[:, :, 1] = 1.0
    pool = box.view(torch.int32).view(n, -1)
    got = S.spectra_paged_select(m, ck, pool, q, ints([0, tokens]), 12, n * 64, first=0, last=0)
    assert torch.equal(got.cpu(), torch.arange(12, dtype=torch.int32).expand(tokens, 1, 12))
    # without that block the definition's choice: the largest remainders, lowest indices first
    box[far, 0, 0, 0, 0, 0] = 0.0
    got = S.spectra_paged_select(m, ck, pool, q, ints([0, tokens]), 12, n * 64, first=0, last=0).cpu().numpy()[:, 0]
    for t in (0, tokens - 1):
        have = -(-(n * 64 - tokens + t + 1) // 64)
        assert np.array_equal(got[t], np.sort(np.argsort(-(np.arange(have) % 50), kind="stable")[:12])), t
