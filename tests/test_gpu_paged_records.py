"""Paged attention over records and codec states at the ends of what they can hold."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_cases import Built, check_split, records_of
from paged_ref import D, G, codec, records

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

B8 = [[5, 1, 0, 0], [4, 2, 0, 0]]
FORMS = [([200, 90], [1, 1], 4), ([200, 90], [40, 7], 4)]   # few rows, chunks


def _run(c):
    lse = torch.empty(c.q.shape[:2], device="cuda")
    return S.spectra_paged_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, max(c.new), max(c.lens), lse=lse), lse


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
