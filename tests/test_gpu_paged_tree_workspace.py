"""Attention of drafted trees in a workspace of exactly the size asked for: nothing is written behind it, and what it held
before reaches no result."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_sparse_ref import cache, check, tree, tree_sees

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new,n_qh", [([3000], [1], 1), ([3000], [16], 1), ([3000, 200], [4, 4], 4), ([3000, 70], [5, 3], 4), ([900], [33], 1),
                                           ([900, 5000, 64], [17, 64, 1], 2), ([900, 5000, 64, 30], [8, 9, 8, 2], 16),
                                           ([20000], [64], 7), ([700] * 40, [3, 1] * 20, 3), ([80] * 300, [2] * 300, 8)])
def test_workspace_of_the_size_asked_for(lens, new, n_qh, f32):
    c = cache(lens, new, n_qh, f32=f32, seed=n_qh)
    p = tree("random", new)
    need = S.spectra_paged_tree_attention_workspace_bytes(len(new), sum(new), 2 * n_qh, 2, max(new), max(lens))
    room = torch.empty(need + 65536, dtype=torch.uint8, device="cuda")
    up, got = torch.tensor(p, dtype=torch.int32, device="cuda"), []
    for fill in (0, 255, 0x7F):
        room.fill_(fill)
        out, lse = torch.full_like(c.q, float("nan")), torch.full(c.q.shape[:2], float("nan"), device="cuda")
        S.spectra_paged_tree_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, up, max(new), max(lens), out=out, lse=lse,
                                       workspace=room[:need])
        assert (room[need:] == fill).all()
        got.append((out, lse))
    if len(new) < 100:
        check(c, tree_sees(lens, new, p), *got[0])
    assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))
    assert np.isfinite(got[0][1].cpu().numpy()).all()
