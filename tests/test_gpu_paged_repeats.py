"""Calls on trees, boxes and lists again and again, whatever their workspaces and outputs held before: every bit alike, and
nothing written behind a workspace of the size asked for. Accepted paths beside pools of no words."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_sparse_ref import cache
from test_gpu_paged_sparse import ints, lists, whole
from test_gpu_paged_tree import Accept, paths

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("lens,new,n_qh,most", [([5000], [1], 4, 60), ([5000] * 20, [1] * 20, 4, 33), ([900, 3000], [40, 300], 4, 12),
                                                ([30000], [2], 16, 400), ([700, 64, 2000], [200, 3, 90], 1, 9), ([4000], [600], 7, 64)])
def test_lists_and_selections_repeat_themselves(lens, new, n_qh, most, f32):
    c = cache(lens, new, n_qh, f32=f32, seed=most)
    n, box, blocks = sum(new), whole(c), ints(lists(c, most, seed=most))
    need = [S.spectra_paged_select_workspace_bytes(n, 2 * n_qh, 2, max(lens)), S.spectra_paged_sparse_attention_workspace_bytes(n, 2 * n_qh, 2, most)]
    room = [torch.empty(b + 65536, dtype=torch.uint8, device="cuda") for b in need]
    got = []
    for fill in (0, 255, 0x7F, 0):
        for r in room:
            r.fill_(fill)
        sel, out = torch.full((n, 2, most), -9, dtype=torch.int32, device="cuda"), torch.full_like(c.q, float("nan"))
        lse = torch.full(c.q.shape[:2], float("nan"), device="cuda")
        S.spectra_paged_select(c.cache, c.ck, box, c.q, c.cu, most, max(lens), out=sel, workspace=room[0][:need[0]])
        S.spectra_paged_sparse_attention(c.cache, c.ck, c.cv, *c.pools, c.q, c.cu, blocks, out=out, lse=lse, workspace=room[1][:need[1]])
        assert all((r[b:] == fill).all() for r, b in zip(room, need))
        again = whole(c)
        assert torch.equal(again, box)
        got.append((sel, out, lse))
    assert torch.isfinite(got[0][1].float()).all() and not (got[0][0] == -9).any()
    for g in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(g, got[0]))


def test_accepted_paths_beside_pools_of_no_words():
    """Several pools of no words have one address, or none; that is no pool listed twice."""
    a = Accept([150, 90, 64, 200], words=(8, 0, 0, 5), seed=6)
    rng = np.random.default_rng(7)
    drafted = [40, 64, 1, 33]
    counts = [11, 64, 0, 5]
    assert min(a.run(np.arange(4), drafted, paths(rng, drafted, counts, 64), counts)) >= 0
