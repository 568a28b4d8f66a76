"""Block selection where its forms meet: one query head to a KV head, and scores that are infinite."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D, codec
from paged_sparse_ref import B8, block_values, box_of, cache
from test_gpu_paged_sparse import select, whole

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


def equal_values(n, seed=0):
    """A map of one sequence of n blocks in a shuffled order, boxes whose bounds are small whole numbers."""
    ck, _ = codec([[4, 0, 0, 0]], 10, 1)
    ck.basis[0] = torch.eye(D)
    m = S.PagedCache(n, 64, 2, n)
    rng = np.random.default_rng(seed)
    order = rng.permutation(n)
    m.table[0] = ints(order)
    m.table[1] = ints(order[::-1].copy())
    vals = rng.integers(0, 9, n)
    box = torch.zeros((n, 1, 1, 4, 2, 32), dtype=torch.float16, device="cuda")
    box[ints(order).long(), 0, 0, 0, 1, 0] = torch.tensor(vals, dtype=torch.float16, device="cuda")
    return ck, m, box.view(torch.int32).view(n, -1), vals


@pytest.mark.parametrize("n,tokens,n_qh", [(17000, 1020, 16), (17000, 17000, 1), (20000, 14000, 3), (4000, 70000, 2), (40000, 7000, 1),
                                          (2000, 140000, 1), (10000, 30000, 1)])
def test_selections_whose_scores_do_not_fit_at_once(n, tokens, n_qh):
    """Calls that keep the scores of some of their tokens at a time: two sequences, whose new tokens meet inside one of
    those parts, the second with a length of its own; exact values. And the workspace of exactly the size asked for."""
    ck, m, pool, vals = equal_values(n, tokens)
    cut = tokens // 3
    ends = [n * 64, max(n * 32 + 17, tokens - cut + 1000)]
    q = torch.zeros((tokens + 3, n_qh, D), device="cuda")
    q[:, :, 0] = 1.0 + torch.arange(tokens + 3, device="cuda")[:, None] % 3
    need = S.spectra_paged_select_workspace_bytes(tokens + 3, n_qh, 1, n * 64)
    row = -(-n // 32) * 32
    assert 4 * tokens * row * (n_qh if tokens <= 1024 else 1) > need  # otherwise nothing is split
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((tokens + 3, 1, 9), 77, dtype=torch.int32, device="cuda")
    S.spectra_paged_select(m, ck, pool, q, ints([0, cut, tokens]), 9, n * 64, first=1, last=2, ends=ints(ends), out=out, workspace=ws[:need])
    assert (ws[need:] == 255).all() and (out[tokens:] == 77).all()
    got = out.cpu().numpy()[:, 0]
    for b, (lo, hi) in enumerate(((0, cut), (cut, tokens))):
        seq = vals if b == 0 else vals[::-1]
        for t in np.unique(np.concatenate([np.linspace(lo, hi - 1, 150).astype(int), np.arange(lo, min(hi, lo + 70)), np.arange(max(lo, hi - 70), hi)])):
            have = -(-(ends[b] - (hi - lo) + (t - lo) + 1) // 64)
            rest = 1 + np.argsort(-seq[1:have - 2], kind="stable")[:6]
            assert got[t].tolist() == sorted([0, have - 2, have - 1, *rest.tolist()]), (b, t)
    # a sequence past the call's bound is left as it was, whatever part its tokens fall into
    out.fill_(77)
    S.spectra_paged_select(m, ck, pool, q, ints([0, cut, tokens]), 9, n * 64 - 1, first=1, last=2, ends=ints(ends), out=out)
    assert (out[:cut] == 77).all() and np.array_equal(out.cpu().numpy()[cut:tokens, 0], got[cut:tokens])


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [5, 600])
def test_queries_that_mostly_lie_in_dropped_directions(tokens, f32):
    """q' of the kept directions is then a small difference of large terms and off by its rotation: three parts of 8 bits and
    at most 24 products of 32 terms, one after the other, summed to 2^-23 each, so 2^-18 of sum_i |q_i V_ij|. No block
    is left out whose value passes a chosen one's by more than what that and the products (2^-20 of sum |q' box|) leave of
    two values and the bests they count from."""
    c = cache([5000], [tokens], 4, f32=f32, seed=21)
    box = whole(c)
    raw, table = box.cpu().numpy(), c.cache.table.cpu().numpy()
    rng = np.random.default_rng(tokens)
    q = np.zeros((tokens, 8, D))
    for h in range(2):
        v = c.state(h)[0]
        amount = np.where(np.arange(D) < 64, rng.standard_normal((tokens, 4, D)), 3e6 * rng.standard_normal((tokens, 4, D)))
        q[:, 4 * h:4 * h + 4] = amount @ v.T
    c.q = torch.from_numpy(q.astype(np.float32)).cuda()
    c.q = c.q if f32 else c.q.bfloat16()
    q = c.q.float().cpu().numpy().astype(np.float64)
    got = select(c, box, 9).cpu().numpy()
    for h in range(2):
        v = c.state(h)[0]
        boxed = np.stack([box_of(raw, table[0], i, 64, h, 2, B8[h])[0] for i in range(79)]) * np.repeat(np.asarray(B8[h]) > 0, 32)
        for i in range(0, tokens, 1 + tokens // 20):
            have = -(-(5000 - tokens + i + 1) // 64)
            rows, mine = q[i, 4 * h:4 * h + 4], got[i, h]
            vals, size = block_values(rows, boxed, v, np.arange(79) < have)
            turn = (np.abs(rows) @ np.abs(v) @ np.abs(boxed[:have]).max(1).T).max()
            taken, left = mine[1:-1], np.setdiff1d(np.arange(have), mine)
            assert (np.diff(mine) > 0).all() and mine[0] == 0 and mine[-1] == have - 1
            assert vals[taken].min() >= vals[left].max() - 4 * (2.0 ** -20 * size + 2.0 ** -18 * turn), (h, i)
