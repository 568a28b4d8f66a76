"""Selections over more blocks than registers hold, with several KV heads and sequences, on both sides of 1024 tokens times
KV heads; and boxes of more sequences than their starts have room for in LDS."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D, codec
from paged_sparse_ref import B8, cache
from test_gpu_paged_sparse import check_boxes, ints

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


@pytest.mark.parametrize("page", [192, 1024])
@pytest.mark.parametrize("new", [(2, 3), (1, 510), (300, 260), (700, 1)])
@pytest.mark.parametrize("blocks", [(16400, 20001), (16384, 3000), (40, 16385)])
def test_long_selection(blocks, new, page):
    """Against the definition in 64 bits, a sample of the tokens: ascending, the forced blocks among them, and no block left
    out whose value passes a chosen one's by more than the products' errors (2^-20 of sum |q' box|, as in check_selection)."""
    bits, n_qh, most = [[4, 4, 0, 0], [0, 5, 0, 1]], 3, 150
    rng = np.random.default_rng(page + sum(new))
    lens = [64 * n - int(rng.integers(0, 64)) for n in blocks]
    new = [min(n, x) for n, x in zip(new, lens)]
    ck, _ = codec(bits, 10, 1)
    pages = [-(-n // page) for n in lens]
    m = S.PagedCache(sum(pages) + 2, page, 3, max(pages))
    ids = rng.permutation(sum(pages) + 2)
    rows = [2, 0]
    for b, r in enumerate(rows):
        m.table[r, :pages[b]] = ints(ids[sum(pages[:b]):sum(pages[:b + 1])])
        m.lens[r] = lens[b]
    gen = torch.Generator(device="cuda").manual_seed(page + sum(new))
    box = torch.randn((m.n_pages, 2, page // 64, 4, 2, 32), generator=gen, device="cuda").sort(-2).values.half().contiguous()
    n = sum(new)
    q = torch.randn((n, 2 * n_qh, D), generator=gen, device="cuda")
    got = S.spectra_paged_select(m, ck, box.view(torch.int32).view(m.n_pages, -1), q, ints([0, new[0], n]), most, max(lens), first=2,
                                 last=3, rows=ints(rows)).cpu().numpy()
    qp = q.double().view(n, 2, n_qh, D) @ ck.basis.double()
    for b, r in enumerate(rows):
        flat = box[m.table[r, :pages[b]].long()].transpose(1, 2).reshape(-1, 2, 4, 2, 32)[:blocks[b]].double()
        for h in range(2):
            kept = np.flatnonzero(bits[h])
            x = flat[:, h, :2].transpose(1, 2).reshape(blocks[b], 2, 64)
            for i in sorted({0, new[b] // 2, new[b] - 1, int(rng.integers(new[b]))}):
                t = sum(new[:b]) + i
                have = -(-(lens[b] - new[b] + i + 1) // 64)
                mine = got[t, h]
                k = min(have, most)
                assert (mine[k:] == -1).all() and (np.diff(mine[:k]) > 0).all() and mine[0] >= 0 and mine[k - 1] < have, (b, h, i)
                if have <= most:
                    continue
                forced = {0, 1, have - 3, have - 2, have - 1}
                assert forced <= set(mine.tolist())
                y = torch.cat([qp[t, h][:, 32 * g:32 * g + 32] for g in kept], 1)
                s = y.clamp(min=0) @ x[:have, 1].T + y.clamp(max=0) @ x[:have, 0].T
                v = (s - s.amax(1, keepdim=True)).amax(0).cpu().numpy()
                size = float((y.abs() @ x[:have].abs().amax(1).T).max())
                taken = [j for j in mine if j not in forced]
                assert v[taken].min() >= v[np.setdiff1d(np.arange(have), mine)].max() - 4 * 2.0 ** -20 * size, (b, h, i)


@pytest.mark.parametrize("batch", [510, 511, 512, 513, 900])
def test_boxes_of_many_sequences(batch):
    """On both sides of 512 starts; one in six sequences has nothing new, and the last starts lie past n_new."""
    rng = np.random.default_rng(batch)
    lens = rng.integers(1, 200, batch)
    new = np.minimum(rng.integers(1, 140, batch), lens) * (rng.random(batch) > 1 / 6)
    c = cache(lens.tolist(), [0] * (batch - 1) + [1], 1, seed=batch)
    cu = np.concatenate([[0], np.cumsum(new)])
    for n in (int(cu[-1]), int(cu[-1]) - int(new[-5:].sum()) - 1):
        box = c.cache.empty_bounds(c.ck).fill_(-7)
        S.spectra_paged_bounds(c.cache, c.ck, c.pools[0], box, ints(cu), n)
        # a block is made by its first new token below n
        first, ends = [], []
        for b in range(batch):
            live = max(0, min(int(cu[b + 1]), n) - int(cu[b]))
            first.append((int(lens[b]) - live) // 64 if live else 99)
            ends.append(int(lens[b]))
        check_boxes(c, box, B8, 64, first, ends)
