"""The paged calls together, as a serving loop runs them: prompts in chunks, decode steps, branches,
dropped sequences, compaction; the contiguous calls over the same records; graphs and streams."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
import synth
from paged_ref import D

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

H, QH = 2, 4


def _ints(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _fitted(seed):
    """Key and value codecs of H heads, fitted on a prefill."""
    w = synth.WORKLOADS["llama_layer_4x"]
    out = []
    for t in (0, 1):
        x = np.stack([synth.numpy_stream(w, seed, 0, h, t, n_tokens=600) for h in range(H)])
        x = torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).cuda().view(torch.bfloat16)
        c = S.Codec(S.Params(ratio=8.0), H)
        S.spectra_fit_basis(c, x)
        out.append((c, x))
    return out


class Server:
    def __init__(self, n_pages=40, rows=8, row_pages=16, page=64, seed=0):
        (self.ck, xk), (self.cv, xv) = _fitted(seed)
        self.map = S.PagedCache(n_pages, page, rows, row_pages)
        self.pools = [self.map.empty_pool(c) for c in (self.ck, self.cv)]
        self.x = [xk.transpose(0, 1).contiguous(), xv.transpose(0, 1).contiguous()]  # [600, H, 128]
        self.q = torch.randn((600, H * QH, D), generator=torch.Generator("cuda").manual_seed(seed), device="cuda").bfloat16()

    def step(self, rows, new, tokens, out=None):
        """new[i] tokens of the prefill, from tokens[i] on, behind row rows[i] -> ends, attention."""
        at = torch.cat([torch.arange(t, t + n) for t, n in zip(tokens, new)]).cuda()
        r = _ints(*rows)
        ends = S.spectra_pages_extend(self.map, r, _ints(*new), self.pools)
        cu = _ints(*np.concatenate([[0], np.cumsum(new)]))
        S.spectra_paged_encode(self.map, self.ck, self.cv, *self.pools, self.x[0][at], self.x[1][at], cu, rows=r, ends=ends)
        q = self.q[at]
        out = S.spectra_paged_attention(self.map, self.ck, self.cv, *self.pools, q, cu, max(new), 600, rows=r, ends=ends,
                                        out=torch.empty(q.shape, device="cuda"))
        return ends.tolist(), out, q

    def contiguous(self, tokens, q):
        """Attention of query rows q [QH * H] over a contiguous cache of the listed tokens."""
        cap = -(-len(tokens) // 64) * 64
        packed = []
        for c, x in zip((self.ck, self.cv), self.x):
            p = c.empty_packed(cap)
            S.spectra_encode(c, x[tokens].transpose(0, 1).contiguous(), 0, p, cap)
            packed.append(p)
        return S.spectra_decode_attention(self.ck, self.cv, *packed, cap, len(tokens), q[None].contiguous(), H)[0]


def _close(a, b):
    # two fp32 paths over the same records: each is good to a few 2^-20 of the values' size
    assert (a - b).abs().max() <= 2.0 ** -16 * b.abs().max()


def test_serving_loop_matches_the_contiguous_calls():
    s = Server()
    held = {r: [] for r in range(8)}  # tokens of each row

    def step(rows, new, tokens):
        ends, out, q = s.step(rows, new, tokens)
        at = 0
        for r, n, t, e in zip(rows, new, tokens, ends):
            if e >= 0:
                before = list(held[r])
                held[r] += list(range(t, t + n))
                assert e == len(held[r])
                for i in (0, n // 2, n - 1):
                    _close(out[at + i], s.contiguous(before + list(range(t, t + i + 1)), q[at + i]))
            else:
                assert (out[at:at + n] == 0).all()
            at += n

    step([0, 1], [100, 37], [0, 200])           # prompts
    step([0, 1], [150, 1], [100, 300])          # a chunk beside a decode step
    for i in range(3):
        step([1, 0], [1, 1], [310 + i, 330 + i])
    ends = S.spectra_pages_fork(s.map, _ints(0, 0, 1), _ints(2, 3, 4))
    assert ends.tolist() == [len(held[0]), len(held[0]), len(held[1])]
    for c, p in ((2, 0), (3, 0), (4, 1)):
        held[c] = list(held[p])
    step([2, 0, 3, 4, 1], [1, 1, 1, 1, 1], [400, 410, 420, 430, 440])  # branches part
    step([2, 3], [30, 70], [450, 500])
    S.spectra_pages_truncate(s.map, _ints(0, 3), _ints(0, 120))
    held[0], held[3] = [], held[3][:120]
    step([3, 4], [5, 1], [580, 590])
    before, refs = [p.clone() for p in s.pools], s.map.refs.clone()
    moved = S.spectra_pages_compact(s.map, s.pools)
    used = int(moved[-1])
    assert used == int((refs > 0).sum()) and (s.map.refs[:used] > 0).all() and (s.map.refs[used:] == 0).all()
    live = (refs > 0).nonzero()[:, 0]
    for p, b in zip(s.pools, before):  # every used page holds in its new place what it held
        assert torch.equal(p[moved[live].long()], b[live])
    step([1, 2, 3, 4], [1, 2, 1, 40], [100, 110, 120, 130])


def test_no_room_leaves_rows_alone():
    s = Server(n_pages=4)
    ends, _, _ = s.step([0, 1], [128, 65], [0, 200])
    assert ends == [128, 65]
    ends, out, _ = s.step([0, 1], [1, 3], [300, 310])   # no page left for row 0
    assert ends == [-1, 68] and (out[0] == 0).all() and not (out[1] == 0).all()
    assert s.map.lens.tolist()[:2] == [128, 68]


def test_a_captured_decode_loop():
    a, b = Server(seed=1), Server(seed=1)
    for s in (a, b):
        s.step([0, 1, 2], [200, 90, 64], [0, 200, 300])
    rows, counts, cu = _ints(0, 1, 2), _ints(1, 1, 1), _ints(0, 1, 2, 3)
    k, v, q = (torch.empty((3, n, D), dtype=torch.bfloat16, device="cuda") for n in (H, H, H * QH))
    ends, out = torch.empty_like(rows), torch.empty_like(q)
    pw = torch.empty(S.spectra_pages_workspace_bytes(a.map), dtype=torch.uint8, device="cuda")
    aw = torch.empty(S.spectra_paged_attention_workspace_bytes(3, 3, H * QH, H, 1, 600), dtype=torch.uint8, device="cuda")

    def work(s, ends, out):
        S.spectra_pages_extend(s.map, rows, counts, s.pools, ends=ends, workspace=pw)
        S.spectra_paged_encode(s.map, s.ck, s.cv, *s.pools, k, v, cu, rows=rows, ends=ends)
        S.spectra_paged_attention(s.map, s.ck, s.cv, *s.pools, q, cu, 1, 600, rows=rows, ends=ends, out=out, workspace=aw)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        work(a, ends, out)
    for i in range(70):  # over a page's end
        at = torch.tensor([i, 100 + i, 400 + i], device="cuda")
        k.copy_(a.x[0][at])
        v.copy_(a.x[1][at])
        q.copy_(a.q[at])
        out.fill_(float("nan"))
        g.replay()
        e2, o2 = torch.empty_like(ends), torch.empty_like(out)
        got = (ends.clone(), out.clone())
        aw.fill_(255)  # the eager call of the other server shares the workspaces, behind the replay
        pw.fill_(255)
        work(b, e2, o2)
        assert torch.equal(got[0], e2) and torch.equal(got[1], o2), i
    torch.cuda.synchronize()
    for x, y in zip((a.map.table, a.map.lens, a.map.refs, *a.pools), (b.map.table, b.map.lens, b.map.refs, *b.pools)):
        assert torch.equal(x, y)


def test_a_captured_chunk_with_parts():
    # a chunk whose slots are split and joined, replayed with garbage in the workspace
    s = Server(n_pages=60, row_pages=60)
    s.step([0], [600], [0])
    for _ in range(4):
        s.step([0], [590], [5])
    assert int(s.map.lens[0]) == 600 + 4 * 590
    q = s.q[:64].contiguous()
    cu = _ints(0, 64)
    args = (s.map, s.ck, s.cv, *s.pools, q, cu, 64, 4096)
    ws = torch.empty(S.spectra_paged_attention_workspace_bytes(1, 64, H * QH, H, 64, 4096), dtype=torch.uint8, device="cuda")
    want = S.spectra_paged_attention(*args)
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.spectra_paged_attention(*args, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_streams_and_their_temporaries():
    a, b = Server(seed=2), Server(seed=3)
    for s in (a, b):
        s.step([0, 1], [300, 70], [0, 300])
    cu, q = _ints(0, 40, 41), [s.q[:41].contiguous() for s in (a, b)]
    want = [S.spectra_paged_attention(s.map, s.ck, s.cv, *s.pools, x, cu, 40, 300) for s, x in zip((a, b), q)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i, (s, x) in enumerate(zip((a, b), q)):
            got[i].append(S.spectra_paged_attention(s.map, s.ck, s.cv, *s.pools, x, cu, 40, 300, stream=streams[i]))
            torch.empty(1 << 22, device="cuda").fill_(float("nan"))  # would land in a workspace freed too early
    torch.cuda.synchronize()
    for i in (0, 1):
        for o in got[i]:
            assert torch.equal(o, want[i])


def test_same_result_twice():
    # no result depends on the order of atomics or workgroups
    s = Server(seed=4)
    s.step([0, 1, 2], [300, 70, 500], [0, 300, 90])
    cu, q = _ints(0, 100, 101, 140), s.q[:140].contiguous()
    outs = [S.spectra_paged_attention(s.map, s.ck, s.cv, *s.pools, q, cu, 100, 512) for _ in range(5)]
    for o in outs[1:]:
        assert torch.equal(o, outs[0])


def test_padded_batch():
    # a call of fixed size whose last sequences are padding: rows of -1, with and without tokens
    a, b = Server(seed=5), Server(seed=5)
    for s in (a, b):
        s.step([0, 1], [130, 70], [0, 200])
    ends, out, _ = a.step([0, 1], [1, 40], [300, 310])
    padded, pout, _ = b.step([0, 1, -1, -1, 8], [1, 40, 0, 2, 30], [300, 310, 0, 5, 7])
    assert padded == ends + [-1, -1, -1]
    # padding of a chunk's rows can change how the slots are split: the order of fp32 sums
    _close(pout[:41], out)
    assert (pout[41:] == 0).all()
    for x, y in zip((a.map.table, a.map.lens, a.map.refs, *a.pools), (b.map.table, b.map.lens, b.map.refs, *b.pools)):
        assert torch.equal(x, y)
    S.spectra_pages_truncate(b.map, _ints(-1, 1, 8, 1), _ints(0, 5, 0, 3))
    assert b.map.lens.tolist() == [131, 3, 0, 0, 0, 0, 0, 0]
    assert S.spectra_pages_fork(b.map, _ints(-1, 0, 8), _ints(2, -1, 3)).tolist() == [-1, -1, -1]
