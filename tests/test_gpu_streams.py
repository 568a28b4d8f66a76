"""Calls on a given stream while the current one has work pending on memory that it has freed: what is
made for a call is not that memory, and is not taken by later work before the call has passed."""
import numpy as np
import pytest

import paper_2608_07915_amd as S
from paged_ref import D, MapModel, codec

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

H, QH = 2, 4
BITS = [[5, 1, 0, 0], [4, 2, 0, 0]]


def _under_pending_work(call, sizes):
    """call(stream) while the current stream is still to fill freed blocks of the given bytes."""
    want = call(None)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for _ in range(3):
        blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
        torch.cuda._sleep(20_000_000)  # some milliseconds
        for b in blocks:
            b.fill_(255)
        del blocks, b
        got = call(stream)
        after = [torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255) for n in sizes]  # would take a freed workspace
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del got, after


def _cache(lens):
    (ck, _), (cv, _) = codec(BITS, 8, 1), codec(BITS, 8, 2)
    m = MapModel(40, 64, 4, 10)
    at = 0
    for b, n in enumerate(lens):
        k = -(-n // 64)
        m.table[b, :k] = range(at, at + k)
        m.refs[at:at + k] = 1
        m.lens[b] = n
        at += k
    cache = m.cache()
    pools = [cache.empty_pool(c) for c in (ck, cv)]
    x = torch.randn((sum(lens), H, D), device="cuda")
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    S.spectra_paged_encode(cache, ck, cv, *pools, x, x, cu)
    return cache, ck, cv, pools


@pytest.mark.parametrize("new", [1, 60])
def test_paged_attention(new):
    cache, ck, cv, pools = _cache([300, 200, 100])
    q = torch.randn((3 * new, H * QH, D), device="cuda")
    cu = torch.arange(4, dtype=torch.int32, device="cuda") * new
    need = S.spectra_paged_attention_workspace_bytes(3, 3 * new, H * QH, H, new, 300)
    _under_pending_work(lambda s: S.spectra_paged_attention(cache, ck, cv, *pools, q, cu, new, 300, stream=s),
                        [q.numel() * 4, need])


def test_map_calls():
    cache, ck, cv, pools = _cache([300, 200, 100])
    state = [t.clone() for t in (cache.table, cache.lens, cache.refs)]
    torch.cuda.synchronize()
    rows = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    children = torch.tensor([3], dtype=torch.int32, device="cuda")

    def again(stream):  # the map as it was, in the call's order
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            for t, old in zip((cache.table, cache.lens, cache.refs), state):
                t.copy_(old)

    def extend(s):
        again(s)
        return S.spectra_pages_extend(cache, rows, rows, pools, stream=s)

    def fork(s):
        again(s)
        return S.spectra_pages_fork(cache, rows[:1], children, stream=s)

    def compact(s):
        again(s)
        return S.spectra_pages_compact(cache, pools, stream=s)
    need = S.spectra_pages_workspace_bytes(cache)
    for call in (extend, fork, compact):
        _under_pending_work(call, [512, need])


def test_contiguous_calls():
    (ck, _), (cv, _) = codec(BITS, 8, 3), codec(BITS, 8, 4)
    cap, T = 320, 300
    x = torch.randn((H, T, D), device="cuda")
    packed = [c.empty_packed(cap) for c in (ck, cv)]
    for c, p in zip((ck, cv), packed):
        S.spectra_encode(c, x, 0, p, cap)
    q = torch.randn((1, H * QH, D), device="cuda")
    need = S.spectra_attention_workspace_bytes(1, H * QH, H, T)
    freq = torch.rand(D // 2, device="cuda")
    new = [x[:, i][None].contiguous() for i in (0, 1)]
    _under_pending_work(lambda s: S.spectra_decode_attention(ck, cv, *packed, cap, T, q, H, stream=s), [q.numel() * 4, need])
    _under_pending_work(lambda s: S.spectra_decode_attention_rope(ck, cv, *packed, cap, T, q, H, freq, stream=s),
                        [q.numel() * 4, need])
    _under_pending_work(lambda s: S.spectra_decode_step(ck, cv, *packed, cap, T, *new, q, H, stream=s),
                        [q.numel() * 4, need])
    _under_pending_work(lambda s: S.spectra_decode(cv, packed[1], cap, 0, T, stream=s), [H * T * D * 4])
    _under_pending_work(lambda s: S.spectra_unpack_codes(cv, packed[1], cap, T, stream=s)[1], [H * T * D, H * T * 4 * 4])


def test_captured_with_the_stream_given():
    # outputs and workspaces made during the capture, two graphs replayed in turn
    cache, ck, cv, pools = _cache([300, 200, 100])
    graphs = []
    for new in (1, 60):
        q = torch.randn((3 * new, H * QH, D), device="cuda")
        cu = torch.arange(4, dtype=torch.int32, device="cuda") * new
        call = lambda s: S.spectra_paged_attention(cache, ck, cv, *pools, q, cu, new, 300, stream=s)  # noqa: E731
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call(torch.cuda.current_stream())
        graphs.append((g, q, out, cu, new))
    for _ in range(3):
        for g, q, out, cu, new in graphs:
            q.normal_()
            g.replay()
            got = out.clone()
            assert torch.equal(got, S.spectra_paged_attention(cache, ck, cv, *pools, q, cu, new, 300))


def test_two_captured_calls_share_a_workspace():
    # single tokens, and chunks whose slots are split, with their log-sum-exp
    (ck, _), (cv, _) = codec(BITS, 8, 1), codec(BITS, 8, 2)
    cache = S.PagedCache(50, 64, 1, 50)
    cache.table[0, :47] = torch.randperm(47).int()
    cache.lens[0] = 3000
    pools = [cache.empty_pool(c) for c in (ck, cv)]
    x = torch.randn((3000, H, D), device="cuda")
    S.spectra_paged_encode(cache, ck, cv, *pools, x, x, torch.tensor([0, 3000], dtype=torch.int32, device="cuda"))
    need = S.spectra_paged_attention_workspace_bytes(1, 64, H * QH, H, 64, 3000)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    graphs = []
    for new in (1, 64):
        for dtype in (torch.float32, torch.bfloat16):
            q = torch.randn((new, H * QH, D), device="cuda").to(dtype)
            cu = torch.tensor([0, new], dtype=torch.int32, device="cuda")
            out, lse = torch.empty_like(q), torch.empty((new, H * QH), device="cuda")
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                S.spectra_paged_attention(cache, ck, cv, *pools, q, cu, new, 3000, out=out, lse=lse, workspace=ws)
            graphs.append((g, q, cu, out, lse, new))
    for _ in range(3):
        for g, q, cu, out, lse, new in graphs:
            q.normal_()
            ws.fill_(255)
            g.replay()
            want_lse = torch.empty_like(lse)
            want = S.spectra_paged_attention(cache, ck, cv, *pools, q, cu, new, 3000, lse=want_lse)
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
