"""Arguments that the calls on drafted trees, boxes and listed blocks refuse on the host, before anything is launched.
No GPU is needed (pointers are never followed)."""
import ctypes

import pytest

import paper_2608_07915_amd as S
from paper_2608_07915_amd import _lib
from paper_2608_07915_amd._lib import spectra_pool
from test_paged_refusals import BAD_MAPS, EINVAL, EUNSUPPORTED, EWORKSPACE, P, _cache_args, _call, _codec, _map

TREE = ["m", "ck", "cv", "pool_k", "pool_v", "rows", "ends", "cu", "parents", "batch", "n_new", "max_new", "max_tokens", "q", "q_dt",
        "qts", "qhs", "heads", "scale", "out", "out_dt", "lse", "ws", "ws_bytes", "stream"]
SPARSE = ["m", "ck", "cv", "pool_k", "pool_v", "rows", "ends", "cu", "batch", "n_new", "blocks", "n_blocks", "q", "q_dt", "qts", "qhs",
          "heads", "scale", "out", "out_dt", "lse", "ws", "ws_bytes", "stream"]
SELECT = ["m", "ck", "bounds", "rows", "ends", "cu", "batch", "n_new", "max_tokens", "q", "q_dt", "qts", "qhs", "heads", "n_blocks",
          "first", "last", "blocks", "ws", "ws_bytes", "stream"]
BOUNDS = ["m", "ck", "pool_k", "bounds", "rows", "ends", "cu", "batch", "n_new", "stream"]
QUERY = dict(q=P, q_dt=1, qts=1024, qhs=128, heads=8)


def _args(*names, **more):
    a = dict(_cache_args(), **more)
    return {k: v for k, v in a.items() if k in names}


def tree(**bad):
    return _call("spectra_paged_tree_attention", _args(*TREE, parents=P, max_new=4, max_tokens=300, scale=0.0, out=P, out_dt=1, lse=None,
                                                       ws=P, ws_bytes=1 << 30, **QUERY), TREE, **bad)


def sparse(**bad):
    return _call("spectra_paged_sparse_attention", _args(*SPARSE, blocks=P, n_blocks=9, scale=0.0, out=P, out_dt=1, lse=None, ws=P,
                                                         ws_bytes=1 << 30, **QUERY), SPARSE, **bad)


def select(**bad):
    return _call("spectra_paged_select", _args(*SELECT, bounds=P, max_tokens=300, n_blocks=9, first=1, last=2, blocks=P, ws=P,
                                               ws_bytes=1 << 30, **QUERY), SELECT, **bad)


def bounds(**bad):
    return _call("spectra_paged_bounds", _args(*BOUNDS, bounds=P), BOUNDS, **bad)


SHARED = [dict(batch=-1), dict(batch=16385), dict(batch=9), dict(n_new=-1), dict(n_new=2 ** 31), dict(cu=None), dict(cu=P + 2),
          dict(rows=P + 1), dict(ends=P + 1)]


@pytest.mark.parametrize("call", [tree, sparse, select, bounds])
def test_sequences(call):
    for bad in BAD_MAPS:
        assert call(m=_map(**bad)) == EINVAL, bad
    for bad in SHARED:
        assert call(**bad) == EINVAL, bad
    layer = _codec(2, head_dim=256, group_size=64)
    assert call(ck=layer, **({"cv": layer} if call in (tree, sparse) else {})) == EUNSUPPORTED
    broken = _codec()
    broken.bits = P + 2
    assert call(ck=broken) == EINVAL
    assert call(batch=0) == 0 and call(n_new=0) == 0  # nothing to do


@pytest.mark.parametrize("call", [tree, sparse])
def test_attention_arguments(call):
    for bad in (dict(heads=0), dict(heads=7), dict(q=None), dict(q=P + 4), dict(q_dt=2), dict(out_dt=2), dict(qts=9), dict(qhs=-8),
                dict(out=None), dict(out=P + 8), dict(lse=P + 1), dict(ws=None), dict(ws=P + 16), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(pool_k=None), dict(pool_v=P + 8), dict(ck=_codec(3)), dict(n_new=2 ** 21 + 1)):
        assert call(**bad) == EINVAL, bad
    assert call(heads=34) == EUNSUPPORTED
    assert call(ws_bytes=255) == EWORKSPACE
    many = dict(m=_map(rows=65535), ck=_codec(32), cv=_codec(32), heads=32)
    assert call(batch=2 ** 13, **many) == EINVAL and b"2^18" in _lib.get().spectra_last_error()


def test_tree_arguments():
    for bad in (dict(parents=None), dict(parents=P + 2), dict(max_new=-1), dict(max_tokens=-1), dict(max_tokens=2 ** 30 + 1)):
        assert tree(**bad) == EINVAL, bad
    assert tree(max_new=65) == EUNSUPPORTED and b"64" in _lib.get().spectra_last_error()
    assert tree(max_new=0) == 0 and tree(max_tokens=0) == 0
    need = S.spectra_paged_tree_attention_workspace_bytes
    assert need(0, 5, 8, 2, 4, 300) == need(3, 5, 7, 2, 4, 300) == need(3, 5, 8, 2, 0, 300) == need(3, 2 ** 22, 8, 2, 4, 300) == 0


def test_sparse_arguments():
    for bad in (dict(blocks=None), dict(blocks=P + 2), dict(n_blocks=0), dict(n_blocks=4097), dict(n_new=2 ** 20, n_blocks=4096)):
        assert sparse(**bad) == EINVAL, bad
    need = S.spectra_paged_sparse_attention_workspace_bytes
    assert need(0, 8, 2, 9) == need(5, 7, 2, 9) == need(5, 8, 2, 0) == need(5, 8, 2, 4097) == 0


def test_select_arguments():
    for bad in (dict(bounds=None), dict(bounds=P + 8), dict(q=None), dict(q=P + 8), dict(q_dt=5), dict(qts=4), dict(qhs=-8), dict(heads=7),
                dict(max_tokens=-1), dict(max_tokens=2 ** 31), dict(n_blocks=-1), dict(n_blocks=4097), dict(first=-1), dict(last=-1),
                dict(first=5, last=5), dict(blocks=None), dict(blocks=P + 1), dict(ws=None), dict(ws=P + 128), dict(n_new=2 ** 21 + 1)):
        assert select(**bad) == EINVAL, bad
    assert select(heads=34) == EUNSUPPORTED
    assert select(ws_bytes=3) == EWORKSPACE
    assert select(max_tokens=0) == 0 and select(n_blocks=0, first=0, last=0) == 0
    need = S.spectra_paged_select_workspace_bytes
    assert need(0, 8, 2, 300) == need(5, 7, 2, 300) == need(5, 8, 2, 0) == 0


def test_bounds_arguments():
    for bad in (dict(pool_k=None), dict(pool_k=P + 8), dict(bounds=None), dict(bounds=P + 4), dict(n_new=2 ** 29 + 1)):
        assert bounds(**bad) == EINVAL, bad
    words = _lib.get().spectra_paged_bounds_words
    assert words(ctypes.byref(_map(page_tokens=128)), 3) == 100 * 3 * 2 * 128
    assert words(None, 3) == words(ctypes.byref(_map()), 0) == 0


def test_accept_arguments():
    pools = (spectra_pool * 2)(spectra_pool(P, 64 * 3 * 8), spectra_pool(P, 64 * 3 * 5))

    def accept(m=None, rows=P, drafted=P, path=P, stride=8, counts=P, n=4, pools=pools, n_pools=2, kv=3, ends=P):
        return _lib.get().spectra_pages_accept(ctypes.byref(m or _map()), rows, drafted, path, stride, counts, n, pools, n_pools, kv, ends,
                                               None)

    for bad in BAD_MAPS + [dict(refs=None), dict(refs=P + 3)]:
        assert accept(m=_map(**bad)) == EINVAL, bad
    for a in ("rows", "drafted", "path", "counts", "ends"):
        assert accept(**{a: None}) == EINVAL and accept(**{a: P + 2}) == EINVAL, a
    for bad in (dict(n=-1), dict(n=1025), dict(stride=-1), dict(stride=65), dict(kv=0), dict(kv=65536), dict(n_pools=-1), dict(kv=2, n_pools=1, pools=(spectra_pool * 1)(spectra_pool(P, 64 * 3)))):
        assert accept(**bad) == EINVAL, bad
    for p in (spectra_pool(P, 64 * 8), spectra_pool(P + 8, 192), spectra_pool(None, 192), spectra_pool(P, -192), spectra_pool(P, 2 ** 40)):
        assert accept(pools=(spectra_pool * 1)(p), n_pools=1) == EINVAL
    assert accept(n=0) == 0 and accept(n=0, rows=None, path=None) == 0


def test_workspaces_never_fall():
    sizes = [1, 2, 3, 7, 16, 60, 300, 5000]
    for kv, q in ((1, 1), (2, 8), (4, 28), (8, 128), (300, 300)):
        last = 0
        for n in sizes:
            b = S.spectra_paged_tree_attention_workspace_bytes(n, n, q, kv, 64, 1000)
            assert b >= last and b >= S.spectra_paged_tree_attention_workspace_bytes(max(1, n // 2), n, q, kv, 9, 10)
            last = b
        last = 0
        for n in sizes:
            for k in (1, 4, 64, 4096):
                b = S.spectra_paged_sparse_attention_workspace_bytes(n, q, kv, k)
                assert b >= S.spectra_paged_sparse_attention_workspace_bytes(max(1, n // 2), q, kv, max(1, k // 3))
            assert b >= last
            last = b
        last = 0
        for t in (1, 63, 64, 65, 1000, 10 ** 6):
            b = S.spectra_paged_select_workspace_bytes(5, q, kv, t)
            assert b >= last and b >= S.spectra_paged_select_workspace_bytes(4, q, kv, t)
            last = b


def test_binding_refuses_wrong_tensors():
    torch = pytest.importorskip("torch")
    c = S.PagedCache(10, 64, 2, 4, device="cpu")
    ck, cv = S.Codec(S.Params(), 2, device="cpu"), S.Codec(S.Params(), 2, device="cpu")
    pools = [c.empty_pool(x) for x in (ck, cv)]
    box = c.empty_bounds(ck)
    assert tuple(box.shape) == (10, 2 * 128)
    q, one = torch.zeros(1, 4, 128), torch.zeros(1, dtype=torch.int32)
    cu, path = torch.tensor([0, 1], dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)
    blocks = torch.zeros(1, 2, 3, dtype=torch.int32)
    for call in (lambda: S.spectra_paged_tree_attention(c, ck, cv, *pools, q, cu, one, 1, 1),
                 lambda: S.spectra_pages_accept(c, one, one, path, one, pools, 2),
                 lambda: S.spectra_paged_bounds(c, ck, pools[0], box, cu, 1),
                 lambda: S.spectra_paged_select(c, ck, box, q, cu, 3, 100),
                 lambda: S.spectra_paged_sparse_attention(c, ck, cv, *pools, q, cu, blocks)):
        with pytest.raises(ValueError, match="on a device"):
            call()
    for call, text in ((lambda: S.spectra_paged_tree_attention(c, ck, cv, *pools, q, cu, one.long(), 1, 1), "parents"),
                       (lambda: S.spectra_paged_tree_attention(c, ck, cv, *pools, q, cu, cu, 1, 1), "parents"),
                       (lambda: S.spectra_pages_accept(c, one, one, path.long(), one, pools, 2), "path"),
                       (lambda: S.spectra_paged_bounds(c, ck, pools[0], box[:9], cu, 1), "bounds"),
                       (lambda: S.spectra_paged_bounds(c, ck, pools[0][:9], box, cu, 1), "pool_k holds"),
                       (lambda: S.spectra_paged_select(c, ck, box, q[:, :3], cu, 3, 100), "multiple of the codec"),
                       (lambda: S.spectra_paged_sparse_attention(c, ck, cv, *pools, q, cu, blocks[:, :1]), "blocks"),
                       (lambda: S.spectra_paged_sparse_attention(c, ck, cv, *pools, q, cu, blocks, lse=torch.zeros(1, 3)), "lse")):
        with pytest.raises(ValueError, match=text):
            call()
