"""Arguments that the paged cache's entry points refuse on the host, before anything is launched:
each call is right but for one argument. No GPU is needed (pointers are never followed)."""
import ctypes

import pytest

import paper_2608_07915_amd as S
from paper_2608_07915_amd import _lib
from paper_2608_07915_amd._lib import spectra_pages, spectra_pool

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -4
P = 1 << 20            # an aligned address that nothing follows
OK = object()


def _codec(heads=2, **kw):
    c = _lib.spectra_codec()
    p = S.Params(**kw).c()
    _lib.check(_lib.get().spectra_codec_init(ctypes.byref(c), ctypes.byref(p), heads))
    c.basis = c.mean = c.var = c.bits = P
    return c


def _map(**kw):
    m = spectra_pages(100, 64, 8, 10, 0, P, P, P)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


BAD_MAPS = [dict(n_pages=0), dict(n_pages=2 ** 31), dict(page_tokens=0), dict(page_tokens=96), dict(rows=0), dict(rows=65536),
            dict(row_pages=0), dict(row_pages=2 ** 25), dict(table=None), dict(table=P + 2), dict(lens=None), dict(lens=P + 1)]


def _call(name, args, order, **bad):
    assert set(bad) <= set(order), bad
    vals = {**args, **bad}
    keep = []

    def c(v):
        if isinstance(v, ctypes.Structure):
            keep.append(v)
            return ctypes.byref(v)
        return v
    return getattr(_lib.get(), name)(*[c(vals[k]) for k in order])


ENCODE = ["m", "ck", "cv", "pool_k", "pool_v", "rows", "ends", "cu", "batch", "n_new", "k", "kts", "khs", "v", "vts", "vhs", "dt", "stream"]
ATTEND = ["m", "ck", "cv", "pool_k", "pool_v", "rows", "ends", "cu", "batch", "n_new", "max_new", "max_tokens", "q", "q_dt", "qts", "qhs",
          "heads", "scale", "out", "out_dt", "lse", "ws", "ws_bytes", "stream"]


def _cache_args():
    return dict(m=_map(), ck=_codec(), cv=_codec(), pool_k=P, pool_v=P, rows=None, ends=None, cu=P, batch=3, n_new=5, stream=None)


def encode(**bad):
    return _call("spectra_paged_encode", dict(_cache_args(), k=P, kts=256, khs=128, v=P, vts=256, vhs=128, dt=1), ENCODE, **bad)


def attend(**bad):
    return _call("spectra_paged_attention", dict(_cache_args(), max_new=4, max_tokens=300, q=P, q_dt=1, qts=1024, qhs=128, heads=8,
                                                 scale=0.0, out=P, out_dt=1, lse=None, ws=P, ws_bytes=1 << 30), ATTEND, **bad)


SHARED = [dict(ck=_codec(3)), dict(batch=-1), dict(batch=16385), dict(batch=9), dict(n_new=-1), dict(n_new=2 ** 31), dict(cu=None),
          dict(cu=P + 2), dict(rows=P + 1), dict(ends=P + 1), dict(pool_k=None), dict(pool_v=P + 8)]


@pytest.mark.parametrize("call", [encode, attend])
def test_cache_arguments(call):
    for bad in BAD_MAPS:
        assert call(m=_map(**bad)) == EINVAL, bad
    for bad in SHARED:
        assert call(**bad) == EINVAL, bad
    layer = _codec(2, head_dim=256, group_size=64)
    assert call(ck=layer, cv=layer) == EUNSUPPORTED
    broken = _codec()
    broken.basis = P + 4
    assert call(cv=broken) == EINVAL
    assert b"basis" in _lib.get().spectra_last_error()
    assert call(batch=0) == 0 and call(n_new=0) == 0  # nothing to do


def test_encode_arguments():
    for bad in (dict(k=None), dict(k=P + 8), dict(v=P + 2), dict(dt=7), dict(kts=-8), dict(khs=4), dict(vts=12), dict(vhs=-128)):
        assert encode(**bad) == EINVAL, bad
    assert encode(dt=0, kts=6) == EINVAL


def test_attention_arguments():
    for bad in (dict(heads=0), dict(heads=7), dict(max_new=-1), dict(max_tokens=-1), dict(max_new=2 ** 30), dict(n_new=2 ** 28),
                dict(q=None), dict(q=P + 4), dict(q_dt=2), dict(out_dt=2), dict(qts=9), dict(qhs=-8), dict(out=None), dict(out=P + 8),
                dict(lse=P + 1), dict(ws=None), dict(ws=P + 16), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attend(**bad) == EINVAL, bad
    assert attend(heads=34) == EUNSUPPORTED
    assert attend(ws_bytes=255) == EWORKSPACE
    assert attend(max_new=0) == 0 and attend(max_tokens=0) == 0
    need = S.spectra_paged_attention_workspace_bytes
    assert need(0, 5, 8, 2, 4, 300) == need(3, 5, 7, 2, 4, 300) == need(3, 5, 8, 2, 0, 300) == 0
    assert need(3, 5, 8, 2, 4, 300) % 256 == 0


def test_map_calls():
    lib = _lib.get()
    pools = (spectra_pool * 2)(spectra_pool(P, 1024), spectra_pool(P, 0))
    none = ctypes.POINTER(spectra_pool)()

    def extend(m=None, rows=P, counts=P, n=4, pools=pools, n_pools=2, ends=P, ws=P, ws_bytes=1 << 20):
        return lib.spectra_pages_extend(ctypes.byref(m or _map()), rows, counts, n, pools, n_pools, ends, ws, ws_bytes, None)

    def fork(m=None, parents=P, children=P, n=4, ends=P):
        return lib.spectra_pages_fork(ctypes.byref(m or _map()), parents, children, n, ends, None)

    def truncate(m=None, rows=P, keep=P, n=4):
        return lib.spectra_pages_truncate(ctypes.byref(m or _map()), rows, keep, n, None)

    def compact(m=None, pools=pools, n_pools=2, moved=P, ws=P, ws_bytes=1 << 20):
        return lib.spectra_pages_compact(ctypes.byref(m or _map()), pools, n_pools, moved, ws, ws_bytes, None)

    for call in (extend, fork, truncate, compact):
        for bad in BAD_MAPS + [dict(refs=None), dict(refs=P + 3)]:
            assert call(m=_map(**bad)) == EINVAL, (call.__name__, bad)
    for call, lists in ((extend, ("rows", "counts", "ends")), (fork, ("parents", "children", "ends")), (truncate, ("rows",))):
        for a in lists:
            assert call(**{a: None}) == EINVAL and call(**{a: P + 2}) == EINVAL, (call.__name__, a)
        assert call(n=-1) == EINVAL and call(n=1025) == EINVAL
        assert call(n=0) == 0
    assert truncate(keep=P + 1) == EINVAL
    for call in (extend, compact):
        for bad in (spectra_pool(P, 100), spectra_pool(P, -64), spectra_pool(P + 8, 64), spectra_pool(None, 64)):
            assert call(pools=(spectra_pool * 1)(bad), n_pools=1) == EINVAL
        assert call(pools=none, n_pools=1) == EINVAL and call(n_pools=-1) == EINVAL
        assert call(ws=None) == EINVAL and call(ws=P + 64) == EINVAL and call(ws_bytes=256) == EWORKSPACE
    assert compact(moved=None) == EINVAL and compact(moved=P + 2) == EINVAL
    assert lib.spectra_pages_extend(None, P, P, 1, pools, 2, P, P, 1 << 20, None) == EINVAL


def test_sizes():
    lib = _lib.get()
    m, c = _map(), _codec(3, ratio=8.0)
    assert lib.spectra_paged_pool_words(ctypes.byref(m), ctypes.byref(c)) == 100 * 64 * 3 * 8
    assert lib.spectra_pages_workspace_bytes(ctypes.byref(m)) >= 2 * 100 * 4
    assert lib.spectra_paged_pool_words(None, ctypes.byref(c)) == 0 and lib.spectra_pages_workspace_bytes(None) == 0


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    c = S.PagedCache(10, 64, 2, 4, device="cpu")
    ck, cv = S.Codec(S.Params(), 2, device="cpu"), S.Codec(S.Params(), 2, device="cpu")
    rows = torch.zeros(1, dtype=torch.int32)
    pools = [c.empty_pool(x) for x in (ck, cv)]
    x = torch.zeros(1, 2, 128)
    cu = torch.tensor([0, 1], dtype=torch.int32)
    for call in (lambda: S.spectra_pages_extend(c, rows, rows, pools), lambda: S.spectra_pages_fork(c, rows, rows),
                 lambda: S.spectra_pages_truncate(c, rows), lambda: S.spectra_pages_compact(c, pools),
                 lambda: S.spectra_paged_encode(c, ck, cv, *pools, x, x, cu),
                 lambda: S.spectra_paged_attention(c, ck, cv, *pools, x, cu, 1, 1)):
        with pytest.raises(ValueError, match="on a device"):
            call()
    with pytest.raises(ValueError, match="multiple of 64"):
        S.PagedCache(10, 100, 2, 4, device="cpu")
    with pytest.raises(ValueError, match="pool_k holds"):
        S.spectra_paged_encode(c, ck, cv, pools[0][:5], pools[1], x, x, cu)
    with pytest.raises(ValueError, match="k must be"):
        S.spectra_paged_encode(c, ck, cv, *pools, x[:, :1], x, cu)
    with pytest.raises(ValueError, match="int32"):
        S.spectra_paged_encode(c, ck, cv, *pools, x, x, cu.long())
    with pytest.raises(ValueError, match="multiple of the codec"):
        S.spectra_paged_attention(c, ck, cv, *pools, torch.zeros(1, 3, 128), cu, 1, 1)
    with pytest.raises(ValueError, match="lse"):
        S.spectra_paged_attention(c, ck, cv, *pools, x, cu, 1, 1, lse=torch.zeros(1, 3))


def test_sizes_that_kernels_count_in_32_bits():
    for call in (encode, attend):
        assert call(m=_map(page_tokens=2 ** 20 + 64, row_pages=1)) == EINVAL
        assert call(m=_map(row_pages=2 ** 24 + 1)) == EINVAL
        assert call(m=_map(row_pages=2 ** 24), batch=0) == 0
    assert attend(max_tokens=2 ** 30 + 1) == EINVAL
    assert attend(n_new=2 ** 27 + 1) == EINVAL and attend(max_new=2 ** 27 + 1) == EINVAL
    many = dict(m=_map(rows=65535), ck=_codec(32), cv=_codec(32), heads=32)
    assert attend(batch=2 ** 13, **many) == EINVAL and b"2^18" in _lib.get().spectra_last_error()
