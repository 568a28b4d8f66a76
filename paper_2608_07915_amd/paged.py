"""Binding of the paged cache (argument marshalling only): many sequences' records in pools of
pages under one page map, their appends and the attention over them. Function names match the C
ABI in ``include/spectra.h``.

``stream`` (default: the current one) is where a call runs. Outputs and workspaces that are made for
a call belong to that stream; other streams that use an output wait for it first.
"""
from __future__ import annotations

import ctypes

from . import _lib
from ._lib import check, spectra_pages, spectra_pool
from .codec import Codec, _dtype_code, _made, _need


class PagedCache:
    """Page map of a set of sequences, on the device: ``table`` [rows, row_pages], ``lens``
    [rows] and ``refs`` [n_pages] (int32), all pages free. The pools it maps are the caller's
    (``empty_pool``, one per layer and tensor)."""

    def __init__(self, n_pages: int, page_tokens: int, rows: int, row_pages: int, device="cuda"):
        import torch
        self.n_pages, self.page_tokens, self.rows, self.row_pages = int(n_pages), int(page_tokens), int(rows), int(row_pages)
        _need(self.n_pages > 0 and self.rows > 0 and self.row_pages > 0, "n_pages, rows and row_pages must be positive")
        _need(self.page_tokens > 0 and self.page_tokens % 64 == 0, f"page_tokens={page_tokens} must be a multiple of 64")
        self.table = torch.full((self.rows, self.row_pages), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(self.rows, dtype=torch.int32, device=device)
        self.refs = torch.zeros(self.n_pages, dtype=torch.int32, device=device)
        self.struct = spectra_pages(self.n_pages, self.page_tokens, self.rows, self.row_pages, 0, self.table.data_ptr(),
                                    self.lens.data_ptr(), self.refs.data_ptr())
        self.ref = ctypes.byref(self.struct)

    def empty_pool(self, codec: Codec):
        """A pool for the codec's records: int32 [n_pages, words of a page], zeros."""
        import torch
        words = int(_lib.get().spectra_paged_pool_words(self.ref, ctypes.byref(codec.struct)))
        return torch.zeros((self.n_pages, words // self.n_pages), dtype=torch.int32, device=self.table.device)


class _Call:
    """The call's stream, with the cache's device current while the call is made."""
    __slots__ = ("handle", "ctx")

    def __init__(self, device, stream):
        import torch
        _need(device.type == "cuda", "the page map must be on a device")
        _need(stream is None or stream.device == device, f"the stream belongs to another device than the page map's {device}")
        self.handle = stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device.index)
        self.ctx = None if torch.cuda.current_device() == device.index else torch.cuda.device(device)

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        return self

    def __exit__(self, *exc):
        return self.ctx.__exit__(*exc) if self.ctx is not None else None


def _ints(t, name: str, device, n=None):
    """Pointer of a contiguous int32 tensor on the device, of n elements (None: no tensor)."""
    import torch
    if t is None:
        return None
    if not (t.device == device and t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous one-dimensional int32 tensor on {device}")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} must have {n} elements, got {t.numel()}")
    return t.data_ptr()


def _pools(cache: PagedCache, pools):
    import torch
    pools = [pools] if isinstance(pools, torch.Tensor) else pools
    dev, n_pages, flat = cache.table.device, cache.n_pages, []
    for i, p in enumerate(pools):
        n = p.numel()
        if not (p.device == dev and p.dtype == torch.int32 and p.is_contiguous()):
            raise ValueError(f"pool {i} must be a contiguous int32 tensor on {dev}")
        if n % (64 * n_pages):
            raise ValueError(f"pool {i}: {n} words are not {n_pages} pages of whole tiles")
        flat.append((p.data_ptr(), n // n_pages))
    return (spectra_pool * max(len(flat), 1))(*flat), len(flat)


def _workspace(cache: PagedCache, workspace, need: int, stream):
    import torch
    if workspace is None:
        return _made(stream, max(need, 1), torch.uint8, cache.table.device)
    _need(workspace.device == cache.table.device and workspace.is_contiguous(),
          f"workspace must be contiguous and on {cache.table.device}")
    return workspace


def _bytes(t) -> int:
    return t.numel() * t.element_size()


def spectra_pages_workspace_bytes(cache: PagedCache) -> int:
    return int(_lib.get().spectra_pages_workspace_bytes(cache.ref))


def spectra_pages_extend(cache: PagedCache, rows, counts, pools, ends=None, workspace=None, stream=None):
    """Room for counts[i] more tokens in row rows[i] -> ends (int32): the new lengths, -1 where
    refused. ``pools``: every pool of the map (shared last pages are copied in all of them)."""
    import torch
    dev = cache.table.device
    n = rows.numel()
    with _Call(dev, stream) as s:
        args = (_ints(rows, "rows", dev), _ints(counts, "counts", dev, n))
        made, n_pools = _pools(cache, pools)
        ends = _made(stream, n, torch.int32, dev) if ends is None else ends
        ws = _workspace(cache, workspace, spectra_pages_workspace_bytes(cache), stream)
        check(_lib.get().spectra_pages_extend(cache.ref, *args, n, made, n_pools,
                                              _ints(ends, "ends", dev, n), ws.data_ptr(), _bytes(ws), s.handle))
    return ends


def spectra_pages_fork(cache: PagedCache, parents, children, ends=None, stream=None):
    """Rows ``children`` (empty) become copies of rows ``parents`` that share their pages -> ends
    (int32): the children's lengths, -1 where refused."""
    import torch
    dev = cache.table.device
    n = parents.numel()
    with _Call(dev, stream) as s:
        ends = _made(stream, n, torch.int32, dev) if ends is None else ends
        check(_lib.get().spectra_pages_fork(cache.ref, _ints(parents, "parents", dev),
                                            _ints(children, "children", dev, n), n, _ints(ends, "ends", dev, n), s.handle))
    return ends


def spectra_pages_truncate(cache: PagedCache, rows, keep=None, stream=None) -> None:
    """Row rows[i] keeps its first keep[i] slots (keep None: the rows are emptied)."""
    dev = cache.table.device
    n = rows.numel()
    with _Call(dev, stream) as s:
        check(_lib.get().spectra_pages_truncate(cache.ref, _ints(rows, "rows", dev),
                                                _ints(keep, "keep", dev, n), n, s.handle))


def spectra_pages_compact(cache: PagedCache, pools, moved=None, workspace=None, stream=None):
    """Used pages to the front of every pool -> moved (int32 [n_pages + 1]): every page's place
    afterwards, then the number of used pages."""
    import torch
    dev = cache.table.device
    with _Call(dev, stream) as s:
        made, n_pools = _pools(cache, pools)
        moved = _made(stream, cache.n_pages + 1, torch.int32, dev) if moved is None else moved
        ws = _workspace(cache, workspace, spectra_pages_workspace_bytes(cache), stream)
        check(_lib.get().spectra_pages_compact(cache.ref, made, n_pools,
                                               _ints(moved, "moved", dev, cache.n_pages + 1), ws.data_ptr(), _bytes(ws),
                                               s.handle))
    return moved


def _sequences(cache: PagedCache, ck: Codec, cv: Codec, pool_k, pool_v, cu_new, rows, ends):
    """Checks of what append and attention share -> (batch, pointers of the C call's head)."""
    import torch
    dev = cache.table.device
    _need(cu_new.numel() >= 1, "cu_new must have batch + 1 elements")
    batch = cu_new.numel() - 1
    for codec, pool, name in ((ck, pool_k, "pool_k"), (cv, pool_v, "pool_v")):
        _need(codec.basis.device == dev, f"the codecs must be on {dev}")
        _need(pool.device == dev and pool.dtype == torch.int32 and pool.is_contiguous(),
              f"{name} must be a contiguous int32 tensor on {dev}")
        need = int(_lib.get().spectra_paged_pool_words(cache.ref, ctypes.byref(codec.struct)))
        _need(pool.numel() == need, f"{name} holds {pool.numel()} words, the map and codec need {need}")
    return batch, (cache.ref, ctypes.byref(ck.struct), ctypes.byref(cv.struct), pool_k.data_ptr(),
                   pool_v.data_ptr(), _ints(rows, "rows", dev, batch), _ints(ends, "ends", dev, batch),
                   _ints(cu_new, "cu_new", dev), batch)


def _rows(x, name: str, device, heads: int, n=None):
    """x [n, heads, 128] on the device, unit stride along the channels; strides may vary."""
    _need(x.device == device and x.dim() == 3 and x.shape[1] == heads and x.shape[2] == 128 and x.stride(2) == 1,
          f"{name} must be [n, {heads}, 128] on {device} with unit stride along the channels, got {tuple(x.shape)}")
    _need(n is None or x.shape[0] == n, f"{name} must have {n} tokens, got {x.shape[0]}")


def spectra_paged_encode(cache: PagedCache, ck: Codec, cv: Codec, pool_k, pool_v, k, v, cu_new, rows=None, ends=None,
                         stream=None) -> None:
    """New tokens k, v [n, n_kv_heads, 128] of the sequences into their pages: tokens cu_new[b] ..
    cu_new[b + 1] go to the last slots of sequence b, which is map row rows[b] (default b) and has
    ends[b] slots (default ``cache.lens`` of its row) with them."""
    dev = cache.table.device
    batch, head = _sequences(cache, ck, cv, pool_k, pool_v, cu_new, rows, ends)
    _rows(k, "k", dev, ck.n_streams)
    _rows(v, "v", dev, ck.n_streams, k.shape[0])
    _need(k.dtype == v.dtype, "k and v must have one dtype")
    with _Call(dev, stream) as s:
        check(_lib.get().spectra_paged_encode(*head, k.shape[0], k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(),
                                              v.stride(0), v.stride(1), _dtype_code(k), s.handle))


def spectra_paged_attention_workspace_bytes(batch: int, n_new: int, n_q_heads: int, n_kv_heads: int, max_new: int,
                                            max_tokens: int) -> int:
    return int(_lib.get().spectra_paged_attention_workspace_bytes(int(batch), int(n_new), int(n_q_heads), int(n_kv_heads),
                                                                  int(max_new), int(max_tokens)))


def spectra_paged_attention(cache: PagedCache, ck: Codec, cv: Codec, pool_k, pool_v, q, cu_new, max_new: int,
                            max_tokens: int, rows=None, ends=None, softmax_scale: float = 0.0, out=None, lse=None,
                            workspace=None, stream=None):
    """Causal attention of the new tokens q [n, n_q_heads, 128] over their sequences' pages -> out
    [n, n_q_heads, 128] of q's dtype (or a given float32 or bfloat16 ``out``). Sequences as in
    spectra_paged_encode, none with more than max_new new tokens or max_tokens slots. ``lse``: a
    float32 [n, n_q_heads] tensor that takes the log-sum-exp of the scores."""
    import torch
    dev = cache.table.device
    batch, head = _sequences(cache, ck, cv, pool_k, pool_v, cu_new, rows, ends)
    n, n_q_heads = q.shape[0], q.shape[1]
    _rows(q, "q", dev, n_q_heads)
    _need(n_q_heads % ck.n_streams == 0, f"n_q_heads={n_q_heads} is not a multiple of the codec's {ck.n_streams} KV heads")
    _need(lse is None or (lse.device == dev and lse.dtype == torch.float32 and lse.is_contiguous()
                          and tuple(lse.shape) == (n, n_q_heads)), f"lse must be a contiguous float32 tensor {(n, n_q_heads)}")
    with _Call(dev, stream) as s:
        out = _made(stream, (n, n_q_heads, 128), q.dtype, dev) if out is None else out
        _need(out.device == dev and out.is_contiguous() and tuple(out.shape) == (n, n_q_heads, 128),
              f"out must be a contiguous tensor {(n, n_q_heads, 128)} on {dev}")
        ws = _workspace(cache, workspace, spectra_paged_attention_workspace_bytes(batch, n, n_q_heads, ck.n_streams,
                                                                                  max_new, max_tokens), stream)
        check(_lib.get().spectra_paged_attention(*head, n, int(max_new), int(max_tokens), q.data_ptr(), _dtype_code(q),
                                                 q.stride(0), q.stride(1), n_q_heads, float(softmax_scale), out.data_ptr(),
                                                 _dtype_code(out), lse.data_ptr() if lse is not None else None,
                                                 ws.data_ptr(), _bytes(ws), s.handle))
    return out
