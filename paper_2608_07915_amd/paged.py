"""Binding of the paged cache (argument marshalling only): many sequences' records in pools of
pages under one page map, their appends and the attention over them. Function names match the C
ABI in ``include/spectra.h``.

``stream`` (default: the current one) is where a call runs. Outputs and workspaces that are made for
a call belong to that stream; other streams that use an output wait for it first.
"""
from __future__ import annotations

import ctypes
from array import array

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

    def empty_bounds(self, codec: Codec):
        """A box pool for the keys' codec (``spectra_paged_bounds``): int32 [n_pages, words of a page],
        zeros. As float16 it is [n_pages, KV head, tile, place of a kept group, least / largest, 32]."""
        import torch
        words = int(_lib.get().spectra_paged_bounds_words(self.ref, codec.n_streams))
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
    dev, n_pages, flat = cache.table.device, cache.n_pages, array("q")
    for p in pools:
        n = p.numel()
        if p.device != dev or p.dtype != torch.int32 or not p.is_contiguous():
            raise ValueError(f"pool {len(flat) // 2} must be a contiguous int32 tensor on {dev}")
        if n % (64 * n_pages):
            raise ValueError(f"pool {len(flat) // 2}: {n} words are not {n_pages} pages of whole tiles")
        flat.append(p.data_ptr())
        flat.append(n // n_pages)
    made = (spectra_pool * max(len(flat) // 2, 1))()
    if flat:
        ctypes.memmove(made, flat.buffer_info()[0], ctypes.sizeof(made))
    return made, len(flat) // 2


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


def _records(cache: PagedCache, codec: Codec, pool, name: str) -> None:
    import torch
    dev = cache.table.device
    _need(codec.basis.device == dev, f"the codecs must be on {dev}")
    _need(pool.device == dev and pool.dtype == torch.int32 and pool.is_contiguous(),
          f"{name} must be a contiguous int32 tensor on {dev}")
    need = int(_lib.get().spectra_paged_pool_words(cache.ref, ctypes.byref(codec.struct)))
    _need(pool.numel() == need, f"{name} holds {pool.numel()} words, the map and codec need {need}")


def _sequences(cache: PagedCache, ck: Codec, cv: Codec, pool_k, pool_v, cu_new, rows, ends):
    """Checks of what append and attention share -> (batch, pointers of the C call's head)."""
    dev = cache.table.device
    _need(cu_new.numel() >= 1, "cu_new must have batch + 1 elements")
    batch = cu_new.numel() - 1
    _records(cache, ck, pool_k, "pool_k")
    _records(cache, cv, pool_v, "pool_v")
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


def spectra_pages_accept(cache: PagedCache, rows, drafted, path, counts, pools, n_kv_heads: int, ends=None, stream=None):
    """One path of each drafted tree stays: of the last drafted[i] slots of row rows[i] those at path[i, j], j <
    counts[i] (ascending, from 0), move to the front of them in every pool, and the row ends behind them -> ends
    (int32): the new lengths, -1 where refused. ``pools``: the record pools of n_kv_heads KV heads each; boxes
    of the kept slots' blocks are made again by spectra_paged_bounds."""
    import torch
    dev = cache.table.device
    n = rows.numel()
    _need(path.device == dev and path.dtype == torch.int32 and path.dim() == 2 and path.is_contiguous() and path.shape[0] == n,
          f"path must be a contiguous int32 tensor [{n}, most] on {dev}")
    with _Call(dev, stream) as s:
        made, n_pools = _pools(cache, pools)
        ends = _made(stream, n, torch.int32, dev) if ends is None else ends
        check(_lib.get().spectra_pages_accept(cache.ref, _ints(rows, "rows", dev), _ints(drafted, "drafted", dev, n),
                                              path.data_ptr(), path.shape[1], _ints(counts, "counts", dev, n), n, made, n_pools,
                                              int(n_kv_heads), _ints(ends, "ends", dev, n), s.handle))
    return ends


def _attended(cache: PagedCache, ck: Codec, q, lse):
    """Queries and log-sum-exp of an attention call -> (tokens, query heads)."""
    import torch
    dev = cache.table.device
    n, n_q_heads = q.shape[0], q.shape[1]
    _rows(q, "q", dev, n_q_heads)
    _need(n_q_heads % ck.n_streams == 0, f"n_q_heads={n_q_heads} is not a multiple of the codec's {ck.n_streams} KV heads")
    _need(lse is None or (lse.device == dev and lse.dtype == torch.float32 and lse.is_contiguous()
                          and tuple(lse.shape) == (n, n_q_heads)), f"lse must be a contiguous float32 tensor {(n, n_q_heads)}")
    return n, n_q_heads


def _output(out, q, stream):
    shape = tuple(q.shape)
    if out is None:
        return _made(stream, shape, q.dtype, q.device)
    _need(out.device == q.device and out.is_contiguous() and tuple(out.shape) == shape,
          f"out must be a contiguous tensor {shape} on {q.device}")
    return out


def spectra_paged_tree_attention_workspace_bytes(batch: int, n_new: int, n_q_heads: int, n_kv_heads: int, max_new: int,
                                                 max_tokens: int) -> int:
    return int(_lib.get().spectra_paged_tree_attention_workspace_bytes(int(batch), int(n_new), int(n_q_heads),
                                                                       int(n_kv_heads), int(max_new), int(max_tokens)))


def spectra_paged_tree_attention(cache: PagedCache, ck: Codec, cv: Codec, pool_k, pool_v, q, cu_new, parents, max_new: int,
                                 max_tokens: int, rows=None, ends=None, softmax_scale: float = 0.0, out=None, lse=None,
                                 workspace=None, stream=None):
    """Attention of drafted tokens: as spectra_paged_attention, but of its sequence's new tokens a token sees
    itself and its ancestors only. ``parents`` (int32 [n]): the place of each token's parent among the new tokens
    of its sequence, -1 where it continues the history. At most 64 new tokens of a sequence."""
    dev = cache.table.device
    batch, head = _sequences(cache, ck, cv, pool_k, pool_v, cu_new, rows, ends)
    n, n_q_heads = _attended(cache, ck, q, lse)
    up = _ints(parents, "parents", dev, n)
    with _Call(dev, stream) as s:
        out = _output(out, q, stream)
        ws = _workspace(cache, workspace, spectra_paged_tree_attention_workspace_bytes(batch, n, n_q_heads, ck.n_streams, max_new,
                                                                                       max_tokens), stream)
        check(_lib.get().spectra_paged_tree_attention(*head[:-1], up, batch, n, int(max_new), int(max_tokens), q.data_ptr(),
                                                      _dtype_code(q), q.stride(0), q.stride(1), n_q_heads,
                                                      float(softmax_scale), out.data_ptr(), _dtype_code(out),
                                                      lse.data_ptr() if lse is not None else None, ws.data_ptr(), _bytes(ws),
                                                      s.handle))
    return out


def _keys(cache: PagedCache, ck: Codec, bounds, cu_new, rows, ends):
    """Checks of the calls on boxes -> (batch, pointers of the sequences)."""
    import torch
    dev = cache.table.device
    _need(cu_new.numel() >= 1, "cu_new must have batch + 1 elements")
    batch = cu_new.numel() - 1
    _need(ck.basis.device == dev, f"the codecs must be on {dev}")
    need = int(_lib.get().spectra_paged_bounds_words(cache.ref, ck.n_streams))
    _need(bounds.device == dev and bounds.dtype == torch.int32 and bounds.is_contiguous() and bounds.numel() == need,
          f"bounds must be a contiguous int32 tensor of {need} elements on {dev}")
    return batch, (_ints(rows, "rows", dev, batch), _ints(ends, "ends", dev, batch), _ints(cu_new, "cu_new", dev))


def spectra_paged_bounds(cache: PagedCache, ck: Codec, pool_k, bounds, cu_new, n_new: int, rows=None, ends=None,
                         stream=None) -> None:
    """Boxes (least and largest key coefficients of 64 slots) of the blocks that hold the sequences' new tokens, from
    their records in pool_k. Sequences as in spectra_paged_encode; n_new: tokens of cu_new."""
    batch, seqs = _keys(cache, ck, bounds, cu_new, rows, ends)
    _records(cache, ck, pool_k, "pool_k")
    with _Call(cache.table.device, stream) as s:
        check(_lib.get().spectra_paged_bounds(cache.ref, ctypes.byref(ck.struct), pool_k.data_ptr(), bounds.data_ptr(), *seqs,
                                              batch, int(n_new), s.handle))


def spectra_paged_select_workspace_bytes(n_new: int, n_q_heads: int, n_kv_heads: int, max_tokens: int) -> int:
    return int(_lib.get().spectra_paged_select_workspace_bytes(int(n_new), int(n_q_heads), int(n_kv_heads), int(max_tokens)))


def spectra_paged_select(cache: PagedCache, ck: Codec, bounds, q, cu_new, n_blocks: int, max_tokens: int, first: int = 1,
                         last: int = 1, rows=None, ends=None, out=None, workspace=None, stream=None):
    """The blocks that each new token q [n, n_q_heads, 128] attends over -> int32 [n, n_kv_heads, n_blocks], ascending, -1
    behind the last: its first ``first`` and last ``last`` and those whose boxes bound the largest scores.
    Sequences as in spectra_paged_encode, none with more than max_tokens slots."""
    import torch
    dev = cache.table.device
    batch, seqs = _keys(cache, ck, bounds, cu_new, rows, ends)
    n, n_q_heads = _attended(cache, ck, q, None)
    shape = (n, ck.n_streams, int(n_blocks))
    with _Call(dev, stream) as s:
        out = _made(stream, shape, torch.int32, dev) if out is None else out
        _need(out.device == dev and out.dtype == torch.int32 and out.is_contiguous() and tuple(out.shape) == shape,
              f"out must be a contiguous int32 tensor {shape} on {dev}")
        ws = _workspace(cache, workspace, spectra_paged_select_workspace_bytes(n, n_q_heads, ck.n_streams, max_tokens), stream)
        check(_lib.get().spectra_paged_select(cache.ref, ctypes.byref(ck.struct), bounds.data_ptr(), *seqs, batch, n,
                                              int(max_tokens), q.data_ptr(), _dtype_code(q), q.stride(0), q.stride(1),
                                              n_q_heads, int(n_blocks), int(first), int(last), out.data_ptr(), ws.data_ptr(),
                                              _bytes(ws), s.handle))
    return out


def spectra_paged_sparse_attention_workspace_bytes(n_new: int, n_q_heads: int, n_kv_heads: int, n_blocks: int) -> int:
    return int(_lib.get().spectra_paged_sparse_attention_workspace_bytes(int(n_new), int(n_q_heads), int(n_kv_heads),
                                                                         int(n_blocks)))


def spectra_paged_sparse_attention(cache: PagedCache, ck: Codec, cv: Codec, pool_k, pool_v, q, cu_new, blocks, rows=None,
                                   ends=None, softmax_scale: float = 0.0, out=None, lse=None, workspace=None, stream=None):
    """Causal attention of the new tokens q [n, n_q_heads, 128] over listed blocks of their sequences: ``blocks`` (int32
    [n, n_kv_heads, most]) as spectra_paged_select returns them, 64 slots each. The rest as spectra_paged_attention."""
    import torch
    dev = cache.table.device
    batch, head = _sequences(cache, ck, cv, pool_k, pool_v, cu_new, rows, ends)
    n, n_q_heads = _attended(cache, ck, q, lse)
    _need(blocks.device == dev and blocks.dtype == torch.int32 and blocks.dim() == 3 and blocks.is_contiguous()
          and tuple(blocks.shape[:2]) == (n, ck.n_streams),
          f"blocks must be a contiguous int32 tensor {(n, ck.n_streams, 'most')} on {dev}")
    with _Call(dev, stream) as s:
        out = _output(out, q, stream)
        ws = _workspace(cache, workspace, spectra_paged_sparse_attention_workspace_bytes(n, n_q_heads, ck.n_streams,
                                                                                         blocks.shape[2]), stream)
        check(_lib.get().spectra_paged_sparse_attention(*head, n, blocks.data_ptr(), blocks.shape[2], q.data_ptr(), _dtype_code(q),
                                                        q.stride(0), q.stride(1), n_q_heads, float(softmax_scale),
                                                        out.data_ptr(), _dtype_code(out),
                                                        lse.data_ptr() if lse is not None else None, ws.data_ptr(), _bytes(ws),
                                                        s.handle))
    return out
