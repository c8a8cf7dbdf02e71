"""ctypes binding of include/aatc_sparse.h: bounds of the pages' keys, and attention over the pages
that can score most.

As in ``_paged``: device buffers are torch tensors on the current device, the kernels run on the
current stream (or `stream`), and what the C side cannot see is checked here.
"""
from __future__ import annotations

import ctypes

from . import _lib, _paged
from ._lib import HEAD_DIM, AatcError
from ._paged import (PagedCache, _dtype, _floats, _list, _on_device, _ptr, _refuse, _row_stride, _space,
                     _table, _tokens)

_vp, _i32, _i64, _sz, _f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                              ctypes.c_float)
_int = ctypes.c_int

_SIGNATURES = {
    "aatc_page_bounds": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "aatc_paged_sparse_workspace_bytes": (_sz, [_i32, _i32, _i32, _i64]),
    "aatc_paged_sparse_attention": (_int, [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _int, _i64, _f32,
                                           _i32, _i32, _i32, _f32, _vp, _vp, _vp, _vp, _sz, _vp]),
}
_bound = {}


def entry_point(name: str):
    """The C function `name` of the library, with its argument types."""
    f = _bound.get(name)
    if f is None:
        f = getattr(_lib.library(), name)
        f.restype, f.argtypes = _SIGNATURES[name]
        _bound[name] = f
    return f


def _bounds(func: str, cache: PagedCache, codes, scales):
    """codes int8 [n_pages][n_kv_heads][2][128], scales float32 [n_pages][n_kv_heads]."""
    pairs = cache.n_pages * cache.n_kv_heads
    if codes.dtype != _paged._TORCH.int8 or not codes.is_contiguous() or \
            codes.numel() < pairs * 2 * HEAD_DIM:
        _refuse(func, "codes must be a contiguous int8 tensor [n_pages][n_kv_heads][2][128]")
    _floats(func, "scales", scales, pairs)


def aatc_page_bounds(cache: PagedCache, table, held, wanted, codes, scales, stream=None):
    """Bounds of the pages that the tokens held[b] .. wanted[b] - 1 (int32; held None: from 0) of
    every row of the table fall into."""
    f = "aatc_page_bounds"
    device = _on_device(f, held, wanted, codes, scales, cache.tensors[0])
    t, rows = _table(f, table, device)
    if held is not None:
        _list(f, "held", held, rows)
    _list(f, "wanted", wanted, rows)
    _bounds(f, cache, codes, scales)
    status = entry_point(f)(cache.address, t, _ptr(held), wanted.data_ptr(), codes.data_ptr(),
                            scales.data_ptr(),
                            _paged._raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


def aatc_paged_sparse_workspace_bytes(batch: int, n_q_heads: int, n_kv_heads: int,
                                      max_pages: int) -> int:
    return int(entry_point("aatc_paged_sparse_workspace_bytes")(batch, n_q_heads, n_kv_heads,
                                                                max_pages))


def aatc_paged_sparse_attention(cache: PagedCache, table, seq_len, codes, scales, batch: int,
                                n_q_heads: int, q, softmax_scale: float, picked, out, workspace,
                                first: int = 1, last: int = 1, softcap: float = 0.0, lse=None,
                                q_stride: int = None, stream=None):
    """Attention of one token per sequence (q as in aatc_paged_decode_attention) over the pages that
    each KV head picks by their bounds: picked int32 [batch][n_kv_heads][most], most pages at most,
    among them the first `first` and the last `last`."""
    f = "aatc_paged_sparse_attention"
    device = _on_device(f, seq_len, codes, scales, q, picked, out, workspace, lse, cache.tensors[0])
    _list(f, "seq_len", seq_len, batch)
    _bounds(f, cache, codes, scales)
    if picked.dim() != 3 or picked.shape[0] < batch or picked.shape[1] != cache.n_kv_heads:
        _refuse(f, "picked must be an int32 tensor [batch][n_kv_heads][most]")
    most = picked.shape[2]
    _list(f, "picked", picked, batch * cache.n_kv_heads * most)
    _floats(f, "out", out, batch * n_q_heads * HEAD_DIM)
    if lse is not None:
        _floats(f, "lse", lse, batch * n_q_heads)
    stride = _row_stride(f, q, batch, n_q_heads) if q_stride is None else q_stride
    _tokens(f, "q", q, batch, stride, n_q_heads)
    t, _ = _table(f, table, device)
    status = entry_point(f)(cache.address, t, seq_len.data_ptr(), codes.data_ptr(), scales.data_ptr(),
                            batch, n_q_heads, q.data_ptr(), _dtype(q), stride, softmax_scale, most,
                            first, last, softcap, picked.data_ptr(), out.data_ptr(), _ptr(lse),
                            workspace.data_ptr(), _space(f, workspace),
                            _paged._raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)
