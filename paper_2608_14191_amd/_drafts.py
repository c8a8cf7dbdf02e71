"""ctypes binding of include/aatc_drafts.h: attention of drafted tokens over the paged cache, and the
acceptance of a path of them.

As in ``_paged``: device buffers are torch tensors on the current device, the kernels run on the
current stream (or `stream`), and what the C side cannot see is checked here.
"""
from __future__ import annotations

import ctypes

from . import _lib, _paged
from ._lib import HEAD_DIM, AatcError
from ._paged import (PagedCache, _dtype, _floats, _list, _on_device, _ptr, _refuse, _space, _table,
                     _tokens)

MAX_DRAFTS = 64

_vp, _i32, _i64, _sz, _f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                              ctypes.c_float)
_int = ctypes.c_int

_SIGNATURES = {
    "aatc_paged_tree_workspace_bytes": (_sz, [_i32, _i32, _i32, _i32]),
    "aatc_paged_tree_attention": (_int, [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _vp, _int, _i64,
                                         _f32, _i32, _i32, _f32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "aatc_paged_tree_accept": (_int, [_vp, _i32, _i64, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp,
                                      _vp, _vp, _vp, _vp]),
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


def aatc_paged_tree_workspace_bytes(batch: int, max_draft: int, n_q_heads: int,
                                    n_kv_heads: int) -> int:
    return int(entry_point("aatc_paged_tree_workspace_bytes")(batch, max_draft, n_q_heads,
                                                              n_kv_heads))


def _trees(func: str, seq_len, n_draft, parent, batch: int, max_draft: int):
    _list(func, "seq_len", seq_len, batch)
    if n_draft is not None:
        _list(func, "n_draft", n_draft, batch)
    if parent is not None:
        _list(func, "parent", parent, batch * max_draft)


def _draft_stride(func: str, q, batch: int, max_draft: int, heads: int) -> int:
    """Elements between the drafts of a tensor that lies packed, or whose first dimension is tokens,
    [tokens][heads][128], or its first two are sequences and drafts, [batch][max_draft][...]; with
    more heads than are read, each draft's first ones."""
    n, width, packed = batch * max_draft, heads * HEAD_DIM, q.is_contiguous()
    if n <= 1 or (packed and q.numel() == n * width):
        return width
    while q.dim() > 1 and q.shape[0] == 1:
        q = q[0]
    shape, dim = q.shape, q.dim()
    if packed and (dim == 1 or q.stride(0) <= width):          # (tokens, or parts of them)
        return width
    two = dim > 3 or (packed and dim == 3 and not (shape[2] == HEAD_DIM and shape[0] >= n))
    if not two or max_draft == 1:
        if shape[0] < n:
            _refuse(func, f"q has {shape[0]} tokens of {n}")
        return q.stride(0)
    if shape[0] < batch or shape[1] != max_draft or \
            (batch > 1 and q.stride(0) != max_draft * q.stride(1)):
        _refuse(func, f"q's {batch} x {max_draft} drafts do not lie at equal steps")
    return q.stride(1)


def aatc_paged_tree_attention(cache: PagedCache, table, seq_len, batch: int, max_draft: int,
                              n_q_heads: int, q, softmax_scale: float, out, workspace,
                              q_tok_stride: int = None, n_draft=None, parent=None, window: int = 0,
                              sink: int = 0, softcap: float = 0.0, slopes=None, lse=None,
                              stream=None):
    """Attention of max_draft drafted tokens per sequence (q: batch * max_draft tokens of
    [n_q_heads][128], q_tok_stride elements apart, by default as the tensor has them:
    [tokens][n_q_heads][128], or [batch][max_draft][n_q_heads][128])
    over the pages; parent int32 [batch][max_draft] or None (a chain); out
    [batch][max_draft][n_q_heads][128] and lse [batch][max_draft][n_q_heads] in float32."""
    f = "aatc_paged_tree_attention"
    device = _on_device(f, seq_len, n_draft, parent, q, out, workspace, slopes, lse,
                        cache.tensors[0])
    n = batch * max_draft
    _trees(f, seq_len, n_draft, parent, batch, max_draft)
    _floats(f, "out", out, n * n_q_heads * HEAD_DIM)
    if lse is not None:
        _floats(f, "lse", lse, n * n_q_heads)
    if slopes is not None:
        _floats(f, "slopes", slopes, n_q_heads)
    stride = _draft_stride(f, q, batch, max_draft, n_q_heads) if q_tok_stride is None else q_tok_stride
    _tokens(f, "q", q, n, stride, n_q_heads)
    t, _ = _table(f, table, device)
    status = entry_point(f)(cache.address, t, seq_len.data_ptr(), _ptr(n_draft), _ptr(parent), batch,
                            max_draft, n_q_heads, q.data_ptr(), _dtype(q), stride, softmax_scale,
                            window, sink, softcap, _ptr(slopes), out.data_ptr(), _ptr(lse),
                            workspace.data_ptr(), _space(f, workspace),
                            _paged._raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


def aatc_paged_tree_accept(cache: PagedCache, table, seq_len, batch: int, max_draft: int, drafted,
                           chosen, path, accepted, next, len_out, n_draft=None, parent=None,
                           n_layers: int = 1, layer_stride: int = 0, stream=None):
    """Walks each sequence's tree along the tokens chosen: path [batch][max_draft], accepted, next
    and len_out [batch] (int32), and moves the accepted tokens up in every layer: `cache` is the
    first layer's, of tensors whose storage has the others layer_stride elements behind."""
    f = "aatc_paged_tree_accept"
    device = _on_device(f, seq_len, n_draft, parent, drafted, chosen, path, accepted, next, len_out,
                        cache.tensors[0])
    _trees(f, seq_len, n_draft, parent, batch, max_draft)
    for name, t in (("drafted", drafted), ("chosen", chosen), ("path", path)):
        _list(f, name, t, batch * max_draft)
    for name, t in (("accepted", accepted), ("next", next), ("len_out", len_out)):
        _list(f, name, t, batch)
    if n_layers > 1:
        pages = cache.tensors[0]
        first = sum((s - 1) * d for s, d in zip(pages.shape, pages.stride())) + 1   # layer 0's elements
        for name, t in zip(("k_pages", "v_pages"), cache.tensors):
            have = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
            if layer_stride <= 0 or have < (n_layers - 1) * layer_stride + first:
                _refuse(f, f"{name} holds no {n_layers} layers, {layer_stride} elements apart")
    t, _ = _table(f, table, device)
    status = entry_point(f)(cache.address, n_layers, layer_stride, t, seq_len.data_ptr(),
                            _ptr(n_draft), _ptr(parent), batch, max_draft, drafted.data_ptr(),
                            chosen.data_ptr(), path.data_ptr(), accepted.data_ptr(), next.data_ptr(),
                            len_out.data_ptr(),
                            _paged._raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)
