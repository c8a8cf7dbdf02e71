"""ctypes binding of include/aatc_paged.h: rotary positions, the paged cache at input precision
and its page tables.

As in ``_lib``: every function has the name of the C entry point it calls, device buffers are
torch tensors, and the kernels run on the current stream (or `stream`).  What the C side cannot
see is checked here: that tensors are on the current device and of the type and size that the
call reads or writes.  Entry points are bound at their first use.
"""
from __future__ import annotations

import ctypes

import numpy as np

from . import _lib
from ._lib import BF16, E_INVALID, F16, F32, HEAD_DIM, AatcError, _check

ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_NTK, ROPE_BANDS, ROPE_YARN = range(5)

_vp, _i32, _i64, _sz, _f32, _f64 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                    ctypes.c_size_t, ctypes.c_float, ctypes.c_double)
_int = ctypes.c_int


class Rope(ctypes.Structure):
    """aatc_rope_spec.  freq: float64 tensor [rot_dim / 2] on the device, kept alive here."""

    _fields_ = [("freq", _vp), ("rot_dim", _i32), ("layout", _i32), ("factor", _f32)]

    def __init__(self, freq, layout: int = ROPE_HALF, factor: float = 1.0):
        import torch
        if freq.dtype != torch.float64 or freq.dim() != 1 or not freq.is_contiguous():
            raise TypeError("freq must be a contiguous float64 tensor [rot_dim / 2]")
        _on_device("Rope", freq)
        super().__init__(freq.data_ptr(), 2 * freq.numel(), int(layout), float(factor))
        self.tensor = freq


class PagedCache(ctypes.Structure):
    """aatc_paged_cache of two tensors seen as [page][KV head][token][128], in any order in
    memory (token-major pages: a transposed view); the tensors are kept alive here."""

    _fields_ = [("k_pages", _vp), ("v_pages", _vp), ("dtype", _i32), ("n_kv_heads", _i32),
                ("d", _i32), ("page_tokens", _i32), ("n_pages", _i64), ("page_stride", _i64),
                ("head_stride", _i64), ("tok_stride", _i64)]

    def __init__(self, k_pages, v_pages):
        if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype:
            raise ValueError("k_pages and v_pages must be [page][KV head][token][128], alike")
        if k_pages.stride() != v_pages.stride() or k_pages.stride(3) != 1:
            raise ValueError("k_pages and v_pages must be laid out alike, channels contiguous")
        _on_device("PagedCache", k_pages, v_pages)
        n_pages, heads, tokens, d = k_pages.shape
        # (a stride of a dimension of one has no meaning: the smallest that is allowed)
        page, head, tok = (s if n > 1 else HEAD_DIM for s, n in zip(k_pages.stride(), k_pages.shape[:3]))
        super().__init__(k_pages.data_ptr(), v_pages.data_ptr(), _dtype(k_pages), heads, d, tokens,
                         n_pages, page, head, tok)
        self.tensors = (k_pages, v_pages)


class PageTable(ctypes.Structure):
    """aatc_page_table of an int32 tensor [rows][max_pages] (rows may be padded)."""

    _fields_ = [("table", _vp), ("stride", _i64), ("rows", _i32), ("max_pages", _i32)]

    def __init__(self, table):
        rows, entries = table.shape
        if table.dtype != _torch().int32 or (entries > 1 and table.stride(1) != 1):
            raise TypeError("a page table must be an int32 tensor [rows][max_pages], rows contiguous")
        _on_device("PageTable", table)
        super().__init__(table.data_ptr(), table.stride(0) if rows > 1 else entries, rows, entries)


_TORCH = None
_DTYPES = {}


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
        _DTYPES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    return _TORCH


def _dtype(t) -> int:
    _torch()
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _on_device(func: str, *tensors):
    """Tensors (None allowed) must be on the current device: kernels are launched there."""
    device = _torch().cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise AatcError(f"{func} (a tensor is on {t.device}, the current device is cuda:{device})",
                            E_INVALID)


def _want(func: str, what: str, ok: bool):
    if not ok:
        raise AatcError(f"{func} ({what})", E_INVALID)


def _list(func: str, name: str, t, n: int):
    """An int32 tensor that n numbers are read from or written to."""
    _want(func, f"{name} must be a contiguous int32 tensor of at least {n}",
          t.dtype == _TORCH.int32 and t.is_contiguous() and t.numel() >= n)


def _tokens(func: str, name: str, t, n_tok: int, stride: int, heads: int):
    """A view whose first element is token 0's: the storage must reach the last token's end."""
    need = (n_tok - 1) * stride + heads * HEAD_DIM if n_tok > 0 else 0
    have = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
    _want(func, f"{name} holds {have} elements from its first on, {need} are used", have >= need)


_SIGNATURES = {
    "aatc_rope_frequencies": (_int, [_i32, _f64, _int, _f64, _i64, _f64, _f64, _vp, _vp]),
    "aatc_rope": (_int, [_vp, _int, _i64, _i32, _i32, _i64, _vp, _vp, _i32, _vp, _i64, _vp]),
    "aatc_paged_append": (_int, [_vp, _vp, _i64, _int, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _i32,
                                 _vp, _i64, _vp, _i64, _vp]),
    "aatc_paged_decode_workspace_bytes": (_sz, [_i32, _i32, _i32]),
    "aatc_paged_decode_attention": (_int, [_vp, _vp, _vp, _i32, _i32, _vp, _int, _i64, _f32, _i32,
                                           _i32, _f32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "aatc_decode_paged_workspace_bytes": (_sz, [_i32, _i32, _i32, _i64]),
    "aatc_decode_attention_paged": (_int, [_vp, _vp, _i32, _i32, _i32, _i32, _vp, _int, _vp, _vp,
                                           _vp, _vp, _vp, _i64, _i32, _i32, _f32, _vp, _vp, _vp,
                                           _vp, _vp, _sz, _vp]),
    "aatc_pages_fork": (_int, [_vp, _vp, _vp, _i64, _vp, _i64, _vp]),
    "aatc_pages_free": (_int, [_vp, _vp, _i64, _vp, _i64, _vp]),
    "aatc_pages_workspace_bytes": (_sz, [_i64, _i64]),
    "aatc_pages_reserve": (_int, [_vp, _vp, _i64, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "aatc_pages_compact": (_int, [_vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "aatc_pages_copy": (_int, [_vp, _i64, _i64, _i64, _i64, _vp, _i64, _vp, _vp]),
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


def _ptr(t):
    return None if t is None else t.data_ptr()


def aatc_rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: int = ROPE_PLAIN,
                          scale: float = 1.0, trained: int = 1, low: float = 1.0,
                          high: float = 4.0):
    """(angles per position [rot_dim / 2] as a float64 numpy array, factor); host only."""
    freq = np.zeros(max(1, int(rot_dim) // 2), dtype=np.float64)
    factor = _f32()
    if int(rot_dim) > HEAD_DIM:                       # (the C side refuses it before writing)
        raise AatcError("aatc_rope_frequencies", E_INVALID)
    _check("aatc_rope_frequencies",
           entry_point("aatc_rope_frequencies")(int(rot_dim), float(base), int(scaling),
                                                float(scale), int(trained), float(low),
                                                float(high), freq.ctypes.data,
                                                ctypes.addressof(factor)))
    return freq, float(factor.value)


def aatc_rope(x, n_tok: int, n_heads: int, x_tok_stride: int, pos, rope: Rope, out,
              out_tok_stride: int, inverse: bool = False, stream=None):
    """Rotates n_tok tokens of x ([n_heads][128] at every x_tok_stride elements) into out."""
    f = "aatc_rope"
    _on_device(f, x, pos, out, rope.tensor)
    _want(f, "x and out differ in type", x.dtype == out.dtype)
    _list(f, "pos", pos, n_tok)
    _tokens(f, "x", x, n_tok, x_tok_stride, n_heads)
    _tokens(f, "out", out, n_tok, out_tok_stride, n_heads)
    _check(f, entry_point(f)(_ptr(x), _dtype(x), n_tok, n_heads, HEAD_DIM, x_tok_stride, _ptr(pos),
                             ctypes.addressof(rope), 1 if inverse else 0, _ptr(out),
                             out_tok_stride, _lib._stream(stream)))


def aatc_paged_append(cache: PagedCache, table, n_tok: int, k, v, k_tok_stride: int,
                      v_tok_stride: int, seq, pos, rope: Rope = None, n_q_heads: int = 0, q=None,
                      q_tok_stride: int = 0, q_out=None, q_out_tok_stride: int = 0, stream=None):
    """Stores n_tok new tokens in the pages of their sequences, keys (and q, into q_out) rotated."""
    f = "aatc_paged_append"
    _on_device(f, k, v, seq, pos, q, q_out, cache.tensors[0], rope.tensor if rope else None)
    _want(f, "q, k and v differ in type", k.dtype == v.dtype and
          (q is None or (q.dtype == k.dtype and q_out is not None and q_out.dtype == k.dtype)))
    _list(f, "pos", pos, n_tok)
    if seq is not None:
        _list(f, "seq", seq, n_tok)
    _tokens(f, "k", k, n_tok, k_tok_stride, cache.n_kv_heads)
    _tokens(f, "v", v, n_tok, v_tok_stride, cache.n_kv_heads)
    if q is not None:
        _tokens(f, "q", q, n_tok, q_tok_stride, n_q_heads)
        _tokens(f, "q_out", q_out, n_tok, q_out_tok_stride, n_q_heads)
    t = PageTable(table)
    _check(f, entry_point(f)(ctypes.addressof(cache), ctypes.addressof(t), n_tok, _dtype(k),
                             _ptr(k), k_tok_stride, _ptr(v), v_tok_stride, _ptr(seq), _ptr(pos),
                             ctypes.addressof(rope) if rope else None, n_q_heads, _ptr(q),
                             q_tok_stride, _ptr(q_out), q_out_tok_stride, _lib._stream(stream)))


def aatc_paged_decode_workspace_bytes(batch: int, n_q_heads: int, n_kv_heads: int) -> int:
    return int(entry_point("aatc_paged_decode_workspace_bytes")(batch, n_q_heads, n_kv_heads))


def _bytes(workspace) -> int:
    return workspace.numel() * workspace.element_size()


def aatc_paged_decode_attention(cache: PagedCache, table, seq_len, batch: int, n_q_heads: int, q,
                                softmax_scale: float, out, workspace, q_stride: int = None,
                                window: int = 0, sink: int = 0, softcap: float = 0.0, slopes=None,
                                lse=None, stream=None):
    """Attention of one token per sequence (q: [batch][n_q_heads][128], rows q_stride elements
    apart) over the pages; out [batch][n_q_heads][128] and lse [batch][n_q_heads] in float32."""
    f = "aatc_paged_decode_attention"
    _on_device(f, seq_len, q, out, workspace, slopes, lse, cache.tensors[0])
    fp32 = _TORCH.float32
    _list(f, "seq_len", seq_len, batch)
    _want(f, "out must be a contiguous float32 tensor [batch][n_q_heads][128]",
          out.dtype == fp32 and out.is_contiguous() and out.numel() >= batch * n_q_heads * HEAD_DIM)
    for name, t, n in (("lse", lse, batch * n_q_heads), ("slopes", slopes, n_q_heads)):
        if t is not None:
            _want(f, f"{name} must be a contiguous float32 tensor of at least {n}",
                  t.dtype == fp32 and t.is_contiguous() and t.numel() >= n)
    stride = n_q_heads * HEAD_DIM if q_stride is None else q_stride
    _tokens(f, "q", q, batch, stride, n_q_heads)
    t = PageTable(table)
    _check(f, entry_point(f)(ctypes.addressof(cache), ctypes.addressof(t), _ptr(seq_len), batch,
                             n_q_heads, _ptr(q), _dtype(q), stride, softmax_scale, window, sink,
                             softcap, _ptr(slopes), _ptr(out), _ptr(lse), _ptr(workspace),
                             _bytes(workspace), _lib._stream(stream)))


def aatc_decode_paged_workspace_bytes(batch: int, n_q_heads: int, n_kv_heads: int,
                                      cap: int) -> int:
    return int(entry_point("aatc_decode_paged_workspace_bytes")(batch, n_q_heads, n_kv_heads, cap))


def aatc_decode_attention_paged(dev_params_k, dev_params_v, batch: int, n_q_heads: int,
                                n_kv_heads: int, q, k_codes, k_alpha, v_codes, v_alpha, seq_len,
                                cap: int, k_record_bytes: int, v_record_bytes: int,
                                softmax_scale: float, cache: PagedCache, table, page_len, out,
                                workspace, stream=None):
    """Decode attention over the compressed caches plus the page_len tokens of the pages."""
    f = "aatc_decode_attention_paged"
    _on_device(f, dev_params_k, dev_params_v, q, k_codes, k_alpha, v_codes, v_alpha, seq_len,
               page_len, out, workspace, cache.tensors[0])
    _list(f, "seq_len", seq_len, batch)
    _list(f, "page_len", page_len, batch)
    _want(f, "out must be a contiguous float32 tensor [batch][n_q_heads][128]",
          out.dtype == _TORCH.float32 and out.is_contiguous() and
          out.numel() >= batch * n_q_heads * HEAD_DIM)
    _tokens(f, "q", q, batch, n_q_heads * HEAD_DIM, n_q_heads)
    t = PageTable(table)
    _check(f, entry_point(f)(
        _ptr(dev_params_k), _ptr(dev_params_v), batch, n_q_heads, n_kv_heads, HEAD_DIM, _ptr(q),
        _dtype(q), _ptr(k_codes), _ptr(k_alpha), _ptr(v_codes), _ptr(v_alpha), _ptr(seq_len), cap,
        k_record_bytes, v_record_bytes, softmax_scale, ctypes.addressof(cache),
        ctypes.addressof(t), _ptr(page_len), _ptr(out), _ptr(workspace), _bytes(workspace),
        _lib._stream(stream)))


# Page tables: `table` int32 [rows][max_pages], `ref` int32 [n_pages] (include/aatc_paged.h).
def _pairs(func: str, name: str, t, n: int):
    _want(func, f"{name} must be a contiguous int32 tensor [{n}][2]",
          t.dtype == _TORCH.int32 and t.is_contiguous() and t.numel() >= 2 * n)


def aatc_pages_fork(src_table, dst_table, ref, pairs, stream=None):
    """dst_table's rows pairs[:, 1] become copies of src_table's rows pairs[:, 0]."""
    f = "aatc_pages_fork"
    _on_device(f, ref, pairs)
    n = pairs.shape[0]
    _pairs(f, "pairs", pairs, n)
    _list(f, "ref", ref, 1)
    src, dst = PageTable(src_table), PageTable(dst_table)
    _check(f, entry_point(f)(ctypes.addressof(src), ctypes.addressof(dst), _ptr(ref), ref.numel(),
                             _ptr(pairs) or None, n, _lib._stream(stream)) if n else 0)


def aatc_pages_free(table, ref, rows, stream=None):
    """Empties the rows listed (int32 tensor)."""
    f = "aatc_pages_free"
    _on_device(f, ref, rows)
    n = rows.numel()
    _list(f, "rows", rows, n)
    _list(f, "ref", ref, 1)
    t = PageTable(table)
    _check(f, entry_point(f)(ctypes.addressof(t), _ptr(ref), ref.numel(), _ptr(rows), n,
                             _lib._stream(stream)) if n else 0)


def aatc_pages_workspace_bytes(rows: int, n_pages: int) -> int:
    return int(entry_point("aatc_pages_workspace_bytes")(rows, n_pages))


def aatc_pages_reserve(table, ref, page_tokens: int, held, wanted, pairs, lacking, workspace,
                       stream=None):
    """Pages for the tokens held[b] .. wanted[b] - 1 of every row; pairs [rows][2] to copy,
    lacking [1]."""
    f = "aatc_pages_reserve"
    _on_device(f, ref, held, wanted, pairs, lacking, workspace)
    rows = table.shape[0]
    for name, t in (("held", held), ("wanted", wanted)):
        _list(f, name, t, rows)
    _list(f, "ref", ref, 1)
    _list(f, "lacking", lacking, 1)
    _pairs(f, "pairs", pairs, rows)
    t = PageTable(table)
    _check(f, entry_point(f)(ctypes.addressof(t), _ptr(ref), ref.numel(), page_tokens, _ptr(held),
                             _ptr(wanted), _ptr(pairs), _ptr(lacking), _ptr(workspace),
                             _bytes(workspace), _lib._stream(stream)))


def aatc_pages_compact(table, ref, table_out, ref_out, pairs, moves, workspace, stream=None):
    """The table and counts with the pages in use moved to the front, and the moves
    (pairs [n_pages / 2][2], moves [1]) for aatc_pages_copy."""
    f = "aatc_pages_compact"
    _on_device(f, ref, ref_out, pairs, moves, workspace)
    n_pages = ref.numel()
    _list(f, "ref", ref, 1)
    _list(f, "ref_out", ref_out, n_pages)
    _list(f, "moves", moves, 1)
    _pairs(f, "pairs", pairs, n_pages // 2)
    t, o = PageTable(table), PageTable(table_out)
    _check(f, entry_point(f)(ctypes.addressof(t), _ptr(ref), n_pages, ctypes.addressof(o),
                             _ptr(ref_out), _ptr(pairs), _ptr(moves), _ptr(workspace),
                             _bytes(workspace), _lib._stream(stream)))


def aatc_pages_copy(pools, pairs, n_pairs=None, stream=None):
    """Copies page pairs[i][0] to pairs[i][1] in every pool of `pools` ([pool][page][...], pages
    contiguous); n_pairs: int32 tensor [1], copy no more pairs than that."""
    f = "aatc_pages_copy"
    _on_device(f, pools, pairs, n_pairs)
    n = pairs.shape[0]
    _pairs(f, "pairs", pairs, n)
    if n_pairs is not None:
        _list(f, "n_pairs", n_pairs, 1)
    _want(f, "pools must be [pool][page][...] with contiguous pages, one behind the other",
          pools.dim() >= 3 and pools[0].is_contiguous())
    page_bytes = pools[0, 0].numel() * pools.element_size()
    n_pools, n_pages = pools.shape[:2]
    stride = pools.stride(0) * pools.element_size() if n_pools > 1 else n_pages * page_bytes
    _check(f, entry_point(f)(_ptr(pools), n_pools, stride, n_pages, page_bytes, _ptr(pairs), n,
                             _ptr(n_pairs), _lib._stream(stream)) if n else 0)
