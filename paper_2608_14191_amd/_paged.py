"""ctypes binding of include/aatc_paged.h: rotary positions, the paged cache at input precision
and its page tables.

As in ``_lib``: every function has the name of the C entry point it calls, device buffers are
torch tensors, and the kernels run on the current stream (or `stream`).  What the C side cannot
see is checked here: that tensors are on the current device and of the type and size that the
call reads or writes.  Entry points are bound at their first use.
"""
from __future__ import annotations

import ctypes
import struct

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
        self.address = ctypes.addressof(self)


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
        self.address = ctypes.addressof(self)


class PageTable(ctypes.Structure):
    """aatc_page_table of an int32 tensor [rows][max_pages] (rows may be padded), kept alive here.
    The calls below also take the tensor itself."""

    _fields_ = [("table", _vp), ("stride", _i64), ("rows", _i32), ("max_pages", _i32)]

    def __init__(self, table):
        packed, _ = _table("PageTable", table, _on_device("PageTable", table))
        super().__init__(*struct.unpack("=Qqii", packed))
        self.tensor = table


# Marshalling: the shortest kernels take 3 us, so the checks are plain attribute reads, error
# texts are made only when an error is raised, and a page table given as a tensor goes as 24
# packed bytes.
_TORCH = None
_DTYPES = {}
_device = _raw_stream = None
_pack_table = struct.Struct("=Qqii").pack


def _torch():
    global _TORCH, _device, _raw_stream
    if _TORCH is None:
        import torch
        _DTYPES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
        _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
        _TORCH = torch
    return _TORCH


def _dtype(t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        _torch()
        code = _DTYPES.get(t.dtype)
        if code is None:
            raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _on_device(func: str, *tensors) -> int:
    """Tensors (None allowed) must be on the current device, where kernels are launched: its
    index."""
    if not _torch().cuda.is_initialized():
        _TORCH.cuda.init()
    device = _device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            _refuse(func, f"a tensor is on {t.device}, the current device is cuda:{device}")
    return device


def _refuse(func: str, why: str):
    raise AatcError(f"{func} ({why})", E_INVALID)


def _list(func: str, name: str, t, n: int):
    """An int32 tensor that n numbers are read from or written to."""
    if t.dtype != _TORCH.int32 or not t.is_contiguous() or t.numel() < n:
        _refuse(func, f"{name} must be a contiguous int32 tensor of at least {n}")


def _pairs(func: str, pairs) -> int:
    """The number of pairs of an int32 tensor [n][2]."""
    n = len(pairs)
    if n and (pairs.dim() != 2 or pairs.shape[1] != 2):
        _refuse(func, "pairs must be an int32 tensor [n][2]")
    _list(func, "pairs", pairs, 2 * n)
    return n


def _floats(func: str, name: str, t, n: int):
    if t.dtype != _TORCH.float32 or not t.is_contiguous() or t.numel() < n:
        _refuse(func, f"{name} must be a contiguous float32 tensor of at least {n}")


def _tokens(func: str, name: str, t, n_tok: int, stride: int, heads: int):
    """A view whose first element is token 0's: the storage must reach the last token's end."""
    need = (n_tok - 1) * stride + heads * HEAD_DIM
    if n_tok <= 0 or (t.is_contiguous() and t.numel() >= need):
        return
    strides = t.stride()
    if strides == (stride, HEAD_DIM, 1):               # a view [tokens][heads][128]
        shape = t.shape
        if shape[0] >= n_tok and shape[1] >= heads and shape[2] == HEAD_DIM:
            return
    if strides[-1] != 1 or (len(strides) > 2 and t.shape[-2] > 1 and strides[-2] != HEAD_DIM):
        _refuse(func, f"the heads and channels of {name} must be contiguous")
    have = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
    if have < need:
        _refuse(func, f"{name} holds {have} elements from its first on, {need} are used")


def _row_stride(func: str, q, rows: int, heads: int) -> int:
    """Elements between the rows of a tensor that lies packed, or whose first dimension is rows; with
    more heads than are read, each row's first ones."""
    width, packed = heads * HEAD_DIM, q.is_contiguous()
    if rows <= 1 or (packed and q.numel() == rows * width):
        return width
    while packed and q.dim() > 1 and q.shape[0] == 1:
        q = q[0]
    if packed and (q.dim() == 1 or q.stride(0) <= width):      # (rows, or parts of them)
        return width
    if q.shape[0] < rows:
        _refuse(func, f"q has {q.shape[0]} rows of {rows}")
    return q.stride(0)


def _table(func: str, table, device: int):
    """(aatc_page_table as an argument, rows) of a PageTable or an int32 tensor."""
    handle = isinstance(table, PageTable)
    t = table.tensor if handle else table
    if t.get_device() != device:
        _refuse(func, f"the page table is on {t.device}, the current device is cuda:{device}")
    if handle:
        return ctypes.addressof(table), table.rows
    rows, entries = table.shape
    across, along = table.stride()
    if table.dtype != _TORCH.int32 or (entries > 1 and along != 1):
        _refuse(func, "a page table must be an int32 tensor [rows][max_pages], rows contiguous")
    return _pack_table(table.data_ptr(), across if rows > 1 else entries, rows, entries), rows


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
    device = _on_device(f, x, pos, out, rope.tensor)
    if x.dtype != out.dtype:
        _refuse(f, "x and out differ in type")
    _list(f, "pos", pos, n_tok)
    _tokens(f, "x", x, n_tok, x_tok_stride, n_heads)
    _tokens(f, "out", out, n_tok, out_tok_stride, n_heads)
    if n_tok == 0:
        return
    status = entry_point(f)(x.data_ptr(), _dtype(x), n_tok, n_heads, HEAD_DIM, x_tok_stride,
                            pos.data_ptr(), rope.address, 1 if inverse else 0, out.data_ptr(),
                            out_tok_stride, _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


def aatc_paged_append(cache: PagedCache, table, n_tok: int, k, v, k_tok_stride: int,
                      v_tok_stride: int, seq, pos, rope: Rope = None, n_q_heads: int = 0, q=None,
                      q_tok_stride: int = 0, q_out=None, q_out_tok_stride: int = 0, stream=None):
    """Stores n_tok new tokens in the pages of their sequences, keys (and q, into q_out) rotated."""
    f = "aatc_paged_append"
    device = _on_device(f, k, v, seq, pos, q, q_out, cache.tensors[0],
                        None if rope is None else rope.tensor)
    x = k.dtype
    if v.dtype != x:
        _refuse(f, "q, k and v differ in type")
    heads = cache.n_kv_heads
    _list(f, "pos", pos, n_tok)
    if seq is not None:
        _list(f, "seq", seq, n_tok)
    _tokens(f, "k", k, n_tok, k_tok_stride, heads)
    _tokens(f, "v", v, n_tok, v_tok_stride, heads)
    if q is not None:
        if q_out is None or q.dtype != x or q_out.dtype != x:
            _refuse(f, "q, q_out and k differ in type")
        _tokens(f, "q", q, n_tok, q_tok_stride, n_q_heads)
        _tokens(f, "q_out", q_out, n_tok, q_out_tok_stride, n_q_heads)
    t, _ = _table(f, table, device)
    if n_tok == 0:
        return
    status = entry_point(f)(cache.address, t, n_tok, _dtype(k), k.data_ptr(), k_tok_stride,
                            v.data_ptr(), v_tok_stride, _ptr(seq), pos.data_ptr(),
                            None if rope is None else rope.address, n_q_heads, _ptr(q),
                            q_tok_stride, _ptr(q_out), q_out_tok_stride,
                            _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


def aatc_paged_decode_workspace_bytes(batch: int, n_q_heads: int, n_kv_heads: int) -> int:
    return int(entry_point("aatc_paged_decode_workspace_bytes")(batch, n_q_heads, n_kv_heads))


def _space(func: str, workspace) -> int:
    """The bytes of a workspace, for the C side to compare with what the call needs."""
    if not workspace.is_contiguous():
        _refuse(func, "the workspace must be a contiguous tensor")
    return workspace.nbytes


def _buffer(func: str, name: str, t, n: int):
    """A contiguous tensor of any type that holds n bytes."""
    if not t.is_contiguous() or t.nbytes < n:
        _refuse(func, f"{name} must be a contiguous tensor of at least {n} bytes")


def aatc_paged_decode_attention(cache: PagedCache, table, seq_len, batch: int, n_q_heads: int, q,
                                softmax_scale: float, out, workspace, q_stride: int = None,
                                window: int = 0, sink: int = 0, softcap: float = 0.0, slopes=None,
                                lse=None, stream=None):
    """Attention of one token per sequence (q: [batch][n_q_heads][128], rows q_stride elements
    apart, by default as the tensor has them) over the pages; out [batch][n_q_heads][128] and lse
    [batch][n_q_heads] in float32."""
    f = "aatc_paged_decode_attention"
    device = _on_device(f, seq_len, q, out, workspace, slopes, lse, cache.tensors[0])
    _list(f, "seq_len", seq_len, batch)
    _floats(f, "out", out, batch * n_q_heads * HEAD_DIM)
    if lse is not None:
        _floats(f, "lse", lse, batch * n_q_heads)
    if slopes is not None:
        _floats(f, "slopes", slopes, n_q_heads)
    stride = _row_stride(f, q, batch, n_q_heads) if q_stride is None else q_stride
    _tokens(f, "q", q, batch, stride, n_q_heads)
    t, _ = _table(f, table, device)
    status = entry_point(f)(cache.address, t, seq_len.data_ptr(), batch, n_q_heads, q.data_ptr(),
                            _dtype(q), stride, softmax_scale, window, sink, softcap, _ptr(slopes),
                            out.data_ptr(), _ptr(lse), workspace.data_ptr(), _space(f, workspace),
                            _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


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
    device = _on_device(f, dev_params_k, dev_params_v, q, k_codes, k_alpha, v_codes, v_alpha,
                        seq_len, page_len, out, workspace, cache.tensors[0])
    _list(f, "seq_len", seq_len, batch)
    _list(f, "page_len", page_len, batch)
    _floats(f, "out", out, batch * n_q_heads * HEAD_DIM)
    if not q.is_contiguous() or q.numel() < batch * n_q_heads * HEAD_DIM or \
            _row_stride(f, q, batch, n_q_heads) != n_q_heads * HEAD_DIM:
        _refuse(f, "q must be a contiguous tensor [batch][n_q_heads][128]")
    params, tokens = _lib.aatc_params_bytes(n_kv_heads), batch * n_kv_heads * cap
    _buffer(f, "dev_params_k", dev_params_k, params)
    _buffer(f, "dev_params_v", dev_params_v, params)
    _buffer(f, "k_codes", k_codes, tokens * k_record_bytes)
    _buffer(f, "v_codes", v_codes, tokens * v_record_bytes)
    for name, alpha in (("k_alpha", k_alpha), ("v_alpha", v_alpha)):
        if alpha.element_size() != 2:
            _refuse(f, f"{name} must be of a 16-bit type")
        _buffer(f, name, alpha, 2 * tokens)
    t, _ = _table(f, table, device)
    status = entry_point(f)(
        dev_params_k.data_ptr(), dev_params_v.data_ptr(), batch, n_q_heads, n_kv_heads, HEAD_DIM,
        q.data_ptr(), _dtype(q), k_codes.data_ptr(), k_alpha.data_ptr(), v_codes.data_ptr(),
        v_alpha.data_ptr(), seq_len.data_ptr(), cap, k_record_bytes, v_record_bytes, softmax_scale,
        cache.address, t, page_len.data_ptr(), out.data_ptr(), workspace.data_ptr(),
        _space(f, workspace), _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


# Page tables: `table` int32 [rows][max_pages] (or a PageTable), `ref` int32 [n_pages]
# (include/aatc_paged.h).
def aatc_pages_fork(src_table, dst_table, ref, pairs, stream=None):
    """dst_table's rows pairs[:, 1] become copies of src_table's rows pairs[:, 0]."""
    f = "aatc_pages_fork"
    device = _on_device(f, ref, pairs)
    n = _pairs(f, pairs)
    _list(f, "ref", ref, 1)
    src, _ = _table(f, src_table, device)
    dst, _ = _table(f, dst_table, device)
    if n == 0:
        return
    status = entry_point(f)(src, dst, ref.data_ptr(), ref.numel(), pairs.data_ptr(), n,
                            _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


def aatc_pages_free(table, ref, rows, stream=None):
    """Empties the rows listed (int32 tensor)."""
    f = "aatc_pages_free"
    device = _on_device(f, ref, rows)
    n = rows.numel()
    _list(f, "rows", rows, n)
    _list(f, "ref", ref, 1)
    t, _ = _table(f, table, device)
    if n == 0:
        return
    status = entry_point(f)(t, ref.data_ptr(), ref.numel(), rows.data_ptr(), n,
                            _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


def aatc_pages_workspace_bytes(rows: int, n_pages: int) -> int:
    return int(entry_point("aatc_pages_workspace_bytes")(rows, n_pages))


def aatc_pages_reserve(table, ref, page_tokens: int, held, wanted, pairs, lacking, workspace,
                       stream=None):
    """Pages for the tokens held[b] .. wanted[b] - 1 of every row; pairs [rows][2] to copy,
    lacking [1]."""
    f = "aatc_pages_reserve"
    device = _on_device(f, ref, held, wanted, pairs, lacking, workspace)
    t, rows = _table(f, table, device)
    _list(f, "held", held, rows)
    _list(f, "wanted", wanted, rows)
    _list(f, "ref", ref, 1)
    _list(f, "lacking", lacking, 1)
    _list(f, "pairs", pairs, 2 * rows)
    status = entry_point(f)(t, ref.data_ptr(), ref.numel(), page_tokens, held.data_ptr(),
                            wanted.data_ptr(), pairs.data_ptr(), lacking.data_ptr(),
                            workspace.data_ptr(), _space(f, workspace),
                            _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


def aatc_pages_compact(table, ref, table_out, ref_out, pairs, moves, workspace, stream=None):
    """The table and counts with the pages in use moved to the front, and the moves
    (pairs [n_pages / 2][2], moves [1]) for aatc_pages_copy."""
    f = "aatc_pages_compact"
    device = _on_device(f, ref, ref_out, pairs, moves, workspace)
    n_pages = ref.numel()
    _list(f, "ref", ref, 1)
    _list(f, "ref_out", ref_out, n_pages)
    _list(f, "moves", moves, 1)
    _list(f, "pairs", pairs, n_pages // 2 * 2)
    t, _ = _table(f, table, device)
    o, _ = _table(f, table_out, device)
    status = entry_point(f)(t, ref.data_ptr(), n_pages, o, ref_out.data_ptr(), pairs.data_ptr(),
                            moves.data_ptr(), workspace.data_ptr(), _space(f, workspace),
                            _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)


def aatc_pages_copy(pools, pairs, n_pairs=None, stream=None):
    """Copies page pairs[i][0] to pairs[i][1] in every pool of `pools` ([pool][page][...], pages
    contiguous); n_pairs: int32 tensor [1], copy no more pairs than that."""
    f = "aatc_pages_copy"
    device = _on_device(f, pools, pairs, n_pairs)
    n = _pairs(f, pairs)
    if n_pairs is not None:
        _list(f, "n_pairs", n_pairs, 1)
    if pools.dim() < 3 or not (pools.is_contiguous() or pools[0].is_contiguous()):
        _refuse(f, "pools must be [pool][page][...] with contiguous pages, one behind the other")
    n_pools, n_pages = pools.shape[:2]
    if n == 0 or pools.numel() == 0:
        return
    size = pools.element_size()
    page_bytes = pools.numel() // (n_pools * n_pages) * size
    stride = pools.stride(0) * size if n_pools > 1 else n_pages * page_bytes
    status = entry_point(f)(pools.data_ptr(), n_pools, stride, n_pages, page_bytes,
                            pairs.data_ptr(), n, _ptr(n_pairs),
                            _raw_stream(device) if stream is None else int(stream))
    if status:
        raise AatcError(f, status)
