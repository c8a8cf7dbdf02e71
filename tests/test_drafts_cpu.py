"""The host side of drafted tokens and of sparse attention without a GPU: exports, and every refusal of
the C ABI (before anything is launched)."""
import ctypes
import os

import paper_2608_14191_amd as P
from paper_2608_14191_amd import _drafts, _sparse
from paper_2608_14191_amd._lib import exported_symbols_declared_in_header
from test_paged_cpu import (A, BAD_CACHES, BAD_TABLES, CACHE, INVALID, ODD, ROOT, TABLE, UNSUPPORTED,
                            WORKSPACE, _fill)

NAN, INF = float("nan"), float("inf")
FAR = 1 << 30                                         # (past every list that begins at A)


def test_exports_and_signatures():
    for header, module in (("aatc_drafts.h", _drafts), ("aatc_sparse.h", _sparse)):
        names = exported_symbols_declared_in_header(os.path.join(ROOT, "include", header))
        assert set(names) == set(module._SIGNATURES)
        for n in names:
            assert hasattr(P.library(), n) and hasattr(P, n), n
    assert P.MAX_DRAFTS == 64


def _call(module, name, args, **change):
    a = dict(args)
    for k, v in change.items():
        assert k in a, k
        a[k] = v
    keep = [_fill(v[0], **v[1]) if isinstance(v, tuple) else v for v in a.values()]
    return module.entry_point(name)(*(ctypes.addressof(v) if isinstance(v, ctypes.Structure) else v
                                      for v in keep))


def _refused(module, name, args, refusals):
    for bad, status in BAD_CACHES:
        assert _call(module, name, args, cache=(P.PagedCache, {**CACHE, **bad})) == status, bad
    for bad, status in BAD_TABLES:
        assert _call(module, name, args, table=(P.PageTable, {**TABLE, **bad})) == status, bad
    for status, change in [(INVALID, dict(cache=None)), (INVALID, dict(table=None)), *refusals]:
        assert _call(module, name, args, **change) == status, change


TREES = [(INVALID, dict(batch=0)), (INVALID, dict(batch=5)), (INVALID, dict(drafts=0)),
         (INVALID, dict(drafts=-1)), (UNSUPPORTED, dict(drafts=65)), (INVALID, dict(len=None)),
         (INVALID, dict(len=A + 2)), (INVALID, dict(counts=A + 1)), (INVALID, dict(parent=A + 2))]

QUERIES = [(INVALID, dict(hq=0)), (INVALID, dict(hq=30)), (INVALID, dict(hq=-8)), (INVALID, dict(q=None)),
           (INVALID, dict(q=ODD)), (INVALID, dict(qd=7)), (INVALID, dict(qd=0, q=A + 2)),
           (INVALID, dict(qs=4095)), (INVALID, dict(qs=1 << 41)), (INVALID, dict(scale=NAN)),
           (INVALID, dict(scale=INF)), (INVALID, dict(cap=-1.0)), (INVALID, dict(cap=NAN)),
           (INVALID, dict(cap=INF)), (INVALID, dict(cap=1e-40)), (INVALID, dict(out=None)),
           (INVALID, dict(out=A + 4)), (INVALID, dict(lse=A + 1)), (INVALID, dict(ws=None)),
           (INVALID, dict(ws=A + 16))]

MANY = dict(table=(P.PageTable, {**TABLE, "max_pages": 1 << 24, "stride": 1 << 24}),
            cache=(P.PagedCache, {**CACHE, "page_tokens": 128}))


def test_tree_attention_refusals():
    name = "aatc_paged_tree_attention"
    args = dict(cache=(P.PagedCache, CACHE), table=(P.PageTable, TABLE), len=A, counts=None, parent=None,
                batch=4, drafts=8, hq=32, q=A, qd=1, qs=4096, scale=0.1, window=0, sink=0, cap=0.0,
                slopes=None, out=A, lse=None, ws=A, ws_bytes=1 << 40, stream=None)
    need = P.aatc_paged_tree_workspace_bytes(4, 8, 32, 8)
    assert need > 0
    _refused(_drafts, name, args, TREES + QUERIES + [
        (INVALID, dict(window=-1)), (INVALID, dict(sink=-1)), (INVALID, dict(slopes=A + 3)),
        (WORKSPACE, dict(ws_bytes=need - 1)), (WORKSPACE, dict(ws_bytes=0)), (UNSUPPORTED, MANY),
        # 64 drafts of 264 heads on a KV head: 16896 columns
        (UNSUPPORTED, dict(hq=264 * 8, drafts=64, qs=264 * 8 * 128))])


def test_tree_workspace_sizes():
    size = P.aatc_paged_tree_workspace_bytes
    for bad in ((0, 8, 32, 8), (-1, 8, 32, 8), (4, 0, 32, 8), (4, 65, 32, 8), (4, 8, 0, 8), (4, 8, 32, 0),
                (4, 8, 30, 8), (4, 64, 264 * 8, 8)):
        assert size(*bad) == 0, bad
    assert size(4, 64, 256 * 8, 8) > 0


def test_tree_accept_refusals():
    name = "aatc_paged_tree_accept"
    args = dict(cache=(P.PagedCache, CACHE), layers=2, layer_stride=1 << 20, table=(P.PageTable, TABLE),
                len=2 * FAR, counts=None, parent=None, batch=4, drafts=8, drafted=3 * FAR, chosen=4 * FAR,
                path=5 * FAR, accepted=6 * FAR, next=7 * FAR, len_out=8 * FAR, stream=None)
    lists = ("drafted", "chosen", "path", "accepted", "next", "len_out")
    _refused(_drafts, name, args, TREES + [
        (INVALID, {k: x}) for k in lists for x in (None, A + 2)] + [
        (INVALID, dict(layers=0)), (INVALID, dict(layers=-1)), (INVALID, dict(layers=65536)),
        (INVALID, dict(layer_stride=0)), (INVALID, dict(layer_stride=127)), (INVALID, dict(layer_stride=132)),
        (INVALID, dict(layer_stride=1 << 40)), (INVALID, dict(layer_stride=-2048)),
        (INVALID, dict(cache=(P.PagedCache, {**CACHE, "n_kv_heads": 65536})))])
    # outputs that overlap an input or one another: the first and the last number of 32, of 4
    ins = dict(drafted=32, chosen=32, len=4, counts=4, parent=32)
    outs = dict(path=32, accepted=4, next=4, len_out=4)
    for out, size in outs.items():
        for x, n in {**ins, **outs}.items():
            if x != out:
                for at in (9 * FAR, 9 * FAR - 4 * (size - 1), 9 * FAR + 4 * (n - 1)):
                    assert _call(_drafts, name, args, **{x: 9 * FAR, out: at}) == INVALID, (out, x)
        for at in (A, A + 4 * (3 * 32 + 31)):         # (the table: rows of 32 entries)
            assert _call(_drafts, name, args, **{out: at}) == INVALID, out


def test_page_bounds_refusals():
    args = dict(cache=(P.PagedCache, CACHE), table=(P.PageTable, TABLE), held=None, wanted=A, codes=A,
                scales=A, stream=None)
    # 4 rows of 2^26 pages of 8 KV heads: 2^31
    most = (P.PageTable, {**TABLE, "max_pages": 1 << 26, "stride": 1 << 26})
    _refused(_sparse, "aatc_page_bounds", args, [
        (INVALID, dict(held=A + 2)), (INVALID, dict(wanted=None)), (INVALID, dict(wanted=A + 1)),
        (INVALID, dict(codes=None)), (INVALID, dict(codes=A + 8)), (INVALID, dict(scales=None)),
        (INVALID, dict(scales=A + 2)), (UNSUPPORTED, dict(table=most))])


def test_sparse_attention_refusals():
    name = "aatc_paged_sparse_attention"
    args = dict(cache=(P.PagedCache, CACHE), table=(P.PageTable, TABLE), len=A, codes=A, scales=A, batch=4,
                hq=32, q=A, qd=1, qs=4096, scale=0.1, most=8, first=1, last=1, cap=0.0, picked=A, out=A,
                lse=None, ws=A, ws_bytes=1 << 40, stream=None)
    need = P.aatc_paged_sparse_workspace_bytes(4, 32, 8, 32)
    assert need > 0
    many = (P.PageTable, {**TABLE, "max_pages": 1 << 26, "stride": 1 << 26})
    _refused(_sparse, name, args, QUERIES + [
        (INVALID, dict(batch=0)), (INVALID, dict(batch=5)), (INVALID, dict(len=None)), (INVALID, dict(len=A + 2)),
        (INVALID, dict(codes=None)), (INVALID, dict(codes=A + 4)), (INVALID, dict(scales=None)),
        (INVALID, dict(scales=A + 1)), (INVALID, dict(most=0)), (INVALID, dict(first=-1)),
        (INVALID, dict(last=-1)), (INVALID, dict(first=4, last=5)),
        (INVALID, dict(first=(1 << 31) - 1, last=(1 << 31) - 1)), (INVALID, dict(picked=None)),
        (INVALID, dict(picked=A + 2)), (WORKSPACE, dict(ws_bytes=need - 1)), (WORKSPACE, dict(ws_bytes=0)),
        (UNSUPPORTED, dict(most=(1 << 20) + 1)), (UNSUPPORTED, MANY), (UNSUPPORTED, dict(table=many)),
        (UNSUPPORTED, dict(hq=257 * 8, qs=257 * 8 * 128))])


def test_sparse_workspace_sizes():
    size = P.aatc_paged_sparse_workspace_bytes
    for bad in ((0, 32, 8, 32), (4, 0, 8, 32), (4, 32, 0, 32), (4, 30, 8, 32), (4, 32, 8, 0),
                (4, 32, 8, -1), (4, 32, 8, 1 << 26), (4, 257 * 8, 8, 32), (1, 8, 8, 1 << 62)):
        assert size(*bad) == 0, bad
    # a key for every page and KV head, at least
    for pages in (1, 32, 4096, 1 << 20):
        assert size(4, 32, 8, pages) >= 4 * 8 * pages * 4
