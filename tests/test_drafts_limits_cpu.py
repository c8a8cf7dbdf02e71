"""What a call of aatc_paged_tree_accept can hold at most: refused among the checks of its arguments, seen
over stand-ins of the launchers (which report a device error for what reaches them)."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2608_14191_amd as P
from paper_2608_14191_amd import _drafts, _sparse
from paper_2608_14191_amd._lib import BF16, E_DEVICE, F16, F32
from test_drafts_cpu import FAR, _call
from test_paged_cpu import A, CACHE, INVALID, ROOT, TABLE, UNSUPPORTED, _fill

DEVICE = E_DEVICE


@pytest.fixture(scope="module")
def accept(tmp_path_factory):
    """accept(n_layers, n_kv_heads, dtype) over the C entry point and a launcher that only reports."""
    if shutil.which("g++") is None:
        pytest.skip("no host C++ compiler")
    csrc = os.path.join(ROOT, "paper_2608_14191_amd", "csrc")
    lib = tmp_path_factory.mktemp("limits") / "libdrafts.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(csrc, "drafts_abi.cpp"), os.path.join(ROOT, "tests", "host_stub", "drafts_stub.cpp"),
                    "-o", str(lib)], check=True)
    f = getattr(ctypes.CDLL(str(lib), mode=os.RTLD_LAZY), "aatc_paged_tree_accept")
    f.restype, f.argtypes = _drafts._SIGNATURES["aatc_paged_tree_accept"]

    def call(layers, heads, dtype):
        cache = _fill(P.PagedCache, **{**CACHE, "n_kv_heads": heads, "dtype": dtype})
        table = _fill(P.PageTable, **TABLE)
        return f(ctypes.addressof(cache), layers, 1 << 20, ctypes.addressof(table), A, None, None, 4, 8, 3 * FAR,
                 4 * FAR, 5 * FAR, 6 * FAR, 7 * FAR, 8 * FAR, None)
    return call


@pytest.mark.parametrize("dtype,most", [(BF16, 1 << 26), (F16, 1 << 26), (F32, 1 << 25)])
def test_layers_and_heads_of_accept(accept, dtype, most):
    """layers * heads * bytes of a head's token: up to 2^34."""
    for layers in (1024, 4096, 32768, 65535):
        heads = most // layers
        if heads <= 65535:
            assert accept(layers, heads, dtype) == DEVICE, (layers, heads)
        if heads + 1 <= 65535:
            assert accept(layers, heads + 1, dtype) == UNSUPPORTED, (layers, heads + 1)
    assert accept(65535, 65535, dtype) == UNSUPPORTED
    assert accept(1, 65535, dtype) == DEVICE
    # (numbers out of their own range are refused as such)
    assert accept(65536, 65535, dtype) == INVALID and accept(65535, 65536, dtype) == INVALID


def test_rows_of_a_launch():
    """Grids of up to 2^22 workgroups: the sizes on either side."""
    tree, sparse = P.aatc_paged_tree_workspace_bytes, P.aatc_paged_sparse_workspace_bytes
    for drafts, group, blocks in ((1, 1, 1), (64, 2, 1), (64, 4, 2), (43, 3, 2), (64, 256, 128)):
        rows = (1 << 22) // blocks - 1032
        assert tree(rows, drafts, group, 1) > 0 and tree(rows + 1, drafts, group, 1) == 0, (drafts, group)
        assert tree(rows // 8, drafts, 8 * group, 8) > 0 and tree(rows // 8 + 1, drafts, 8 * group, 8) == 0
    for pages, group, groups in ((64, 1, 1), (65, 1, 2), (256, 16, 4), (1, 17, 2), (64, 256, 16)):
        rows = (1 << 22) // groups
        assert sparse(rows, group, 1, pages) > 0 and sparse(rows + 1, group, 1, pages) == 0, (pages, group)
    # and the calls themselves
    many = (P.PageTable, {**TABLE, "rows": 1 << 22, "max_pages": 1, "stride": 1})
    attention = dict(cache=(P.PagedCache, CACHE), table=many, len=A, counts=None, parent=None, batch=(1 << 19), drafts=1,
                     hq=8, q=A, qd=1, qs=1024, scale=0.1, window=0, sink=0, cap=0.0, slopes=None, out=A, lse=None, ws=A,
                     ws_bytes=1 << 40, stream=None)
    assert _call(_drafts, "aatc_paged_tree_attention", attention) == UNSUPPORTED
    picked = dict(cache=(P.PagedCache, CACHE), table=many, len=A, codes=A, scales=A, batch=(1 << 19) + 1, hq=8, q=A, qd=1,
                  qs=1024, scale=0.1, most=8, first=1, last=1, cap=0.0, picked=A, out=A, lse=None, ws=A, ws_bytes=1 << 40,
                  stream=None)
    assert _call(_sparse, "aatc_paged_sparse_attention", picked) == UNSUPPORTED
