"""What a call of aatc_paged_tree_accept can hold at most: refused among the checks of its arguments, seen
over stand-ins of the launchers (which report a device error for what reaches them)."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2608_14191_amd as P
from paper_2608_14191_amd import _drafts
from paper_2608_14191_amd._lib import BF16, E_DEVICE, F16, F32
from test_drafts_cpu import FAR
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
