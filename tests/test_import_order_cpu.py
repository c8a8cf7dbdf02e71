"""The package and torch in one process, imported in either order: they have one HIP runtime (torch brings
its own, and kernels launched through another one than their memory's fail)."""
import os
import subprocess
import sys

import pytest

from test_paged_cpu import ROOT

RUNTIMES = """
import importlib.util, sys
if importlib.util.find_spec("torch") is None: sys.exit(77)
{}
maps = {{line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line}}
assert len(maps) == 1, maps
"""


@pytest.mark.parametrize("order", ["import paper_2608_14191_amd, torch", "import torch, paper_2608_14191_amd",
                                   "import paper_2608_14191_amd.build, torch"])
def test_one_runtime(order):
    env = {k: v for k, v in os.environ.items() if k != "AATC_LIBRARY"}
    run = subprocess.run([sys.executable, "-c", RUNTIMES.format(order)], capture_output=True, text=True, cwd=ROOT,
                         env=env, timeout=300)
    if run.returncode == 77:
        pytest.skip("no torch")
    assert run.returncode == 0, run.stderr[-2000:]


def test_torch_is_not_imported():
    """The host's calls (calibration, sizes) do without."""
    code = "import sys, paper_2608_14191_amd as P; assert 'torch' not in sys.modules; P.aatc_params_bytes(8)"
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ROOT, timeout=300)
