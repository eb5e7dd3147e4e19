"""Every vector read of a matrix-core result in the attention kernels of drafted trees is at least
tests.xdl_hazards.MIN_WAIT wait states after the op (CPU: compiles the kernels to AMD assembly)."""
import os
import shutil
import tempfile

import pytest

from tests import xdl_hazards as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.slow
def test_every_xdl_result_read_is_padded_in_the_tree_kernels():
    hipcc = next((c for c in ("/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
    if hipcc is None:
        pytest.skip("hipcc not found")
    with tempfile.TemporaryDirectory() as d:
        asm = X.compile_asm(hipcc, os.path.join(ROOT, "paper_2608_13667_amd", "csrc", "kernels.hip"),
                            os.path.join(ROOT, "include"), os.path.join(d, "kernels.s"))
    kernels = X.kernels(asm, "tree_tiles")
    assert len(kernels) == 12
    for k in kernels:
        pairs = X.scan(asm, k)
        assert pairs, k
        assert min(p[0] for p in pairs) >= X.MIN_WAIT, (k, sorted(pairs)[:3])
