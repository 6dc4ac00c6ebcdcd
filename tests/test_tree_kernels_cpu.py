"""What the compiler says of the tree-attention kernels.  CPU only."""
import os
import re
import shutil
import subprocess

import pytest


@pytest.mark.parametrize("source,kernel", [("tree_attention.hip", "tree_rows_kernel"), ("tree_tile.hip", "tree_tile_kernel")])
def test_no_instance_spills_vector_registers(source, kernel):
    """Both kernels hold their sums in registers through the whole run; a spill would put memory traffic into every step."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    from paper_2605_10453_amd import build as build_mod
    src = os.path.join(build_mod.CSRC, source)
    flags = [f for f in build_mod.flags_of(src) if f not in ("-shared", "-fPIC")]
    out = subprocess.run([hipcc, *flags, "--cuda-device-only", "-c", src, "-o", os.devnull, "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True)
    assert out.returncode == 0, out.stderr[-2000:]
    found = re.findall(r"Function Name: (\S+).*?VGPRs Spill: (\d+)", out.stderr, flags=re.S)
    mine = [(n, int(s)) for n, s in found if kernel in n]
    assert len(mine) >= 10 and all(s == 0 for _, s in mine), mine


def test_reads_of_values_return_before_the_barrier_that_lets_them_be_loaded_over():
    """After a barrier of tree_tile_kernel the other wavefronts load over the stage read last: a wavefront's own reads must have returned before it."""
    from paper_2605_10453_amd import build as build_mod
    text = open(os.path.join(build_mod.CSRC, "tree_tile.hip")).read()
    barriers = [m.start() for m in re.finditer(r"__builtin_amdgcn_s_barrier\(\);", text)]
    assert len(barriers) == 2
    for at in barriers:
        assert "s_waitcnt lgkmcnt(0)" in text[at - 120:at], text[at - 200:at]
