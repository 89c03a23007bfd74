"""The products' kernels give up a wait after a limit and then retire.  Each warp finds
out for itself, between one tile and the next, so no warp may wait for another at a
barrier without a limit before all have left their loops: such a barrier (a named one,
or the block's inside the roles' branches) is where a kernel that gave up would stand."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1807_11091_gb300", "csrc")


def code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


@pytest.mark.parametrize("name", ["tgemm_pair.cu", "tgemm.cu", "tgemm_dev.cuh"])
def test_no_named_barrier(name):
    assert not re.search(r"\bbar(rier)?\.(cta\.)?(sync|red|arrive)|named_barrier", code(name))


@pytest.mark.parametrize("name", ["tgemm_pair.cu", "tgemm.cu"])
def test_block_barriers_are_not_in_loops_or_roles(name):
    """__syncthreads() and cluster_sync() stand at the kernel's own level, or in a branch that is the
    launch's (splits), never deeper."""
    text = code(name)
    for kernel in re.finditer(r"__global__.*?\)\s*\n\{(.*?)\n\}\n", text, flags=re.S):
        for line in kernel.group(1).split("\n"):
            if "__syncthreads()" in line or "cluster_sync()" in line:
                depth = len(line) - len(line.lstrip())
                assert depth == 4 or (depth == 8 and name == "tgemm.cu"), line
