"""Layer norm's kernels in the library, by their names: every instance is one that some call can reach."""
import re
import shutil
import subprocess

import pytest


@pytest.mark.skipif(shutil.which("nm") is None, reason="needs binutils")
@pytest.mark.parametrize("kernel", ["norm_forward_kernel", "norm_backward_kernel"])
def test_instances_that_calls_reach(kernel):
    from paper_1910_02120_b200 import build
    names = subprocess.run(["nm", "-C", build.build()], capture_output=True, text=True, check=True).stdout
    found = set(re.findall(r"\b%s<(\S+), (\S+), (\d+), (\d+), (\d+), \d+, \d+, (\d+), (\d+)>" % kernel, names))
    assert len(found) > 50
    for xt, other, *numbers in found:
        v, nv, tpr, cluster, least = map(int, numbers)
        width = v * nv * tpr                                  # of a block
        if least == width:                                    # for rows of just this width: only those in whole aligned pieces
            assert v > 1, (xt, other, numbers)
        else:                                                 # some width above the next smaller class is a multiple of V
            assert least < width and (cluster > 1 or any(c % v == 0 for c in range(max(least, 17), width))), (xt, other, numbers)
