"""Kernels of a group launch ask for more LDS than a launch may take unless an attribute of the kernel says so.  It is set once for each, by a static
of the launch function: there have to be as many of those as kernels, or whichever of two is launched second goes without.  (ROCm 7.2 launches it all
the same, so that no launch shows it.)"""
import os
import re
import shutil
import subprocess

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2111_05972_amd", "libtp_layer.so")


@pytest.mark.skipif(shutil.which("nm") is None or not os.path.exists(LIB), reason="needs nm and the built library")
def test_a_static_to_each_kernel():
    names = [line.split()[-1] for line in subprocess.run(["nm", LIB], capture_output=True, text=True, check=True).stdout.splitlines()]
    kernels = {n for n in names if re.match(r"_ZN3tpl\d+gemm_bf16_group(_pp)?_kernelI", n)}
    guards = {n for n in names if n.startswith("_ZGVZN3tpl") and "12launch_groupI" in n}          # of function-local statics
    assert len(kernels) >= 8, kernels                                # 192, 128 and 64 a side; three tiles by turns, two of them also scaled
    assert len(guards) == len(kernels), (sorted(guards), sorted(kernels))
