"""Kernels that are on the GPU before the one in front of them is done must not read by loads that take the memory to be unchanged for as
long as the kernel is there: whether such a load finds an old value depends on what else the SM has cached, so the sources are looked at."""
import glob
import os
import re

from paper_2508_19263_b200 import build


def test_kernels_that_start_early_use_ordinary_loads():
    files = sorted(glob.glob(os.path.join(build.CSRC, "zc_fp8*.cu*")))
    assert len(files) == 5
    for path in files:
        with open(path) as f:
            code = re.sub(r"//.*", "", f.read())
        assert not re.search(r"__ldg\(|__ldcs\(|\.global[.\w:]*\.nc|__restrict__", code), path
