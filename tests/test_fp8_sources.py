"""What no run shows for certain, so that the sources of the FP8 operators are looked at.  Kernels that are on the GPU before the one in
front of them is done must not read by loads that take the memory to be unchanged for as long as the kernel is there: whether such
a load finds an old value depends on what else the SM has cached."""
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


def test_launches_say_themselves_how_they_went():
    # the runtime's last error may be another call's: a query on the legacy stream while a stream is captured leaves one
    for path in sorted(glob.glob(os.path.join(build.CSRC, "zc_fp8*.cu*"))):
        with open(path) as f:
            code = re.sub(r"//.*", "", f.read())
        assert "<<<" not in code and "cudaGetLastError" not in code and "cudaPeekAtLastError" not in code, path
