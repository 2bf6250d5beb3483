"""The norm's kernel run on the host, a thread a lane: rows that one workgroup
takes one behind another share its LDS without a race, whichever of them are
padding."""
import os
import re
import shutil

import pytest

from test_sanitizers import CSRC, SAN, run


def kernel_text():
    src = open(os.path.join(CSRC, "rows8.hip")).read()
    args = re.search(r"^struct NormArgs \{.*?^\};\n", src, re.M | re.S).group(0)
    body = re.search(r"^template <typename H, typename T, int N>\n__global__.*? void norm_kernel\(.*?^\}\n", src, re.M | re.S).group(0)
    body, n = re.subn(r"__shared__ float (\w+)", r"static Cell \1", body)
    assert n == 1 and "__shared__" not in body
    return args + body


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
def test_rows_of_a_workgroup_share_lds_without_a_race(tmp_path):
    (tmp_path / "norm_kernel.inc").write_text(kernel_text())
    exe = str(tmp_path / "norm_lanes")
    run(["g++", "-std=c++20", "-O1", "-g", "-ffp-contract=off", "-Wno-unknown-pragmas", "-pthread", "-I", str(tmp_path),
         os.path.join(SAN, "norm_lanes.cpp"), "-o", exe])
    assert run([exe]).stdout.strip().endswith("norm lanes ok")
