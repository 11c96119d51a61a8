"""The dense products' grids over every accepted size (tests/host/dense_grids.cpp; host code only, under
AddressSanitizer and UndefinedBehaviorSanitizer)."""
import os
import shutil

import pytest

from tests.test_host_sanitizers import ROOT, SAN, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_grids_fit_a_launch_at_every_accepted_size(tmp_path):
    exe = str(tmp_path / "dense_grids")
    out = _build_and_run(["g++", "-std=c++17", *SAN,
                          "-I", os.path.join(ROOT, "paper_2106_08846_amd", "csrc"),
                          os.path.join(ROOT, "tests", "host", "dense_grids.cpp"),
                          os.path.join(ROOT, "paper_2106_08846_amd", "csrc", "validate.cpp"),
                          "-o", exe], exe)
    assert int(out.split()[1]) > 1 << 28, "the largest sizes must be reached"
