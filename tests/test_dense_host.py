"""The argument checks of the 8-bit and gated entry points under AddressSanitizer and
UndefinedBehaviorSanitizer (tests/host/dense_validate_fuzz.cpp; host code only)."""
import os
import shutil

import pytest

from tests.test_host_sanitizers import ROOT, SAN, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_dense_validation_under_sanitizers(tmp_path):
    exe = str(tmp_path / "dense_validate_fuzz")
    _build_and_run(["g++", "-std=c++17", *SAN,
                    "-I", os.path.join(ROOT, "paper_2106_08846_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "dense_validate_fuzz.cpp"),
                    os.path.join(ROOT, "paper_2106_08846_amd", "csrc", "validate.cpp"),
                    "-o", exe], exe)
