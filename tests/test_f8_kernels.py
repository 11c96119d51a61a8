"""Every kernel of the 8-bit floating-point product that its launch rules can choose is launched by a GPU test,
with tokens of either format (tests/host/f8_kernels.cpp; host code only, under AddressSanitizer and
UndefinedBehaviorSanitizer)."""
import itertools
import os
import shutil

import pytest

from tests import test_gpu_f8 as G
from tests import test_gpu_f8_forms as M
from tests.test_host_sanitizers import ROOT, SAN, _build_and_run


def parameters(test):
    """The calls of a parametrised test, as dicts."""
    marks = [m for m in test.pytestmark if m.name == "parametrize"]
    for combination in itertools.product(*(m.args[1] for m in marks)):
        call = {}
        for m, values in zip(marks, combination):
            names = m.args[0].split(",")
            call.update(zip(names, values if len(names) > 1 else [values]))
        yield call


def launched_by_tests(x_fmt):
    for test in (G.test_matmul, G.test_matmul_few_tokens, G.test_matmul_large_tiles,
                 G.test_matmul_long_contractions, M.test_few_tokens, M.test_large_tiles,
                 M.test_long_contractions, M.test_middle_tiles):
        for c in parameters(test):
            if c["x_fmt"] != x_fmt:
                continue
            T, N, K, pad = c["T"], c["N"], c["K"], c["pad"]
            out = c["out"] if "out" in c else ["f32", "bf16"][(T + K) % 2]
            aligned = pad < 0 or (K + pad) % 16 == 0 and c.get("shift", 0) % 16 == 0
            yield T, N, K, aligned, out == "f32", c["rows"] == 1


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("x_fmt", ["e4m3", "e5m2"])
def test_every_kernel_is_tested(tmp_path, x_fmt):
    calls = sorted(set(launched_by_tests(x_fmt)))
    header, exe = tmp_path / "calls.h", str(tmp_path / "f8_kernels")
    header.write_text("#define CALLS " + ", ".join(
        "{%s}" % ", ".join(str(int(v)) for v in c) for c in calls) + "\n")
    out = _build_and_run(["g++", "-std=c++17", *SAN, "-Wno-narrowing", "-include", str(header),
                          "-I", os.path.join(ROOT, "paper_2106_08846_amd", "csrc"),
                          os.path.join(ROOT, "tests", "host", "f8_kernels.cpp"), "-o", exe], exe)
    kernels = [line.split(" ", 1) for line in out.splitlines()[1:]]
    assert len(kernels) > 50
    assert [name for n, name in kernels if n == "0"] == []
