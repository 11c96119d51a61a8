"""Refusals of the layer norm's and the 8-bit floating-point entry points, which need no GPU: every case
is rejected on the host before any HIP call.  (Fake device pointers are never dereferenced.)"""
import os
import shutil

import pytest
import torch

from tests.test_dense_abi import ARG, DTYPE, MB, NULL, SHAPE, UNSUPPORTED, WORKSPACE, check
from tests.test_host_sanitizers import ROOT, SAN, _build_and_run

X, R, GAMMA, BETA, Y, S, MEAN, RSTD, DY, DS, DX, DG, DB, WS = (MB * (16 + i) for i in range(14))
W, SX, SW, BIAS, Q, SC, QT, SCT = (MB * (40 + i) for i in range(8))
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    from paper_2106_08846_amd import bsr
    return bsr


@pytest.mark.parametrize("kw,status", [
    ({}, None), ({"dt": 1}, None), ({"R": None, "S": None, "ldr": 0, "lds": 0}, None),
    ({"S": None}, None), ({"gamma": None, "beta": None}, None), ({"mean": None, "rstd": None}, None),
    ({"eps": 0.0}, None), ({"T": 0, "X": None, "Y": None}, 0),
    ({"X": None}, NULL), ({"Y": None}, NULL), ({"mean": None}, NULL), ({"rstd": None}, NULL),
    ({"T": -1}, SHAPE), ({"K": 0}, SHAPE), ({"ldx": 63}, SHAPE), ({"ldr": 63}, SHAPE),
    ({"ldy": 63}, SHAPE), ({"lds": 63}, SHAPE),
    ({"R": None}, ARG), ({"eps": -1e-9}, ARG), ({"eps": NAN}, ARG), ({"eps": INF}, ARG),
    ({"dt": 2}, DTYPE), ({"dt": 3}, ARG), ({"dt": -1}, ARG),
    ({"T": (1 << 24) + 1}, UNSUPPORTED), ({"ldx": MB + 1}, UNSUPPORTED), ({"ldr": MB + 1}, UNSUPPORTED),
    ({"ldy": MB + 1}, UNSUPPORTED), ({"lds": MB + 1}, UNSUPPORTED),
    ({"K": MB + 1, "ldx": MB + 1, "ldr": MB + 1, "ldy": MB + 1, "lds": MB + 1}, UNSUPPORTED),
    ({"Y": X}, ARG), ({"Y": X + 256}, ARG), ({"S": X}, ARG), ({"S": R + 4}, ARG), ({"Y": S}, ARG),
    ({"mean": GAMMA + 252}, ARG), ({"rstd": MEAN + 28}, ARG), ({"Y": BETA}, ARG),
    # columns of one buffer: apart, and one element too near
    ({"Y": X + 256, "ldx": 128, "ldy": 128}, None), ({"Y": X + 252, "ldx": 128, "ldy": 128}, ARG),
])
def test_layer_norm(L, kw, status):
    a = dict(X=X, ldx=64, R=R, ldr=64, T=8, K=64, dt=0, gamma=GAMMA, beta=BETA, eps=1e-5, Y=Y, ldy=64,
             S=S, lds=64, mean=MEAN, rstd=RSTD)
    a.update(kw)
    check(L.library().bsr_layer_norm, (*a.values(), None), status)


@pytest.mark.parametrize("kw,status", [
    ({}, None), ({"dt": 1, "gt": 0}, None), ({"gt": 1}, None), ({"dS": None, "ldds": 0}, None),
    ({"gamma": None}, None), ({"dX": None, "lddx": 0}, None), ({"dg": None}, None),
    ({"dg": None, "db": None, "ws": None, "wsb": 0}, None),
    ({"dX": None, "dg": None, "db": None, "ws": None}, 0),
    ({"T": 0, "dg": None, "db": None}, 0), ({"T": 0, "dY": None, "S": None, "mean": None}, None),
    ({"dY": None}, NULL), ({"S": None}, NULL), ({"mean": None}, NULL), ({"rstd": None}, NULL),
    ({"T": -1}, SHAPE), ({"K": 0}, SHAPE), ({"lddy": 63}, SHAPE), ({"lds": 63}, SHAPE),
    ({"ldds": 63}, SHAPE), ({"lddx": 63}, SHAPE),
    ({"dt": 2}, DTYPE), ({"gt": 2}, DTYPE), ({"dt": 4}, ARG), ({"gt": 4}, ARG),
    ({"T": (1 << 24) + 1}, UNSUPPORTED), ({"lddy": MB + 1}, UNSUPPORTED), ({"ldds": MB + 1}, UNSUPPORTED),
    ({"lds": MB + 1}, UNSUPPORTED), ({"lddx": MB + 1}, UNSUPPORTED),
    ({"ws": None}, WORKSPACE), ({"wsb": 500}, WORKSPACE), ({"ws": WS + 8}, WORKSPACE),
    ({"db": None, "ws": None}, WORKSPACE),
    ({"dX": DY}, ARG), ({"dX": S + 4}, ARG), ({"dX": DS}, ARG), ({"dg": DB + 8}, ARG),
    ({"dg": GAMMA}, ARG), ({"db": MEAN}, ARG), ({"ws": DX}, ARG), ({"ws": S}, ARG), ({"ws": DG}, ARG),
])
def test_layer_norm_backward(L, kw, status):
    a = dict(dY=DY, lddy=64, S=S, lds=64, T=8, K=64, dt=0, gamma=GAMMA, mean=MEAN, rstd=RSTD, dS=DS,
             ldds=64, dX=DX, lddx=64, dg=DG, db=DB, gt=0, ws=WS, wsb=MB)
    a.update(kw)
    check(L.library().bsr_layer_norm_backward, (*a.values(), None), status)


def test_layer_norm_workspace_bytes(L):
    f = L.library().bsr_layer_norm_workspace_bytes
    assert f(0, 64) > 0 and f(1, 1) >= 8 and f(6144, 2048) >= 2 * 2048 * 4
    for bad in ((-1, 64), (8, 0), ((1 << 24) + 1, 64), (8, MB + 1)):
        assert f(*bad) == 0


@pytest.mark.parametrize("kw,status", [
    ({}, None), ({"dt": 1, "f": 1, "rows": 128}, None),
    ({"Q": None, "s": None, "ldq": 0, "lds": 0}, None), ({"QT": None, "st": None, "ldqt": 0}, None),
    ({"T": 0, "X": None, "Q": None, "QT": None}, 0),
    ({"X": None}, NULL), ({"Q": None}, NULL), ({"s": None}, NULL), ({"QT": None}, NULL),
    ({"st": None}, NULL), ({"Q": None, "s": None, "QT": None, "st": None}, NULL),
    ({"T": -1}, SHAPE), ({"K": 0}, SHAPE), ({"ldx": 199}, SHAPE), ({"ldq": 199}, SHAPE),
    ({"lds": 7}, SHAPE), ({"ldqt": 7}, SHAPE), ({"ldst": 199}, SHAPE),
    ({"rows": 128, "lds": 1, "ldst": 1}, SHAPE), ({"rows": 128, "lds": 1, "ldst": 2}, None),
    ({"rows": 2}, ARG), ({"rows": 0}, ARG), ({"f": 2}, ARG), ({"f": -1}, ARG), ({"dt": 3}, ARG),
    ({"dt": 2}, DTYPE),
    ({"ldx": MB + 1}, UNSUPPORTED), ({"ldq": MB + 1}, UNSUPPORTED), ({"ldqt": MB + 1}, UNSUPPORTED),
    ({"T": (1 << 24) + 1, "lds": 1 << 25, "ldqt": 1 << 25}, UNSUPPORTED),
    ({"T": MB + 1, "lds": MB + 1, "ldqt": MB + 1}, UNSUPPORTED),
    ({"lds": (1 << 24) + 1}, UNSUPPORTED), ({"ldst": (1 << 24) + 1}, UNSUPPORTED),
    ({"Q": X}, ARG), ({"QT": Q + 100}, ARG), ({"s": X + 8}, ARG), ({"st": SC + 60}, ARG),
    ({"s": QT + 1500}, ARG),
])
def test_quantize_f8(L, kw, status):
    a = dict(X=X, dt=0, T=8, K=200, ldx=200, rows=1, f=0, Q=Q, ldq=208, s=SC, lds=8, QT=QT, ldqt=16,
             st=SCT, ldst=200)
    a.update(kw)
    check(L.library().bsr_quantize_f8, (*a.values(), None), status)


@pytest.mark.parametrize("kw,status", [
    ({}, None), ({"b": None, "dt": 1, "f": 1}, None), ({"rows": 1, "ldsw": 300}, None),
    ({"T": 0, "X": None, "Y": None}, 0),
    ({"X": None}, NULL), ({"W": None}, NULL), ({"sx": None}, NULL), ({"sw": None}, NULL),
    ({"Y": None}, NULL),
    ({"T": -1}, SHAPE), ({"K": 0}, SHAPE), ({"N": 0}, SHAPE), ({"ldx": 199}, SHAPE),
    ({"ldw": 199}, SHAPE), ({"ldy": 299}, SHAPE), ({"ldsx": 7}, SHAPE), ({"ldsw": 2}, SHAPE),
    ({"rows": 1, "ldsw": 299}, SHAPE),
    ({"rows": 64}, ARG), ({"f": 2}, ARG), ({"dt": 9}, ARG), ({"dt": 2}, DTYPE),
    ({"ldx": MB + 1}, UNSUPPORTED), ({"ldw": MB + 1}, UNSUPPORTED), ({"ldy": MB + 1}, UNSUPPORTED),
    ({"ldsx": (1 << 24) + 1}, UNSUPPORTED), ({"ldsw": (1 << 24) + 1}, UNSUPPORTED),
    ({"T": (1 << 24) + 1, "ldsx": 1 << 25}, UNSUPPORTED),
    ({"T": 1 << 24, "N": 1 << 13, "ldy": 1 << 13, "ldsx": 1 << 24, "ldsw": 64}, UNSUPPORTED),
    ({"Y": X + 1599}, ARG), ({"Y": W}, ARG), ({"Y": SX + 60}, ARG), ({"Y": SW + 20}, ARG),
    ({"Y": BIAS}, ARG),
])
def test_matmul_f8(L, kw, status):
    a = dict(X=X, f=0, T=8, K=200, ldx=200, sx=SX, ldsx=8, W=W, N=300, ldw=200, sw=SW, ldsw=3, rows=128,
             b=BIAS, Y=Y, dt=0, ldy=300)
    a.update(kw)
    if kw.get("N") == 1 << 13:      # 2^37 outputs
        assert a["T"] * a["N"] > 1 << 36
    check(L.library().bsr_matmul_f8, (*a.values(), None), status)


def test_binding_refuses_before_the_library(L):
    """Sizes and types that the C side cannot see."""
    f8, e5 = torch.float8_e4m3fn, torch.float8_e5m2
    x, v4, v64 = torch.zeros(4, 64), torch.zeros(4), torch.zeros(64)
    xq, wq = torch.zeros(4, 200).to(f8), torch.zeros(300, 200).to(f8)
    sx, sw = torch.zeros(2, 4), torch.zeros(2, 3)
    for f in (lambda: L.bsr_layer_norm(v4),
              lambda: L.bsr_layer_norm(x, v4),
              lambda: L.bsr_layer_norm(x, v64, v4),
              lambda: L.bsr_layer_norm(x, R=torch.zeros(4, 63)),
              lambda: L.bsr_layer_norm(x, R=torch.zeros(1, 64).expand(4, 64)),
              lambda: L.bsr_layer_norm(x, S=x),
              lambda: L.bsr_layer_norm(x, mean=v4),
              lambda: L.bsr_layer_norm(x, Y=torch.zeros(3, 64)),
              lambda: L.bsr_layer_norm(torch.zeros(64, 4).t()),
              lambda: L.bsr_layer_norm_backward(x, x, None, None),
              lambda: L.bsr_layer_norm_backward(x, x, v4, v64),
              lambda: L.bsr_layer_norm_backward(x[:, :63], x, v4, v4),
              lambda: L.bsr_layer_norm_backward(x, x, v4, v4, v4),
              lambda: L.bsr_layer_norm_backward(x, x, v4, v4, dS=x[:3]),
              lambda: L.bsr_layer_norm_backward(x, x, v4, v4, dgamma=v4),
              lambda: L.bsr_layer_norm_backward(x, x, v4, v4, workspace=x),
              lambda: L.bsr_quantize_f8(v4),
              lambda: L.bsr_quantize_f8(x, block_rows=64),
              lambda: L.bsr_quantize_f8(x, form="all"),
              lambda: L.bsr_quantize_f8(x, QT=torch.zeros(64, 4).to(f8)),
              lambda: L.bsr_quantize_f8(x, form="columns", Q=x.to(f8)),
              lambda: L.bsr_quantize_f8(x, Q=x[:3].to(f8)),
              lambda: L.bsr_quantize_f8(x, scale=torch.zeros(1, 3)),
              lambda: L.bsr_quantize_f8(x, block_rows=128, scale=torch.zeros(1, 4)),
              lambda: L.bsr_matmul_f8(xq, sx, wq[:, :199], sw),
              lambda: L.bsr_matmul_f8(xq, sx[:1], wq, sw),
              lambda: L.bsr_matmul_f8(xq, sx.t(), wq, sw),
              lambda: L.bsr_matmul_f8(xq, sx, wq, torch.zeros(2, 4)),
              lambda: L.bsr_matmul_f8(xq, sx, wq, torch.zeros(3, 300).t()),
              lambda: L.bsr_matmul_f8(xq, sx, wq, sw, bias=v4),
              lambda: L.bsr_matmul_f8(xq, sx, wq, sw, Y=torch.zeros(4, 299))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: L.bsr_layer_norm(x.half()),
              lambda: L.bsr_layer_norm(x),                    # CPU tensors
              lambda: L.bsr_layer_norm(x, v64.bfloat16()),
              lambda: L.bsr_layer_norm(x, R=x.bfloat16()),
              lambda: L.bsr_layer_norm_backward(x.bfloat16(), x, v4, v4),
              lambda: L.bsr_layer_norm_backward(x, x, v4, v4, grad_dtype=torch.float16),
              lambda: L.bsr_layer_norm_backward(x, x, v4, v4),
              lambda: L.bsr_quantize_f8(x, q_dtype=torch.int8),
              lambda: L.bsr_quantize_f8(x, Q=x.to(e5)),
              lambda: L.bsr_quantize_f8(x.to(f8)),
              lambda: L.bsr_quantize_f8(x),
              lambda: L.bsr_matmul_f8(xq, sx, wq.to(e5), sw),
              lambda: L.bsr_matmul_f8(xq.to(torch.int8), sx, wq, sw),
              lambda: L.bsr_matmul_f8(xq, sx.double(), wq, sw),
              lambda: L.bsr_matmul_f8(xq, sx, wq, sw, out_dtype=torch.float16),
              lambda: L.bsr_matmul_f8(xq, sx, wq, sw)):
        with pytest.raises(TypeError):
            f()


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_validation_under_sanitizers(tmp_path):
    exe = str(tmp_path / "norm_f8_validate_fuzz")
    _build_and_run(["g++", "-std=c++17", *SAN,
                    "-I", os.path.join(ROOT, "paper_2106_08846_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "norm_f8_validate_fuzz.cpp"),
                    os.path.join(ROOT, "paper_2106_08846_amd", "csrc", "validate.cpp"),
                    "-o", exe], exe)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_grids(tmp_path):
    exe = str(tmp_path / "f8_grids")
    _build_and_run(["g++", "-std=c++17", *SAN,
                    "-I", os.path.join(ROOT, "paper_2106_08846_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "f8_grids.cpp"), "-o", exe], exe)
