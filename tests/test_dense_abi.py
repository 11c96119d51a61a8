"""Refusals of the 8-bit and gated entry points, which need no GPU: every case is rejected on the
host before any HIP call.  (Fake device pointers are never dereferenced.)"""
import ctypes

import pytest
import torch

NULL, SHAPE, ARG, DTYPE, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4, 6, 9
PAST_CHECKS = (0, 7, 8)        # no GPU here: a valid call ends in the device check
MB = 1 << 20
X, WG, WU, SX, SG, SU, BG, BU, H, G, U = (MB * (16 + i) for i in range(11))
DH, DX, DWG, DWU, DBG, DBU, WS = (MB * (40 + i) for i in range(7))


@pytest.fixture(scope="module")
def L():
    from paper_2106_08846_amd import bsr
    return bsr


def check(call, args, expected):
    """expected None: a call that passes the checks, which never reaches a GPU with these pointers."""
    if expected is None:
        if torch.cuda.is_available():
            pytest.skip("a GPU is there, and the pointers are not memory")
        assert call(*args) in PAST_CHECKS
    else:
        assert call(*args) == expected


@pytest.mark.parametrize("kw,status", [
    ({}, None), ({"dt": 1}, None), ({"T": 0, "X": None, "Q": None, "s": None}, 0),
    ({"X": None}, NULL), ({"Q": None}, NULL), ({"s": None}, NULL),
    ({"T": -1}, SHAPE), ({"K": 0}, SHAPE), ({"ldx": 63}, SHAPE), ({"ldq": 63}, SHAPE),
    ({"dt": 2}, DTYPE), ({"dt": 3}, ARG), ({"dt": -1}, ARG),
    ({"ldx": MB + 1}, UNSUPPORTED), ({"ldq": MB + 1}, UNSUPPORTED),
    ({"T": (1 << 24) + 1}, UNSUPPORTED),
    ({"Q": X + 100}, ARG), ({"s": X + 1000}, ARG), ({"s": WG + 60}, ARG),
])
def test_quantize_rows(L, kw, status):
    a = dict(X=X, dt=0, T=8, K=64, ldx=64, Q=WG, ldq=64, s=SX)
    a.update(kw)
    check(L.library().bsr_quantize_rows, (*a.values(), None), status)


@pytest.mark.parametrize("kw,status", [
    ({}, None), ({"b": None, "dt": 1}, None), ({"T": 0, "X": None, "Y": None}, 0),
    ({"X": None}, NULL), ({"W": None}, NULL), ({"sx": None}, NULL), ({"sw": None}, NULL),
    ({"Y": None}, NULL),
    ({"T": -1}, SHAPE), ({"K": 0}, SHAPE), ({"N": 0}, SHAPE), ({"ldx": 63}, SHAPE),
    ({"ldw": 63}, SHAPE), ({"ldy": 31}, SHAPE),
    ({"dt": 2}, DTYPE), ({"dt": 9}, ARG),
    ({"K": 131072, "ldx": 131072, "ldw": 131072}, UNSUPPORTED),
    ({"K": 131071, "ldx": 131071, "ldw": 131072, "T": 1, "N": 1, "W": WS, "Y": 2 * WS}, None),
    ({"ldw": MB + 1}, UNSUPPORTED), ({"ldy": MB + 1}, UNSUPPORTED),
    ({"T": (1 << 24) + 1}, UNSUPPORTED), ({"T": 1 << 24, "N": 1 << 14, "ldy": 1 << 14}, UNSUPPORTED),
    ({"Y": X + 511}, ARG), ({"Y": WG + 10}, ARG), ({"Y": SX + 31}, ARG), ({"Y": SG}, ARG),
    ({"Y": BG + 4}, ARG),
])
def test_matmul_i8(L, kw, status):
    a = dict(X=X, T=8, K=64, ldx=64, sx=SX, W=WG, N=32, ldw=64, sw=SG, b=BG, Y=H, dt=0, ldy=32)
    a.update(kw)
    check(L.library().bsr_matmul_i8, (*a.values(), None), status)


def block(L, kw, i8=False):
    a = dict(K=64, F=32, Wg=WG, Wu=WU, ldg=64, ldu=64, sg=SG if i8 else None,
             su=SU if i8 else None, bg=BG, bu=BU, dtype=2 if i8 else 1, act=0)
    a.update({k: kw.pop(k) for k in list(kw) if k in a})
    return L.bsr_gated_t(*a.values())


BLOCK_REFUSALS = [
    ({"Wg": None}, NULL), ({"Wu": None}, NULL), ({"K": 0}, SHAPE), ({"F": 0}, SHAPE),
    ({"ldg": 63}, SHAPE), ({"ldu": 63}, SHAPE), ({"act": 4}, ARG), ({"act": -1}, ARG),
    ({"dtype": 3}, ARG), ({"ldg": MB + 1}, UNSUPPORTED), ({"ldu": MB + 1}, UNSUPPORTED),
    ({"K": MB + 1, "ldg": MB + 1, "ldu": MB + 1, "ldx": MB + 1}, UNSUPPORTED),
    ({"T": -1}, SHAPE), ({"ldx": 63}, SHAPE), ({"T": (1 << 24) + 1}, UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BLOCK_REFUSALS + [
    ({}, None), ({"dtype": 0, "bg": None, "bu": None}, None), ({"G": G, "U": U}, None),
    ({"T": 0, "X": None, "H": None}, 0),
    ({"dtype": 2, "sg": SG, "su": SU}, DTYPE), ({"X": None}, NULL), ({"H": None}, NULL),
    ({"G": G}, NULL), ({"U": U}, NULL), ({"ldh": 31}, SHAPE), ({"G": G, "U": U, "ldp": 31}, SHAPE),
    ({"ldh": MB + 1}, UNSUPPORTED), ({"T": 1 << 24, "F": 1 << 13, "ldh": 1 << 13}, UNSUPPORTED),
    ({"H": X + 64}, ARG), ({"H": WG + 64}, ARG), ({"H": WU}, ARG), ({"H": BG}, ARG),
    ({"H": BU + 100}, ARG), ({"G": G, "U": G + 500}, ARG), ({"G": H + 256, "U": U}, ARG),
    ({"G": G, "U": X}, ARG),
    # columns of one buffer: apart, one byte too near, wrapping into the next row, other pitches
    ({"G": G, "U": G + 32 * 4, "ldp": 64}, None), ({"U": G, "G": G + 32 * 4, "ldp": 64}, None),
    ({"G": G, "U": G + 32 * 4 - 1, "ldp": 64}, ARG), ({"G": G, "U": G + 32 * 4, "ldp": 63}, ARG),
    ({"G": G, "U": G + 32 * 4 + 64 * 4, "ldp": 64}, None), ({"G": G, "U": G + 64 * 4, "ldp": 64}, ARG),
    ({"G": G, "U": G + 33 * 4, "ldp": 64}, ARG), ({"H": X + 64 * 2, "ldx": 96, "ldh": 95}, ARG),
])
def test_gated(L, kw, status):
    kw = dict(kw)
    m = block(L, kw)
    a = dict(X=X, T=8, ldx=64, m=ctypes.byref(m), H=H, ldh=32, G=None, U=None, ldp=32)
    a.update(kw)
    check(L.library().bsr_gated, (*a.values(), None), status)


def test_gated_without_a_block(L):
    lib = L.library()
    assert lib.bsr_gated(X, 8, 64, None, H, 32, None, None, 0, None) == NULL
    assert lib.bsr_gated_i8(X, 8, 64, SX, None, H, 0, 32, None) == NULL
    assert lib.bsr_gated_backward(DH, 32, X, 8, 64, None, G, U, 32, DX, 64, DWG, DWU, 64, None,
                                  None, 0, WS, MB, None) == NULL


@pytest.mark.parametrize("kw,status", BLOCK_REFUSALS + [
    ({}, None), ({"hd": 0}, None), ({"T": 0, "X": None, "H": None}, 0),
    ({"dtype": 1}, DTYPE), ({"hd": 2}, DTYPE), ({"hd": 5}, ARG), ({"sg": None}, NULL),
    ({"su": None}, NULL), ({"sx": None}, NULL), ({"X": None}, NULL), ({"H": None}, NULL),
    ({"K": 131072, "ldg": 131072, "ldu": 131072, "ldx": 131072}, UNSUPPORTED),
    ({"ldh": 31}, SHAPE), ({"ldh": MB + 1}, UNSUPPORTED),
    ({"H": X + 8}, ARG), ({"H": SX}, ARG), ({"H": SG + 4}, ARG), ({"H": SU}, ARG),
    ({"H": WU + 5}, ARG), ({"H": BU}, ARG),
])
def test_gated_i8(L, kw, status):
    kw = dict(kw)
    m = block(L, kw, i8=True)
    a = dict(X=X, T=8, ldx=64, sx=SX, m=ctypes.byref(m), H=H, hd=1, ldh=32)
    a.update(kw)
    check(L.library().bsr_gated_i8, (*a.values(), None), status)


@pytest.mark.parametrize("kw,status", BLOCK_REFUSALS + [
    ({}, None), ({"gd": 0}, None), ({"dX": None}, None), ({"dWg": None, "dWu": None}, None),
    ({"dX": None, "dWg": None, "dWu": None, "dbg": None, "dbu": None}, 0),
    ({"T": 0, "dWg": None, "dWu": None, "dbg": None, "dbu": None}, 0),
    ({"dtype": 2}, DTYPE), ({"gd": 2}, DTYPE), ({"gd": 7}, ARG),
    ({"dH": None}, NULL), ({"X": None}, NULL), ({"G": None}, NULL), ({"U": None}, NULL),
    ({"dWg": None}, NULL), ({"dWu": None}, NULL),
    ({"lddh": 31}, SHAPE), ({"ldp": 31}, SHAPE), ({"lddx": 63}, SHAPE), ({"lddw": 63}, SHAPE),
    ({"T": (1 << 20) + 1}, UNSUPPORTED), ({"lddw": MB + 1}, UNSUPPORTED),
    ({"F": MB // 2 + 1, "lddh": MB, "ldp": MB}, UNSUPPORTED),
    ({"ws": None}, WORKSPACE), ({"wsb": 1000}, WORKSPACE), ({"ws": WS + 8}, WORKSPACE),
    ({"dX": X}, ARG), ({"dWg": WG}, ARG), ({"dWg": DWU + 100}, ARG), ({"dbg": DBU}, ARG),
    ({"dX": DH + 2}, ARG), ({"dWu": G}, ARG), ({"ws": DX}, ARG), ({"ws": U}, ARG),
    ({"dbu": DX + 10}, ARG),
    ({"dWu": DWG + 64 * 2, "lddw": 128}, None), ({"dWu": DWG + 63 * 2, "lddw": 128}, ARG),
])
def test_gated_backward(L, kw, status):
    kw = dict(kw)
    m = block(L, kw)
    a = dict(dH=DH, lddh=32, X=X, T=8, ldx=64, m=ctypes.byref(m), G=G, U=U, ldp=32, dX=DX, lddx=64,
             dWg=DWG, dWu=DWU, lddw=64, dbg=DBG, dbu=DBU, gd=1, ws=WS, wsb=MB)
    a.update(kw)
    check(L.library().bsr_gated_backward, (*a.values(), None), status)


def test_workspace_bytes(L):
    lib = L.library()
    assert lib.bsr_gated_workspace_bytes(8, 64, 32, 1) >= 8 * 64 * 2
    assert lib.bsr_gated_workspace_bytes(0, 64, 32, 1) > 0
    for bad in ((-1, 64, 32, 1), (8, 0, 32, 1), (8, 64, 0, 1), (8, 64, 32, 2), (8, 64, 32, 9),
                ((1 << 20) + 1, 64, 32, 1)):
        assert lib.bsr_gated_workspace_bytes(*bad) == 0


def test_binding_refuses_before_the_library(L):
    """Sizes and types that the C side cannot see."""
    x, w = torch.zeros(4, 64), torch.zeros(8, 64)
    xq, wq = x.to(torch.int8), w.to(torch.int8)
    s4, s8 = torch.zeros(4), torch.zeros(8)
    g = torch.zeros(4, 8)
    for f in (lambda: L.bsr_quantize_rows(torch.zeros(4)),
              lambda: L.bsr_quantize_rows(x, Q=torch.zeros(3, 64, dtype=torch.int8)),
              lambda: L.bsr_quantize_rows(x, scale=torch.zeros(3)),
              lambda: L.bsr_quantize_rows(torch.zeros(64, 4).t()),
              lambda: L.bsr_quantize_rows(torch.zeros(1, 64).expand(4, 64)),
              lambda: L.bsr_matmul_i8(xq, s4, wq[:, :63], s8),
              lambda: L.bsr_matmul_i8(xq, s8, wq, s8),
              lambda: L.bsr_matmul_i8(xq, s4, wq, s4),
              lambda: L.bsr_matmul_i8(xq, s4, wq, None),
              lambda: L.bsr_matmul_i8(xq, s4, wq, s8, bias=torch.zeros(7)),
              lambda: L.bsr_matmul_i8(xq, s4, wq, s8, Y=torch.zeros(4, 9)),
              lambda: L.bsr_gated(x, w, w[:7]),
              lambda: L.bsr_gated(x, w, w, bg=s4),
              lambda: L.bsr_gated(x, w, w, act="tanh"),
              lambda: L.bsr_gated(x, w, w, G=g),
              lambda: L.bsr_gated(x, w, w, H=torch.zeros(4, 9)),
              lambda: L.bsr_gated(x, w, w, G=g, U=torch.zeros(4, 10)[:, :8]),
              lambda: L.bsr_gated_i8(xq, s4, wq, s8, wq, None),
              lambda: L.bsr_gated_i8(xq, s8, wq, s8, wq, s8),
              lambda: L.bsr_gated_backward(g, x, w, w, g, g[:3]),
              lambda: L.bsr_gated_backward(g, x, w, w, g, g, need=("W", "b")),
              lambda: L.bsr_gated_backward(g, x, w, w, g, g, dWg=w),
              lambda: L.bsr_gated_backward(g, x, w, w, g, g, dX=torch.zeros(4, 63)),
              lambda: L.bsr_gated_backward(g, x, w, w, g, g, dbg=s4),
              lambda: L.bsr_gated_backward(g, x, w, w, g, g,
                                           workspace=torch.zeros(4, 4, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: L.bsr_quantize_rows(x.half()),
              lambda: L.bsr_quantize_rows(x),                 # CPU tensors
              lambda: L.bsr_matmul_i8(x, s4, wq, s8),
              lambda: L.bsr_matmul_i8(xq, s4.double(), wq, s8),
              lambda: L.bsr_matmul_i8(xq, s4, wq, s8, out_dtype=torch.float16),
              lambda: L.bsr_matmul_i8(xq, s4, wq, s8),
              lambda: L.bsr_gated(x, w.bfloat16(), w),
              lambda: L.bsr_gated(x, w, w),
              lambda: L.bsr_gated(xq, wq, wq),
              lambda: L.bsr_gated_i8(x, s4, w, s8, w, s8),
              lambda: L.bsr_gated_backward(g.bfloat16(), x, w, w, g, g),
              lambda: L.bsr_gated_backward(g, x, w, w, g, g, grad_dtype=torch.float16),
              lambda: L.bsr_gated_backward(g, x, w, w, g, g)):
        with pytest.raises(TypeError):
            f()
