"""Oracle of the 8-bit floating-point matrices and their product (numpy), from their definitions.  Shares
no code with the library: codes are found by comparison with the format's 256 values.
"""
from __future__ import annotations

import numpy as np

from oracle.dense_oracle import TINY, U32, U_OUT

BLOCK = 128
#            exponent bits, fraction bits, bias, largest value
FORMATS = {"e4m3": (4, 3, 7, 448.0), "e5m2": (5, 2, 15, 57344.0)}


def values(fmt: str) -> np.ndarray:
    """The value of each of the 256 codes (NaN and infinities among them), by sign, exponent and
    fraction."""
    ebits, fbits, bias, largest = FORMATS[fmt]
    v = np.empty(256)
    for code in range(256):
        e, f = (code & 0x7F) >> fbits, code & ((1 << fbits) - 1)
        x = f * 2.0 ** (1 - bias - fbits) if e == 0 else (1 + f / 2.0 ** fbits) * 2.0 ** (e - bias)
        if x > largest:
            x = np.inf if fmt == "e5m2" and f == 0 else np.nan
        v[code] = -x if code & 0x80 else x
    return v


def encode(x: np.ndarray, fmt: str) -> np.ndarray:
    """Codes of fp32 values within the format's range: the nearest value, of two equally near the one
    whose fraction is even; a zero keeps its sign."""
    table = values(fmt)
    grid = table[:0x80][np.isfinite(table[:0x80])]           # ascending with the code
    a = np.abs(np.asarray(x, np.float64))
    hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
    lo = hi - 1
    below, above = a - grid[lo], grid[hi] - a
    code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def quantize(x: np.ndarray, block_rows: int = 1, fmt: str = "e4m3"):
    """(codes uint8 [R, K], scale fp32 [blocks of K, blocks of R]) in the definition's fp32 operations."""
    x = np.asarray(x, np.float32)
    R, K = x.shape
    rb, kb = -(-R // block_rows), -(-K // BLOCK)
    codes, scale = np.zeros((R, K), np.uint8), np.empty((kb, rb), np.float32)
    m = np.float32(FORMATS[fmt][3])
    with np.errstate(all="ignore"):
        for b in range(kb):
            cols = slice(b * BLOCK, min(K, (b + 1) * BLOCK))
            part = x[:, cols]
            pad = np.zeros((rb * block_rows, part.shape[1]), np.float32)
            pad[:R] = part
            top = np.max(np.abs(pad).reshape(rb, -1), axis=1)        # a NaN stays one
            scale[b] = top / m
            lift = np.where(top < np.float32(2.0 ** -64), np.float32(2.0 ** 64), np.float32(1))
            r = m / (top * lift)
            plain = (top > 0) & np.isfinite(top)
            rows = np.arange(R) // block_rows
            v = (part * lift[rows, None]) * r[rows, None]
            codes[:, cols] = np.where(plain[rows, None], encode(np.where(plain[rows, None], v, 0), fmt), 0)
    return codes, scale


def nominal_exponents(codes, fmt):
    """The exponent that a code is held with: of a subnormal value, the format's least; a zero has none."""
    _, fbits, bias, _ = FORMATS[fmt]
    magnitude = (codes & 0x7F).astype(np.int64)
    return np.where(magnitude == 0, -500, np.maximum(magnitude >> fbits, 1) - bias)


def aligned_loss(xq, wq, x_fmt, scales):
    """The most that the 8-bit matrix instructions drop: in every eight consecutive k the products are
    cut off (towards zero) below 2^-13 of the largest nominal exponent among them (products of zero do not
    count), so each of the eight loses less than that, times its block's scales."""
    ex, ew = nominal_exponents(xq, x_fmt), nominal_exponents(wq, "e4m3")
    loss = np.zeros((xq.shape[0], wq.shape[0]))
    for k in range(0, xq.shape[1], 8):
        most = np.full(loss.shape, -500)
        for i in range(k, min(k + 8, xq.shape[1])):
            most = np.maximum(most, ex[:, i, None] + ew[None, :, i])
        loss += 8 * 2.0 ** (most - 13.0) * scales(k // BLOCK)
    return loss


def matmul(xq, sx, wq, sw, block_rows, bias=None, x_fmt="e4m3", out="f32"):
    """(Y, bound): a product of two codes is exact in fp32; the sum of K of them, the products with the
    scales (two roundings each) and the bias round in fp32, the output once more.  With bf16 output
    the sums may be formed by the 8-bit matrix instructions."""
    K, N = xq.shape[1], wq.shape[0]
    at = np.arange(K) // BLOCK
    X = values(x_fmt)[xq] * np.asarray(sx, np.float64)[at].T
    W = values("e4m3")[wq] * np.asarray(sw, np.float64)[at][:, np.arange(N) // block_rows].T
    b = np.zeros(N) if bias is None else np.asarray(bias, np.float64)
    y = X @ W.T + b
    mag = np.abs(X) @ np.abs(W).T + np.abs(b)
    e = (K + 4) * U32 * mag
    if out == "bf16":
        s, v = np.asarray(sx, np.float64), np.asarray(sw, np.float64)
        e = e + aligned_loss(xq, wq, x_fmt,
                             lambda b_: s[b_][:, None] * v[b_][np.arange(N) // block_rows][None, :])
    return y, e + U_OUT[out] * (np.abs(y) + e) * 1.0001 + TINY
