"""Oracle of the dense products in fp64 (numpy), from their formulas: 8-bit rows and their product,
the gated feed-forward block and its gradients.  Shares no code with the library.

Every function also has the elementwise error bound that its fp32 evaluation can be held to:
u = 2^-24 is fp32's unit roundoff, a sum of n fp32 terms in any order is off by at most n u times the
sum of their magnitudes, and a rounding to bf16 by 2^-8 of the value.
"""
from __future__ import annotations

import math

import numpy as np
from scipy.special import erfc, expit

U32 = 2.0 ** -24
U_OUT = {"f32": U32, "bf16": 2.0 ** -8}
TERMS = {"f32": 6.1, "bf16": 1}
TINY = 1e-30          # below every tested quantity; keeps a bound of zero terms positive
ACT_SLOPE = 1.13      # the largest slope of every activation (silu 1.0998, gelu 1.1289)
ACT_CURVE = 1.0       # and of every slope except relu's (gelu 0.798, gelu_tanh 0.80, silu 0.5)
ACT_ULPS = 16         # roundings inside one activation: exp, erfc, a quotient and a few products


def quantize_rows(x: np.ndarray):
    """(q int8, scale fp32) of fp32 rows, in the definition's fp32 operations."""
    x = np.asarray(x, np.float32)
    top = np.max(np.abs(x), axis=1)      # a NaN stays one
    with np.errstate(all="ignore"):
        lift = np.where(top < np.float32(2.0 ** -64), np.float32(2.0 ** 64), np.float32(1))
        r = np.float32(127) / (top * lift)
        v = np.rint((x * lift[:, None]) * r[:, None])
        q = np.where(np.isnan(v), np.float32(0), v).astype(np.int8)
        return q, (top / np.float32(127)).astype(np.float32)


def matmul_i8(xq, sx, wq, sw, bias=None, out="f32"):
    """(Y, bound): the scaled integer product; the fp32 conversion of the sum, two products and an
    addition round once each, the output once more."""
    acc = xq.astype(np.int64) @ wq.astype(np.int64).T
    y = acc.astype(np.float64) * sx.astype(np.float64)[:, None] * sw.astype(np.float64)[None, :]
    b = 0.0 if bias is None else bias.astype(np.float64)[None, :]
    mag = np.abs(y) + np.abs(b)
    return y + b, 5 * U32 * mag + U_OUT[out] * np.abs(y + b) * 1.0001 + TINY


def act(name: str, g: np.ndarray):
    """act(g) and its slope."""
    if name == "silu":
        p = expit(g)
        return g * p, p + g * p * expit(-g)
    if name == "gelu":
        p = 0.5 * erfc(-g / math.sqrt(2.0))
        return g * p, p + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        z = math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)
        t = np.tanh(z)
        dz = math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * g * g)
        return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * dz
    return np.where(g > 0, g, 0.0), np.where(g > 0, 1.0, 0.0)


def gated(X, Wg, Wu, bg=None, bu=None, name="silu", out="f32"):
    """(H, G, U, bound of H, bound of G, bound of U) from fp64 copies of the operands."""
    X, Wg, Wu = (np.asarray(a, np.float64) for a in (X, Wg, Wu))
    bg = np.zeros(len(Wg)) if bg is None else np.asarray(bg, np.float64)
    bu = np.zeros(len(Wu)) if bu is None else np.asarray(bu, np.float64)
    n = TERMS[out] * X.shape[1] + 2
    G, U = X @ Wg.T + bg, X @ Wu.T + bu
    eg = n * U32 * (np.abs(X) @ np.abs(Wg).T + np.abs(bg)) + TINY
    eu = n * U32 * (np.abs(X) @ np.abs(Wu).T + np.abs(bu)) + TINY
    H, e = gated_of(G, U, eg, eu, name, out)
    return H, G, U, e, eg, eu


def gated_of(G, U, eg, eu, name, out):
    """(H, bound) from pre-activations off by at most eg and eu."""
    a, _ = act(name, G)
    H = a * U
    ea = ACT_SLOPE * eg + ACT_ULPS * U32 * np.abs(G)
    e = ea * (np.abs(U) + eu) + np.abs(a) * eu + 2 * U32 * np.abs(H)
    return H, e + U_OUT[out] * (np.abs(H) + e) + TINY


def gated_backward(dH, X, Wg, Wu, G, U, name="silu", dtype="f32", grad="f32"):
    """{name: (gradient, bound)} from fp64 copies of the operands and of the saved G and U.  dG and dU
    are rounded to the block's type before the products (fp32: a rounding already counted)."""
    dH, X, Wg, Wu, G, U = (np.asarray(a, np.float64) for a in (dH, X, Wg, Wu, G, U))
    a, da = act(name, G)
    dG, dU = dH * U * da, dH * a
    eG = np.abs(dH * U) * ACT_ULPS * U32 * (1.0 + np.abs(G)) * 2 + 3 * U32 * np.abs(dG)
    eU = np.abs(dH) * ACT_ULPS * U32 * np.abs(G) + 3 * U32 * np.abs(dU)
    rG, rU = (e + U_OUT[dtype] * (np.abs(d) + e) for e, d in ((eG, dG), (eU, dU)))
    T, F = dH.shape

    def out(v, e, kind):
        return v, e + U_OUT[kind] * (np.abs(v) + e) + TINY

    def product(pairs, n, kind):
        v = sum(p @ q for p, _, q in pairs)
        e = sum(r @ np.abs(q) + n * U32 * ((np.abs(p) + r) @ np.abs(q)) for p, r, q in pairs)
        return out(v, e, kind)

    return {
        "dX": product([(dG, rG, Wg), (dU, rU, Wu)], TERMS[dtype] * 2 * F + 2, dtype),
        "dWg": product([(dG.T, rG.T, X)], TERMS[dtype] * T + 2, grad),
        "dWu": product([(dU.T, rU.T, X)], TERMS[dtype] * T + 2, grad),
        "dbg": out(dG.sum(0), eG.sum(0) + (T + 2) * U32 * (np.abs(dG) + eG).sum(0), grad),
        "dbu": out(dU.sum(0), eU.sum(0) + (T + 2) * U32 * (np.abs(dU) + eU).sum(0), grad),
    }
