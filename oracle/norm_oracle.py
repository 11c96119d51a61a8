"""Oracle of the layer norm and its gradients in fp64 (numpy), from their formulas.  Shares no code
with the library.

The bounds are elementwise: u = 2^-24 is fp32's unit roundoff, a sum of n fp32 terms in any order is off
by at most n u times the sum of their magnitudes, and a rounding to bf16 by 2^-8 of the value.
"""
from __future__ import annotations

import numpy as np

from oracle.dense_oracle import TINY, U32, U_OUT


def residual_sum(X: np.ndarray, R: np.ndarray | None, to_type) -> np.ndarray:
    """S of fp32 arrays that hold values of the type; `to_type` rounds an fp32 array to it."""
    if R is None:
        return np.asarray(X, np.float32)
    return to_type(np.asarray(X, np.float32) + np.asarray(R, np.float32))


def depth(n: int) -> int:
    """The most additions that a term of a row's sum goes through: rows are spread over 64 lanes or more
    in pieces of eight, and the lanes and waves joined in at most 16 more."""
    return 8 * -(-n // 512) + 16


def statistics(S, eps):
    """(mean, rstd, deviations, bound of mean, relative bound of rstd) of rows in fp64.

    With a computed mean that is off by e the squares sum to n (var + e^2) exactly, since the
    deviations sum to 0; each deviation and square rounds once."""
    S = np.asarray(S, np.float64)
    n = S.shape[1]
    mean = S.mean(1, keepdims=True)
    e_mean = (depth(n) + 1) * U32 * np.abs(S).mean(1, keepdims=True) + TINY
    d = S - mean
    var = (d * d).mean(1, keepdims=True)
    e_var = e_mean ** 2 + (depth(n) + 4) * U32 * (var + e_mean ** 2)
    v = var + eps
    rstd = 1.0 / np.sqrt(v)
    # 1 / sqrt(v - e) against 1 / sqrt(v); then the sum with eps, the root and the quotient
    r_rstd = np.sqrt(v / np.maximum(v - e_var, 1e-3 * v)) - 1.0 + 4 * U32
    return mean, rstd, d, e_mean, r_rstd


def layer_norm(S, gamma=None, beta=None, eps=1e-5, out="f32"):
    """(Y, bound)."""
    mean, rstd, d, e_mean, r_rstd = statistics(S, eps)
    n = d.shape[1]
    e_d = e_mean + U32 * (np.abs(d) + e_mean)
    g = np.ones(n) if gamma is None else np.asarray(gamma, np.float64)
    b = np.zeros(n) if beta is None else np.asarray(beta, np.float64)
    h = d * rstd
    e_h = e_d * rstd * (1 + r_rstd) + np.abs(h) * (r_rstd + 2 * U32)
    y = h * g + b
    e = e_h * np.abs(g) + 3 * U32 * (np.abs(h * g) + np.abs(b))
    return y, e + U_OUT[out] * (np.abs(y) + e) * 1.0001 + TINY


def backward(dY, S, mean, rstd, gamma=None, dS=None, out="f32", grad="f32"):
    """{name: (gradient, bound)} from fp64 copies of the operands and of the saved statistics."""
    dY, S, mean, rstd = (np.asarray(a, np.float64) for a in (dY, S, mean, rstd))
    T, n = S.shape
    g = dY if gamma is None else dY * np.asarray(gamma, np.float64)
    h = (S - mean[:, None]) * rstd[:, None]
    e_h = 3 * U32 * np.abs(h)
    e_g = U32 * np.abs(g)
    c1, c2 = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    m1, m2 = np.abs(g).mean(1, keepdims=True), np.abs(g * h).mean(1, keepdims=True)
    e1 = (depth(n) + 3) * U32 * m1
    e2 = (depth(n) + 7) * U32 * m2
    dx = rstd[:, None] * (g - c1 - h * c2)
    parts = np.abs(g) + np.abs(c1) + np.abs(h * c2)
    e = rstd[:, None] * (e_g + e1 + np.abs(h) * e2 + e_h * (np.abs(c2) + e2) + 5 * U32 * parts)
    if dS is not None:
        dx = dx + np.asarray(dS, np.float64)
        e = e + 2 * U32 * np.abs(dx)
    dgamma, dbeta = (dY * h).sum(0), dY.sum(0)
    eg = (T + 6) * U32 * np.abs(dY * h).sum(0)
    eb = (T + 2) * U32 * np.abs(dY).sum(0)

    def rounded(v, bound, kind):
        return v, bound * 1.001 + U_OUT[kind] * (np.abs(v) + bound) * 1.0001 + TINY

    return {"dX": rounded(dx, e, out), "dgamma": rounded(dgamma, eg, grad),
            "dbeta": rounded(dbeta, eb, grad)}
