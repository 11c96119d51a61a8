"""The layer norm's oracle against torch's fp64 autograd and against differences, and the 8-bit
floating-point oracle against torch's own conversions and hand-made values."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as F
from oracle import norm_oracle as N

F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("T,K", [(1, 1), (3, 7), (5, 130)])
@pytest.mark.parametrize("affine", [True, False])
def test_norm_and_gradients_against_autograd(T, K, affine):
    rng = np.random.default_rng(T * 100 + K)
    S, dY, dS = (rng.standard_normal((T, K)) for _ in range(3))
    gamma, beta = (rng.standard_normal(K), rng.standard_normal(K)) if affine else (None, None)
    s = torch.from_numpy(S).requires_grad_()
    g = torch.from_numpy(gamma if affine else np.ones(K)).requires_grad_()
    b = torch.from_numpy(beta if affine else np.zeros(K)).requires_grad_()
    y = torch.nn.functional.layer_norm(s, (K,), g, b, 1e-5)
    grads = torch.autograd.grad(y, (s, g, b), torch.from_numpy(dY))
    Y, bound = N.layer_norm(S, gamma, beta, 1e-5)
    assert np.allclose(Y, y.detach().numpy(), rtol=1e-10, atol=1e-12) and np.all(bound > 0)
    mean, rstd = N.statistics(S, 1e-5)[:2]
    got = N.backward(dY, S, mean[:, 0], rstd[:, 0], gamma, dS)
    assert np.allclose(got["dX"][0], grads[0].numpy() + dS, rtol=1e-9, atol=1e-11)
    assert np.allclose(got["dgamma"][0], grads[1].numpy(), rtol=1e-9, atol=1e-11)
    assert np.allclose(got["dbeta"][0], grads[2].numpy(), rtol=1e-9, atol=1e-11)


def test_gradients_against_differences():
    rng = np.random.default_rng(3)
    S, dY = rng.standard_normal((2, 9)), rng.standard_normal((2, 9))
    gamma, beta = rng.standard_normal(9), rng.standard_normal(9)

    def loss(s, g, b):
        return float((N.layer_norm(s, g, b, 1e-5)[0] * dY).sum())
    mean, rstd = N.statistics(S, 1e-5)[:2]
    got = N.backward(dY, S, mean[:, 0], rstd[:, 0], gamma)
    h = 1e-5
    for k in range(9):
        e = np.eye(9)[k] * h
        assert abs((loss(S, gamma + e, beta) - loss(S, gamma - e, beta)) / (2 * h)
                   - got["dgamma"][0][k]) < 1e-7
        assert abs((loss(S, gamma, beta + e) - loss(S, gamma, beta - e)) / (2 * h)
                   - got["dbeta"][0][k]) < 1e-7
        for t in range(2):
            d = np.zeros_like(S)
            d[t, k] = h
            assert abs((loss(S + d, gamma, beta) - loss(S - d, gamma, beta)) / (2 * h)
                       - got["dX"][0][t, k]) < 1e-6


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_formats_against_torch(fmt):
    codes = torch.arange(256, dtype=torch.uint8).view(F8[fmt]).float().numpy()
    v = F.values(fmt)
    assert np.array_equal(v.astype(np.float32), codes, equal_nan=True)
    rng = np.random.default_rng(1)
    top = F.FORMATS[fmt][3]
    x = rng.standard_normal(20000) * np.exp(rng.uniform(-14, 8, 20000))
    fine = np.sort(v[np.isfinite(v)])
    ties = (fine[1:] + fine[:-1]) / 2
    near = np.concatenate([ties, np.nextafter(ties.astype(np.float32), 1e9),
                           np.nextafter(ties.astype(np.float32), -1e9)])
    x = np.clip(np.concatenate([x, fine, near]), -top, top).astype(np.float32)
    want = torch.from_numpy(x).to(F8[fmt]).view(torch.uint8).numpy()
    assert np.array_equal(F.encode(x, fmt), want)


def test_quantize_by_hand():
    x = np.zeros((3, 130), np.float32)
    x[0, 0], x[0, 1], x[0, 129] = 448.0, -1.0625, 2.0     # scales 1 and 2 / 448
    x[1, 5] = -7.0                                        # scale 7 / 448 = 2^-6
    codes, scale = F.quantize(x, 1, "e4m3")
    assert scale.shape == (2, 3)
    assert scale[0, 0] == 1.0 and scale[1, 0] == np.float32(2) / np.float32(448)
    assert scale[0, 1] == 2.0 ** -6 and scale[1, 1] == 0.0 and scale[0, 2] == 0.0
    v = F.values("e4m3")[codes]
    assert v[0, 0] == 448 and v[0, 1] == -1.0 and v[0, 129] == 448 and v[1, 5] == -448
    assert np.count_nonzero(v) == 4
    codes, scale = F.quantize(x, 128, "e4m3")
    assert scale.shape == (2, 1) and scale[0, 0] == 1.0
    assert F.values("e4m3")[codes][1, 5] == -7.0
    # one of one block by its transpose
    t, ts = F.quantize(x.T.copy(), 128, "e4m3")
    assert np.array_equal(t.T[:, :128], codes[:, :128]) and ts.shape == (1, 2) and ts[0, 0] == 1.0


def test_matmul_against_decoded_operands():
    rng = np.random.default_rng(7)
    X, W = rng.standard_normal((5, 300)).astype(np.float32), rng.standard_normal((200, 300)).astype(np.float32)
    xq, sx = F.quantize(X, 1, "e5m2")
    for rows in (1, 128):
        wq, sw = F.quantize(W, rows, "e4m3")
        Y, bound = F.matmul(xq, sx, wq, sw, rows, x_fmt="e5m2")
        want = np.zeros((5, 200))
        for b in range(3):
            cols = slice(128 * b, min(300, 128 * b + 128))
            part = F.values("e5m2")[xq[:, cols]] @ F.values("e4m3")[wq[:, cols]].T
            want += part * sx[b].astype(float)[:, None] * np.repeat(sw[b].astype(float), rows)[None, :200]
        assert np.allclose(Y, want, rtol=1e-12, atol=1e-12)
        # half a step of each operand: e5m2 2^-3, e4m3 2^-4, and what falls below the least exponents
        mag = np.abs(X.astype(float)) @ np.abs(W.astype(float)).T
        assert np.all(np.abs(Y - X.astype(float) @ W.astype(float).T) < (2 ** -3 + 2 ** -4 + 2 ** -7) * mag
                      + 300 * 1e-2)
