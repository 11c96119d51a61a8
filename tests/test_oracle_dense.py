"""The dense products' oracle against hand values, torch's own activations and central differences."""
import numpy as np
import pytest
import torch

from oracle import dense_oracle as D

ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


@pytest.mark.parametrize("name", ACTS)
def test_activations_match_torch(name):
    g = np.concatenate([np.linspace(-12, 12, 481), [-40.0, 40.0, 0.0]])
    t = torch.from_numpy(g).requires_grad_()
    nn = torch.nn.functional
    ref = {"silu": nn.silu, "gelu": nn.gelu, "relu": nn.relu,
           "gelu_tanh": lambda v: nn.gelu(v, approximate="tanh")}[name](t)
    ref.sum().backward()
    a, da = D.act(name, g)
    # 1 + erf and 1 + tanh cancel in torch's forms: absolute accuracy of g times 2^-52
    assert np.all(np.abs(a - ref.detach().numpy()) <= 1e-14 * (1 + np.abs(g)))
    assert np.all(np.abs(da - t.grad.numpy()) <= 1e-13 * (1 + np.abs(g)))


@pytest.mark.parametrize("name", ACTS)
def test_slopes_stay_below_the_constants_of_the_bounds(name):
    g = np.linspace(-30, 30, 600001)
    a, da = D.act(name, g)
    assert np.max(np.abs(da)) <= D.ACT_SLOPE
    if name != "relu":
        assert np.max(np.abs(np.diff(da) / np.diff(g))) <= D.ACT_CURVE


@pytest.mark.parametrize("name", ACTS)
def test_gradients_match_central_differences(name):
    rng = np.random.default_rng(3)
    T, K, F = 5, 4, 3
    arrs = {"X": rng.standard_normal((T, K)), "Wg": rng.standard_normal((F, K)),
            "Wu": rng.standard_normal((F, K)), "bg": rng.standard_normal(F),
            "bu": rng.standard_normal(F)}
    dH = rng.standard_normal((T, F))

    def loss(a):
        return float(np.sum(dH * D.gated(a["X"], a["Wg"], a["Wu"], a["bg"], a["bu"], name)[0]))

    _, G, U, *_ = D.gated(*arrs.values(), name)
    assert np.min(np.abs(G)) > 1e-3            # away from relu's kink
    grads = D.gated_backward(dH, arrs["X"], arrs["Wg"], arrs["Wu"], G, U, name)
    h = 1e-5
    for key, arr in arrs.items():
        got = grads["d" + key][0]
        for i in np.ndindex(arr.shape):
            hi, lo = ({**arrs, key: arr.copy()} for _ in range(2))
            hi[key][i] += h
            lo[key][i] -= h
            diff = (loss(hi) - loss(lo)) / (2 * h)
            # second-order differences: error about h^2 times the third derivative, plus 1e-16 / h
            assert abs(diff - got[i]) <= 1e-7 * (1 + abs(got[i])), (key, i)


def test_quantize_rows_by_hand():
    x = np.zeros((7, 4), np.float32)
    x[0] = [127.0, -63.5, 0.5, 1.5]              # r = 1: ties to even
    x[1] = [0.0, 0.0, 0.0, 0.0]
    x[2] = [np.inf, 1.0, -1.0, 0.0]
    x[3] = [np.nan, 1.0, -1.0, 0.0]
    x[4] = [-254.0, 254.0, 1.0, 3.0]             # r = 0.5
    x[5] = [2.0 ** -149, 0.0, -2.0 ** -149, 0.0]  # the smallest subnormal
    x[6] = [np.inf, np.nan, 0.0, 0.0]
    q, s = D.quantize_rows(x)
    assert q.tolist() == [[127, -64, 0, 2], [0] * 4, [0] * 4, [0] * 4, [-127, 127, 0, 2],
                          [127, 0, -127, 0], [0] * 4]
    assert s[0] == 1.0 and s[1] == 0.0 and np.isinf(s[2]) and np.isnan(s[3]) and s[4] == 2.0
    assert s[5] == 0.0 and np.isnan(s[6])


def test_matmul_i8_by_hand():
    y, bound = D.matmul_i8(np.array([[127, -128]], np.int8), np.array([0.5], np.float32),
                           np.array([[1, 2], [-127, 1]], np.int8),
                           np.array([2.0, 0.25], np.float32), np.array([1.0, -1.0], np.float32))
    assert y.tolist() == [[-129.0 + 1.0, (-16129 - 128) * 0.125 - 1.0]]
    assert np.all(bound < 1e-3)
