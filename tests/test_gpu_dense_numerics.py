"""The dense products' arithmetic where it is easiest to lose: operands at the ends of fp32's range,
saturated activations, gradients kept in fp32, and results whose every rounding is defined."""
import numpy as np
import pytest
import torch

from oracle import dense_oracle as D
from paper_2106_08846_amd import bsr as B
from tests.test_gpu_dense import DEV, TORCH, f64, frame, held, rand, within

pytestmark = pytest.mark.gpu


# --- fp32 weight gradients of a bf16 block ---------------------------------------------------------

# (T, K, F): one token to several tiles of every kind, and sums over T in slices.
@pytest.mark.parametrize("T,K,F", [(1, 8, 3), (33, 40, 50), (70, 33, 65), (64, 128, 64), (300, 200, 211),
                                   (100, 1000, 400), (5000, 48, 40), (6000, 264, 130),
                                   (2000, 2040, 1030), (4000, 33, 4090)])
def test_fp32_weight_gradients_keep_sixteen_bits_of_the_slopes(T, K, F):
    """dG and dU are whole numbers of up to 16 bits (10 where more tokens are summed): exact in two bf16
    pieces, not in one.  Sums stay below 2^24."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T + K + F)
    most = 181 if T <= 100 else 31          # 181^2 < 2^15; 2 * 181^2 * 100 < 2^24; 2 * 31^2 * 6000 < 2^24

    def ints(n, *shape):
        return torch.randint(-n, n + 1, shape, device=DEV, generator=gen).double()

    x, wg, wu, dh, g, u = (ints(2, T, K), ints(2, F, K), ints(2, F, K), ints(most, T, F),
                           ints(most, T, F), ints(most, T, F))
    bf = torch.bfloat16
    got = B.bsr_gated_backward(dh.to(bf), x.to(bf), wg.to(bf), wu.to(bf), g.float(), u.float(),
                               act="relu", bias=True, need=("W",), grad_dtype=torch.float32)
    dg, du = dh * u * (g > 0), dh * torch.clamp(g, min=0)
    for t, want in zip(got[1:], (dg.t() @ x, du.t() @ x, dg.sum(0), du.sum(0))):
        assert torch.equal(t.double(), want)


@pytest.mark.parametrize("T,K,F", [(1, 64, 96), (16, 100, 257), (65, 96, 33), (130, 257, 100)])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_fp32_weight_gradients_of_a_bf16_block(T, K, F, act):
    """Two bf16 pieces of dG and dU leave at most 2^-16 of them out; the sum has two terms a token."""
    rng = np.random.default_rng(T + K + F)
    x, dh = rand(rng, T, K, dtype="bf16"), rand(rng, T, F, dtype="bf16")
    w = rand(rng, F, K, dtype="bf16")
    g, u = rand(rng, T, F, sigma=2.0), rand(rng, T, F)
    got = B.bsr_gated_backward(*(t.to(DEV) for t in (dh, x, w, w, g, u)), act=act, need=("W",),
                               grad_dtype=torch.float32)
    want = D.gated_backward(f64(dh), f64(x), f64(w), f64(w), f64(g), f64(u), act, "f32", "f32")
    a, da = D.act(act, f64(g))
    for t, name, d in ((got[1], "dWg", f64(dh) * f64(u) * da), (got[2], "dWu", f64(dh) * a)):
        v, e = want[name]                   # counts 6.1 roundings a token, and of dG in fp32
        within(t, v, e + 1.01 * 2.0 ** -16 * np.abs(d).T @ np.abs(f64(x)), name)
