"""The dense products' arithmetic where it is easiest to lose: operands at the ends of fp32's range,
saturated activations, gradients kept in fp32, and results whose every rounding is defined."""
import numpy as np
import pytest
import torch
from scipy.special import erfc, expit

from oracle import dense_oracle as D
from paper_2106_08846_amd import bsr as B
from tests.gpu_common import host
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


# --- fp32 operands at the ends of the range ---------------------------------------------------------

FLT_MAX = 3.4028234663852886e38
# Token counts and widths on both sides of the few-token kernel's rule, in both tile sizes.
ENDS = [(1, 90), (32, 2000), (96, 2000), (200, 2000), (777, 2048)]


@pytest.mark.parametrize("T,F", ENDS)
@pytest.mark.parametrize("K", [100, 101])
def test_fp32_operands_near_the_largest_finite_one(T, F, K):
    """Values from 2^128 (1 - 2^-9) on, which one bf16 piece cannot hold, times small ones."""
    rng = np.random.default_rng(T + F + K)
    x, wg, wu = rand(rng, T, K), rand(rng, F, K), rand(rng, F, K)
    x[:, 3] *= 1e-10                        # times 3.4e38
    wg[5, 3], wu[F - 1, 3], wg[7, 3] = 3.4e38, -FLT_MAX, 2.0 ** 127 * (2 - 2.0 ** -7)
    x[:, 20] = 0.0
    wg[8, 20], wu[9, 20] = FLT_MAX, -3.4e38
    x[T // 2, 90], x[T - 1, K - 1] = -3.4e38, FLT_MAX
    wg[:, 90] *= 1e-12
    wu[:, 90] *= 1e-30
    wg[:, K - 1] *= 1e-25
    wu[:, K - 1] = 0.0
    H, G, U = B.bsr_gated(x.to(DEV), wg.to(DEV), wu.to(DEV), act="relu", save=True)
    with np.errstate(all="ignore"):
        wh, g, u, eh, eg, eu = D.gated(f64(x), f64(wg), f64(wu), name="relu")
    within(G, g, eg, "G")
    within(U, u, eu, "U")
    fits = np.abs(wh) + eh < 1e38
    assert fits.mean() > 0.9
    got = f64(H)
    assert np.all(np.abs(got - wh)[fits] <= eh[fits])
    # the outputs without such an operand are those of a call without any
    for w, channels in ((wg, (5, 7, 8)), (wu, (9, F - 1))):
        w[list(channels)] = 0.0
    x[T // 2] = x[T - 1] = 0.0
    H0, G0, U0 = B.bsr_gated(x.to(DEV), wg.to(DEV), wu.to(DEV), act="relu", save=True)
    t = torch.ones(T, dtype=torch.bool, device=DEV)
    t[[T // 2, T - 1]] = False
    f = torch.ones(F, dtype=torch.bool, device=DEV)
    f[[5, 7, 8, 9, F - 1]] = False
    for a, b in ((H, H0), (G, G0), (U, U0)):
        assert torch.equal(a[t][:, f], b[t][:, f])


@pytest.mark.parametrize("T,K,F", [(1, 90, 40), (70, 100, 900), (70, 2040, 1020), (600, 800, 700)])
def test_fp32_gradients_of_operands_near_the_largest_finite_one(T, K, F):
    rng = np.random.default_rng(T + F + K)
    x, wg, wu, dh = rand(rng, T, K), rand(rng, F, K), rand(rng, F, K), rand(rng, T, F, sigma=1e-3)
    g, u = rand(rng, T, F), rand(rng, T, F)
    dh[:, 7] *= 1e-15                       # times the weights of channel 7, in dX
    wg[7, 11], wu[7, 12] = 3.4e38, -FLT_MAX
    x[T // 2, 30] = -FLT_MAX                # times dG and dU of one token, in dWg and dWu
    dh[T // 2] *= 1e-20
    got = B.bsr_gated_backward(*(t.to(DEV) for t in (dh, x, wg, wu, g, u)), act="gelu")
    want = D.gated_backward(*(f64(t) for t in (dh, x, wg, wu, g, u)), "gelu")
    # dG and dU of the small token and channel 7 are near 1e-38.  An operand below 2^-100 may lose 2^-125
    # (dG and dU are themselves rounded to 2^-150 there), which the other operand multiplies.
    a, da = D.act("gelu", f64(g))
    dg, du, X, Wg, Wu = f64(dh) * f64(u) * da, f64(dh) * a, f64(x), f64(wg), f64(wu)

    def lost(p, q):
        return 2.0 ** -125 * ((np.abs(p) < 2.0 ** -100) @ np.abs(q))

    more = {"dX": lost(dg, Wg) + lost(du, Wu), "dWg": lost(dg.T, X), "dWu": lost(du.T, X)}
    for name, t in zip(("dX", "dWg", "dWu"), got):
        v, e = want[name]
        within(t, v, e + more[name], name)


@pytest.mark.parametrize("T,F", ENDS)
@pytest.mark.parametrize("small", [2.0 ** -98, 2.0 ** -104, 2.0 ** -112, 2.0 ** -124])
def test_fp32_operands_near_the_smallest_ones(T, F, small):
    """Pieces below 2^-126 may be lost, at most 2^-125 of an operand in all: small tokens times large
    weights, and the other way round."""
    K = 96
    rng = np.random.default_rng(T + F)
    for sx, sw in ((small, 2.0 ** 50), (2.0 ** 50, small)):
        x, wg, wu = rand(rng, T, K, sigma=sx), rand(rng, F, K, sigma=sw), rand(rng, F, K, sigma=sw)
        _, G, U = B.bsr_gated(x.to(DEV), wg.to(DEV), wu.to(DEV), act="relu", save=True)
        _, g, u, _, eg, eu = D.gated(f64(x), f64(wg), f64(wu), name="relu")
        for got, want, e, w in ((G, g, eg, wg), (U, u, eu, wu)):
            operand = w if sx == small else x
            size = np.abs(f64(operand)).sum(1)
            within(got, want, e + 2.0 ** -125 * (size[None, :] if sx == small else size[:, None]), "small")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,F,K", [(96, 2000, 104), (300, 2000, 101), (777, 2048, 96), (2050, 2300, 72),
                                   (2050, 2300, 75)])
def test_non_finite_operands_in_tiles(dtype, T, F, K):
    """Sizes beyond the few-token kernel's: an infinity or a NaN reaches its token's or channel's outputs
    and leaves the other ones of its tile as they are."""
    rng = np.random.default_rng(T + F + K)
    x, wg, wu = (rand(rng, n, K, dtype=dtype).to(DEV) for n in (T, F, F))
    clean = B.bsr_gated(x, wg, wu, save=True)
    x[0, 17], x[T - 2, K - 1] = float("nan"), float("-inf")
    wg[7, 3], wu[50, K - 1], wg[F - 1, 0] = float("inf"), float("nan"), float("-inf")
    H, G, U = B.bsr_gated(x, wg, wu, save=True)
    t = torch.ones(T, dtype=torch.bool, device=DEV)
    t[[0, T - 2]] = False
    assert torch.isnan(G[0]).all() and torch.isnan(U[0]).all() and torch.isnan(H[0]).all()
    assert not torch.isfinite(G[T - 2]).any() and not torch.isfinite(U[T - 2]).any()
    f = torch.ones(F, dtype=torch.bool, device=DEV)
    f[[7, 50, F - 1]] = False
    for a, b in zip((H, G, U), clean):
        assert torch.equal(a[t][:, f], b[t][:, f])
    assert not torch.isfinite(G[:, [7, F - 1]]).any() and torch.isnan(U[:, 50]).all()
    assert torch.equal(G[t][:, 50], clean[1][t][:, 50]) and torch.equal(U[t][:, 7], clean[2][t][:, 7])


# --- saturated activations -------------------------------------------------------------------------

def wide_range():
    big = [16.7, 17.5, 30.0, 60.0, 86.5, 87.0, 87.25, 87.5, 88.0, 88.5, 89.0, 104.0, 1e3, 1e4, 1e10, 1e19,
           1.9e19, 1e20, 1e30, 3e38]
    small = [1e-38, 1e-30, 1e-10, 1e-3, 0.1, 1.0, 3.0, 5.5, 9.0, 10.5, 12.0, 13.5, 14.5]
    return torch.tensor([s * v for v in big + small for s in (1.0, -1.0)] + [0.0], dtype=torch.float32)


def act64(name, g):
    """act(g), its slope and the exponent of its negative tail, in forms that do not cancel."""
    with np.errstate(all="ignore"):
        if name == "silu":
            p = expit(g)
            return g * p, p * (1 + g * expit(-g)), np.zeros_like(g)
        if name == "gelu":
            p = 0.5 * erfc(-g / np.sqrt(2.0))
            return g * p, p + g * np.exp(-0.5 * g * g) / np.sqrt(2 * np.pi), g * g
        if name == "gelu_tanh":
            c = np.sqrt(2.0 / np.pi)
            z = c * g * (1 + 0.044715 * g * g)
            p, q = expit(2 * z), expit(-2 * z)
            slope = np.where(p * q == 0, p, p + g * p * q * 2 * c * (1 + 3 * 0.044715 * g * g))
            return g * p, slope, 2 * np.abs(z)
        return np.maximum(g, 0), np.where(g > 0, 1.0, 0.0), np.zeros_like(g)


# What an activation may be off by where its probability lies below 2^-126, for |g| < 2^8; farther out the
# exact value is below 2^-200.
TAIL = 2.0 ** -118


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_activations_far_out(act, dtype):
    """A relative error of 16 roundings and of the rounded argument of the tail's exponential (4 roundings
    of up to 200, beyond which the tail is below 2^-126)."""
    g = wide_range().to(TORCH[dtype])
    n = len(g)
    x = torch.zeros(n, 128, dtype=TORCH[dtype])
    x[:, :n] = torch.eye(n)
    wg = torch.zeros(24, 128, dtype=TORCH[dtype])
    wg[:, :n] = g
    wu = torch.full((24, 128), 0.75, dtype=TORCH[dtype])
    H, G, U = B.bsr_gated(x.to(DEV), wg.to(DEV), wu.to(DEV), act=act, save=True)
    v = f64(g)[:, None] * np.ones((1, 24))
    assert np.array_equal(f64(G), v) and torch.all(U == 0.75)
    a, _, zeta = act64(act, v)
    want = 0.75 * a
    e = D.U32 * np.abs(want) * (20 + 4 * np.minimum(zeta, 200.0)) + TAIL
    within(H, want, e + D.U_OUT[dtype] * (np.abs(want) + e) * 1.0001, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_slopes_far_out(act, dtype):
    """One token with dH = U = 1: the bias gradients are the slopes and the activations.  A slope's
    summands, of at most 1 + |g| while it is neither 0 nor 1 (|g| < 20), are off by 32 roundings."""
    g = wide_range()
    F = len(g)
    one = torch.ones(1, F, device=DEV)
    dt = TORCH[dtype]
    zero = torch.zeros(F, 8, dtype=dt, device=DEV)
    out = B.bsr_gated_backward(one.to(dt), torch.ones(1, 8, dtype=dt, device=DEV), zero, zero,
                               g[None].to(DEV), one, act=act, bias=True, grad_dtype=torch.float32)
    a, da, zeta = act64(act, f64(g))
    within(out[3], da, 32 * D.U32 * (1 + np.minimum(np.abs(f64(g)), 20.0)), "slope")
    within(out[4], a, D.U32 * np.abs(a) * (20 + 4 * np.minimum(zeta, 200.0)) + TAIL, "activation")
    assert all(torch.isfinite(t).all() for t in out)


# --- defined roundings ---------------------------------------------------------------------------

# Few-token kernel (one token, one round), ring tiles and tiles of unaligned rows.
I8_SIZES = [(1, 100, 1000), (1, 100, 1001), (16, 257, 256), (30, 257, 255), (33, 6000, 64), (33, 6000, 65),
            (300, 513, 96), (300, 513, 97), (1100, 1300, 192), (1100, 1300, 191), (4000, 2900, 64),
            (4000, 2900, 66)]


def scaled(xq, sx, wq, sw, bias):
    """The definition in fp32, one operation after the other."""
    y = (xq.astype(np.int64) @ wq.astype(np.int64).T).astype(np.float32)
    return ((y * sx[:, None]) * sw[None, :]) + bias[None, :]


@pytest.mark.parametrize("T,N,K", I8_SIZES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_matmul_i8_rounds_as_defined(T, N, K, out):
    rng = np.random.default_rng(T + N + K)
    xq, wq = (rng.integers(-128, 128, s).astype(np.int8) for s in ((T, K), (N, K)))
    sx, sw = (rng.uniform(0.001, 0.1, n).astype(np.float32) for n in (T, N))
    bias = rng.standard_normal(N).astype(np.float32)
    y = B.bsr_matmul_i8(*(torch.from_numpy(a).to(DEV) for a in (xq, sx, wq, sw, bias)),
                        out_dtype=TORCH[out])
    want = torch.from_numpy(scaled(xq, sx, wq, sw, bias)).to(TORCH[out])
    assert torch.equal(y.cpu(), want)


@pytest.mark.parametrize("T,F,K", [(t, n // 2, k) for t, n, k in I8_SIZES])
def test_gated_i8_rounds_as_defined(T, F, K):
    """With relu everything after the integer sums is a defined fp32 operation."""
    rng = np.random.default_rng(T + F + K)
    xq, gq, uq = (rng.integers(-127, 128, s).astype(np.int8) for s in ((T, K), (F, K), (F, K)))
    sx, sg, su = (rng.uniform(0.001, 0.1, n).astype(np.float32) for n in (T, F, F))
    bg, bu = (rng.standard_normal(F).astype(np.float32) for _ in range(2))
    t = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    h = B.bsr_gated_i8(t(xq), t(sx), t(gq), t(sg), t(uq), t(su), t(bg), t(bu), act="relu",
                       out_dtype=torch.float32)
    want = np.maximum(scaled(xq, sx, gq, sg, bg), np.float32(0)) * scaled(xq, sx, uq, su, bu)
    assert np.array_equal(host(h), want)


# --- offsets past 32 bits --------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_past_32_bits_of_offset(dtype):
    """Every matrix of a backward call that has a pitch, in turn, with rows that start more than 2^32
    bytes into it; all rows differ, so that one read or written 2^31 or 2^32 bytes off shows."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    pitch, T, K = 1 << 20, 2200, 40
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    dt = TORCH[dtype]

    def ints(n, *shape):
        return torch.randint(-n, n + 1, shape, device=DEV, generator=gen).double()

    def far(t, dtype):
        view = torch.empty(t.shape[0], pitch, dtype=dtype, device=DEV)[:, :t.shape[1]]
        view.copy_(t)
        return view

    # tokens far apart: X, dH, dX (bf16 2 MiB a row, fp32 4), then G and U (4 MiB)
    F = 48
    x, wg, wu, dh, g, u = (ints(2, T, K), ints(2, F, K), ints(2, F, K), ints(1, T, F), ints(3, T, F),
                           ints(3, T, F))
    dg, du = dh * u * (g > 0), dh * torch.clamp(g, min=0)
    want = [dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dg.sum(0), du.sum(0)]

    def call(X, Wg, Wu, dH, G, U, **outs):
        got = B.bsr_gated_backward(dH, X, Wg, Wu, G, U, act="relu", bias=True,
                                   grad_dtype=torch.float32, **outs)
        for t, w, name in zip(got, want, ("dX", "dWg", "dWu", "dbg", "dbu")):
            assert torch.equal(t, w.float().to(t.dtype)), name

    near = [t.to(dt) for t in (wg, wu)]
    dX = torch.empty(T, pitch, dtype=dt, device=DEV)[:, :K]
    assert dX.stride(0) == pitch
    call(far(x, dt), *near, far(dh, dt), g.float(), u.float(), dX=dX)
    del dX
    call(x.to(dt), *near, dh.to(dt), far(g, torch.float32), far(u, torch.float32))
    # channels far apart: the weights and their gradients
    T, F = 96, 2200
    x, wg, wu, dh, g, u = (ints(2, T, K), ints(2, F, K), ints(2, F, K), ints(1, T, F), ints(3, T, F),
                           ints(3, T, F))
    dg, du = dh * u * (g > 0), dh * torch.clamp(g, min=0)
    want = [dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dg.sum(0), du.sum(0)]
    dW = [torch.empty(F, pitch, device=DEV)[:, :K] for _ in range(2)]
    call(x.to(dt), far(wg, dt), far(wu, dt), dh.to(dt), g.float(), u.float(), dWg=dW[0], dWu=dW[1])


def test_transposes_of_more_tiles_than_workgroups():
    """fp32 weights of 2 x 192 x 192 tiles of 64 x 64, more than the 2^16 workgroups that transpose."""
    T, K, F = 5, 12270, 12250
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)
    x, wg, wu, dh, g, u = (torch.randint(-n, n + 1, s, device=DEV, generator=gen).float() for n, s in
                           ((2, (T, K)), (2, (F, K)), (2, (F, K)), (1, (T, F)), (3, (T, F)), (3, (T, F))))
    got = B.bsr_gated_backward(dh, x, wg, wu, g, u, act="relu")
    dg, du = (dh * u * (g > 0)).double(), (dh * torch.clamp(g, min=0)).double()
    for t, want in zip(got, (dg @ wg.double() + du @ wu.double(), dg.t() @ x.double(), du.t() @ x.double())):
        assert torch.equal(t.double(), want)          # below 2^24: exact
