"""The 8-bit and gated products on the GPU against the fp64 oracle, within bounds that count the
roundings of fp32 sums and of the outputs (oracle/dense_oracle.py), and bit for bit where every
operation is exact.  Sizes straddle the kernels' tiles, rows start at no particular alignment, pitches
exceed widths, and the gaps between rows hold NaN on the way in and a sentinel on the way out."""
import numpy as np
import pytest
import torch

from oracle import dense_oracle as D
from paper_2106_08846_amd import bsr as B
from tests.gpu_common import host

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


def f64(t):
    return t.detach().to("cpu").double().numpy()


def held(a, pad=0, shift=0, gap=float("nan")):
    """A device tensor equal to `a` with row pitch width + pad, starting `shift` elements into its
    storage; what lies between the rows is `gap`."""
    T, K = a.shape
    gap = 99 if a.dtype == torch.int8 else gap
    buf = torch.full((T * (K + pad) + shift + 8,), gap, dtype=a.dtype, device=DEV)
    view = buf[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K]
    view.copy_(a)
    return view


def frame(T, K, dtype, pad=0, shift=0):
    """An output view of that layout in a buffer of sentinels, and a check that nothing but the view
    was written."""
    buf = torch.full((T * (K + pad) + shift + 64,), 77, dtype=dtype, device=DEV)
    view = buf[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K]

    def untouched():
        copy = buf.clone()
        copy[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K] = 77
        return bool((copy == 77).all())
    return view, untouched


def rand(rng, *shape, sigma=1.0, dtype="f32"):
    return torch.from_numpy((rng.standard_normal(shape) * sigma).astype(np.float32)).to(TORCH[dtype])


def within(got, want, bound, what):
    err = np.abs(f64(got) - want)
    assert np.all(np.isfinite(f64(got))), what
    assert np.all(err <= bound), (what, float(np.max(err / bound)))


# --- rows in 8 bits -----------------------------------------------------------------------------

@pytest.mark.parametrize("T,K", [(1, 1), (3, 7), (1, 1024), (5, 255), (17, 256), (4, 4096),
                                 (2, 4099), (3, 20000), (1000, 64), (65, 513), (2, 70001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1), (16, 8)])
def test_quantize_rows(T, K, dtype, pad, shift):
    rng = np.random.default_rng(T * 100003 + K)
    x = rand(rng, T, K, dtype=dtype) * torch.from_numpy(
        np.exp(rng.uniform(-20, 20, (T, 1))).astype(np.float32)).to(TORCH[dtype])
    X = held(x, pad, shift)
    Q, clean = frame(T, K, torch.int8, pad, shift)
    q, s = B.bsr_quantize_rows(X, Q=Q)
    wq, ws = D.quantize_rows(x.float().numpy())
    assert np.array_equal(host(q), wq)
    assert np.array_equal(host(s).view(np.uint32), ws.view(np.uint32))
    assert clean()
    q2, s2 = B.bsr_quantize_rows(X)
    assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [5, 640, 9001])
def test_quantize_rows_special_values(dtype, K):
    x = np.random.default_rng(5).standard_normal((9, K)).astype(np.float32)
    x[0] = 0.0
    x[1, K - 1] = np.inf
    x[2, 0] = -np.inf
    x[3, K // 2] = np.nan
    x[4] *= np.float32(2.0 ** -130)                  # subnormal rows
    x[5] = np.float32(2.0 ** -133)                   # (bf16's smallest)
    x[6] *= np.float32(1e37)
    x[7, 0], x[7, K - 1] = np.inf, np.nan
    x[8] = -0.0
    t = torch.from_numpy(x).to(TORCH[dtype])
    q, s = B.bsr_quantize_rows(t.to(DEV))
    wq, ws = D.quantize_rows(t.float().numpy())
    assert np.array_equal(host(q), wq)
    gs = host(s)
    assert np.array_equal(np.isnan(gs), np.isnan(ws))
    ok = ~np.isnan(ws)
    assert np.array_equal(gs[ok].view(np.uint32), ws[ok].view(np.uint32))


# --- 8-bit product ------------------------------------------------------------------------------

# Token counts around the small-batch and tile sizes; widths around the depth of one step.
I8_SIZES = [(1, 1, 1), (1, 64, 64), (1, 100, 1000), (2, 33, 770), (4, 4096, 64), (7, 16, 4096),
            (16, 257, 256), (17, 129, 255), (32, 64, 2048), (33, 96, 128), (63, 100, 96),
            (64, 256, 384), (65, 255, 130), (128, 128, 1024), (130, 640, 48), (257, 130, 514),
            (300, 513, 1), (512, 1024, 256), (1100, 1300, 192), (3, 5, 20001)]


@pytest.mark.parametrize("T,N,K", I8_SIZES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 3), (16, 16)])
def test_matmul_i8(T, N, K, out, pad, shift):
    rng = np.random.default_rng(T * 7919 + N * 31 + K)
    xq = torch.from_numpy(rng.integers(-128, 128, (T, K)).astype(np.int8))
    wq = torch.from_numpy(rng.integers(-128, 128, (N, K)).astype(np.int8))
    sx = torch.from_numpy(rng.uniform(0.001, 0.1, T).astype(np.float32))
    sw = torch.from_numpy(rng.uniform(0.001, 0.1, N).astype(np.float32))
    bias = rand(rng, N) if (T + N) % 2 else None
    Y, clean = frame(T, N, TORCH[out], pad, shift)
    B.bsr_matmul_i8(held(xq, pad, shift), sx.to(DEV), held(wq, pad, shift), sw.to(DEV),
                    None if bias is None else bias.to(DEV), Y=Y)
    want, bound = D.matmul_i8(xq.numpy(), sx.numpy(), wq.numpy(), sw.numpy(),
                              None if bias is None else bias.numpy(), out)
    within(Y, want, bound, "Y")
    assert clean()
    # unit scales and no bias: the integer itself (exact in fp32 below 2^24)
    one = torch.ones(max(T, N), device=DEV)
    y = B.bsr_matmul_i8(held(xq, pad, shift), one[:T], held(wq, pad, shift), one[:N])
    exact = xq.numpy().astype(np.int64) @ wq.numpy().astype(np.int64).T
    assert np.array_equal(host(y), exact.astype(np.float32))


# Outputs large enough for the largest tiles: ragged in both directions, a depth that ends inside a
# step, rows on and off 16-byte boundaries.
LARGE = [(3330, 4100, 144), (3330, 4100, 130), (4000, 2900, 64), (6100, 2048, 200), (6100, 2048, 208),
         (4090, 2040, 96), (4090, 2040, 99), (2040, 2044, 160), (2040, 2044, 167), (1020, 1024, 80),
         (1020, 1024, 77), (100, 1000, 2064), (64, 512, 1000), (127, 256, 777), (2040, 20470, 64),
         (4096, 5000, 64)]


@pytest.mark.parametrize("T,N,K", LARGE)
def test_matmul_i8_large(T, N, K):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T + K)
    xq, wq = (torch.randint(-128, 128, s, dtype=torch.int8, device=DEV, generator=gen)
              for s in ((T, K), (N, K)))
    one = torch.ones(max(T, N), device=DEV)
    Y, clean = frame(T, N, torch.float32, 4, 0)
    B.bsr_matmul_i8(xq, one[:T], wq, one[:N], Y=Y)
    assert torch.equal(Y.double(), xq.double() @ wq.double().t())      # below 2^24: exact
    assert clean()


@pytest.mark.parametrize("T,F,K", [(t, n // 2, k) for t, n, k in LARGE])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "i8"])
def test_gated_large(T, F, K, dtype):
    """Whole numbers, exact in every type, through forward and backward."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(F + K)
    x, wg, wu = (torch.randint(-2, 3, s, device=DEV, generator=gen).double()
                 for s in ((T, K), (F, K), (F, K)))
    g, u = x @ wg.t(), x @ wu.t()
    h = torch.clamp(g, min=0) * u
    assert h.abs().max() < 2 ** 24          # exact in fp32
    if dtype == "i8":
        one = torch.ones(max(T, F), device=DEV)
        H = B.bsr_gated_i8(x.to(torch.int8), one[:T], wg.to(torch.int8), one[:F], wu.to(torch.int8),
                           one[:F], act="relu", out_dtype=torch.float32)
        assert torch.equal(H.double(), h)
        return
    dt = TORCH[dtype]
    H, G, U = B.bsr_gated(x.to(dt), wg.to(dt), wu.to(dt), act="relu", save=True)
    assert torch.equal(G.double(), g) and torch.equal(U.double(), u)
    assert torch.equal(H, h.float().to(dt))


# Gradients whose outputs meet every tile (dX: T x K, the weights' 2 F x K), and some whose outputs are
# so few that their contraction is sliced (over F, or over T).
GRADIENTS = [(4090, 4088, 33), (6100, 2048, 20), (4090, 2040, 33), (2040, 2040, 17), (40, 4090, 2040),
             (50, 2040, 3050), (33, 2040, 2040), (70, 2040, 1020), (70, 40, 5000), (1, 264, 4100),
             (5000, 48, 40), (9000, 33, 30), (300, 200, 2111), (4096, 5000, 33), (2048, 20480, 24)]


@pytest.mark.parametrize("T,K,F", GRADIENTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_backward_large(T, K, F, dtype):
    """Whole numbers small enough that every sum is exact."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T + K + F)
    dt = TORCH[dtype]

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi + 1, shape, device=DEV, generator=gen).double()

    x, wg, wu, dh = ints(-2, 2, T, K), ints(-2, 2, F, K), ints(-2, 2, F, K), ints(-1, 1, T, F)
    g, u = ints(-3, 3, T, F), ints(-3, 3, T, F)
    dX, clean = frame(T, K, dt, 8, 0)
    got = B.bsr_gated_backward(dh.to(dt), x.to(dt), wg.to(dt), wu.to(dt), g.float(), u.float(),
                               act="relu", bias=True, grad_dtype=torch.float32, dX=dX)
    dg, du = dh * u * (g > 0), dh * torch.clamp(g, min=0)
    for t, want in zip(got, (dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dg.sum(0), du.sum(0))):
        assert torch.equal(t, want.float().to(t.dtype))
    assert clean()


def test_matmul_i8_longest_rows():
    """K = 131071 with every product at its largest: the sum comes to 2^31 - 2^14."""
    K = 131071
    x = torch.full((3, K), -128, dtype=torch.int8, device=DEV)
    w = torch.full((70, K), -128, dtype=torch.int8, device=DEV)
    one = torch.ones(70, device=DEV)
    y = B.bsr_matmul_i8(x, one[:3], w, one)
    assert torch.all(y == float(np.float32(16384 * K)))
    w.fill_(127)
    y = B.bsr_matmul_i8(x, one[:3], w, one)
    assert torch.all(y == float(np.float32(-16256 * K)))
    with pytest.raises(B.BSRError) as e:
        B.bsr_matmul_i8(torch.zeros((1, K + 1), dtype=torch.int8, device=DEV), one[:1],
                        torch.zeros((1, K + 1), dtype=torch.int8, device=DEV), one[:1])
    assert e.value.status == 9


def test_matmul_i8_row_scales_that_are_not_numbers():
    x = torch.randn(40, 96, device=DEV)
    x[3, 5], x[20, 0], x[7] = float("inf"), float("nan"), 0.0
    q, s = B.bsr_quantize_rows(x)
    wq, sw = B.bsr_quantize_rows(torch.randn(50, 96, device=DEV))
    y = B.bsr_matmul_i8(q, s, wq, sw)
    bad = torch.zeros(40, dtype=torch.bool, device=DEV)
    bad[[3, 20]] = True
    assert torch.equal(torch.isnan(y).all(1), bad) and torch.equal(torch.isnan(y).any(1), bad)
    assert torch.all(y[7] == 0)


# --- the gated block ----------------------------------------------------------------------------

GATED_SIZES = [(1, 1, 1), (1, 64, 96), (2, 33, 70), (4, 256, 64), (7, 1000, 40), (16, 100, 257),
               (17, 64, 129), (33, 48, 80), (64, 130, 64), (65, 96, 33), (128, 128, 128),
               (130, 257, 100), (257, 65, 160), (300, 72, 513), (512, 128, 384), (700, 320, 520)]


def block_inputs(T, K, F, dtype, bias):
    rng = np.random.default_rng(T * 7919 + K * 31 + F)
    x = rand(rng, T, K, dtype=dtype)
    wg, wu = (rand(rng, F, K, sigma=2.0 / K ** 0.5, dtype=dtype) for _ in range(2))
    b = [rand(rng, F) if bias else None for _ in range(2)]
    return rng, x, wg, wu, *b


@pytest.mark.parametrize("T,K,F", GATED_SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 3), (16, 8)])
def test_gated(T, K, F, dtype, pad, shift):
    act = ACTS[(T + K + F) % 4]
    _, x, wg, wu, bg, bu = block_inputs(T, K, F, dtype, T % 2 == 1)
    H, cleanh = frame(T, F, TORCH[dtype], pad, shift)
    G, cleang = frame(T, F, torch.float32, pad, shift)
    U, cleanu = frame(T, F, torch.float32, pad, shift)
    args = (held(x, pad, shift), held(wg, pad, shift), held(wu, pad, shift),
            *(None if b is None else b.to(DEV) for b in (bg, bu)))
    B.bsr_gated(*args, act=act, H=H, G=G, U=U)
    wh, wg_, wu_, eh, eg, eu = D.gated(f64(x), f64(wg), f64(wu), *(None if b is None else f64(b)
                                                                  for b in (bg, bu)), act, dtype)
    within(G, wg_, eg, "G")
    within(U, wu_, eu, "U")
    within(H, wh, eh, "H")
    assert cleanh() and cleang() and cleanu()
    assert torch.equal(B.bsr_gated(*args, act=act), H)      # without saving: the same values


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_activations(act, dtype):
    """Every activation over a wide range of pre-activations, exact ones (a one-hot product)."""
    F = 128
    g = torch.linspace(-30, 30, 96 * F).view(96, F).to(TORCH[dtype])
    x = torch.cat([torch.eye(96), torch.zeros(96, 32)], 1).to(TORCH[dtype])
    wg = torch.zeros(F, 128, dtype=TORCH[dtype])
    wg[:, :96] = g.t()
    wu = torch.full((F, 128), 0.75, dtype=TORCH[dtype])
    H, G, U = B.bsr_gated(x.to(DEV), wg.to(DEV), wu.to(DEV), act=act, save=True)
    assert np.array_equal(f64(G), f64(g)) and torch.all(U == 0.75)
    want, bound = D.gated_of(f64(g), np.full((96, F), 0.75), 0.0, 0.0, act, dtype)
    within(H, want, bound, act)


@pytest.mark.parametrize("T,K,F", GATED_SIZES)
@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                        ("f32", "bf16")])
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 3)])
def test_gated_backward(T, K, F, dtype, grad, pad, shift):
    act = ACTS[(T + K + F) % 4]
    rng, x, wg, wu, _, _ = block_inputs(T, K, F, dtype, False)
    dh = rand(rng, T, F, dtype=dtype)
    g, u = rand(rng, T, F, sigma=2.0), rand(rng, T, F)
    outs = {"dX": frame(T, K, TORCH[dtype], pad, shift), "dWg": frame(F, K, TORCH[grad], pad, shift),
            "dWu": frame(F, K, TORCH[grad], pad, shift)}
    args = (held(dh, pad, shift), held(x, pad, shift), held(wg, pad, shift), held(wu, pad, shift),
            held(g, pad, shift), held(u, pad, shift))
    got = B.bsr_gated_backward(*args, act=act, bias=True, grad_dtype=TORCH[grad],
                               **{k: v[0] for k, v in outs.items()})
    want = D.gated_backward(f64(dh), f64(x), f64(wg), f64(wu), f64(g), f64(u), act, dtype, grad)
    for name, t in zip(("dX", "dWg", "dWu", "dbg", "dbu"), got):
        assert t.dtype == TORCH[dtype if name == "dX" else grad]
        within(t, *want[name], name)
    assert all(v[1]() for v in outs.values())
    again = B.bsr_gated_backward(*args, act=act, bias=True, grad_dtype=TORCH[grad])
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    # what is not wanted does not change the rest
    only = B.bsr_gated_backward(*args, act=act, need=("X",), grad_dtype=TORCH[grad])
    assert torch.equal(only[0], got[0]) and only[1:] == (None, None, None, None)
    only = B.bsr_gated_backward(*args, act=act, need=("W",), grad_dtype=TORCH[grad])
    assert only[0] is None and torch.equal(only[1], got[1]) and torch.equal(only[2], got[2])
    only = B.bsr_gated_backward(*args, act=act, need=(), bias=True, grad_dtype=TORCH[grad])
    assert torch.equal(only[3], got[3]) and torch.equal(only[4], got[4]) and only[0] is None


@pytest.mark.parametrize("T", [1, 63, 1024, 1025, 5000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", [1, 37])
def test_bias_gradients_of_many_tokens_are_exact(T, F, dtype):
    """Whole numbers of at most 4 and relu: every partial sum is a whole number below 2^24."""
    rng = np.random.default_rng(T + F)
    x, wg, wu, dh, g, u = (torch.from_numpy(rng.integers(-2, 3, s).astype(np.float32)) for s in
                           ((T, 3), (F, 3), (F, 3), (T, F), (T, F), (T, F)))
    b = lambda t: t.to(TORCH[dtype]).to(DEV)  # noqa: E731
    out = B.bsr_gated_backward(b(dh), b(x), b(wg), b(wu), g.to(DEV), u.to(DEV), act="relu", bias=True,
                               need=(), grad_dtype=torch.float32)
    dH, G, U = (t.double().numpy() for t in (dh, g, u))
    assert np.array_equal(f64(out[3]), (dH * U * (G > 0)).sum(0))
    assert np.array_equal(f64(out[4]), (dH * np.maximum(G, 0)).sum(0))


@pytest.mark.parametrize("T,K,F", [(5, 7, 9), (64, 64, 64), (100, 130, 70), (260, 200, 300)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_integers_are_exact(T, K, F, dtype):
    """Small integers and relu: every sum and product is exact, so a misplaced, doubled or missing
    term shows in the last bit."""
    rng = np.random.default_rng(T)
    ints = [torch.from_numpy(rng.integers(-2, 3, s).astype(np.float32)) for s in
            ((T, K), (F, K), (F, K), (T, F))]
    x, wg, wu, dh = (held(t.to(TORCH[dtype]), 1, 1) for t in ints)
    X, Wg, Wu, dH = (t.double().numpy() for t in ints)
    H, G, U = B.bsr_gated(x, wg, wu, act="relu", save=True)
    g, u = X @ Wg.T, X @ Wu.T
    assert np.array_equal(f64(G), g) and np.array_equal(f64(U), u)
    h = torch.from_numpy(np.maximum(g, 0) * u).float().to(TORCH[dtype])
    assert torch.equal(H.cpu(), h)
    # saved values small enough that dG and dU are whole numbers below 2^8, exact in bf16
    gi, ui = np.clip(g, -3, 3), np.clip(u, -3, 3)
    to = lambda a: torch.from_numpy(a).float().to(DEV)  # noqa: E731
    out = B.bsr_gated_backward(dh, x, wg, wu, to(gi), to(ui), act="relu", bias=True,
                               grad_dtype=torch.float32)
    dG, dU = dH * ui * (gi > 0), dH * np.maximum(gi, 0)
    for t, want in zip(out, (dG @ Wg + dU @ Wu, dG.T @ X, dU.T @ X, dG.sum(0), dU.sum(0))):
        want = torch.from_numpy(want).float().to(t.dtype)
        assert torch.equal(t.cpu(), want)


def test_no_tokens():
    w = torch.randn(24, 40, device=DEV)
    x, e = torch.zeros(0, 40, device=DEV), torch.zeros(0, 24, device=DEV)
    assert B.bsr_gated(x, w, w).shape == (0, 24)
    dX, dWg, dWu, dbg, dbu = B.bsr_gated_backward(e, x, w, w, e, e, bias=True)
    assert dX.shape == (0, 40)
    assert all(torch.all(t == 0) for t in (dWg, dWu, dbg, dbu))
    q, s = B.bsr_quantize_rows(x)
    wq, sw = B.bsr_quantize_rows(w)
    assert q.shape == (0, 40) and s.shape == (0,)
    assert B.bsr_matmul_i8(q, s, wq, sw).shape == (0, 24)
    assert B.bsr_gated_i8(q, s, wq, sw, wq, sw).shape == (0, 24)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 40, 300])
def test_gated_non_finite_values_stay_in_their_rows(dtype, T):
    """An infinity or a NaN in a token reaches that token's outputs and no other's."""
    rng = np.random.default_rng(11)
    x, w = rand(rng, T, 96, dtype=dtype), rand(rng, 80, 96, dtype=dtype)
    clean = B.bsr_gated(x.to(DEV), w.to(DEV), w.to(DEV))
    x[0, 17] = float("nan")
    if T > 1:
        x[T - 2, 95] = float("inf")
    H, G, U = B.bsr_gated(x.to(DEV), w.to(DEV), w.to(DEV), save=True)
    assert torch.isnan(H[0]).all()
    keep = [t for t in range(T) if t not in (0, T - 2)]
    assert torch.equal(H[keep], clean[keep])
    if T > 1:
        assert not torch.isfinite(G[T - 2]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 40, 300])
def test_gated_non_finite_weights_stay_in_their_channels(dtype, T):
    rng = np.random.default_rng(12)
    x = rand(rng, T, 100, dtype=dtype).to(DEV)
    wg, wu = (rand(rng, 90, 100, dtype=dtype).to(DEV) for _ in range(2))
    clean, G0, U0 = B.bsr_gated(x, wg, wu, save=True)
    wg[7, 3], wu[50, 99], wu[89, 0] = float("inf"), float("nan"), -3.4e38
    H, G, U = B.bsr_gated(x, wg, wu, save=True)
    assert not torch.isfinite(G[:, 7]).any() and torch.isnan(U[:, 50]).all()
    keep = [f for f in range(90) if f not in (7, 50, 89)]
    assert torch.equal(H[:, keep], clean[:, keep])
    assert torch.equal(G[:, 50], G0[:, 50]) and torch.equal(U[:, 7], U0[:, 7])


def test_offsets_past_32_bits():
    """Rows that start more than 2^31 and 2^32 bytes into their matrices."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    pitch, T, K, F = 1 << 20, 2200, 40, 48                # int8 rows a MiB apart; bf16 two
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    ints = lambda *s: torch.randint(-2, 3, s, device=DEV, generator=gen)  # noqa: E731
    small, w = ints(T, K), ints(F, K)
    one = torch.ones(T, device=DEV)
    want = small.double() @ w.double().t()
    x8 = torch.empty(T, pitch, dtype=torch.int8, device=DEV)[:, :K]
    x8.copy_(small)
    y = torch.empty(T, pitch, dtype=torch.bfloat16, device=DEV)[:, :F]
    B.bsr_matmul_i8(x8, one, w.to(torch.int8), one[:F], Y=y)
    assert torch.equal(y.double(), want)
    q, s = B.bsr_quantize_rows(y)
    wq, ws = D.quantize_rows(y.float().cpu().numpy())
    assert np.array_equal(host(q), wq) and np.array_equal(host(s), ws)
    del x8
    x = torch.empty(T, pitch, dtype=torch.bfloat16, device=DEV)[:, :K]
    x.copy_(small)
    wb = w.to(torch.bfloat16)
    H, G, U = B.bsr_gated(x, wb, wb, act="relu", save=True, H=y)
    assert torch.equal(G.double(), want) and torch.equal(U.double(), want)
    assert torch.equal(H, (torch.clamp(want, min=0) * want).float().to(torch.bfloat16))
    y.fill_(1)
    grads = B.bsr_gated_backward(y, x, wb, wb, torch.ones_like(G), torch.ones_like(U), act="relu",
                                 grad_dtype=torch.float32, dX=x.clone())
    ones = torch.ones(T, F, dtype=torch.float64, device=DEV)
    assert torch.equal(grads[0].double(), 2 * ones @ w.double())
    assert torch.equal(grads[1].double(), ones.t() @ small.double())


@pytest.mark.parametrize("T,K,F", GATED_SIZES + [(16, 2048, 512)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 3), (16, 16)])
def test_gated_i8(T, K, F, out, pad, shift):
    act = ACTS[(T + K + F) % 4]
    rng = np.random.default_rng(T * 7919 + K * 31 + F)
    xq, wgq, wuq = (torch.from_numpy(rng.integers(-127, 128, s).astype(np.int8))
                    for s in ((T, K), (F, K), (F, K)))
    scale = 1.0 / (73.0 * K ** 0.5)
    sx = torch.from_numpy(rng.uniform(0.5, 2.0, T).astype(np.float32))
    sg, su = (torch.from_numpy((rng.uniform(0.5, 2.0, F) * scale / 73.0).astype(np.float32))
              for _ in range(2))
    bg, bu = (rand(rng, F) if F % 2 else None for _ in range(2))
    H, clean = frame(T, F, TORCH[out], pad, shift)
    dev = [None if t is None else t.to(DEV) for t in (sx, sg, su, bg, bu)]
    B.bsr_gated_i8(held(xq, pad, shift), dev[0], held(wgq, pad, shift), dev[1],
                   held(wuq, pad, shift), dev[2], dev[3], dev[4], act=act, H=H)
    G, eg = D.matmul_i8(xq.numpy(), sx.numpy(), wgq.numpy(), sg.numpy(),
                        None if bg is None else bg.numpy())
    U, eu = D.matmul_i8(xq.numpy(), sx.numpy(), wuq.numpy(), su.numpy(),
                        None if bu is None else bu.numpy())
    want, bound = D.gated_of(G, U, eg, eu, act, out)
    within(H, want, bound, "H")
    assert clean()


# --- streams, graphs, devices -------------------------------------------------------------------

def _step(x, wg, wu, dh, ws):
    H, G, U = B.bsr_gated(x, wg, wu, save=True)
    grads = B.bsr_gated_backward(dh, x, wg, wu, G, U, bias=True, workspace=ws)
    q, s = B.bsr_quantize_rows(x)
    gq, gs = B.bsr_quantize_rows(wg)
    uq, us = B.bsr_quantize_rows(wu)
    h8 = B.bsr_gated_i8(q, s, gq, gs, uq, us)
    y8 = B.bsr_matmul_i8(q, s, gq, gs)
    return [H, *grads, h8, y8]


@pytest.mark.parametrize("T,K,F", [(3, 40, 24), (70, 33, 65), (150, 64, 128)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_arrays_side_by_side_in_one_buffer(T, K, F, dtype):
    """X beside H, G beside U, dWg beside dWu and dH beside dX, as columns of one buffer each, give what
    arrays of their own give."""
    rng, x, wg, wu, _, _ = block_inputs(T, K, F, dtype, False)
    dt = TORCH[dtype]
    x, wg, wu, dh = (t.to(dt).to(DEV) for t in (x, wg, wu, rand(rng, T, F, dtype=dtype)))
    want = B.bsr_gated(x, wg, wu, save=True)
    want += B.bsr_gated_backward(dh, x, wg, wu, want[1], want[2])[:3]
    xh, gu = torch.zeros(T, K + F, dtype=dt, device=DEV), torch.zeros(T, 2 * F, device=DEV)
    dw, dd = torch.zeros(F, 2 * K, dtype=dt, device=DEV), torch.zeros(T, F + K, dtype=dt, device=DEV)
    xh[:, :K] = x
    dd[:, :F] = dh
    got = B.bsr_gated(xh[:, :K], wg, wu, H=xh[:, K:], G=gu[:, :F], U=gu[:, F:])
    got += B.bsr_gated_backward(dd[:, :F], xh[:, :K], wg, wu, gu[:, :F], gu[:, F:], dX=dd[:, F:],
                                dWg=dw[:, :K], dWu=dw[:, K:])[:3]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(xh[:, :K], x) and torch.equal(dd[:, :F], dh)


@pytest.mark.parametrize("T", [3, 150])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(T, dtype):
    K, F = 200, 168
    rng = np.random.default_rng(4)
    x, wg, wu, dh = (rand(rng, *s, dtype=dtype).to(DEV) for s in
                     ((T, K), (F, K), (F, K), (T, F)))
    ws = torch.empty(B.bsr_gated_workspace_bytes(T, K, F, TORCH[dtype]), dtype=torch.uint8,
                     device=DEV)
    _step(x, wg, wu, dh, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _step(x, wg, wu, dh, ws)
    for n in range(4):
        x.copy_(rand(rng, T, K, dtype=dtype))
        dh.copy_(rand(rng, T, F, dtype=dtype))
        graph.replay()
        got = [t.clone() for t in outs]
        torch.cuda.synchronize()
        want = _step(x, wg, wu, dh, None)          # eager work between the replays
        assert all(torch.equal(a, b) for a, b in zip(got, want)), n


def test_side_streams():
    """Calls on streams of their own, by object and by handle, at the same time as each other."""
    rng = np.random.default_rng(8)
    K, F = 320, 256
    sets = [tuple(rand(rng, *s, dtype="bf16").to(DEV) for s in ((T, K), (F, K), (F, K), (T, F)))
            for T in (100, 37)]
    want = [_step(*s, None) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for (x, wg, wu, dh), st in zip(sets, (streams[0], streams[1].cuda_stream)):
        H, G, U = B.bsr_gated(x, wg, wu, save=True, stream=st)
        grads = B.bsr_gated_backward(dh, x, wg, wu, G, U, bias=True, stream=st)
        q, s = B.bsr_quantize_rows(x, stream=st)
        gq, gs = B.bsr_quantize_rows(wg, stream=st)
        uq, us = B.bsr_quantize_rows(wu, stream=st)
        got.append([H, *grads, B.bsr_gated_i8(q, s, gq, gs, uq, us, stream=st),
                    B.bsr_matmul_i8(q, s, gq, gs, stream=st)])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_trained_pruned_and_served():
    """The operators as they are used together: gradients of the block feed fp32 master weights, the
    trained gate projection is pruned by the library's block prune, the dense block is served in 8
    bits, its down projection as a block-sparse product and as an 8-bit one."""
    rng = np.random.default_rng(21)
    T, K, F = 192, 128, 256
    x = rand(rng, T, K).to(DEV)
    wg, wu = (rand(rng, F, K, sigma=0.1).to(DEV) for _ in range(2))
    wd = rand(rng, K, F, sigma=0.1).to(DEV)
    dh = rand(rng, T, F, sigma=0.1).to(DEV)
    H, G, U = B.bsr_gated(x, wg, wu, act="gelu", save=True)
    _, dwg, dwu, _, _ = B.bsr_gated_backward(dh, x, wg, wu, G, U, act="gelu",
                                             grad_dtype=torch.float32)
    # W - eta grad by the library's update (its gradient operand is stored K x F)
    zero = torch.zeros(K, F, device=DEV)
    new = B.bsr_iht_update(wg, dwg.t().contiguous(), zero, 0.01)
    want = D.gated_backward(f64(dh), f64(x), f64(wg), f64(wu), f64(G), f64(U), "gelu")["dWg"]
    step = f64(wg) - 0.01 * want[0]
    within(new, step, 0.01 * want[1] + 3 * D.U32 * (np.abs(f64(wg)) + np.abs(step)), "update")
    M = B.bsr_prune_from_dense(new, 16, 16, density=0.5)
    Wp = B.bsr_to_dense(M)
    hp = B.bsr_gated(x, Wp, wu, act="gelu")               # pruned gate, dense form
    gate = B.bsr_spmm(x, M)                               # and its block-sparse product
    want_h, _, _, eh, _, _ = D.gated(f64(x), f64(Wp), f64(wu), name="gelu")
    within(hp, want_h, eh, "pruned block")
    eg = (K + 2) * D.U32 * (np.abs(f64(x)) @ np.abs(f64(Wp)).T) + D.TINY
    within(gate, f64(x) @ f64(Wp).T, eg, "block-sparse gate")
    # served: 8-bit rows in and out of the block
    xq, sx = B.bsr_quantize_rows(x)
    gq, sg = B.bsr_quantize_rows(Wp)
    uq, su = B.bsr_quantize_rows(wu)
    dq, sd = B.bsr_quantize_rows(wd)
    h8 = B.bsr_gated_i8(xq, sx, gq, sg, uq, su, act="gelu")
    hq, sh = B.bsr_quantize_rows(h8)
    y8 = B.bsr_matmul_i8(hq, sh, dq, sd)
    full = B.bsr_prune_from_dense(wd, 16, 16, density=1.0)
    y = B.bsr_spmm(hp, full)
    # each operand is off by at most half a step of its row's scale: sum of (max|a| |b| + |a| max|b|)
    # / 254 over the terms, for both layers
    def layer(a, w, ea):
        ea = np.broadcast_to(ea, a.shape)
        ra = ea + np.max(np.abs(a) + ea, 1, keepdims=True) / 254 * 1.0001
        rw = np.broadcast_to(np.max(np.abs(w), 1, keepdims=True) / 254 * 1.0001, w.shape)
        return ra @ np.abs(w).T + (np.abs(a) + ra) @ rw.T
    X, P, Wu_, Wd = f64(x), f64(Wp), f64(wu), f64(wd)
    Gp, Up = X @ P.T, X @ Wu_.T
    e_g, e_u = layer(X, P, 0.0), layer(X, Wu_, 0.0)
    a, _ = D.act("gelu", Gp)
    e_h = D.ACT_SLOPE * e_g * (np.abs(Up) + e_u) + np.abs(a) * e_u
    e_h = e_h * 1.01 + 2.0 ** -8 * np.abs(a * Up)
    assert np.all(np.abs(f64(h8) - want_h) <= e_h + 1e-5)
    e_y = layer(a * Up, Wd, e_h)
    assert np.all(np.abs(f64(y8) - f64(y)) <= 1.01 * e_y + 1e-4)
