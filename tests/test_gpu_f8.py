"""Matrices in 8-bit floating point and their product on the GPU: codes and scales bit for bit as the
oracle defines them, products within bounds that count the roundings of fp32 (oracle/f8_oracle.py) and bit
for bit where every operation is exact."""
import numpy as np
import pytest
import torch

from oracle import f8_oracle as F
from paper_2106_08846_amd import bsr as B
from tests.gpu_common import host
from tests.test_gpu_dense import DEV, TORCH, f64, held, rand, within

pytestmark = pytest.mark.gpu

F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def bits(t):
    return host(t.contiguous().view(torch.uint8))


def codes(q, fmt, pad=0, shift=0, gap=0x7F):
    """Codes (uint8) on the device at pitch width + pad, `shift` bytes into their storage; NaN between."""
    T, K = q.shape
    buf = torch.full((T * (K + pad) + shift + 8,), gap, dtype=torch.uint8, device=DEV)
    view = buf[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K]
    view.copy_(torch.from_numpy(q))
    return view.view(F8[fmt])


def code_frame(T, K, fmt, pad, shift):
    buf = torch.full((T * (K + pad) + shift + 64,), 77, dtype=torch.uint8, device=DEV)
    view = buf[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K]

    def untouched():
        copy = buf.clone()
        copy[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K] = 77
        return bool((copy == 77).all())
    return view.view(F8[fmt]), untouched


def check_codes(x, q, scale, rows, fmt):
    want, want_s = F.quantize(x, rows, fmt)
    assert np.array_equal(bits(q), want)
    got = host(scale)
    assert got.shape == want_s.shape
    assert np.array_equal(np.isnan(got), np.isnan(want_s))
    ok = ~np.isnan(want_s)
    assert np.array_equal(got[ok].view(np.uint32), want_s[ok].view(np.uint32))


@pytest.mark.parametrize("T,K", [(1, 1), (1, 128), (2, 129), (3, 770), (16, 512), (17, 513), (128, 128),
                                 (129, 127), (300, 1000), (5, 4096), (127, 259), (256, 384)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,fmt", [(1, "e4m3"), (1, "e5m2"), (128, "e4m3"), (128, "e5m2")])
def test_quantize(T, K, dtype, rows, fmt):
    rng = np.random.default_rng(T * 100003 + K)
    x = rand(rng, T, K, dtype=dtype) * torch.from_numpy(
        np.exp(rng.uniform(-20, 20, (T, 1))).astype(np.float32)).to(TORCH[dtype])
    xn = x.float().numpy()
    for pad, shift in ((0, 0), (3, 1)):
        X = held(x, pad, shift)
        q, clean = code_frame(T, K, fmt, pad, shift)
        qt, clean_t = code_frame(K, T, fmt, pad, shift)
        Q, s, QT, st = B.bsr_quantize_f8(X, rows, F8[fmt], "both", Q=q, QT=qt)
        check_codes(xn, Q, s, rows, fmt)
        check_codes(np.ascontiguousarray(xn.T), QT, st, rows, fmt)
        assert clean() and clean_t()
        only, only_s = B.bsr_quantize_f8(X, rows, F8[fmt])
        assert np.array_equal(bits(only), bits(Q)) and torch.equal(only_s, s)
        only, only_s = B.bsr_quantize_f8(X, rows, F8[fmt], "columns")
        assert np.array_equal(bits(only), bits(QT)) and torch.equal(only_s, st)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_special_values(dtype, fmt, rows):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((9 * rows, 300)).astype(np.float32)
    at = lambda i: i * rows                           # noqa: E731  the first row of block row i
    x[at(0):at(1)] = 0.0
    x[at(1), 299] = np.inf
    x[at(2), 0] = -np.inf
    x[at(3), 130] = np.nan
    x[at(4):at(5)] *= np.float32(2.0 ** -130)         # subnormal blocks
    x[at(5):at(6)] = np.float32(2.0 ** -133)
    x[at(6):at(7)] *= np.float32(1e37)
    x[at(7), 0], x[at(7), 5] = np.inf, np.nan
    x[at(8):] = -0.0
    # ties and the largest value exactly: 448 and 57344 are 1.75 times a power of two
    x[at(6), :128] = np.arange(128, dtype=np.float32) * np.float32(1.75 / 127)
    t = torch.from_numpy(x).to(TORCH[dtype])
    Q, s, QT, st = B.bsr_quantize_f8(t.to(DEV), rows, F8[fmt], "both")
    check_codes(t.float().numpy(), Q, s, rows, fmt)
    check_codes(np.ascontiguousarray(t.float().numpy().T), QT, st, rows, fmt)


def test_quantize_long_offsets():
    T, K, pitch = 2200, 200, 1 << 20
    x = rand(np.random.default_rng(9), T, K, dtype="bf16")
    buf = torch.empty(T * pitch, dtype=torch.bfloat16, device=DEV)
    X = buf.view(T, pitch)[:, :K]
    X.copy_(x)
    out = torch.empty(T * pitch, dtype=torch.uint8, device=DEV).view(T, pitch)[:, :K].view(F8["e4m3"])
    Q, s, QT, st = B.bsr_quantize_f8(X, form="both", Q=out)
    check_codes(x.float().numpy(), Q, s, 1, "e4m3")
    check_codes(np.ascontiguousarray(x.float().numpy().T), QT, st, 1, "e4m3")


# --- product ------------------------------------------------------------------------------------

# Token counts around the small-batch and tile sizes; widths around blocks of 128 and chunks of 16.
SIZES = [(1, 1, 1), (1, 64, 128), (1, 100, 1000), (2, 33, 770), (4, 4096, 64), (7, 16, 4096),
         (16, 257, 256), (17, 129, 255), (32, 64, 2048), (33, 96, 129), (63, 100, 96), (64, 256, 384),
         (65, 255, 130), (128, 128, 1024), (130, 640, 48), (257, 130, 514), (300, 513, 1),
         (512, 1024, 256), (1100, 1300, 192), (3, 5, 20001)]


def random_codes(rng, T, K, fmt):
    """Any finite code."""
    table = F.values(fmt)
    fine = np.nonzero(np.isfinite(table))[0].astype(np.uint8)
    return fine[rng.integers(0, len(fine), (T, K))]


def product_case(rng, T, N, K, rows, x_fmt):
    xq, wq = random_codes(rng, T, K, x_fmt), random_codes(rng, N, K, "e4m3")
    kb = -(-K // 128)
    sx = np.exp(rng.uniform(-8, 2, (kb, T))).astype(np.float32)
    sw = np.exp(rng.uniform(-8, 2, (kb, -(-N // rows)))).astype(np.float32)
    return xq, sx, wq, sw


@pytest.mark.parametrize("T,N,K", SIZES)
@pytest.mark.parametrize("rows,x_fmt", [(128, "e4m3"), (1, "e4m3"), (128, "e5m2"), (1, "e5m2")])
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 3), (16, 16), (-1, 0)])
def test_matmul(T, N, K, rows, x_fmt, pad, shift):
    """pad -1: rows on 16-byte boundaries, whatever their width."""
    rng = np.random.default_rng(T * 7919 + N * 31 + K + rows)
    xq, sx, wq, sw = product_case(rng, T, N, K, rows, x_fmt)
    pad = -K % 16 if pad < 0 else pad
    bias = rand(rng, N) if (T + N) % 2 else None
    out = ["f32", "bf16"][(T + K) % 2]
    buf = torch.full((T * (N + 5) + 64,), 77, dtype=TORCH[out], device=DEV)
    Y = buf[3:3 + T * (N + 5)].view(T, N + 5)[:, :N]
    y = B.bsr_matmul_f8(codes(xq, x_fmt, pad, shift), held(torch.from_numpy(sx), 2, 1),
                        codes(wq, "e4m3", pad, shift), held(torch.from_numpy(sw), 1, 3),
                        None if bias is None else bias.to(DEV), Y=Y)
    want, bound = F.matmul(xq, sx, wq, sw, rows, None if bias is None else bias.numpy(), x_fmt, out)
    within(y, want, bound, "Y")
    copy = buf.clone()
    copy[3:3 + T * (N + 5)].view(T, N + 5)[:, :N] = 77
    assert bool((copy == 77).all())
    again = B.bsr_matmul_f8(codes(xq, x_fmt, pad, shift), torch.from_numpy(sx).to(DEV),
                            codes(wq, "e4m3", pad, shift), torch.from_numpy(sw).to(DEV),
                            None if bias is None else bias.to(DEV), out_dtype=TORCH[out])
    assert torch.equal(again, y)


@pytest.mark.parametrize("T,N,K", [(1, 4500, 4301), (16, 5000, 4232), (17, 4201, 2500), (32, 9000, 301),
                                   (5, 5003, 130), (32, 64, 9001), (64, 500, 4500), (2, 12300, 512)])
@pytest.mark.parametrize("rows,x_fmt", [(128, "e4m3"), (1, "e5m2")])
@pytest.mark.parametrize("pad,shift", [(1, 3), (-1, 0)])
def test_matmul_few_tokens(T, N, K, rows, x_fmt, pad, shift):
    """More channels than a round of the chip holds, more blocks than a workgroup's waves take at once."""
    test_matmul(T, N, K, rows, x_fmt, pad, shift)


@pytest.mark.parametrize("T,N,K", [(4096, 4096, 272), (1536, 8192, 389), (2050, 4099, 389), (4900, 4096, 272),
                                   (4096, 4096, 2064), (1536, 8192, 2053), (2048, 4096, 4112),
                                   (3136, 8192, 2053)])
@pytest.mark.parametrize("rows,x_fmt", [(128, "e4m3"), (1, "e5m2")])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 7, -1])
def test_matmul_large_tiles(T, N, K, rows, x_fmt, out, pad):
    """Sizes that take each of the larger tiles, on and off 16-byte boundaries (pad -1: on), and two
    launches; tokens from every part of the grid."""
    rng = np.random.default_rng(T + N + K)
    pad = -K % 16 if pad < 0 else pad
    xq, sx, wq, sw = product_case(rng, T, N, K, rows, x_fmt)
    bias = rand(rng, N)
    y = B.bsr_matmul_f8(codes(xq, x_fmt, pad), torch.from_numpy(sx).to(DEV), codes(wq, "e4m3", pad),
                        torch.from_numpy(sw).to(DEV), bias.to(DEV), out_dtype=TORCH[out])
    t = np.unique(np.concatenate([np.arange(0, T, 167 if K < 1000 else 977), [T - 1, 127, 128, 191, 255, 256]]))
    want, bound = F.matmul(xq[t], sx[:, t], wq, sw, rows, bias.numpy(), x_fmt, out)
    within(y[torch.from_numpy(t).to(DEV)], want, bound, "Y")
    # the codes of integers, whose sums are exact, over the whole of it
    x, w = (torch.from_numpy(rng.integers(-4, 5, s).astype(np.float32)) for s in ((T, K), (N, K)))
    sx[:], sw[:] = 0.5, 0.25

    def small(v, fmt):
        return codes(v.to(F8[fmt]).view(torch.uint8).numpy(), fmt, pad)
    one = B.bsr_matmul_f8(small(x, x_fmt), torch.from_numpy(sx).to(DEV), small(w, "e4m3"),
                          torch.from_numpy(sw).to(DEV), out_dtype=TORCH[out])
    exact = (x.to(DEV) @ w.to(DEV).t()) * 0.125
    assert torch.equal(one, exact.to(TORCH[out]))


@pytest.mark.parametrize("T,N,K", [(200, 1000, 2048), (257, 520, 2170), (150, 1100, 2200), (513, 1024, 8700),
                                   (512, 1000, 8200), (130, 2050, 8400), (193, 900, 8500)])
@pytest.mark.parametrize("rows,x_fmt", [(128, "e4m3"), (1, "e5m2")])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, -1])
def test_matmul_long_contractions(T, N, K, rows, x_fmt, out, pad):
    """Few tiles and many blocks of columns, whose number parts of a workgroup's waves may not divide."""
    rng = np.random.default_rng(T + N + K)
    pad = -K % 16 if pad < 0 else pad
    xq, sx, wq, sw = product_case(rng, T, N, K, rows, x_fmt)
    bias = rand(rng, N)
    y = B.bsr_matmul_f8(codes(xq, x_fmt, pad), torch.from_numpy(sx).to(DEV), codes(wq, "e4m3", pad),
                        torch.from_numpy(sw).to(DEV), bias.to(DEV), out_dtype=TORCH[out])
    t = np.unique(np.append(np.arange(0, T, 41), [63, 64, 127, 128, T - 1]))
    want, bound = F.matmul(xq[t], sx[:, t], wq, sw, rows, bias.numpy(), x_fmt, out)
    within(y[torch.from_numpy(t).to(DEV)], want, bound, "Y")
    # integers and powers of two, whose sums are exact, over the whole of it
    x, w = (torch.from_numpy(rng.integers(-4, 5, s).astype(np.float32)) for s in ((T, K), (N, K)))
    sx[:], sw[:] = 0.5, 0.25
    x8, w8 = (codes(v.to(F8[f]).view(torch.uint8).numpy(), f, pad) for v, f in ((x, x_fmt), (w, "e4m3")))
    one = B.bsr_matmul_f8(x8, torch.from_numpy(sx).to(DEV), w8, torch.from_numpy(sw).to(DEV),
                          out_dtype=TORCH[out])
    exact = (x.to(DEV) @ w.to(DEV).t()) * 0.125
    assert torch.equal(one, exact.to(TORCH[out]))


@pytest.mark.parametrize("T,N,K", [(8, 40, 2170), (200, 1000, 2170), (300, 700, 8200), (1100, 1300, 700)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("pad", [3, -1])
def test_scales_whose_product_overflows(T, N, K, out, rows, pad):
    """sx sw is formed first: where it passes the largest fp32 value the outputs are infinite, not NaN."""
    pad = -K % 16 if pad < 0 else pad
    kb = -(-K // 128)
    sx = torch.ones(kb, T, device=DEV)
    sw = torch.ones(kb, -(-N // rows), device=DEV)
    sx[kb - 1], sw[kb - 1] = 2.0 ** 70, 2.0 ** 70
    x, w = (codes(F.encode(np.ones(s, np.float32), "e4m3"), "e4m3", pad) for s in ((T, K), (N, K)))
    y = B.bsr_matmul_f8(x, sx, w, sw, out_dtype=TORCH[out])
    assert bool((y == float("inf")).all())


@pytest.mark.parametrize("T,N,K", [(1, 48, 4096), (19, 70, 770), (200, 300, 1000), (600, 700, 512)])
@pytest.mark.parametrize("rows", [1, 128])
def test_matmul_exact(T, N, K, rows):
    """Small integers and scales that are powers of two: every product and sum is exact."""
    rng = np.random.default_rng(K)
    x, w = (rng.integers(-4, 5, s).astype(np.float32) for s in ((T, K), (N, K)))
    kb = -(-K // 128)
    sx = (2.0 ** rng.integers(-1, 2, (kb, T))).astype(np.float32)
    sw = (2.0 ** rng.integers(-1, 2, (kb, -(-N // rows)))).astype(np.float32)
    xq, wq = F.encode(x, "e4m3"), F.encode(w, "e4m3")
    Y = B.bsr_matmul_f8(codes(xq, "e4m3"), torch.from_numpy(sx).to(DEV), codes(wq, "e4m3"),
                        torch.from_numpy(sw).to(DEV))
    want, _ = F.matmul(xq, sx, wq, sw, rows)
    assert np.array_equal(f64(Y), want)


@pytest.mark.parametrize("T,N,K", [(5, 40, 300), (150, 200, 300), (700, 600, 1024)])
def test_matmul_not_finite(T, N, K):
    """A NaN or infinite scale, or a NaN code, reaches every output of its token or channel and no other;
    what lies between the rows reaches none."""
    rng = np.random.default_rng(3)
    xq, sx, wq, sw = product_case(rng, T, N, K, 1, "e5m2")
    clean = F.matmul(xq, sx, wq, sw, 1, x_fmt="e5m2")
    sx[0, 1], sx[1, 3], sw[2, 7] = np.nan, np.inf, np.nan
    xq[1], xq[3], xq[4, K - 1], wq[11, 17] = 0, 0, 0x7F, 0x7F
    Y = f64(B.bsr_matmul_f8(codes(xq, "e5m2", 5), torch.from_numpy(sx).to(DEV), codes(wq, "e4m3", 5),
                            torch.from_numpy(sw).to(DEV)))
    bad = np.zeros((T, N), bool)
    bad[[1, 3, 4]] = True
    bad[:, [7, 11]] = True
    assert np.array_equal(np.isnan(Y), bad)
    assert np.all((np.abs(Y - clean[0]) <= clean[1])[~bad])


@pytest.mark.parametrize("T,N,K", [(5, 40, 300), (150, 200, 300), (260, 600, 2300), (700, 1500, 200)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [5, -1])
def test_codes_that_are_not_finite(T, N, K, out, pad):
    """A NaN code of a token or a channel gives NaN there; an infinite code of a token (E5M2) infinities of
    its products' signs, NaN where the channel's code is 0; the rest stays within its bound."""
    rng = np.random.default_rng(T + K)
    pad = -K % 16 if pad < 0 else pad
    xq, sx, wq, sw = product_case(rng, T, N, K, 128, "e5m2")
    nan_k, inf_k, w_k = K - 1, K // 2, 17
    wq[:, inf_k] = F.encode(np.where(np.arange(N) % 3 == 0, 0.0, np.where(np.arange(N) % 3 == 1, 1.5, -2.0))
                            .astype(np.float32), "e4m3")
    xq[:, [inf_k, nan_k, w_k]] = 0
    clean, bound = F.matmul(xq, sx, wq, sw, 128, None, "e5m2", out)
    xq[2, inf_k], xq[3, inf_k], xq[4, nan_k], wq[11, w_k] = 0x7C, 0xFC, 0x7F, 0x7F
    want = clean.copy()
    sign = np.array([np.nan, 1.0, -1.0])[np.arange(N) % 3]
    want[2], want[3], want[4], want[:, 11] = np.inf * sign, -np.inf * sign, np.nan, np.nan
    y = f64(B.bsr_matmul_f8(codes(xq, "e5m2", pad), torch.from_numpy(sx).to(DEV), codes(wq, "e4m3", pad),
                            torch.from_numpy(sw).to(DEV), out_dtype=TORCH[out]))
    special = ~np.isfinite(want)
    assert np.array_equal(y[special], want[special], equal_nan=True)
    assert np.all((np.abs(y - clean) <= bound)[~special])


def test_matmul_of_views():
    """Tokens, blocks and channels cut out of larger matrices, with the scales' views."""
    rng = np.random.default_rng(8)
    xq, sx, wq, sw = product_case(rng, 96, 512, 1024, 128, "e4m3")
    X, SX = codes(xq, "e4m3"), torch.from_numpy(sx).to(DEV)
    W, SW = codes(wq, "e4m3"), torch.from_numpy(sw).to(DEV)
    t, k, n = slice(5, 78), slice(256, 1000), slice(128, 470)
    Y = B.bsr_matmul_f8(X[t, k], SX[2:8, t], W[n, k], SW[2:8, 1:4])
    want, bound = F.matmul(xq[t, k], sx[2:8, t], wq[n, k], sw[2:8, 1:4], 128)
    within(Y, want, bound, "Y")
    assert B.bsr_matmul_f8(X[:0], SX[:, :0], W, SW).shape == (0, 512)


@pytest.mark.parametrize("T,N", [(3, 130), (260, 130)])
def test_matmul_long_offsets(T, N):
    """Rows and outputs beyond 2^31 bytes from the first, for the tokens and the channels."""
    rng = np.random.default_rng(12)
    K, pitch = 272, 1 << 20
    rows_x, rows_w = (T, 2600) if T < 100 else (2600, 130)
    xq, wq = random_codes(rng, rows_x, K, "e4m3"), random_codes(rng, rows_w, K, "e4m3")

    def far(q):
        buf = torch.full((len(q) * pitch,), 0x7F, dtype=torch.uint8, device=DEV).view(len(q), pitch)[:, :K]
        buf.copy_(torch.from_numpy(q))
        return buf.view(F8["e4m3"])
    sx = np.exp(rng.uniform(-3, 0, (3, rows_x))).astype(np.float32)
    sw = np.exp(rng.uniform(-3, 0, (3, -(-rows_w // 128)))).astype(np.float32)
    Y = B.bsr_matmul_f8(far(xq), torch.from_numpy(sx).to(DEV), far(wq), torch.from_numpy(sw).to(DEV))
    want, bound = F.matmul(xq, sx, wq, sw, 128)
    within(Y, want, bound, "Y")


def test_matmul_many_columns_of_scales():
    """Scales whose pitch puts a block's beyond 2^31 bytes from the first."""
    rng = np.random.default_rng(13)
    T, N, K, pitch = 40, 70, 128 * 40, 1 << 24
    xq, sx, wq, sw = product_case(rng, T, N, K, 1, "e4m3")
    buf = torch.empty(40 * pitch, device=DEV).view(40, pitch)
    S, SW = buf[:, :T], buf[:, 1 << 20:(1 << 20) + N]
    S.copy_(torch.from_numpy(sx))
    SW.copy_(torch.from_numpy(sw))
    want, bound = F.matmul(xq, sx, wq, sw, 1)
    within(B.bsr_matmul_f8(codes(xq, "e4m3"), S, codes(wq, "e4m3"), SW), want, bound, "Y")
    T2 = 12                                           # few tokens
    within(B.bsr_matmul_f8(codes(xq[:T2], "e4m3"), S[:, :T2], codes(wq, "e4m3"), SW), want[:T2],
           bound[:T2], "Y")


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_products_beside_a_large_one(out):
    """1 - 1 + 2^-s in one group of eight: fp32 output keeps every s, bf16 output, whose sums the 8-bit matrix
    instructions form, down to 2^-13 of the largest product; products in other groups are kept in both."""
    T = N = 512                                        # enough for tiles
    for s in range(4, 15):
        for at in (2, 7, 8, 100):
            x, w = np.zeros((T, 128), np.float32), np.zeros((N, 128), np.float32)
            x[:, 0], w[:, 0], x[:, 1], w[:, 1] = 1, 1, -1, 1
            x[:, at], w[:, at] = 2.0 ** -(s // 2), 2.0 ** -(s - s // 2)
            one = torch.ones(1, T, device=DEV)
            y = B.bsr_matmul_f8(codes(F.encode(x, "e4m3"), "e4m3"), one, codes(F.encode(w, "e4m3"), "e4m3"),
                                one, out_dtype=TORCH[out])
            kept = out == "f32" or s <= 13 or at >= 8
            assert bool((y == (2.0 ** -s if kept else 0.0)).all()), (s, at)


@pytest.mark.parametrize("x_fmt,x0,w0,cut", [
    ("e4m3", 1.75, 1.75, -13),                         # 2^0 2^0, less 13: the fractions do not count
    ("e4m3", 2.0 ** -9, 448.0, -11), ("e4m3", 448.0, 2.0 ** -9, -11),     # 2^-6 2^8
    ("e5m2", 57344.0, 2.0 ** -9, -4),                  # 2^15 2^-6
    ("e4m3", 0.0, 448.0, None), ("e4m3", 448.0, 0.0, None), ("e5m2", 57344.0, 0.0, None)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T", [20, 512])
def test_products_beside_a_large_subnormal_or_zero(x_fmt, x0, w0, cut, out, T):
    """x0 w0 - x0 w0 + 2^s in one group of eight: the 8-bit instructions that make bf16 output in tiles keep 2^s
    from 2^-13 of the pair's exponents on, where a subnormal code's exponent is its format's least normal
    one; beside products of zero they keep it all.  So do fp32 output and the kernel for few tokens.  The
    sums of two groups side by side (2^s at 8) meet with the 24 bits of fp32: from 2^-24 of those exponents
    on, 11 places further down."""
    N = 512
    ones_x, ones_w = torch.ones(1, T, device=DEV), torch.ones(1, N, device=DEV)

    def rows(n, fmt, at, *v):
        q = np.zeros((n, 128), np.uint8)
        q[:, [0, 1, at]] = F.encode(np.array(v, np.float32), fmt)
        return codes(q, fmt)
    for s in range(-16, 0):
        for at in (2, 7, 8, 100):
            y = B.bsr_matmul_f8(rows(T, x_fmt, at, x0, -x0, 2.0 ** (s // 2)), ones_x,
                                rows(N, "e4m3", at, w0, w0, 2.0 ** (s - s // 2)), ones_w, out_dtype=TORCH[out])
            least = -99 if out == "f32" or T == 20 or cut is None else {2: cut, 7: cut, 8: cut - 11, 100: -99}[at]
            assert bool((y == (2.0 ** s if s >= least else 0.0)).all()), (s, at)


@pytest.mark.parametrize("T,N,K", [(1000003, 24, 64), (40, 100003, 48), (70001, 72, 130)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_matmul_long_and_narrow(T, N, K, out):
    rng = np.random.default_rng(31)
    x, w = (rng.integers(-4, 5, s).astype(np.float32) for s in ((T, K), (N, K)))
    kb = -(-K // 128)
    sx = (2.0 ** rng.integers(-1, 2, (kb, T))).astype(np.float32)
    sw = (2.0 ** rng.integers(-1, 2, (kb, N))).astype(np.float32)
    y = B.bsr_matmul_f8(codes(F.encode(x, "e4m3"), "e4m3"), torch.from_numpy(sx).to(DEV),
                        codes(F.encode(w, "e4m3"), "e4m3"), torch.from_numpy(sw).to(DEV),
                        out_dtype=TORCH[out])
    want = 0
    for b in range(kb):
        k = slice(128 * b, 128 * b + 128)
        part = torch.from_numpy(x[:, k]).to(DEV) @ torch.from_numpy(w[:, k]).to(DEV).t()
        want = want + part * torch.from_numpy(sx[b]).to(DEV)[:, None] * torch.from_numpy(sw[b]).to(DEV)
    assert torch.equal(y, want.to(TORCH[out]))        # integers and powers of two: exact


def test_calls_side_by_side():
    """Products and quantisations on two streams at once."""
    rng = np.random.default_rng(15)
    w = B.bsr_quantize_f8(rand(rng, 1100, 1024, sigma=0.02).to(DEV), 128)
    xs = [rand(rng, T, 1024, dtype="bf16").to(DEV) for T in (900, 7)]
    want = [B.bsr_matmul_f8(*B.bsr_quantize_f8(x), *w) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, (x, s) in enumerate(zip(xs, streams)):
            with torch.cuda.stream(s):
                got[i].append(B.bsr_matmul_f8(*B.bsr_quantize_f8(x), *w))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_streams_and_graphs():
    rng = np.random.default_rng(14)
    xs = [rand(rng, 300, 640, dtype="bf16").to(DEV) for _ in range(3)]
    w = B.bsr_quantize_f8(rand(rng, 256, 640, sigma=0.02).to(DEV), 128)
    eager = [B.bsr_matmul_f8(*B.bsr_quantize_f8(x), *w) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = B.bsr_matmul_f8(*B.bsr_quantize_f8(xs[0], stream=side), *w, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(other, eager[0])
    X = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = B.bsr_matmul_f8(*B.bsr_quantize_f8(X), *w)
    for i in (1, 2, 0, 1):
        X.copy_(xs[i])
        graph.replay()
        again = B.bsr_matmul_f8(*B.bsr_quantize_f8(xs[i]), *w)
        torch.cuda.synchronize()
        assert torch.equal(Y, eager[i]) and torch.equal(again, eager[i])


# --- a layer with its norm, as it is trained -----------------------------------------------------

def test_layer_step():
    """h = norm(x + r), y = h W^T in 8 bits, and from dy the gradients of W, x, gamma and beta: every stage
    against its oracle on the stage's own inputs, and the ends against the step without rounding to 8
    bits, whose codes are off by at most 2^-4 of their value, or 2^-10 of the block's scale below the
    least exponent."""
    rng = np.random.default_rng(21)
    T, K, Nn = 333, 770, 520
    x, r = rand(rng, T, K).to(DEV), rand(rng, T, K).to(DEV)
    gamma, beta = (rand(rng, K, sigma=0.1) + 1.0).to(DEV), rand(rng, K, sigma=0.1).to(DEV)
    W, dy = rand(rng, Nn, K, sigma=0.02).to(DEV), rand(rng, T, Nn, sigma=0.1).to(DEV)
    h, s, mean, rstd = B.bsr_layer_norm(x, gamma, beta, R=r, save=True)
    hq, sh, hqt, sht = B.bsr_quantize_f8(h, form="both")
    wq, sw, wqt, swt = B.bsr_quantize_f8(W, 128, form="both")
    y = B.bsr_matmul_f8(hq, sh, wq, sw)
    dq, sd, dqt, sdt = B.bsr_quantize_f8(dy, form="both")
    dh = B.bsr_matmul_f8(dq, sd, wqt, swt)
    dW = B.bsr_matmul_f8(dqt, sdt, hqt, sht)
    dx, dgamma, dbeta = B.bsr_layer_norm_backward(dh, s, mean, rstd, gamma)
    for got, ops, rows in ((y, (hq, sh, wq, sw), 128), (dh, (dq, sd, wqt, swt), 128),
                           (dW, (dqt, sdt, hqt, sht), 1)):
        a = [bits(t) if i % 2 == 0 else host(t) for i, t in enumerate(ops)]
        within(got, *F.matmul(*a, rows), "product")
    from oracle import norm_oracle as N
    want = N.backward(f64(dh), f64(s), f64(mean), f64(rstd), f64(gamma))
    for name, got in (("dX", dx), ("dgamma", dgamma), ("dbeta", dbeta)):
        within(got, *want[name], name)

    def off(a, scale, rows):        # how far the codes of a may be from it
        at, to = np.arange(a.shape[1]) // 128, np.arange(a.shape[0]) // rows
        return 2.0 ** -4 * np.abs(a) + 2.0 ** -10 * host(scale).astype(np.float64)[at][:, to].T

    for got, (a, sa, ra), (b, sb, rb) in (
            (y, (f64(h), sh, 1), (f64(W), sw, 128)), (dh, (f64(dy), sd, 1), (f64(W).T, swt, 128)),
            (dW, (f64(dy).T, sdt, 1), (f64(h).T, sht, 1))):
        ea, eb = off(a, sa, ra) * 1.001, off(b, sb, rb) * 1.001
        bound = ea @ np.abs(b).T + np.abs(a) @ eb.T + ea @ eb.T
        bound += (a.shape[1] + 4) * 2.0 ** -24 * ((np.abs(a) + ea) @ (np.abs(b) + eb).T)
        within(got, a @ b.T, bound, "step")
