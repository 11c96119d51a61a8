"""The 8-bit floating-point product's kernels with every pair of token format and scales: dY in E5M2 with a
weight's 128-row scales, the way back to the inputs, and E4M3 with a scale for each row beside the pairs of a
forward product and a weight's gradient."""
import pytest

from tests import test_gpu_f8 as G

pytestmark = pytest.mark.gpu

FORMS = [(128, "e5m2"), (1, "e4m3")]


@pytest.mark.parametrize("T,N,K", [(1, 4500, 4301), (16, 5000, 4232), (17, 4201, 2500), (32, 9000, 301)])
@pytest.mark.parametrize("rows,x_fmt", FORMS)
@pytest.mark.parametrize("pad,shift", [(1, 3), (-1, 0)])
def test_few_tokens(T, N, K, rows, x_fmt, pad, shift):
    G.test_matmul(T, N, K, rows, x_fmt, pad, shift)


@pytest.mark.parametrize("T,N,K", [(4096, 4096, 272), (1536, 8192, 389), (2050, 4099, 389), (4900, 4096, 272),
                                   (4096, 4096, 2064), (1536, 8192, 2053), (2048, 4096, 4112),
                                   (3136, 8192, 2053)])
@pytest.mark.parametrize("rows,x_fmt", FORMS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [7, -1])
def test_large_tiles(T, N, K, rows, x_fmt, out, pad):
    G.test_matmul_large_tiles(T, N, K, rows, x_fmt, out, pad)


@pytest.mark.parametrize("T,N,K", [(200, 1000, 2048), (257, 520, 2170), (513, 1024, 8700), (193, 900, 8500)])
@pytest.mark.parametrize("rows,x_fmt", FORMS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [7, -1])
def test_long_contractions(T, N, K, rows, x_fmt, out, pad):
    G.test_matmul_long_contractions(T, N, K, rows, x_fmt, out, pad)


@pytest.mark.parametrize("T,N,K", [(2048, 2048, 2064), (3300, 2400, 4112)])
@pytest.mark.parametrize("rows,x_fmt", [(128, "e4m3"), (1, "e5m2"), *FORMS])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [7, -1])
def test_middle_tiles(T, N, K, rows, x_fmt, out, pad):
    """One and two rounds of 128 x 128 tiles."""
    G.test_matmul_large_tiles(T, N, K, rows, x_fmt, out, pad)
