"""The layer norm and its gradients on the GPU against the fp64 oracle, within bounds that count the
roundings (oracle/norm_oracle.py).  Sizes straddle what a wave and a workgroup hold, rows start at no
particular alignment, pitches exceed widths, and the gaps between rows hold NaN on the way in and a
sentinel on the way out."""
import numpy as np
import pytest
import torch

from oracle import norm_oracle as N
from paper_2106_08846_amd import bsr as B
from tests.test_gpu_dense import DEV, TORCH, f64, frame, held, rand

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 7), (3, 64), (5, 511), (4, 512), (17, 768), (2, 1024), (9, 1025), (33, 4096),
         (6, 4097), (3, 16384), (2, 16385), (2, 70001), (1000, 96), (2053, 24)]


def to_type(dtype):
    return lambda a: torch.from_numpy(a).to(TORCH[dtype]).float().numpy()


def within(got, want, bound, what):
    err = np.abs(f64(got) - want)
    assert np.all(np.isfinite(f64(got))), what
    assert np.all(err <= bound), (what, float(np.max(err / bound)))


def operands(rng, T, K, dtype, affine=True):
    x = rand(rng, T, K, dtype=dtype) + 0.5
    r = rand(rng, T, K, sigma=2.0, dtype=dtype)
    gamma = rand(rng, K) + 1.0 if affine else None
    beta = rand(rng, K) if affine else None
    return x, r, gamma, beta


def dev(t):
    return None if t is None else t.to(DEV)


@pytest.mark.parametrize("T,K", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift,residual", [(0, 0, True), (3, 1, False), (16, 8, True), (1, 3, True)])
def test_norm(T, K, dtype, pad, shift, residual):
    rng = np.random.default_rng(T * 100003 + K)
    affine = (T + K) % 3 > 0
    x, r, gamma, beta = operands(rng, T, K, dtype, affine)
    R = held(r, pad, shift) if residual else None
    Y, clean = frame(T, K, TORCH[dtype], pad, shift)
    S, clean_s = frame(T, K, TORCH[dtype], pad + 1, shift) if residual else (None, None)
    y, s, mean, rstd = B.bsr_layer_norm(held(x, pad, shift), dev(gamma), dev(beta), R=R, eps=1e-5,
                                        save=True, Y=Y, S=S)
    want_s = N.residual_sum(x.float().numpy(), r.float().numpy() if residual else None, to_type(dtype))
    assert np.array_equal(f64(s).astype(np.float32), want_s)
    want, bound = N.layer_norm(want_s, None if gamma is None else gamma.numpy(),
                               None if beta is None else beta.numpy(), 1e-5, dtype)
    within(y, want, bound, "Y")
    m, rs, _, e_mean, r_rstd = N.statistics(want_s, 1e-5)
    within(mean, m[:, 0], e_mean[:, 0], "mean")
    within(rstd, rs[:, 0], (rs * r_rstd)[:, 0], "rstd")
    assert clean() and (clean_s is None or clean_s())
    # without the statistics, and with outputs of the binding: the same bits
    again = B.bsr_layer_norm(held(x, 0, 0), dev(gamma), dev(beta), R=R)
    assert torch.equal(again, y)


@pytest.mark.parametrize("T,K", SIZES)
@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("pad,shift,extra", [(0, 0, True), (3, 1, False), (16, 8, True)])
def test_backward(T, K, dtype, grad, pad, shift, extra):
    rng = np.random.default_rng(T * 7919 + K)
    affine = (T + K) % 3 > 0
    x, dy, gamma, beta = operands(rng, T, K, dtype, affine)
    ds = rand(rng, T, K, sigma=0.3, dtype=dtype)
    X = held(x, pad, shift)
    _, S, mean, rstd = B.bsr_layer_norm(X, dev(gamma), dev(beta), save=True)
    assert S is X
    dX, clean = frame(T, K, TORCH[dtype], pad, shift)
    got = dict(zip(("dX", "dgamma", "dbeta"), B.bsr_layer_norm_backward(
        held(dy, pad, shift), S, mean, rstd, dev(gamma), dS=held(ds, pad, shift) if extra else None,
        dX=dX, grad_dtype=TORCH[grad])))
    want = N.backward(f64(dy), f64(x), f64(mean), f64(rstd), None if gamma is None else gamma.numpy(),
                      f64(ds) if extra else None, dtype, grad)
    for name, (value, bound) in want.items():
        within(got[name], value, bound, name)
    assert clean()


# Several rounds over the rows for a workgroup of the backward pass; forward, rows of up to 4096 columns on a
# wave.  Every width of a workgroup, and every end of a row.
MANY_ROWS = [(4103, 96), (6151, 520), (4099, 1024), (2051, 1531), (2049, 2056), (2050, 4096), (1031, 4095),
             (771, 5000), (514, 4099), (515, 8192), (259, 16383), (201, 16392)]


@pytest.mark.parametrize("T,K", MANY_ROWS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows(T, K, dtype):
    test_norm(T, K, dtype, 8, 0, True)
    test_backward(T, K, dtype, "f32", 8, 0, (T + K) % 2 == 0)


@pytest.mark.parametrize("T,K", [(37, 768), (9, 2050), (4, 20000)])
def test_parts_of_the_gradients(T, K):
    """Each gradient alone has the bits of all of them together; the workspace may be the caller's."""
    rng = np.random.default_rng(11)
    x, dy, gamma, _ = operands(rng, T, K, "bf16")
    X, dY, g = dev(x), dev(dy), dev(gamma)
    _, S, mean, rstd = B.bsr_layer_norm(X, g, save=True)
    dX, dg, db = B.bsr_layer_norm_backward(dY, S, mean, rstd, g, grad_dtype=torch.float32)
    only, none, none2 = B.bsr_layer_norm_backward(dY, S, mean, rstd, g, affine=False)
    assert none is None and none2 is None and torch.equal(only, dX)
    ws = torch.full((B.bsr_layer_norm_workspace_bytes(T, K) + 64,), 255, dtype=torch.uint8, device=DEV)
    none, dg2, db2 = B.bsr_layer_norm_backward(dY, S, mean, rstd, g, grad_dtype=torch.float32,
                                               need_dX=False, workspace=ws)
    assert none is None and torch.equal(dg2, dg) and torch.equal(db2, db)
    assert bool((ws[-64:] == 255).all())
    db3 = torch.empty(K, device=DEV)
    _, none, db4 = B.bsr_layer_norm_backward(dY, S, mean, rstd, g, affine=False, dbeta=db3, need_dX=False)
    assert none is None and db4 is db3 and torch.equal(db3, db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens(dtype):
    X = torch.empty(0, 96, dtype=TORCH[dtype], device=DEV)
    Y, S, mean, rstd = B.bsr_layer_norm(X, save=True)
    assert Y.shape == (0, 96) and mean.shape == (0,)
    dX, dg, db = B.bsr_layer_norm_backward(X, S, mean, rstd)
    assert dX.shape == (0, 96) and not bool(dg.any()) and not bool(db.any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [5, 768, 4500])
def test_special_rows(dtype, K):
    x = np.random.default_rng(5).standard_normal((10, K)).astype(np.float32)
    x[0] = 3.0                                       # no variance: Y is beta
    x[1] = 0.0
    x[2, K - 1] = np.inf
    x[3, 0] = np.nan
    x[4, 0], x[4, 1] = np.inf, -np.inf
    x[5] *= np.float32(2.0 ** -70)                   # squares that vanish beside eps
    x[6] *= np.float32(2.0 ** 90)                    # squares beyond fp32: rstd is 0
    x[7] += 1000.0                                   # far from zero
    t = torch.from_numpy(x).to(TORCH[dtype])
    beta = torch.linspace(-1, 1, K)
    Y, S, mean, rstd = B.bsr_layer_norm(t.to(DEV), None, beta.to(DEV), save=True)
    y = f64(Y)
    with np.errstate(all="ignore"):                  # the rows that are not finite
        want, bound = N.layer_norm(t.double().numpy(), None, beta.numpy(), 1e-5, dtype)
    for row in (0, 1, 5, 7, 8, 9):
        assert np.all(np.abs(y[row] - want[row]) <= bound[row]), row
    assert np.all(np.isnan(y[2:5]).any(1)) and np.all(np.isnan(f64(rstd)[2:5]))
    assert f64(rstd)[6] == 0.0 and np.array_equal(y[6], f64(beta.to(TORCH[dtype])))
    dX = B.bsr_layer_norm_backward(torch.ones_like(S), S, mean, rstd)[0]
    assert np.all(np.isfinite(f64(dX)[[0, 1, 5, 6, 7, 8, 9]]))


def test_offset_rows_keep_their_variance():
    """Rows of 4096 values 1000 from zero with deviations of 2^-6: the mean of the squares alone would
    lose the variance in fp32."""
    rng = np.random.default_rng(2)
    x = (1000.0 + rng.integers(-4, 5, (3, 4096)) * 2.0 ** -8).astype(np.float32)
    Y = B.bsr_layer_norm(torch.from_numpy(x).to(DEV))
    want, bound = N.layer_norm(x)
    # the computed mean is off by up to e_mean of the magnitude 1000; the rest of the bound is small
    within(Y, want, bound, "Y")
    assert abs(float(Y.double().std()) - float(want.std())) < 0.01


@pytest.mark.parametrize("T,K", [(3, 5), (5, 200), (9, 768), (2100, 520), (5, 1030), (5, 1032), (7, 2056),
                                 (3, 4500), (3, 4504), (2, 16380), (2, 20000), (2, 20001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("affine", [True, False])
def test_gradients_of_a_large_constant_row(T, K, dtype, affine):
    """A row of 2^110 among ordinary ones, with eps 2^-40: its sum K 2^110 is exact, so mean is 2^110, rstd 2^20
    and h 0 at every column.  mean * rstd is beyond fp32, and nothing but the row's own columns, whose
    deviations are 0, may meet it."""
    rng = np.random.default_rng(T + K)
    x, dy, gamma, _ = operands(rng, T, K, dtype, affine)
    ds = rand(rng, T, K, dtype=dtype)
    x[1] = 2.0 ** 110
    Y, S, mean, rstd = B.bsr_layer_norm(dev(x), dev(gamma), eps=2.0 ** -40, save=True)
    assert not bool(Y[1].any()) and float(mean[1]) == 2.0 ** 110 and float(rstd[1]) == 2.0 ** 20
    got = B.bsr_layer_norm_backward(dev(dy), S, mean, rstd, dev(gamma), dS=dev(ds), grad_dtype=torch.float32)
    want = N.backward(f64(dy), f64(x), f64(mean), f64(rstd), None if gamma is None else gamma.numpy(),
                      f64(ds), dtype)
    for name, g in zip(("dX", "dgamma", "dbeta"), got):
        within(g, *want[name], name)


@pytest.mark.parametrize("T,K,step", [(3, 64, 2.0 ** -8), (5, 512, 2.0 ** -5), (4, 768, 2.0 ** -4),
                                      (3, 1531, 2.0 ** -3), (3, 4096, 2.0 ** -2), (2100, 4096, 2.0 ** -2),
                                      (3, 5000, 0.5), (2, 32768, 2.0), (2, 70001, 8.0)])
def test_statistics_far_from_zero(T, K, step):
    """Rows of 1000 (1000 to within a step where that is not one) and up to four steps to either side, with
    steps so large that K times the largest value is below 2^24 of them: every sum of a row's values is
    exact, in any order, so the mean is off by its quotient's rounding alone, half a step of fp32 below
    1024 (2^-15).  Deviations and outputs follow it to fp32's rounding."""
    rng = np.random.default_rng(K)
    x = 1000.0 // step * step + rng.integers(-4, 5, (T, K)) * step
    assert np.max(np.abs(x)) * K < 2 ** 24 * step and np.all(x.astype(np.float32) == x)
    Y, _, mean, rstd = B.bsr_layer_norm(torch.from_numpy(x.astype(np.float32)).to(DEV), save=True)
    m = x.mean(1)
    e_mean = 2.0 ** -15
    assert np.all(np.abs(f64(mean) - m) <= e_mean)
    d = x - m[:, None]
    var = (d * d).mean(1)
    # from a mean off by e: n (var + e^2) in squares; each deviation and square rounds once, as their sums do
    e_var = e_mean ** 2 + (N.depth(K) + 4) * N.U32 * (var + e_mean ** 2)
    want = 1.0 / np.sqrt(var + 1e-5)
    r = np.sqrt((var + 1e-5) / (var + 1e-5 - e_var)) - 1.0 + 4 * N.U32
    assert np.all(np.abs(f64(rstd) - want) <= want * r)
    h = d * want[:, None]
    e_d = e_mean + N.U32 * (np.abs(d) + e_mean)
    bound = e_d * (want * (1 + r))[:, None] + np.abs(h) * (r + 2 * N.U32)[:, None]
    assert np.max(bound) < 0.01 * np.std(h)          # a shift of the row would show
    within(Y, h, bound, "Y")


def test_long_offsets():
    """Rows beyond 2^31 elements from the first."""
    T, K, pitch = 2200, 72, 1 << 20
    rng = np.random.default_rng(9)
    x = rand(rng, T, K, dtype="bf16")
    buf = torch.empty(T * pitch, dtype=torch.bfloat16, device=DEV)
    out = torch.empty(T * pitch, dtype=torch.bfloat16, device=DEV)
    X, Y = buf.view(T, pitch)[:, :K], out.view(T, pitch)[:, :K]
    X.copy_(x)
    _, S, mean, rstd = B.bsr_layer_norm(X, Y=Y, save=True)
    want, bound = N.layer_norm(x.double().numpy(), out="bf16")
    within(Y, want, bound, "Y")
    dX, dg, db = B.bsr_layer_norm_backward(Y, S, mean, rstd, dX=Y[:, :K].clone(), grad_dtype=torch.float32)
    got = N.backward(f64(Y), x.double().numpy(), f64(mean), f64(rstd), out="bf16")
    within(dX, *got["dX"], "dX")
    within(dg, *got["dgamma"], "dgamma")
    within(db, *got["dbeta"], "dbeta")


def test_more_rows_than_a_launch():
    T, K = (1 << 21) + 37, 8
    rng = np.random.default_rng(10)
    x = rand(rng, T, K, dtype="bf16")
    X = x.to(DEV)
    gamma = rand(rng, K) + 1.0
    Y, S, mean, rstd = B.bsr_layer_norm(X, gamma.to(DEV), R=X, save=True)
    s = x.float().numpy() * 2
    want, bound = N.layer_norm(s, gamma.numpy(), out="bf16")
    within(Y, want, bound, "Y")
    dX, dg, db = B.bsr_layer_norm_backward(X, S, mean, rstd, gamma.to(DEV), grad_dtype=torch.float32)
    got = N.backward(f64(x), s, f64(mean), f64(rstd), gamma.numpy(), out="bf16")
    within(dX, *got["dX"], "dX")
    within(dg, *got["dgamma"], "dgamma")
    within(db, *got["dbeta"], "dbeta")


def test_backward_side_by_side():
    """Backward passes on two streams at once, with a workspace each."""
    rng = np.random.default_rng(12)
    T, K = 1100, 2304
    sides = []
    for i in range(2):
        x, dy, gamma, _ = operands(rng, T, K, "bf16")
        X, dY, g = dev(x), dev(dy), dev(gamma)
        _, S, mean, rstd = B.bsr_layer_norm(X, g, save=True)
        want = B.bsr_layer_norm_backward(dY, S, mean, rstd, g, grad_dtype=torch.float32)
        ws = torch.empty(B.bsr_layer_norm_workspace_bytes(T, K), dtype=torch.uint8, device=DEV)
        sides.append((torch.cuda.Stream(), (dY, S, mean, rstd, g), ws, want, []))
    torch.cuda.synchronize()
    for _ in range(8):
        for stream, ops, ws, _, got in sides:
            with torch.cuda.stream(stream):
                got.append(B.bsr_layer_norm_backward(*ops, grad_dtype=torch.float32, workspace=ws))
    torch.cuda.synchronize()
    for _, _, _, want, got in sides:
        for g in got:
            assert all(torch.equal(p, q) for p, q in zip(g, want))


def test_repeated_calls_and_streams():
    rng = np.random.default_rng(4)
    x, dy, gamma, beta = operands(rng, 1500, 1030, "bf16")
    X, dY, g, b = dev(x), dev(dy), dev(gamma), dev(beta)
    first = B.bsr_layer_norm(X, g, b, R=dY, save=True)
    grads = B.bsr_layer_norm_backward(dY, *first[1:], g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        again = B.bsr_layer_norm(X, g, b, R=dY, save=True, stream=stream)
        more = B.bsr_layer_norm_backward(dY, *again[1:], g, stream=stream)
        torch.cuda.synchronize()
        for p, q in zip((*first, *grads), (*again, *more)):
            assert torch.equal(p, q)


def test_captured_steps():
    """Forward and backward in a graph, replayed on other inputs with eager work between, two graphs with a
    workspace each."""
    rng = np.random.default_rng(6)
    T, K = 700, 1536
    g = dev(rand(rng, K) + 1.0)
    xs = [dev(rand(rng, T, K, dtype="bf16")) for _ in range(4)]
    graphs = []
    for _ in range(2):
        X, dY = torch.empty_like(xs[0]), torch.empty_like(xs[0])
        X.copy_(xs[0])
        dY.copy_(xs[1])
        ws = torch.empty(B.bsr_layer_norm_workspace_bytes(T, K), dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = B.bsr_layer_norm(X, g, save=True)
            grads = B.bsr_layer_norm_backward(dY, *out[1:], g, grad_dtype=torch.float32, workspace=ws)
        graphs.append((graph, X, dY, out, grads))
    for i in range(4):
        for n, (graph, X, dY, out, grads) in enumerate(graphs):
            x, dy = xs[(i + n) % 4], xs[(i + n + 1) % 4]
            X.copy_(x)
            dY.copy_(dy)
            graph.replay()
            want = B.bsr_layer_norm(x, g, save=True)
            more = B.bsr_layer_norm_backward(dy, *want[1:], g, grad_dtype=torch.float32)
            torch.cuda.synchronize()
            for p, q in zip((out[0], *out[2:], *grads), (want[0], *want[2:], *more)):
                assert torch.equal(p, q)
