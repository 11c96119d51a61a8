"""The norm between the products of a layer and the products in 8-bit floating point, as programs
call them: the residual sum with its layer norm, in inference and in training; the codes and scales of
a matrix in blocks of 128; and the product of two such matrices.

Every case is a dict of plain values.  `prepare` makes what such a program holds before the call,
`run` is one pass: the library's entry points where `own` is true, the same formulas in elementary
torch operations in 32 bits where it is false.  `exact` is the result from the definitions in 64
bits.

Kinds of case:
  norm       S = X + R (rounded to the type of X; without a residual S = X),
             Y[t][k] = (S[t][k] - mean_t) rstd_t gamma[k] + beta[k].
  train      the same forward pass, and from dY and the gradient that reaches S by its other path the
             gradients of X, gamma and beta.
  quantize   blocks of 1 x 128 (a row of activations) or 128 x 128 (a weight): scale = max|x| / m,
             code = x (m / max|x|) in 8-bit floating point, m its largest value; each operation rounded
             to fp32.  "rows": as the matrix lies; "both": its transpose too, with blocks of its own.
  matmul     Y[t][n] = sum over blocks b of sx[b][t] sw[b][n] sum over k in b of Xq[t][k] Wq[n][k],
             + bias[n].
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5
BLOCK = 128
W_SIGMA = 0.02      # an initialiser's scale, for weights and biases

# The most multiply-adds (times two) and the most bytes of one pass among the listed cases.
MAX_FLOPS = 11e11
MAX_BYTES = 2.72e8


def listed():
    return [
        # The norm before a feed-forward block: a prefill that adds the attention's output to the
        # residual stream, and one token, where latency is all.
        {"name": "norm_bf16_8192x4096", "kind": "norm", "dtype": "bf16", "T": 8192, "K": 4096,
         "residual": True, "affine": True, "pad": 0},
        {"name": "norm_f32_1x1024", "kind": "norm", "dtype": "f32", "T": 1, "K": 1024,
         "residual": False, "affine": True, "pad": 0},
        # Training steps through it: 16 sequences of 384 tokens in bf16, and a small fp32 step of odd
        # width whose rows start at no 16-byte boundary.
        {"name": "train_bf16_6144x2048", "kind": "train", "dtype": "bf16", "T": 6144, "K": 2048,
         "residual": True, "affine": True, "pad": 0},
        {"name": "train_f32_777x1531", "kind": "train", "dtype": "f32", "T": 777, "K": 1531,
         "residual": False, "affine": True, "pad": 1},
        # Codes and scales: a prefill's activations; a training step's, which the forward product
        # takes by rows and the weights' gradient by columns; a weight after its update, for the
        # forward product and the one back to the inputs; one token of a server.
        {"name": "quantize_bf16_8192x4096", "kind": "quantize", "dtype": "bf16", "q": "e4m3",
         "T": 8192, "K": 4096, "rows": 1, "form": "rows", "pad": 0},
        {"name": "quantize_both_bf16_6144x2048", "kind": "quantize", "dtype": "bf16", "q": "e5m2",
         "T": 6144, "K": 2048, "rows": 1, "form": "both", "pad": 0},
        {"name": "quantize_weight_f32_2304x770", "kind": "quantize", "dtype": "f32", "q": "e4m3",
         "T": 2304, "K": 770, "rows": 128, "form": "both", "pad": 0},
        {"name": "quantize_bf16_1x4096", "kind": "quantize", "dtype": "bf16", "q": "e4m3", "T": 1,
         "K": 4096, "rows": 1, "form": "rows", "pad": 0},
        # Products: one token through a 4096 x 4096 layer; a ragged batch with rows of 770 bytes, whose
        # last block is two wide; the largest prefill; the gradient of an 8192 x 2048 weight over 6144
        # tokens, where both operands have a scale for each row and the other format carries dY.
        {"name": "matmul_1x4096x4096", "kind": "matmul", "x": "e4m3", "T": 1, "N": 4096, "K": 4096,
         "rows": 128, "out": "f32", "bias": False, "pad": 0},
        {"name": "matmul_333x2304x770", "kind": "matmul", "x": "e4m3", "T": 333, "N": 2304, "K": 770,
         "rows": 128, "out": "bf16", "bias": True, "pad": 0},
        {"name": "matmul_8192x8192x8192", "kind": "matmul", "x": "e4m3", "T": 8192, "N": 8192,
         "K": 8192, "rows": 128, "out": "bf16", "bias": False, "pad": 0},
        {"name": "matmul_gradient_8192x2048x6144", "kind": "matmul", "x": "e5m2", "T": 8192,
         "N": 2048, "K": 6144, "rows": 1, "out": "f32", "bias": False, "pad": 0},
    ]


def draw(rng):
    def size(lo, hi, step):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5:                      # a round size, else any size at all
            n = (n + step - 1) // step * step
        return max(lo, min(hi, n))

    while True:
        kind = rng.choice(["norm", "train", "quantize", "matmul"])
        c = {"kind": kind, "T": size(1, 16384, 16), "K": size(64, 8192, 64)}
        c["pad"] = rng.choice([0, 0, 0, 1, 16])     # the row pitch of X beyond its width
        if kind in ("norm", "train"):
            c.update(dtype=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.5,
                     affine=rng.random() < 0.8)
        elif kind == "quantize":
            c.update(dtype=rng.choice(["bf16", "f32"]), q=rng.choice(["e4m3", "e5m2"]),
                     rows=rng.choice([1, 128]), form=rng.choice(["rows", "both"]))
        else:
            c.update(x=rng.choice(["e4m3", "e4m3", "e5m2"]), N=size(64, 12288, 64),
                     rows=rng.choice([1, 128]), out=rng.choice(["bf16", "f32"]),
                     bias=rng.random() < 0.5)
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return c


def work(case):
    T, K, kind = case["T"], case["K"], case["kind"]
    blocks = _blocks(K)
    if kind == "matmul":
        N = case["N"]
        rows_w = N if case["rows"] == 1 else _blocks(N)
        return {"bytes": T * K + N * K + 4 * blocks * (T + rows_w) + 4 * N * case["bias"]
                + T * N * _bytes(case["out"]), "flops": 2 * T * N * K}
    e = _bytes(case["dtype"])
    if kind == "quantize":
        rows_x = T if case["rows"] == 1 else _blocks(T)
        out = T * K + 4 * blocks * rows_x
        if case["form"] == "both":
            out += T * K + 4 * _blocks(T) * (K if case["rows"] == 1 else blocks)
        return {"bytes": T * K * e + out, "flops": 3 * T * K}
    residual, vectors = case["residual"], 8 * K * case["affine"]
    if kind == "norm":                              # X (and R) read, Y (and S) written
        return {"bytes": T * K * e * (2 + 2 * residual) + vectors, "flops": 8 * T * K}
    # also dY (and the gradient of S) read, the gradients written
    return {"bytes": T * K * e * (4 + 3 * residual) + 2 * vectors, "flops": 20 * T * K}


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _bytes(dtype):
    return 4 if dtype == "f32" else 2


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _q_dtype(name):
    return torch.float8_e4m3fn if name == "e4m3" else torch.float8_e5m2


def _largest(name):
    return 448.0 if name == "e4m3" else 57344.0


def _tokens(gen, T, K, pad):
    """Hidden states: about unit size per token, a few channels an order larger."""
    x = torch.randn((T, K + pad), generator=gen, device=DEVICE)
    size = torch.exp(0.3 * torch.randn((T, 1), generator=gen, device=DEVICE))
    wide = 1.0 + 9.0 * (torch.rand((1, K + pad), generator=gen, device=DEVICE) < 0.004).float()
    return x.mul_(size).mul_(wide)


def _vector(gen, n, mean=0.0):
    return torch.randn((n,), generator=gen, device=DEVICE).mul_(W_SIGMA).add_(mean)


def _quantize_plain(x, rows, name):
    """Codes [R, K] of x's blocks and their scales [blocks of K, blocks of R]."""
    R, K = x.shape
    rb, kb = -(-R // rows), _blocks(K)
    m = _largest(name)
    p = torch.nn.functional.pad(x.float(), (0, kb * BLOCK - K, 0, rb * rows - R))
    p = p.view(rb, rows, kb, BLOCK)
    amax = p.abs().amax(dim=(1, 3), keepdim=True)
    lift = torch.where(amax < 2.0 ** -64, torch.full_like(amax, 2.0 ** 64),
                       torch.ones_like(amax))      # keeps m / max finite
    r = torch.div(torch.full_like(amax, m), amax * lift)
    r = torch.where(torch.isfinite(r) & torch.isfinite(amax), r, torch.zeros_like(r))
    q = (p * lift) * r
    q = torch.where(torch.isnan(q), torch.zeros_like(q), q).to(_q_dtype(name))
    scale = torch.div(amax, torch.full_like(amax, m))[:, 0, :, 0]
    return q.view(rb * rows, kb * BLOCK)[:R, :K], scale.t()


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind, T, K, pad = case["kind"], case["T"], case["K"], case["pad"]
    s = {"case": case}
    if kind == "matmul":
        N = case["N"]

        def codes(x, rows, name):
            q, scale = _quantize_plain(x, rows, name)
            held = torch.zeros((x.shape[0], K + pad), dtype=torch.uint8, device=DEVICE)
            held[:, :K] = q.view(torch.uint8)
            return held.view(_q_dtype(name))[:, :K], scale.contiguous()

        s["X"], s["sx"] = codes(_tokens(gen, T, K, 0), 1, case["x"])
        if case["rows"] == 1:                      # the other operand of a weight's gradient
            s["W"], s["sw"] = codes(_tokens(gen, N, K, 0), 1, "e4m3")
        else:                                      # a server quantises its weights once
            W = torch.randn((N, K), generator=gen, device=DEVICE).mul_(W_SIGMA)
            s["W"], s["sw"] = codes(W, 128, "e4m3")
        s["b"] = _vector(gen, N) if case["bias"] else None
        return s
    dt = _dtype(case["dtype"])
    if kind == "quantize":
        if case["rows"] == 128:
            x = torch.randn((T, K + pad), generator=gen, device=DEVICE).mul_(W_SIGMA)
        else:
            x = _tokens(gen, T, K, pad)
        s["X"] = x.to(dt)[:, :K]
        return s
    s["X"] = _tokens(gen, T, K, pad).add_(0.25).to(dt)[:, :K]
    s["R"] = _tokens(gen, T, K, pad).to(dt)[:, :K] if case["residual"] else None
    s["gamma"] = _vector(gen, K, 1.0) if case["affine"] else None
    s["beta"] = _vector(gen, K) if case["affine"] else None
    if kind == "train":
        def gradient():
            return torch.randn((T, K), generator=gen, device=DEVICE).mul_(0.1).to(dt)

        s["dY"] = gradient()
        s["dS"] = gradient() if case["residual"] else None
    return s


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2106_08846_amd import bsr

    c = s["case"]
    kind = c["kind"]
    if kind == "matmul":
        return bsr.bsr_matmul_f8(s["X"], s["sx"], s["W"], s["sw"], s["b"],
                                 out_dtype=_dtype(c["out"]))
    if kind == "quantize":
        return bsr.bsr_quantize_f8(s["X"], block_rows=c["rows"], q_dtype=_q_dtype(c["q"]),
                                   form=c["form"])
    if kind == "norm":
        out = bsr.bsr_layer_norm(s["X"], s["gamma"], s["beta"], R=s["R"], eps=EPS,
                                 keep_sum=c["residual"])
        return _outputs(s, *out) if c["residual"] else _outputs(s, out, None)
    Y, S, mean, rstd = bsr.bsr_layer_norm(s["X"], s["gamma"], s["beta"], R=s["R"], eps=EPS,
                                          save=True)
    grads = bsr.bsr_layer_norm_backward(s["dY"], S, mean, rstd, s["gamma"], dS=s["dS"],
                                        affine=c["affine"], grad_dtype=torch.float32)
    return _outputs(s, Y, S, *grads)


def _outputs(s, Y, S, dX=None, dgamma=None, dbeta=None):
    out = {"Y": Y}
    if s["R"] is not None:
        out["S"] = S
    if dX is not None:
        out["dX"] = dX
    if dgamma is not None:
        out.update(dgamma=dgamma, dbeta=dbeta)
    return out


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "matmul":
        K, N = c["K"], c["N"]
        X = s["X"].float() * s["sx"].repeat_interleave(BLOCK, dim=0)[:K].t()
        sw = s["sw"].repeat_interleave(BLOCK, dim=0)[:K]
        if c["rows"] > 1:
            sw = sw.repeat_interleave(BLOCK, dim=1)[:, :N]
        y = torch.matmul(X, (s["W"].float() * sw.t()).t())
        return (y if s["b"] is None else y + s["b"]).to(_dtype(c["out"]))
    if kind == "quantize":
        out = _quantize_plain(s["X"], c["rows"], c["q"])
        if c["form"] == "both":
            out += _quantize_plain(s["X"].t(), c["rows"], c["q"])
        return out
    dt = _dtype(c["dtype"])
    S = s["X"] if s["R"] is None else (s["X"].float() + s["R"].float()).to(dt)
    x = S.float()
    d = x - x.mean(dim=1, keepdim=True)
    rstd = 1.0 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    xhat = d * rstd
    y = xhat if s["gamma"] is None else xhat * s["gamma"] + s["beta"]
    if kind == "norm":
        return _outputs(s, y.to(dt), S)
    dy = s["dY"].float()
    g = dy if s["gamma"] is None else dy * s["gamma"]
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    if s["dS"] is not None:
        dx = dx + s["dS"].float()
    grads = ((dy * xhat).sum(dim=0), dy.sum(dim=0)) if c["affine"] else (None, None)
    return _outputs(s, y.to(dt), S, dx.to(dt), *grads)


def _rounded(v, name):
    """v to the nearest value of the 8-bit format, ties to even, from its significand's width and its
    least exponent."""
    bits, least = (3, -6) if name == "e4m3" else (2, -14)
    exponent = (torch.frexp(v)[1] - 1).clamp(min=least).to(torch.int64) - bits
    step = ((exponent + 1023) << 52).view(torch.float64)       # 2^exponent, from its bits
    return torch.round(v / step) * step


def _quantize_exact(x, rows, name):
    # The definition rounds every operation to 32 bits; a quotient or a product of two fp32 values
    # formed in 64 bits and rounded is the correctly rounded one.
    R, K = x.shape
    rb, kb = -(-R // rows), _blocks(K)
    a = torch.zeros((rb * rows, kb * BLOCK), dtype=torch.float64, device=x.device)
    a[:R, :K] = x.to(torch.float64)
    a = a.view(rb, rows, kb, BLOCK)
    top = a.abs().amax(dim=(1, 3), keepdim=True)
    r = (_largest(name) / top).float().to(torch.float64)
    q = _rounded((a * r).float().to(torch.float64).nan_to_num(0.0), name)
    scale = (top / _largest(name)).float()[:, 0, :, 0]
    return q.view(rb * rows, kb * BLOCK)[:R, :K], scale.t()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    d = torch.float64
    if kind == "matmul":
        at = torch.arange(case["K"], device=DEVICE) // BLOCK
        to = torch.arange(case["N"], device=DEVICE) // case["rows"]
        X = s["X"].to(d) * s["sx"].to(d)[at].t()
        W = s["W"].to(d) * s["sw"].to(d)[at][:, to].t()
        y = X @ W.t()
        return y if s["b"] is None else y + s["b"].to(d)[None, :]
    if kind == "quantize":
        out = _quantize_exact(s["X"], case["rows"], case["q"])
        if case["form"] == "both":
            out += _quantize_exact(s["X"].t(), case["rows"], case["q"])
        return out
    S = s["X"].to(d)
    if s["R"] is not None:                          # the sum is kept in the type of X
        S = (S + s["R"].to(d)).float().to(_dtype(case["dtype"])).to(d)
    K = case["K"]
    gamma = torch.ones(K, dtype=d, device=DEVICE) if s["gamma"] is None else s["gamma"].to(d)
    beta = torch.zeros(K, dtype=d, device=DEVICE) if s["beta"] is None else s["beta"].to(d)
    train = kind == "train"
    leaves = [S, gamma, beta]
    with torch.set_grad_enabled(train):
        for v in leaves:
            v.requires_grad_(train)
        y = torch.nn.functional.layer_norm(S, (K,), gamma, beta, EPS)
        if not train:
            return _outputs(s, y, S)
        dx, dgamma, dbeta = torch.autograd.grad(y, leaves, s["dY"].to(d))
    if s["dS"] is not None:
        dx = dx + s["dS"].to(d)
    return _outputs(s, y.detach(), S.detach(), dx, *((dgamma, dbeta) if case["affine"] else ()))
