"""The operators of a layer in bf16 and of the update of its weight, as they are timed.

`kind` of a case:

  linear       linear: x W^T with bias, activation and residual in the product's epilogue, from one token to a
               training micro-batch; with `pre` the pre-activation is written too, as the backward pass needs it;
  linear_grad  linear_backward: the gradients of that layer with respect to its input, its weight and its bias;
  ortho        orthogonalize: Newton-Schulz steps on the short side's Gram matrix, which bring the singular values of an
               update (of one matrix or of several of a shape) near one.

Sizes are those of the repository's workloads (hidden sizes of 4,096 and 2,048; 4 x 256 tokens) and generic ones around
them, odd ones among them.  All values are drawn from the seed."""

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
ACTS = ["relu", "gelu", "gelu_tanh", "silu"]
STEPS, EPS = 5, 1e-7
QUINTIC = (3.4445, -4.7750, 2.0315)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MOST_LINEAR, MOST_GRAD, MOST_ORTHO = 5.4e11, 2.1e12, 4.0e12    # flops of a drawn case


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------

def _linear(M, K, N, **more):
    return {"kind": "linear", "M": M, "K": K, "N": N, "act": None, "bias": "f32", "residual": None, "pre": False, "out": "bf16",
            **more}


def _grad(M, K, N, **more):
    return {"kind": "linear_grad", "M": M, "K": K, "N": N, "act": None, "bias": True, "dw": "bf16", **more}


def _ortho(B, m, n, **more):
    return {"kind": "ortho", "B": B, "m": m, "n": n, "dtype": "f32", **more}


def listed():
    return [
        # one token through a square layer: latency, and the weight's bytes
        _linear(1, 4096, 4096, act="silu", name="linear_token"),
        # a handful of tokens through the widening layer of a block
        _linear(7, 2048, 8200, act="gelu_tanh", bias="bf16", name="linear_few"),
        # a batch of single tokens, one for each response, back to the residual stream
        _linear(48, 16384, 4096, residual="bf16", name="linear_decode"),
        # odd sizes throughout, the sum kept in 32 bits
        _linear(1003, 1027, 2051, act="relu", residual="f32", out="f32", name="linear_ragged"),
        # a training micro-batch of 4,096 tokens through the widening layer, its pre-activation kept
        _linear(4096, 4096, 16384, act="gelu", bias="bf16", pre=True, name="linear_train"),
        # the gradients of a small layer of the smallest batch, 4 x 256 tokens
        _grad(1024, 1024, 1024, act="silu", name="grad_small"),
        # odd rows, no activation, the weight's gradient in 32 bits for an fp32 master copy
        _grad(2507, 2048, 4104, dw="f32", name="grad_ragged"),
        # a micro-batch of 8,192 tokens through the widening layer, backwards
        _grad(8192, 4096, 16384, act="gelu", name="grad_large"),
        # one small matrix: latency
        _ortho(1, 256, 256, name="ortho_small"),
        # the square projections of all blocks at once, momentum in bf16
        _ortho(24, 1024, 1024, dtype="bf16", name="ortho_batch"),
        # a tall matrix of odd sizes
        _ortho(1, 2051, 1000, name="ortho_tall"),
        # the widening layer of a large block
        _ortho(1, 4096, 16384, name="ortho_large"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_grad", "ortho"])
    if kind == "ortho":
        m, n = _log_int(rng, 64, 4096), _log_int(rng, 64, 16384)
        if rng.random() < 0.5:
            m, n = m // 8 * 8, n // 8 * 8
        B = rng.choice([1, 1, 1, _log_int(rng, 2, 32)])
        if rng.random() < 0.4:
            m, n = n, m
        B = max(1, min(B, int(MOST_ORTHO / _ortho_flops(1, m, n)), 300_000_000 // (m * n)))
        return _ortho(B, m, n, dtype=rng.choice(["f32", "bf16"]))
    K, N = _log_int(rng, 64, 8192), _log_int(rng, 64, 16384)
    if rng.random() < 0.6:
        K, N = (K + 7) // 8 * 8, (N + 7) // 8 * 8
    act = rng.choice([None] + ACTS)
    if kind == "linear":
        M = _log_int(rng, 1, max(1, min(8192, int(MOST_LINEAR / (2 * K * N)))))
        return _linear(M, K, N, act=act, bias=rng.choice([None, "f32", "bf16"]), residual=rng.choice([None, "f32", "bf16"]),
                       pre=act is not None and rng.random() < 0.4, out=rng.choice(["bf16", "bf16", "f32"]))
    M = _log_int(rng, 16, max(16, min(8192, int(MOST_GRAD / (4 * K * N)))))
    return _grad(M, K, N, act=act, bias=rng.random() < 0.7, dw="bf16" if act else rng.choice(["bf16", "f32"]))


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _matrix(R, C, gen, std, outliers=False):
    """Normal values in bf16 whose rows start on 16 bytes; with `outliers` rows that differ in size and a few larger columns."""
    x = torch.empty((R, (C + 7) // 8 * 8), device=DEV).normal_(0.0, std, generator=gen)
    if outliers:
        x.mul_(torch.exp(0.3 * torch.randn((R, 1), generator=gen, device=DEV)))
        x[:, :: 97].mul_(6.0)
    return x.to(torch.bfloat16)[:, :C]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = SimpleNamespace(case=case, kind=case["kind"])
    if s.kind == "ortho":
        # a weight's momentum: a few strong directions, many weak ones
        B, m, n = case["B"], case["m"], case["n"]
        r = min(32, m, n)
        size = 0.7 ** torch.arange(r, device=DEV)
        left = torch.randn((B, m, r), generator=gen, device=DEV) * size
        g = left @ torch.randn((B, r, n), generator=gen, device=DEV)
        g += 0.2 * torch.randn((B, m, n), generator=gen, device=DEV)
        s.g = (g * 1e-3).to(DTYPES[case["dtype"]])
        if B == 1:
            s.g = s.g[0]
        return s
    M, K, N = case["M"], case["K"], case["N"]
    s.x = _matrix(M, K, gen, 1.0, outliers=True)
    s.w = _matrix(N, K, gen, K ** -0.5)
    if s.kind == "linear":
        s.bias = s.residual = None
        if case["bias"]:
            s.bias = (0.1 * torch.randn(N, generator=gen, device=DEV)).to(DTYPES[case["bias"]])
        if case["residual"]:
            s.residual = torch.empty((M, (N + 7) // 8 * 8), device=DEV).normal_(generator=gen).to(DTYPES[case["residual"]])[:, :N]
        return s
    s.dy = _matrix(M, N, gen, 1e-3, outliers=True)
    s.pre = _matrix(M, N, gen, 1.2) if case["act"] else None
    return s


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------

def _sigmoid(x):
    return 1 / (1 + torch.exp(-x))


def _plain_act(act, x):
    if act is None:
        return x
    if act == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x))
    if act == "silu":
        return x * _sigmoid(x)
    if act == "gelu":
        return 0.5 * x * torch.erfc(-x * math.sqrt(0.5))
    return x * _sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x))


def _plain_slope(act, x):
    """The activation's derivative."""
    if act == "relu":
        return (x > 0).float()
    if act == "silu":
        p = _sigmoid(x)
        return p * (1 + x * (1 - p))
    if act == "gelu":
        return 0.5 * torch.erfc(-x * math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    k = 2 * math.sqrt(2 / math.pi)
    p = _sigmoid(k * (x + 0.044715 * x * x * x))
    return p + x * p * (1 - p) * k * (1 + 3 * 0.044715 * x * x)


def _plain(s):
    case = s.case
    if s.kind == "linear":
        pre = s.x.float() @ s.w.float().t()
        if s.bias is not None:
            pre = pre + s.bias.float()
        y = _plain_act(case["act"], pre)
        if s.residual is not None:
            y = y + s.residual.float()
        out = {"out": y.to(DTYPES[case["out"]])}
        if case["pre"]:
            out["pre"] = pre.to(torch.bfloat16)
        return out
    if s.kind == "linear_grad":
        g = s.dy.float()
        if case["act"]:
            g = g * _plain_slope(case["act"], s.pre.float())
        out = {"dx": (g @ s.w.float()).to(torch.bfloat16), "dw": (g.t() @ s.x.float()).to(DTYPES[case["dw"]])}
        if case["bias"]:
            out["dbias"] = g.double().sum(0).float()      # long sums
        return out
    x = s.g.float()
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-1, -2)
    norm = torch.sqrt((x.double() * x.double()).sum((-2, -1), keepdim=True))
    x = (x.double() / (norm + EPS)).float()
    a, b, c = QUINTIC
    for _ in range(STEPS):
        gram = x @ x.transpose(-1, -2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return {"out": (x.transpose(-1, -2) if tall else x).to(torch.bfloat16).contiguous()}


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def _framework(s):
    import paper_2607_24062_gb300 as acrl

    case = s.case
    if s.kind == "linear":
        pre = None
        if case["pre"]:
            N = case["N"]
            pre = torch.empty((case["M"], (N + 7) // 8 * 8), dtype=torch.bfloat16, device=DEV)[:, :N]
        out = {"out": acrl.linear(s.x, s.w, s.bias, act=case["act"], residual=s.residual, pre_out=pre, out_dtype=DTYPES[case["out"]])}
        if case["pre"]:
            out["pre"] = pre
        return out
    if s.kind == "linear_grad":
        dx, dw, dbias = acrl.linear_backward(s.dy, s.x, s.w, act=case["act"], pre=s.pre, bias=case["bias"], dw_dtype=DTYPES[case["dw"]])
        return {"dx": dx, "dw": dw, "dbias": dbias} if case["bias"] else {"dx": dx, "dw": dw}
    return {"out": acrl.orthogonalize(s.g, steps=STEPS, coeffs=QUINTIC, eps=EPS)}


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------
# work
# ---------------------------------------------------------------------------------------------------------------

def _ortho_flops(B, m, n):
    m, n = min(m, n), max(m, n)
    # a step: the Gram matrix and its square, half of each for symmetry, and the product with the iterate
    return B * STEPS * (m * m * n + m * m * m + 2 * m * m * n)


def work(case):
    size = {"bf16": 2, "f32": 4, None: 0}
    if case["kind"] == "ortho":
        B, m, n = case["B"], case["m"], case["n"]
        return {"bytes": B * m * n * (size[case["dtype"]] + 2), "flops": _ortho_flops(B, m, n)}
    M, K, N = case["M"], case["K"], case["N"]
    if case["kind"] == "linear":
        each = size[case["out"]] + size[case["residual"]] + (2 if case["pre"] else 0)
        return {"bytes": 2 * M * K + 2 * N * K + N * size[case["bias"]] + each * M * N, "flops": 2 * M * N * K}
    read = 2 * M * N * (2 if case["act"] else 1) + 2 * M * K + 2 * N * K
    return {"bytes": read + 2 * M * K + size[case["dw"]] * N * K + (4 * N if case["bias"] else 0), "flops": 4 * M * N * K}


# ---------------------------------------------------------------------------------------------------------------
# 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------

def _exact_act(act, x):
    """f(x) and f'(x)."""
    one = torch.ones_like(x)
    if act is None:
        return x, one
    if act == "relu":
        return x.clamp(min=0), (x > 0).double()
    if act == "silu":
        p = torch.sigmoid(x)
        return x * p, p + x * p * torch.sigmoid(-x)
    if act == "gelu":
        phi = (1 + torch.erf(x / 2 ** 0.5)) / 2
        return x * phi, phi + x * torch.exp(-x ** 2 / 2) / (2 * math.pi) ** 0.5
    u = (2 / math.pi) ** 0.5 * (x + 0.044715 * x ** 3)
    t = torch.tanh(u)
    return x * (1 + t) / 2, (1 + t) / 2 + x / 2 * (1 - t * t) * (2 / math.pi) ** 0.5 * (1 + 0.134145 * x ** 2)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if work(case)["flops"] > 8e12:
        return None
    if kind == "linear":
        pre = torch.einsum("mk,nk->mn", s.x.double(), s.w.double())
        if s.bias is not None:
            pre += s.bias.double()[None]
        y = _exact_act(case["act"], pre)[0]
        if s.residual is not None:
            y = y + s.residual.double()
        return {"out": y, "pre": pre} if case["pre"] else {"out": y}
    if kind == "linear_grad":
        g = s.dy.double()
        if case["act"]:
            g = g * _exact_act(case["act"], s.pre.double())[1]
        out = {"dx": torch.einsum("mn,nk->mk", g, s.w.double()), "dw": torch.einsum("mn,mk->nk", g, s.x.double())}
        if case["bias"]:
            out["dbias"] = torch.einsum("mn->n", g)
        return out
    # every iterate is a polynomial of the first Gram matrix times the first iterate: P_k(H) X, with Gram matrix P H P
    g = s.g.double()
    if g.dim() == 2:
        g = g[None]
    wide = g.shape[1] <= g.shape[2]
    x = g if wide else g.mT
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + EPS)
    a, b, c = QUINTIC
    gram = x @ x.mT
    eye = torch.eye(x.shape[1], dtype=torch.float64, device=x.device)
    P = eye.expand_as(gram)
    for _ in range(STEPS):
        Q = a * eye + gram @ (b * eye + c * gram)
        P, gram = Q @ P, Q @ gram @ Q
    out = P @ x
    out = out if wide else out.mT
    return {"out": (out if s.g.dim() == 3 else out[0]).contiguous()}
