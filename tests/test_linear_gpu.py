"""The bf16 layer and its gradients against the definitions in 64 bits."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2607_24062_gb300 as acrl  # noqa: E402
from paper_2607_24062_gb300 import api  # noqa: E402

DEV = "cuda"
ACTS = [None, "relu", "gelu", "gelu_tanh", "silu"]
BF, F32 = torch.bfloat16, torch.float32


def _matrix(R, C, seed, std=1.0, gap=0, dtype=BF):
    """Normal values, rows on 16 bytes; what lies between the rows is NaN."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.full((R, (C + 7) // 8 * 8 + gap), float("nan"), device=DEV, dtype=dtype)
    x[:, :C] = torch.randn((R, C), generator=g, device=DEV) * std
    return x[:, :C]


def _f(act, u):
    """The activation and its derivative in 64 bits."""
    one = torch.ones_like(u)
    if act is None:
        return u, one
    if act == "relu":
        return u.clamp(min=0), (u > 0).double()
    if act == "silu":
        p = torch.sigmoid(u)
        return u * p, p + u * p * torch.sigmoid(-u)
    if act == "gelu":
        p = torch.special.ndtr(u)
        return u * p, p + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (u + 0.044715 * u ** 3))
    return u * (1 + t) / 2, (1 + t) / 2 + u * (1 - t * t) / 2 * k * (1 + 3 * 0.044715 * u * u)


def _sum_error(K):
    """Of an fp32 sum of K terms, relative to the sum of their sizes: the tensor cores add sixteen terms at a time and may cut
    each partial sum off after its 24 bits (an error of 2^-23 of it for each sixteen, so K / 8 times 2^-24), and the sixteen and
    a few joins of partial sums among themselves."""
    return 2.0 ** -24 * (16 + K / 8)


def _between(got, exact, off, what=""):
    """Rounding is monotone: a result whose unrounded value is within `off` of the exact one lies between the roundings of the
    interval's ends."""
    lo, hi = (exact - off).to(got.dtype), (exact + off).to(got.dtype)
    bad = ~((got >= lo) & (got <= hi))
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:4], got[bad][:4], lo[bad][:4], hi[bad][:4])


def _check_linear(x, w, bias, act, residual, out, pre=None):
    X, W = x.double(), w.double()
    u, size = X @ W.t(), X.abs() @ W.abs().t()
    if bias is not None:
        u, size = u + bias.double(), size + bias.double().abs()
    off = _sum_error(x.shape[1]) * size + 1e-37
    if pre is not None:
        _between(pre, u, off, "pre")
    y = _f(act, u)[0]
    # the derivatives stay below 1.13, and the function is evaluated to a few units of 2^-24 of u
    off = 1.13 * off + (0.0 if act is None else 2.0 ** -20) * u.abs()
    if residual is not None:
        y = y + residual.double()
        off = off + 2.0 ** -23 * (y.abs() + residual.double().abs())
    _between(out, y, off, "out")


SIZES = [(1, 1, 1), (1, 130, 64), (1, 4096, 1024), (1, 1003, 4104), (2, 515, 1027), (3, 8, 8), (5, 300, 129), (8, 2051, 200),
         (16, 257, 640), (17, 128, 1000), (33, 4099, 72), (64, 515, 513), (128, 129, 2300), (129, 130, 65), (200, 300, 520),
         (256, 256, 4104), (257, 513, 63), (515, 1030, 264), (1300, 264, 2056), (131, 20000, 136), (3000, 520, 72)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_linear(M, N, K, dtype):
    x, w = _matrix(M, K, 1), _matrix(N, K, 2, std=K ** -0.5)
    _check_linear(x, w, None, None, None, acrl.linear(x, w, out_dtype=dtype))


@pytest.mark.parametrize("M,N,K", [(17, 33, 7), (24, 2051, 1030), (31, 520, 2051), (47, 1000, 1003), (60, 70, 9), (64, 2048, 2048), (64, 264, 520),
                                   (20, 16384, 1027), (48, 4100, 4104), (65, 264, 520), (100, 1000, 520), (128, 515, 513),
                                   (70, 20003, 1032), (128, 23000, 1500), (40, 12290, 200), (100, 6000, 515), (128, 8200, 40),
                                   (65, 131, 9000), (129, 264, 520), (200, 700, 77), (256, 768, 768), (255, 37, 1003)])
def test_up_to_256_rows(M, N, K):
    """What one kernel does in registers and the other in tensor memory, by size, with everything that follows the sum."""
    x, w = _matrix(M, K, 1, gap=8), _matrix(N, K, 2, std=K ** -0.5, gap=16)
    b, r = torch.randn(N, device=DEV), _matrix(M, N, 5, gap=8)
    pre = torch.full((M + 1, (N + 7) // 8 * 8 + 8), 7.0, dtype=BF, device=DEV)
    y = torch.full((M + 1, (N + 7) // 8 * 8 + 8), 7.0, dtype=F32, device=DEV)
    got = acrl.linear(x, w, b, act="silu", residual=r, pre_out=pre[:M, :N], out=y[:M, :N])
    _check_linear(x, w, b, "silu", r, got, pre[:M, :N])
    for t in (y, pre):
        assert bool((t[M:] == 7.0).all()) and bool((t[:, N:] == 7.0).all())


@pytest.mark.parametrize("M,N,K", [(3, 40, 264), (8, 130, 1003), (20, 40, 264), (30, 40, 1003), (64, 40, 268)])
def test_infinities_stay_in_their_row_and_column(M, N, K):
    """An infinity anywhere in a row, its first numbers included, makes its own results infinite or NaN and no others."""
    for k in (0, K - 1, K // 2):
        x, w = _matrix(M, K, 3), _matrix(N, K, 4)
        x[M // 2, k] = float("inf")
        w[N // 3, k] = float("-inf")
        y = acrl.linear(x, w, out_dtype=F32)
        want = x.float() @ w.float().t()
        assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(torch.isinf(y), torch.isinf(want))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias,residual,out,keep", [(F32, BF, BF, True), (BF, F32, F32, False), (F32, None, F32, True),
                                                    (None, BF, F32, False), (BF, BF, BF, True), (None, F32, BF, True)])
@pytest.mark.parametrize("M,N,K", [(1, 1031, 520), (6, 200, 1032), (40, 515, 300), (300, 515, 136)])
def test_epilogue(act, bias, residual, out, keep, M, N, K):
    x, w = _matrix(M, K, 3, gap=8), _matrix(N, K, 4, std=2 * K ** -0.5, gap=16)
    b = None if bias is None else torch.randn(N + 1, device=DEV).to(bias)[1:]      # no alignment but its own
    r = None if residual is None else _matrix(M, N, 5, gap=8, dtype=residual)
    pre = torch.full((M + 1, (N + 7) // 8 * 8 + 8), 7.0, dtype=BF, device=DEV) if keep else None
    y = torch.full((M + 1, (N + 7) // 8 * 8 + 8), 7.0, dtype=out, device=DEV)
    got = acrl.linear(x, w, b, act=act, residual=r, pre_out=pre[:M, :N] if keep else None, out=y[:M, :N])
    assert got.data_ptr() == y.data_ptr()
    _check_linear(x, w, b, act, r, got, pre[:M, :N] if keep else None)
    for t in (y, pre):
        if t is not None:    # nothing beyond the matrix is written
            assert bool((t[M:] == 7.0).all()) and bool((t[:, N:] == 7.0).all())


@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (16, 300, 4096), (300, 520, 264)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_residual_in_place(M, N, K, dtype):
    x, w, r = _matrix(M, K, 3), _matrix(N, K, 4, std=K ** -0.5), _matrix(M, N, 5, dtype=dtype)
    want = acrl.linear(x, w, act="silu", residual=r, out_dtype=dtype)
    acrl.linear(x, w, act="silu", residual=r, out=r)
    assert torch.equal(r, want)


@pytest.mark.parametrize("act", ACTS[1:])
def test_activations_over_their_range(act):
    """f and f' at values of every size, through products with the identity."""
    v = torch.cat([torch.linspace(-30, 30, 4001), torch.logspace(-30, 30, 121), -torch.logspace(-30, 30, 121),
                   torch.tensor([0.0, -0.0])]).to(DEV).to(BF)
    v = torch.nn.functional.pad(v, (0, -len(v) % 64)).view(-1, 64)
    one = torch.eye(64, device=DEV).to(BF)
    u = v.double()
    # the identity's other terms are zeros: u is exact
    y, slope = _f(act, u)
    out = acrl.linear(v, one, act=act, out_dtype=F32)
    _between(out, y, 2.0 ** -20 * u.abs() + 1e-37)
    ones = torch.ones_like(v)
    dx, dw, db = acrl.linear_backward(ones, v, one, act=act, pre=v, bias=True, dx_dtype=F32)
    # f' is a sum of terms of size 1 or u phi(u) and alike, and rounded to bf16 on the way
    at = 2.0 ** -19 * torch.ones_like(u)
    lo, hi = (slope - at).to(BF).double(), (slope + at).to(BF).double()
    assert bool(((dx.double() >= lo) & (dx.double() <= hi)).all())
    assert bool(((db.double() - slope.sum(0)).abs() <= (2.0 ** -19 + 2.0 ** -24 * len(v)) * len(v)).all())


def test_infinities_and_nan():
    """They reach what they touch and nothing else."""
    for M in (1, 4, 40, 300):
        x, w = _matrix(M, 200, 1), _matrix(150, 200, 2)
        x[M // 2, 7] = float("nan")
        nan = acrl.linear(x, w, act="relu").isnan()
        assert bool(nan[M // 2].all()) and int(nan.sum()) == 150
        x = _matrix(M, 200, 1)
        w[33, 5] = float("inf")
        y = acrl.linear(x, w)
        assert bool(y[:, 33].isinf().all()) and int(y.isfinite().sum()) == M * 149
        b = torch.zeros(150, device=DEV)
        b[149] = float("nan")
        w = _matrix(150, 200, 2)
        nan = acrl.linear(x, w, b, act="gelu").isnan()
        assert bool(nan[:, 149].all()) and int(nan.sum()) == M


BACK = [(1, 1, 1), (1, 130, 257), (3, 130, 257), (64, 64, 64), (129, 100, 40), (203, 328, 136), (600, 70, 1000), (257, 515, 130),
        (1300, 264, 300), (5000, 136, 72), (130, 2051, 520)]


def _check_backward(dy, x, w, act, pre, dx, dw, dbias):
    slope = torch.ones_like(dy.double()) if act is None else _f(act, pre.double())[1]
    g = dy.double() * slope
    # with an activation: its derivative's evaluation, and g's rounding to bf16 (2^-8) in the products
    each = torch.zeros_like(g) if act is None else 2.0 ** -19 * dy.double().abs()
    once = each if act is None else each + 2.0 ** -8 * g.abs()
    X, W = x.double(), w.double()
    M, N = dy.shape
    if dx is not None:
        _between(dx, g @ W, once @ W.abs() + _sum_error(N) * (g.abs() @ W.abs()) + 1e-37, "dx")
    if dw is not None:
        _between(dw, g.t() @ X, once.t() @ X.abs() + _sum_error(M) * (g.abs().t() @ X.abs()) + 1e-37, "dw")
    if dbias is not None:
        off = each.sum(0) + 2.0 ** -24 * (256 + M / 128) * g.abs().sum(0) + 1e-37
        _between(dbias, g.sum(0), off, "dbias")


@pytest.mark.parametrize("M,N,K", BACK)
@pytest.mark.parametrize("dx_dtype,dw_dtype", [(BF, F32), (F32, BF)])
def test_backward(M, N, K, dx_dtype, dw_dtype):
    dy, x, w = _matrix(M, N, 8, std=1e-3, gap=8), _matrix(M, K, 9), _matrix(N, K, 10, std=0.02, gap=8)
    dx, dw, db = acrl.linear_backward(dy, x, w, bias=True, dx_dtype=dx_dtype, dw_dtype=dw_dtype)
    _check_backward(dy, x, w, None, None, dx, dw, db)


@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("M,N,K", [(1, 130, 72), (70, 515, 200), (300, 264, 520)])
def test_backward_through_activations(act, M, N, K):
    dy, x, w = _matrix(M, N, 8, std=1e-3), _matrix(M, K, 9), _matrix(N, K, 10, std=0.02)
    pre = _matrix(M, N, 11, std=1.5, gap=8)
    dx, dw, db = acrl.linear_backward(dy, x, w, act=act, pre=pre, bias=True)
    _check_backward(dy, x, w, act, pre, dx, dw, db)
    # each gradient alone is the same
    only = acrl.linear_backward(dy, x, w, act=act, pre=pre, need_dw=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    only = acrl.linear_backward(dy, x, w, act=act, pre=pre, need_dx=False)
    assert only[0] is None and torch.equal(only[1], dw)
    only = acrl.linear_backward(dy, x, w, act=act, pre=pre, need_dx=False, need_dw=False, bias=True)
    assert only[:2] == (None, None) and torch.equal(only[2], db)


@pytest.mark.parametrize("M,N,K", [(70, 37, 44), (300, 264, 250)])
def test_backward_writes_nothing_beyond_the_gradients(M, N, K):
    dy, x, w = _matrix(M, N, 8), _matrix(M, K, 9), _matrix(N, K, 10)
    for t in (BF, F32):
        dx = torch.full((M + 1, (K + 7) // 8 * 8 + 8), 3.0, dtype=t, device=DEV)
        dw = torch.full((N + 1, (K + 7) // 8 * 8 + 8), 3.0, dtype=t, device=DEV)
        db = torch.full((N + 1,), 3.0, device=DEV)
        acrl.linear_backward(dy, x, w, bias=True, dx=dx[:M, :K], dw=dw[:N, :K], dbias=db)
        _check_backward(dy, x, w, None, None, dx[:M, :K], dw[:N, :K], db[:N])
        for b, R in ((dx, M), (dw, N)):
            assert bool((b[R:] == 3.0).all()) and bool((b[:, K:] == 3.0).all())
        assert float(db[N]) == 3.0


def test_backward_against_differences():
    """Central differences of a loss of the layer's output, computed in 64 bits."""
    M, N, K = 37, 50, 40
    x, w, b, dy = _matrix(M, K, 1), _matrix(N, K, 2, std=0.3), torch.randn(N, device=DEV), _matrix(M, N, 3)
    for act in ACTS:
        pre = torch.empty((M, 56), dtype=BF, device=DEV)[:, :N]
        acrl.linear(x, w, b, act=act, pre_out=pre)
        dx, dw, db = acrl.linear_backward(dy, x, w, act=act, pre=None if act is None else pre, bias=True, dx_dtype=F32)
        loss = lambda X, W, B: (dy.double() * _f(act, X @ W.t() + B)[0]).sum()   # noqa: E731
        X, W, B = x.double(), w.double(), b.double()
        gen = torch.Generator(device=DEV).manual_seed(5)
        for name, t, grad in (("x", X, dx), ("w", W, dw), ("b", B, db)):
            d = torch.randn(t.shape, generator=gen, device=DEV, dtype=torch.float64)
            h = 1e-4
            at = lambda s: loss(*(v + s * h * d if v is t else v for v in (X, W, B)))   # noqa: E731
            diff = float((at(1) - at(-1)) / (2 * h))
            got = float((grad.double() * d).sum())
            # pre is rounded to bf16 (its error, 2^-8 |u|, times the second derivative, at most 1.2, shifts f'; relu's jumps
            # where u is near 0) and so is g: a part in 2^-7 or so of each term's size, with random signs; and h^2 terms
            size = float((grad.double() * d).norm()) + 1e-9
            assert abs(got - diff) <= 16 * 2.0 ** -8 * size + 1e-6 * abs(diff), (act, name, got, diff, size)


def test_nothing():
    w = _matrix(20, 64, 1)
    assert acrl.linear(_matrix(3, 64, 2)[:0], w).shape == (0, 20)
    assert acrl.linear(_matrix(3, 64, 2), w[:0]).shape == (3, 0)
    x0, w0 = torch.empty((3, 0), dtype=BF, device=DEV), torch.empty((5, 0), dtype=BF, device=DEV)
    b = torch.arange(5.0, device=DEV) - 2
    assert torch.equal(acrl.linear(x0, w0, b, act="relu", out_dtype=F32), b.clamp(min=0).expand(3, 5))
    dx, dw, db = acrl.linear_backward(_matrix(3, 20, 2)[:0], _matrix(3, 64, 3)[:0], w, bias=True)
    assert dx.shape == (0, 64) and dw.shape == (20, 64) and not bool(dw.any()) and db.shape == (20,) and not bool(db.any())
    dx, dw, db = acrl.linear_backward(_matrix(3, 20, 2)[:, :0], _matrix(3, 64, 3), w[:0], bias=True)
    assert dx.shape == (3, 64) and not bool(dx.any()) and dw.shape == (0, 64) and db.shape == (0,)
    dx, dw, db = acrl.linear_backward(_matrix(3, 20, 2), x0, torch.empty((20, 0), dtype=BF, device=DEV), bias=True)
    assert dx.shape == (3, 0) and dw.shape == (20, 0) and db.shape == (20,) and bool(db.any())


def _same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


def test_equal_inputs_give_equal_outputs():
    for M, N, K in ((1, 4096, 4096), (40, 300, 8192), (700, 520, 1032)):
        x, w, dy = _matrix(M, K, 1), _matrix(N, K, 2, std=0.02), _matrix(M, N, 3)
        first = acrl.linear(x, w, act="gelu"), *acrl.linear_backward(dy, x, w, bias=True)
        for _ in range(3):
            assert _same(first, (acrl.linear(x, w, act="gelu"), *acrl.linear_backward(dy, x, w, bias=True)))


def test_other_stream_and_its_memory():
    """On another stream, what a call allocates is that stream's: memory that the current one still writes is not used."""
    M, N, K = 300, 520, 1032
    x, w, dy, pre = _matrix(M, K, 1), _matrix(N, K, 2, std=0.02), _matrix(M, N, 3), _matrix(M, N, 4)
    x1 = _matrix(40, K, 5)
    calls = lambda **kw: (acrl.linear(x, w, act="silu", **kw), acrl.linear(x1, w, **kw),   # noqa: E731
                          *acrl.linear_backward(dy, x, w, act="silu", pre=pre, bias=True, **kw))
    want = [t.clone() for t in calls()]
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    for _ in range(20):
        big = torch.tanh(big @ big)
    for size in (api.linear_workspace_bytes(40, N, K), api.linear_backward_workspace_bytes(M, N, K), M * N * 2, M * K * 2, N * K * 4):
        for _ in range(3):
            torch.empty(max(size, 1), dtype=torch.uint8, device=DEV).fill_(255)
    got = calls(stream=side)
    torch.cuda.synchronize()
    assert _same(want, got)


def test_captured_and_replayed():
    """Two graphs, each with the workspaces of its own pool, replayed by turns and at once."""
    M, N, K = 260, 300, 1032
    sets = [(_matrix(M, K, i), _matrix(N, K, i + 10, std=0.02), _matrix(M, N, i + 20), _matrix(M, N, i + 30)) for i in (1, 2)]
    run = lambda x, w, dy, pre: (acrl.linear(x, w, act="gelu", residual=pre), acrl.linear(x[:9], w),   # noqa: E731
                                 *acrl.linear_backward(dy, x, w, act="gelu", pre=pre, bias=True))
    want = [[t.clone() for t in run(*s)] for s in sets]
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(*s))
        graphs.append(g)
    for _ in range(2):
        for o in outs:
            for t in o:
                t.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(_same(w, o) for w, o in zip(want, outs))
    side = torch.cuda.Stream()
    for _ in range(5):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
    torch.cuda.synchronize()
    assert all(_same(w, o) for w, o in zip(want, outs))


def test_layer_captured_with_its_backward():
    """A forward and its backward in one graph, replayed on other values, gives what the same calls give eagerly."""
    M, N, K = 70, 264, 136
    x, w = _matrix(M, K, 1).requires_grad_(), _matrix(N, K, 2, std=0.1).requires_grad_()
    b, r = torch.randn(N, device=DEV).requires_grad_(), _matrix(M, N, 3).requires_grad_()
    dy = _matrix(M, N, 4)
    run = lambda: torch.autograd.grad(acrl.linear_layer(x, w, b, "gelu", r), (x, w, b, r), dy)   # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for seed in (5, 6):
        with torch.no_grad():
            x.copy_(_matrix(M, K, seed))
            w.copy_(_matrix(N, K, seed + 2, std=0.1))
            dy.copy_(_matrix(M, N, seed + 4))
        g.replay()
        torch.cuda.synchronize()
        assert _same(run(), got)


def test_more_than_two_to_the_31_elements():
    """An output whose offsets pass 32 bits, of rows that hold one value each."""
    M, N, K = 70000, 32768, 8
    x, w = torch.zeros((M, K), dtype=BF, device=DEV), torch.zeros((N, K), dtype=BF, device=DEV)
    x[:, 0] = (torch.arange(M, device=DEV) % 251).to(BF)
    w[:, 0] = 1.0
    y = acrl.linear(x, w)
    for i in range(0, M, 10000):
        assert bool((y[i: i + 10000] == x[i: i + 10000, :1]).all())
    dx, dw, db = acrl.linear_backward(y, x, w, bias=True, dx_dtype=F32)
    assert torch.equal(dx[:, 0], x[:, 0].float() * N)                             # whole numbers, exact in fp32
    total = float((x[:, 0].double() ** 2).sum())
    assert bool(((dw[:, 0].double() - total).abs() <= _sum_error(M) * total).all()) and not bool(dw[:, 1:].any())
    assert bool((db.double() == float(x[:, 0].double().sum())).all())             # below 2^24


@pytest.mark.parametrize("M,K", [(1, 2 ** 31 - 8200), (17, 2 ** 28 + 8)])
def test_the_longest_sums(M, K):
    """A few terms at both ends and in the middle of rows as long as the call takes; fewer rows of it where 17 would not fit."""
    x, w = torch.zeros((M, K), dtype=BF, device=DEV), torch.zeros((3, K), dtype=BF, device=DEV)
    for i, k in enumerate((0, 5000, K // 2, K - 1)):
        x[:, k], w[1, k] = i + 1.0, 2.0 ** i
    y = acrl.linear(x, w, out_dtype=F32)
    assert bool((y[:, 1] == 1 + 4 + 12 + 32).all()) and not bool(y[:, 0].any()) and not bool(y[:, 2].any())


@pytest.mark.parametrize("M", [5, 60, 300])
def test_long_sums_of_one_sign(M):
    """Terms that are all alike add up without a drift: every partial sum is rounded, or short enough.  (Cut off after its 24
    bits at each step of sixteen terms, a sum of 2^17 ones and a bit would lose up to 2^13 times 2^-24 of it.)"""
    K = 2 ** 17
    x, w = torch.full((M, K), 1.0 + 2.0 ** -7, dtype=BF, device=DEV), torch.full((70, K), 1.0 - 2.0 ** -8, dtype=BF, device=DEV)
    exact = K * (1.0 + 2.0 ** -7) * (1.0 - 2.0 ** -8)
    y = acrl.linear(x, w, out_dtype=F32).double()
    # runs of 512 terms at most are exact to 2^-23 of themselves a step (32 steps), and at most 256 of them, or 1,024, add up
    assert bool(((y - exact).abs() <= exact * (2.0 ** -23 * 32 + 2.0 ** -24 * 1024)).all())
    # the same in bf16, of runs of 32,768: 2,048 steps
    y = acrl.linear(x, w).double()
    assert bool(((y - exact).abs() <= exact * (2.0 ** -8 + 2.0 ** -23 * 2048)).all())


def test_refusals():
    x, w = _matrix(8, 64, 1), _matrix(16, 64, 2)
    dy = _matrix(8, 16, 3)
    wide = torch.empty((8, 40), dtype=BF, device=DEV)
    for call in (lambda: acrl.linear(x.float(), w), lambda: acrl.linear(x, w.half()), lambda: acrl.linear(x.cpu(), w),
                 lambda: acrl.linear(x, w[:, :32]), lambda: acrl.linear(x, w.t()), lambda: acrl.linear(x[None], w),
                 lambda: acrl.linear(torch.empty((4, 9), dtype=BF, device=DEV), torch.empty((4, 9), dtype=BF, device=DEV)),
                 lambda: acrl.linear(x, w, act="tanh"), lambda: acrl.linear(x, w, out_dtype=torch.float16),
                 lambda: acrl.linear(x, w, torch.zeros(15, device=DEV)), lambda: acrl.linear(x, w, torch.zeros(16)),
                 lambda: acrl.linear(x, w, torch.zeros(16, device=DEV, dtype=torch.float64)),
                 lambda: acrl.linear(x, w, torch.zeros(32, device=DEV)[::2]),
                 lambda: acrl.linear(x, w, residual=dy.half()), lambda: acrl.linear(x, w, residual=dy[:4]),
                 lambda: acrl.linear(x, w, residual=dy[:1].expand(8, 16)), lambda: acrl.linear(x, w, residual=wide[:, 4:20]),
                 lambda: acrl.linear(x, w, pre_out=dy.float()), lambda: acrl.linear(x, w, out=wide[:, 1:17]),
                 lambda: acrl.linear(x, w, out=torch.empty((8, 8), dtype=BF, device=DEV)),
                 lambda: acrl.linear_backward(dy, x, w, act="gelu"), lambda: acrl.linear_backward(dy, x, w, pre=dy),
                 lambda: acrl.linear_backward(dy, x[:4], w), lambda: acrl.linear_backward(dy, x, w[:8]),
                 lambda: acrl.linear_backward(dy.float(), x, w), lambda: acrl.linear_backward(dy, x, w, dw_dtype=torch.float16),
                 lambda: acrl.linear_backward(dy, x, w, need_dx=False, dx=torch.empty_like(x)),
                 lambda: acrl.linear_backward(dy, x, w, dbias=torch.empty(16, device=DEV)),
                 lambda: acrl.linear_backward(dy, x, w, bias=True, dbias=torch.empty(8, device=DEV)),
                 lambda: acrl.linear_backward(dy, x, w, act="relu", pre=dy,
                                              workspace=torch.empty(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(acrl.AcrlError):
            call()


def test_layer_in_a_graph():
    """linear_layer for autograd: rows of no particular alignment, a broadcast residual, each gradient against the entry points."""
    M, N, K = 33, 131, 70
    x, w = (torch.randn((r, K), device=DEV).to(BF).requires_grad_() for r in (M, N))
    b = torch.randn(N, device=DEV).requires_grad_()
    r = torch.randn((1, N), device=DEV).requires_grad_()
    for act in ACTS:
        for t in (x, w, b, r):
            t.grad = None
        y = acrl.linear_layer(x, w, b, act, r.expand(M, N))
        _check_linear(x.detach(), w.detach(), b.detach(), act, r.detach().expand(M, N), y.detach())
        dy = torch.randn((M, N), device=DEV).to(BF)
        y.backward(dy)
        pre = _matrix(M, N, 1)
        pad = lambda t: torch.nn.functional.pad(t.detach(), (0, -t.shape[1] % 8))[:, : t.shape[1]]   # noqa: E731
        acrl.linear(pad(x), pad(w), b.detach(), pre_out=pre)
        dx, dw, db = acrl.linear_backward(pad(dy), pad(x), pad(w), act=act, pre=None if act is None else pre, bias=True, dw_dtype=BF)
        assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw) and torch.equal(b.grad, db)
        assert bool(((r.grad.double() - dy.double().sum(0)).abs() <= 2.0 ** -24 * M * dy.double().abs().sum(0)).all())
    # bf16 bias, no gradient for the input; and none for anything but the residual
    b16 = b.detach().to(BF).requires_grad_()
    acrl.linear_layer(x.detach(), w, b16, "relu").sum().backward()
    assert b16.grad.dtype == BF and b16.grad.shape == (N,)
    res = torch.randn((M, N), device=DEV).to(BF).requires_grad_()
    acrl.linear_layer(x.detach(), w.detach(), None, "silu", res).backward(dy)
    assert torch.equal(res.grad, dy)


def test_layer_keeps_its_gradient_when_replayed_or_repeated():
    x, w = _matrix(40, 64, 1).contiguous().requires_grad_(), _matrix(24, 64, 2).contiguous().requires_grad_()
    y = acrl.linear_layer(x, w, act="gelu")
    dy = torch.ones_like(y)
    a = torch.autograd.grad(y, (x, w), dy, retain_graph=True)
    for t in a:
        t.add_(1.0)
    b = torch.autograd.grad(y, (x, w), dy)
    assert all(torch.equal(p - 1.0, q) or bool(((p.double() - 1.0 - q.double()).abs() <= 2.0 ** -7 * (p.double().abs() + 1)).all())
               for p, q in zip(a, b))
    y = acrl.linear_layer(x, w, act="gelu")
    dx, = torch.autograd.grad(y.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dx.float().sum().backward()
