"""8-bit matrices and their products against the definitions in 64 bits."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2607_24062_gb300 as acrl  # noqa: E402
from paper_2607_24062_gb300 import api  # noqa: E402

DEV = "cuda"
FORMATS = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}


def _plain_quantize(x, block, fmt, transpose=False):
    """(values of q, scales) of a float64 numpy matrix, from the definition."""
    top, bits, low = FORMATS[fmt]
    x = x.T if transpose else x
    R, C = x.shape
    h = 128 if block == "tile" else 1
    q = np.zeros((R, C))
    scale = np.zeros(((R + h - 1) // h, (C + 127) // 128))
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            at = (slice(i * h, (i + 1) * h), slice(j * 128, (j + 1) * 128))
            b = x[at]
            a = np.abs(b).max()
            if not np.isfinite(a):
                q[at], scale[i, j] = np.nan, np.nan
                continue
            e = -127
            while a > top * 2.0 ** e:
                e += 1
            scale[i, j] = 2.0 ** e if a > 0 else 1.0
            y = b / scale[i, j]
            step = 2.0 ** (np.maximum(np.frexp(np.abs(y))[1] - 1, low) - bits)
            q[at] = np.round(y / step) * step          # numpy rounds halves to even
    return q, scale


def _scales(t):
    e = t.scale.cpu().numpy().astype(np.float64)
    return np.where(e == 255, np.nan, 2.0 ** (e - 127))


def _matrix(R, C, seed, dtype=torch.bfloat16, std=1.0, gap=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ld = (C + 7) // 8 * 8 + gap
    x = torch.randn((R, ld), generator=g, device=DEV) * std * torch.exp2(torch.randint(-9, 9, (R, ld), generator=g, device=DEV) * 0.5)
    return x.to(dtype)[:, :C]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block,transpose", [("row", False), ("row", True), ("tile", False), ("tile", True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,C,gap", [(1, 1, 0), (1, 128, 8), (3, 129, 0), (130, 257, 16), (257, 1000, 8), (129, 17, 0)])
def test_quantize(fmt, block, transpose, dtype, R, C, gap):
    x = _matrix(R, C, 11 * R + C, dtype, gap=gap)
    t = acrl.fp8_quantize(x, block=block, fmt=fmt, transpose=transpose)
    q, s = _plain_quantize(x.double().cpu().numpy(), block, fmt, transpose)
    assert np.array_equal(t.q.float().cpu().numpy().astype(np.float64), q)
    assert np.array_equal(_scales(t), s)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantize_extremes(fmt):
    """Blocks of zeros, of subnormals, of the type's largest, at the edge of a scale, and with an infinity or a NaN."""
    top = FORMATS[fmt][0]
    x = torch.zeros((9, 256), device=DEV)
    x[1, :128] = 1e-40
    x[2, 5] = 3.3895e38
    x[2, 6] = 1e-30
    x[3, 7], x[3, 8] = top * 2.0 ** -20, -top * 2.0 ** -21
    x[4, 7] = float(np.nextafter(np.float32(top * 2.0 ** -20), np.float32(np.inf)))
    x[5, 9] = float("inf")
    x[6, 9] = float("nan")
    x[7, 130], x[7, 131] = -float("inf"), 1.0
    x[8] = 2.0 ** -126
    flags = api.new_flags()
    t = acrl.fp8_quantize(x, fmt=fmt, flags=flags)
    q, s = _plain_quantize(x.double().cpu().numpy(), "row", fmt)
    assert np.array_equal(t.q.float().cpu().numpy().astype(np.float64), q, equal_nan=True)
    assert np.array_equal(_scales(t), s, equal_nan=True)
    assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE
    flags = api.new_flags()
    acrl.fp8_quantize(x[:5], fmt=fmt, flags=flags)
    assert acrl.read_flags(flags) == 0


def test_quantize_writes_nothing_beyond_the_matrix():
    x = _matrix(37, 100, 5)
    q = torch.full((40, 112), 0x55, dtype=torch.uint8, device=DEV)
    s = torch.full((40, 4), 0x55, dtype=torch.uint8, device=DEV)
    acrl.fp8_quantize(x, out=acrl.Fp8Tensor(q[:37, :100].view(torch.float8_e4m3fn), s[:37, :1]))
    assert bool((q[37:] == 0x55).all()) and bool((q[:, 100:] == 0x55).all())
    assert bool((s[37:] == 0x55).all()) and bool((s[:, 1:] == 0x55).all())
    qt = torch.full((101, 48), 0x55, dtype=torch.uint8, device=DEV)
    st = torch.full((101, 4), 0x55, dtype=torch.uint8, device=DEV)
    acrl.fp8_quantize(x, transpose=True, out=acrl.Fp8Tensor(qt[:100, :37].view(torch.float8_e4m3fn), st[:100, :1]))
    assert bool((qt[100:] == 0x55).all()) and bool((qt[:, 37:] == 0x55).all())
    assert bool((st[100:] == 0x55).all()) and bool((st[:, 1:] == 0x55).all())


def _product(a, b):
    """The exact product in float64 and the sum of the terms' absolute values."""
    A, B = a.values().double().cpu().numpy(), b.values().double().cpu().numpy()
    return A @ B.T, np.abs(A) @ np.abs(B).T


def _check_product(out, a, b):
    """fp32 sums of K terms: an error of at most 2^-24 max(4, sqrt(K)) sum |terms| before the one rounding to the output's
    type, so the output lies between the roundings of the ends of that interval (rounding is monotone)."""
    exact, size = _product(a, b)
    off = 2.0 ** -24 * max(4.0, np.sqrt(a.shape[1])) * size + 1e-37
    lo, hi = (torch.from_numpy(v).to(DEV).to(out.dtype) for v in (exact - off, exact + off))
    bad = ~((out >= lo) & (out <= hi))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4], out[bad][:4], lo[bad][:4], hi[bad][:4])


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 130, 128), (5, 300, 129), (16, 257, 640), (17, 128, 1000), (64, 515, 513),
                                   (128, 129, 300), (3, 200, 4100), (128, 300, 2100), (100, 64, 9001), (2, 5000, 2600),
                                   (129, 16, 256), (257, 500, 640), (513, 449, 384), (2100, 700, 130), (200, 300, 520), (300, 257, 2047), (1000, 1111, 1280)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matmul(M, N, K, dtype):
    a = acrl.fp8_quantize(_matrix(M, K, 1))
    b = acrl.fp8_quantize(_matrix(N, K, 2, std=0.02), block="tile")
    _check_product(acrl.fp8_matmul(a, b, out_dtype=dtype), a, b)


@pytest.mark.parametrize("M,N,K", [(2500, 2001, 1500), (517, 8203, 1500), (260, 33003, 1300), (513, 24001, 1700)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_matmul_of_many_columns(M, N, K, dtype):
    """Tiles of more columns than an instruction's, once and several times over; nothing beyond the matrix is written."""
    a = acrl.fp8_quantize(_matrix(M, K, 31))
    b = acrl.fp8_quantize(_matrix(N, K, 32, std=0.02))
    out = torch.full((M + 1, (N + 7) // 8 * 8), 7.0, dtype=dtype, device=DEV)
    _check_product(acrl.fp8_matmul(a, b, out=out[:M]), a, b)
    assert bool((out[M:] == 7.0).all()) and bool((out[:, N:] == 7.0).all())


@pytest.mark.parametrize("fa,fb", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("ba,bb", [("row", "row"), ("tile", "row"), ("tile", "tile")])
@pytest.mark.parametrize("M,N,K", [(40, 200, 700), (333, 140, 900)])
def test_matmul_formats_and_blocks(fa, fb, ba, bb, M, N, K):
    a = acrl.fp8_quantize(_matrix(M, K, 3), fmt=fa, block=ba)
    b = acrl.fp8_quantize(_matrix(N, K, 4), fmt=fb, block=bb)
    _check_product(acrl.fp8_matmul(a, b, out_dtype=torch.float32), a, b)


@pytest.mark.parametrize("M,N,K,gap", [(1, 1000, 520, 0), (1, 1, 1, 7), (2, 17000, 136, 0), (3, 301, 4104, 8), (4, 77, 1000, 0),
                                       (4, 40, 4104, 0), (7, 300, 1032, 8), (130, 513, 264, 16)])
def test_linear_is_quantise_then_product(M, N, K, gap):
    x = _matrix(M, K, 6, gap=gap)
    w = acrl.fp8_quantize(_matrix(N, K, 7, std=0.02), block="tile")
    got = acrl.fp8_linear(x, w)
    assert torch.equal(got, acrl.fp8_matmul(acrl.fp8_quantize(x), w))
    _check_product(got, acrl.fp8_quantize(x), w)


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (3, 130, 257), (129, 100, 40), (203, 328, 136), (600, 70, 1000)])
@pytest.mark.parametrize("fmt,x_fmt", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")])
def test_linear_backward(M, N, K, fmt, x_fmt):
    x, dy, w = _matrix(M, K, 8, gap=8), _matrix(M, N, 9, std=1e-3), _matrix(N, K, 10, std=0.02)
    wt = acrl.fp8_quantize(w, block="tile", transpose=True)
    dx, dw = acrl.fp8_linear_backward(dy, x, wt, fmt=fmt, x_fmt=x_fmt)
    # the products of what fp8_quantize makes, to the last bit
    assert torch.equal(dx, acrl.fp8_matmul(acrl.fp8_quantize(dy, fmt=fmt), wt))
    _check_product(dx, acrl.fp8_quantize(dy, fmt=fmt), wt)
    a, b = acrl.fp8_quantize(dy, fmt=fmt, transpose=True), acrl.fp8_quantize(x, fmt=x_fmt, transpose=True)
    assert torch.equal(dw, acrl.fp8_matmul(a, b, out_dtype=torch.float32))
    _check_product(dw, a, b)
    # the 8-bit weight is the same matrix either way round
    assert torch.equal(wt.values().t(), acrl.fp8_quantize(w, block="tile").values())


def test_linear_backward_of_nothing():
    wt = acrl.fp8_quantize(_matrix(30, 20, 1), block="tile", transpose=True)
    dx, dw = acrl.fp8_linear_backward(_matrix(3, 30, 2)[:0], _matrix(3, 20, 3)[:0], wt)
    assert dx.shape == (0, 20) and dw.shape == (30, 20) and not bool(dw.any())


def test_layer_in_a_graph():
    M, N, K = 33, 131, 72       # rows of N are no multiple of eight
    x, w = _matrix(M, K, 8).contiguous().requires_grad_(), _matrix(N, K, 10, std=0.02).contiguous().requires_grad_()
    y = acrl.fp8_layer(x, w)
    assert torch.equal(y, acrl.fp8_linear(x.detach(), acrl.fp8_quantize(w.detach(), block="tile")))
    dy = torch.randn((M, N), device=DEV).to(torch.bfloat16)
    y.backward(dy)
    wide = torch.zeros((M, 136), dtype=torch.bfloat16, device=DEV)
    wide[:, :N] = dy
    dx, dw = acrl.fp8_linear_backward(wide[:, :N], x.detach(), acrl.fp8_quantize(w.detach(), block="tile", transpose=True))
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw.to(torch.bfloat16))
    # near the gradients of the product in full precision: two operands, each within 2^-4 of its elements (e4m3)
    full = dy.double() @ w.detach().double()
    assert bool(((x.grad - full).abs() <= 0.13 * (dy.double().abs() @ w.detach().double().abs())).all())


def test_nan_blocks_reach_what_they_touch():
    for M in (4, 5):
        x = _matrix(M, 300, 12)
        x[2, 200] = float("nan")
        w = acrl.fp8_quantize(_matrix(140, 300, 13), block="tile")
        flags = api.new_flags()
        out = acrl.fp8_linear(x, w, flags=flags)
        assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE
        nan = out.isnan()
        assert bool(nan[2].all()) and not bool(nan[[0, 1, 3]].any())
        bad = _matrix(140, 300, 13)
        bad[130, 5] = float("inf")
        out = acrl.fp8_linear(_matrix(M, 300, 12), acrl.fp8_quantize(bad, block="tile"))
        assert bool(out[:, 128:].isnan().all()) and not bool(out[:, :128].isnan().any())


def test_products_of_nothing():
    w = acrl.fp8_quantize(_matrix(20, 64, 1), block="tile")
    assert acrl.fp8_linear(_matrix(3, 64, 2)[:0], w).shape == (0, 20)
    x0 = torch.empty((3, 0), dtype=torch.bfloat16, device=DEV)
    e = acrl.fp8_quantize(x0)
    assert e.shape == (3, 0)
    w0 = acrl.fp8_quantize(torch.empty((5, 0), dtype=torch.bfloat16, device=DEV))
    assert bool((acrl.fp8_matmul(e, w0) == 0).all())


def test_output_keeps_what_is_beyond_the_product():
    a = acrl.fp8_quantize(_matrix(300, 256, 3))
    for M in (1, 3, 70, 300):   # one row; both ways round inside the kernel
        for N in (37, 36, 250):
            for dtype in (torch.bfloat16, torch.float32):
                am = acrl.Fp8Tensor(a.q[:M], a.scale[:M])
                b = acrl.fp8_quantize(_matrix(N, 256, 4), block="tile")
                big = torch.full((M + 2, 264), 7.0, dtype=dtype, device=DEV)
                out = acrl.fp8_matmul(am, b, out=big[:M])
                _check_product(out, am, b)
                assert bool((big[M:] == 7).all()) and bool((big[:, N:] == 7).all())


def test_other_stream():
    x, w = _matrix(64, 512, 1), _matrix(700, 512, 2, std=0.02)
    want = acrl.fp8_linear(x, acrl.fp8_quantize(w, block="tile"))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = acrl.fp8_linear(x, acrl.fp8_quantize(w, block="tile", stream=s), stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_refusals():
    x = _matrix(8, 64, 1)
    w = acrl.fp8_quantize(x, block="tile")
    for call in (lambda: acrl.fp8_quantize(x.half()), lambda: acrl.fp8_quantize(x.cpu()), lambda: acrl.fp8_quantize(x, fmt="e3m4"),
                 lambda: acrl.fp8_quantize(x, block="column"), lambda: acrl.fp8_quantize(x.t()),
                 lambda: acrl.fp8_quantize(torch.empty((4, 9), dtype=torch.bfloat16, device=DEV)),     # row stride of 9
                 lambda: acrl.fp8_quantize(x, out=acrl.fp8_quantize(x, fmt="e5m2")),
                 lambda: acrl.Fp8Tensor(x, w.scale), lambda: acrl.Fp8Tensor(w.q, w.scale.float()),
                 lambda: acrl.Fp8Tensor(w.q, w.scale.repeat(3, 1)),
                 lambda: acrl.fp8_matmul(w, acrl.fp8_quantize(_matrix(8, 72, 1))), lambda: acrl.fp8_matmul(w, x),
                 lambda: acrl.fp8_matmul(w, w, out_dtype=torch.float16),
                 lambda: acrl.fp8_matmul(w, w, out=torch.empty((8, 12), dtype=torch.bfloat16, device=DEV)),
                 lambda: acrl.fp8_linear_backward(x, x, w), lambda: acrl.fp8_linear_backward(x.float(), x, w),
                 lambda: acrl.fp8_linear(x.float(), w), lambda: acrl.fp8_linear(x[:, :32], w),
                 lambda: acrl.fp8_linear(x, w, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(acrl.AcrlError):
            call()


@pytest.mark.parametrize("M,N,K", [(200, 300, 520), (515, 1030, 264), (1300, 264, 2056), (131, 20000, 136), (3000, 520, 520)])
@pytest.mark.parametrize("dx_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dw_dtype", [torch.bfloat16, torch.float32])
def test_both_gradients_are_the_products(M, N, K, dx_dtype, dw_dtype):
    """The two gradients of one call, bit for bit those of two calls on the quantised matrices; nothing beyond them is written."""
    dy, x, w = _matrix(M, N, 41), _matrix(M, K, 42), _matrix(N, K, 43, std=0.02)
    wt = acrl.fp8_quantize(w, block="tile", transpose=True)
    dx, dw = torch.full((M + 1, K), 3.0, dtype=dx_dtype, device=DEV), torch.full((N + 1, K), 3.0, dtype=dw_dtype, device=DEV)
    acrl.fp8_linear_backward(dy, x, wt, fmt="e5m2", dx_dtype=dx_dtype, dw_dtype=dw_dtype, dx=dx[:M], dw=dw[:N])
    by_rows = acrl.fp8_quantize(dy, fmt="e5m2")
    turned, xt = acrl.fp8_quantize(dy, fmt="e5m2", transpose=True), acrl.fp8_quantize(x, transpose=True)
    assert torch.equal(dx[:M], acrl.fp8_matmul(by_rows, wt, out_dtype=dx_dtype))
    assert torch.equal(dw[:N], acrl.fp8_matmul(turned, xt, out_dtype=dw_dtype))
    assert bool((dx[M:] == 3.0).all()) and bool((dw[N:] == 3.0).all())


def test_what_a_call_allocates_belongs_to_its_stream():
    """Memory that the current stream has freed but still writes is not what a call on another stream works in."""
    x, dy = _matrix(300, 1000, 51), _matrix(300, 520, 52)
    w = _matrix(520, 1000, 53, std=0.02)
    w8, wt = acrl.fp8_quantize(w, block="tile"), acrl.fp8_quantize(w, block="tile", transpose=True)
    n = api.fp8_linear_workspace_bytes(300, 520, 1000)
    nb = api.fp8_linear_backward_workspace_bytes(300, 520, 1000)
    want = acrl.fp8_linear(x, w8), *acrl.fp8_linear_backward(dy, x, wt), acrl.fp8_quantize(x).q.view(torch.uint8)
    want = [t.clone() for t in want]
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    for _ in range(20):                       # tens of milliseconds of the current stream
        big = torch.tanh(big @ big)
    for size in (n, nb, 300 * 520 * 2, 300 * 1000 * 2, 520 * 1000 * 4, 300 * 1008, 300 * 8):
        for _ in range(3):
            torch.empty(size, dtype=torch.uint8, device=DEV).fill_(255)   # freed at once, written when the stream gets there
    got = acrl.fp8_linear(x, w8, stream=side), *acrl.fp8_linear_backward(dy, x, wt, stream=side), \
        acrl.fp8_quantize(x, stream=side).q.view(torch.uint8)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("M,N", [(1, 140), (1, 5000), (200, 140)])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_nan_blocks_of_one_row_and_of_many(M, N, fmt):
    """As test_nan_blocks_reach_what_they_touch, on the one-row kernel and on pairs, quantised in the call and before."""
    K, row = 1301, M // 2
    x = _matrix(M, K, 12)
    x[row, 700] = float("nan") if fmt == "e4m3" else float("-inf")
    w = acrl.fp8_quantize(_matrix(N, K, 13), block="tile", fmt=fmt)
    flags = api.new_flags()
    outs = [acrl.fp8_linear(x, w, fmt=fmt, flags=flags)]
    assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE
    outs.append(acrl.fp8_matmul(acrl.fp8_quantize(x, fmt=fmt), w))
    for out in outs:
        nan = out.isnan()
        assert bool(nan[row].all()) and int(nan.sum()) == N
    bad = _matrix(N, K, 13)
    bad[130, 5] = float("inf")
    flags = api.new_flags()
    out = acrl.fp8_linear(_matrix(M, K, 12), acrl.fp8_quantize(bad, block="tile", fmt=fmt), fmt=fmt, flags=flags)
    assert acrl.read_flags(flags) == 0                     # the activations are fine
    assert bool(out[:, 128:256].isnan().all()) and not bool(out[:, :128].isnan().any()) and not bool(out[:, 256:].isnan().any())


@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("ba,bb", [("row", "row"), ("tile", "row"), ("row", "tile")])
@pytest.mark.parametrize("N,K", [(1, 17), (203, 900), (130, 2051), (5001, 1337)])
def test_one_row_formats_and_blocks(fa, fb, ba, bb, N, K):
    x = _matrix(1, K, 3)
    a, b = acrl.fp8_quantize(x, fmt=fa, block=ba), acrl.fp8_quantize(_matrix(N, K, 4), fmt=fb, block=bb)
    for dtype in (torch.float32, torch.bfloat16):
        out = acrl.fp8_matmul(a, b, out_dtype=dtype)
        _check_product(out, a, b)
        assert torch.equal(acrl.fp8_linear(x, b, fmt=fa, out_dtype=dtype), out)


@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")])
@pytest.mark.parametrize("M", [1, 2, 150])
def test_scales_of_any_size(fa, fb, M):
    """Factors near the ends of their range whose products are ordinary: a row as large as fp32 allows and a small matrix, and the
    other way round."""
    K, N = 700, 300
    for up in (118, -118):
        a, b = acrl.fp8_quantize(_matrix(M, K, 61), fmt=fa), acrl.fp8_quantize(_matrix(N, K, 62), fmt=fb, block="tile")
        a = acrl.Fp8Tensor(a.q, (a.scale.int() + up).clamp(0, 254).to(torch.uint8))
        b = acrl.Fp8Tensor(b.q, (b.scale.int() - up).clamp(0, 254).to(torch.uint8))
        sa, sb = (torch.exp2(t.scale.double() - 127).cpu().numpy() for t in (a, b))
        A = a.q.float().cpu().numpy().astype(np.float64) * np.repeat(sa, 128, 1)[:, :K]
        B = b.q.float().cpu().numpy().astype(np.float64) * np.repeat(np.repeat(sb, 128, 1)[:, :K], 128, 0)[:N]
        exact, off = A @ B.T, 2.0 ** -24 * np.sqrt(K) * (np.abs(A) @ np.abs(B).T)
        assert np.abs(exact).max() < 1e30
        out = acrl.fp8_matmul(a, b, out_dtype=torch.float32).double().cpu().numpy()
        assert (np.abs(out - exact) <= off * (1 + 2.0 ** -20) + 2.0 ** -24 * np.abs(exact)).all()


def test_one_row_of_activations_at_the_ends_of_their_range():
    K, N = 700, 300
    for size in (2.0 ** 120, 2.0 ** -120):
        x = torch.zeros((2, 704), dtype=torch.bfloat16, device=DEV)
        w = torch.zeros((N, 704), dtype=torch.bfloat16, device=DEV)
        x[:, :K], w[:, :K] = _matrix(1, K, 63).double() * size, _matrix(N, K, 64).double() / size
        w8 = acrl.fp8_quantize(w[:, :K], block="tile")
        one = acrl.fp8_linear(x[:1, :K], w8, out_dtype=torch.float32)
        two = acrl.fp8_linear(x[:, :K], w8, out_dtype=torch.float32)
        assert bool(one.isfinite().all())
        assert bool(((one[0] - two[0]).abs() <= 2.0 ** -18 * two.abs().max()).all())


def test_quantize_the_longest_rows():
    """A row of as many columns as the call takes, the largest number of all just beyond them."""
    C = 2 ** 31 - 1
    x = torch.zeros((1, C + 1), dtype=torch.bfloat16, device=DEV)
    x[0, C], x[0, C - 1], x[0, 5] = 1e30, 3.0, 5.0
    t = acrl.fp8_quantize(x[:, :C])
    assert float(t.q[0, C - 1].float()) == 384.0 and int(t.scale[0, -1]) == 120     # 3 = 384 2^-7
    assert float(t.q[0, 5].float()) == 320.0 and int(t.scale[0, 0]) == 121          # 5 = 320 2^-6
    assert bool((t.scale[0, 1:-1] == 127).all())


def test_layer_has_no_second_derivative():
    """Its backward's products have no backward: a graph of the gradients is refused, not left without their part."""
    x = _matrix(9, 64, 8).contiguous().requires_grad_()
    w = _matrix(40, 64, 10, std=0.02).contiguous().requires_grad_()
    y = acrl.fp8_layer(x, w)
    dx, = torch.autograd.grad(y.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dx.float().sum().backward()
