"""The bf16 layer, its gradients and the update at the edges of what their entry points accept."""

import ctypes
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2607_24062_gb300 as acrl  # noqa: E402
from paper_2607_24062_gb300 import _abi, api  # noqa: E402

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
MOST = 2 ** 31 - 8193    # rows or columns of a call


@pytest.mark.parametrize("M,N", [(1, MOST), (2, MOST - 100000), (3, 131073), (200, 5000)])
def test_column_sums_alone_up_to_the_most_columns(M, N):
    """dbias without a product beside it: whole numbers, whose sums are exact; nothing beyond the columns is written.  (About 50 GB
    for a row of the most columns.)"""
    dy = torch.empty((M, (N + 7) // 8 * 8), dtype=BF, device=DEV)
    at = torch.arange(dy.shape[1], device=DEV, dtype=torch.int32) % 251
    for i in range(M):
        dy[i] = (at + 3 * i).to(torch.uint8).to(BF)    # up to 255: exact in bf16
    del at
    dy = dy[:, :N]
    x, w = torch.empty((M, 0), dtype=BF, device=DEV), torch.empty((N, 0), dtype=BF, device=DEV)
    db = torch.full((N + 32,), -7.0, device=DEV)
    dx, dw, out = acrl.linear_backward(dy, x, w, bias=True, need_dx=False, need_dw=False, dbias=db)
    assert dx is None and dw is None and out.data_ptr() == db.data_ptr()
    step = 1 << 27
    for c in range(0, N, step):
        assert torch.equal(db[c: min(N, c + step)], dy[:, c: c + step].float().sum(0))
    assert bool((db[N:] == -7.0).all())


def _entry(name, args, **changed):
    assert not set(changed) - set(args)
    torch.cuda.synchronize()
    st = getattr(_abi.lib(), name)(*{**args, **changed}.values())
    torch.cuda.synchronize()
    return st


def _filled(*shape, dtype=BF):
    return torch.ones(shape, dtype=dtype, device=DEV)


@pytest.mark.parametrize("M,N,K", [(5, 24, 40), (48, 264, 16384), (300, 264, 520), (3, 24, 0)])
def test_operands_elsewhere_are_refused(M, N, K):
    """Host memory, or an address that is not its type's, in the place of each operand of a call that is accepted."""
    here = dict(x=_filled(M, K), w=_filled(N, K), bias=_filled(N, dtype=F32), r=_filled(M, N, dtype=F32), pre=_filled(M, N), out=_filled(M, N),
                ws=torch.empty(api.linear_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV))
    at = {k: t.data_ptr() or None for k, t in here.items()}
    ok = dict(x=at["x"], M=M, K=K, ldx=K, w=at["w"], N=N, ldw=K, bias=at["bias"], tb=1, act=2, r=at["r"], tr=1, ldr=N, pre=at["pre"], ldp=N,
              out=at["out"], to=0, ldo=N, ws=at["ws"], n=here["ws"].numel(), flags=None, stream=None)
    assert _entry("acrl_linear", ok) == _abi.OK
    assert _entry("acrl_linear", ok, bias=None, r=None, pre=None) == _abi.OK
    host = torch.zeros(M * max(N, K) + N * K + here["ws"].numel() + 64, dtype=F32)    # room for any of them
    base = host.data_ptr() + 15 & ~15
    for name in (k for k in at if at[k] is not None):
        assert _entry("acrl_linear", ok, **{name: base}) == _abi.ERR_INVALID_ARG, name
    assert _entry("acrl_linear", ok, bias=at["bias"] + 2) == _abi.ERR_INVALID_ARG
    assert _entry("acrl_linear", ok, bias=at["bias"] + 1, tb=0) == _abi.ERR_INVALID_ARG
    assert _entry("acrl_linear", ok, bias=at["bias"] + 2, tb=0, N=N - 8) == _abi.OK


@pytest.mark.parametrize("M,N,K", [(5, 24, 40), (300, 264, 520), (0, 24, 40), (3, 24, 0)])
def test_gradients_operands_elsewhere_are_refused(M, N, K):
    here = dict(dy=_filled(M, N), x=_filled(M, K), w=_filled(N, K), pre=_filled(M, N), dx=_filled(M, K), dw=_filled(N, K, dtype=F32),
                db=_filled(N, dtype=F32), ws=torch.empty(api.linear_backward_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV))
    at = {k: t.data_ptr() or None for k, t in here.items()}
    ok = dict(dy=at["dy"], M=M, N=N, lddy=N, x=at["x"], K=K, ldx=K, w=at["w"], ldw=K, act=2, pre=at["pre"], ldp=N, dx=at["dx"], tx=0,
              lddx=K, dw=at["dw"], tw=1, lddw=K, db=at["db"], ws=at["ws"], n=here["ws"].numel(), flags=None, stream=None)
    assert _entry("acrl_linear_backward", ok) == _abi.OK
    host = torch.zeros(M * max(N, K) + N * K + here["ws"].numel() + 64, dtype=F32)
    base = host.data_ptr() + 15 & ~15
    # what a call without rows, or without columns of x, has no use for is not looked at
    used = {"db"} | ({"dw"} if K else set()) | ({"dy", "pre", "ws"} if M else set()) | ({"x", "w", "dx"} if M and K else set())
    for name in used:
        assert _entry("acrl_linear_backward", ok, **{name: base}) == _abi.ERR_INVALID_ARG, name
    assert _entry("acrl_linear_backward", ok, db=at["db"] + 2) == _abi.ERR_INVALID_ARG


ROOM = 1 << 16    # elements of each buffer below: more than any stride that is refused would reach


def _refused(name, ok, bad):
    """`ok` is accepted, and with each of the changes refused."""
    assert _entry(name, ok) == _abi.OK
    for changed in bad:
        assert _entry(name, ok, **changed) == _abi.ERR_INVALID_ARG, changed
    assert _entry(name, ok) == _abi.OK


@pytest.mark.parametrize("M", [5, 300])
def test_strides_and_alignments_that_are_refused(M):
    N, K = 24, 40
    b = {k: torch.ones(ROOM, dtype=F32, device=DEV) for k in ("x", "w", "bias", "r", "pre", "out", "dy", "dx", "dw", "db")}
    p = {k: t.data_ptr() for k, t in b.items()}
    n = api.linear_workspace_bytes(M, N, K)
    assert n == 0
    ok = dict(x=p["x"], M=M, K=K, ldx=40, w=p["w"], N=N, ldw=48, bias=p["bias"] + 2, tb=0, act=2, r=p["r"], tr=1, ldr=24, pre=p["pre"], ldp=24,
              out=p["out"], to=0, ldo=24, ws=None, n=0, flags=None, stream=None)
    _refused("acrl_linear", ok, [dict(x=None), dict(w=None), dict(out=None), dict(ldx=32), dict(ldx=44), dict(ldw=36), dict(ldw=32), dict(ldo=16),
                                 dict(ldo=28), dict(ldr=20), dict(ldr=16), dict(ldp=20), dict(ldp=16), dict(x=p["x"] + 8), dict(w=p["w"] + 2),
                                 dict(out=p["out"] + 8), dict(r=p["r"] + 4), dict(pre=p["pre"] + 2), dict(act=5), dict(to=2), dict(tb=2),
                                 dict(tr=2), dict(n=-1)])
    n = api.linear_backward_workspace_bytes(M, N, K)
    ws = torch.empty(n + 16, dtype=torch.uint8, device=DEV)
    ok = dict(dy=p["dy"], M=M, N=N, lddy=24, x=p["x"], K=K, ldx=40, w=p["w"], ldw=40, act=1, pre=p["pre"], ldp=24, dx=p["dx"], tx=0, lddx=40,
              dw=p["dw"], tw=1, lddw=40, db=p["db"], ws=ws.data_ptr(), n=n, flags=None, stream=None)
    _refused("acrl_linear_backward", ok, [dict(dy=None), dict(x=None), dict(w=None), dict(pre=None), dict(ws=None), dict(n=n - 1), dict(lddy=20),
                                          dict(ldx=36), dict(ldw=32), dict(ldp=28), dict(lddx=32), dict(lddw=44), dict(act=5), dict(act=0),
                                          dict(tx=2), dict(tw=-1), dict(dy=p["dy"] + 2), dict(x=p["x"] + 8), dict(w=p["w"] + 4),
                                          dict(pre=p["pre"] + 8), dict(dx=p["dx"] + 4), dict(dw=p["dw"] + 2), dict(ws=ws.data_ptr() + 8)])


@pytest.mark.parametrize("M,N,K", [(48, 1024, 16384), (129, 256, 8192)])
def test_a_split_sums_workspace(M, N, K):
    x, w, out = _filled(M, K), _filled(N, K), _filled(M, N, dtype=F32)
    n = api.linear_workspace_bytes(M, N, K)
    assert n > 0
    ws = torch.full((n + 64,), 255, dtype=torch.uint8, device=DEV)
    ok = dict(x=x.data_ptr(), M=M, K=K, ldx=K, w=w.data_ptr(), N=N, ldw=K, bias=None, tb=0, act=0, r=None, tr=0, ldr=0, pre=None, ldp=0,
              out=out.data_ptr(), to=1, ldo=N, ws=ws.data_ptr(), n=n, flags=None, stream=None)
    _refused("acrl_linear", ok, [dict(n=n - 1), dict(n=0, ws=None), dict(ws=None), dict(ws=ws.data_ptr() + 8), dict(n=-1)])
    assert bool((out == K).all()) and bool((ws[n:] == 255).all())


def test_updates_that_are_refused():
    B, m, n = 2, 24, 40
    g, out = (torch.ones(ROOM, dtype=t, device=DEV) for t in (F32, BF))
    size = api.orthogonalize_workspace_bytes(B, m, n)
    ws = torch.empty(size + 16, dtype=torch.uint8, device=DEV)
    c = (ctypes.c_float * 15)(*[3.4445, -4.775, 2.0315] * 5)
    ok = dict(g=g.data_ptr(), t=1, B=B, m=m, n=n, ldg=40, gs=24 * 40, c=c, steps=5, eps=1e-7, scale=1.0, out=out.data_ptr(), ldo=40,
              os=24 * 40, ws=ws.data_ptr(), bytes=size, flags=None, stream=None)
    host = torch.zeros(ROOM)
    base = host.data_ptr() + 15 & ~15
    _refused("acrl_orthogonalize", ok, [dict(g=None), dict(out=None), dict(ws=None), dict(c=None), dict(t=2), dict(ldg=36), dict(gs=24 * 40 - 1),
                                        dict(ldo=32), dict(os=24 * 40 - 1), dict(g=g.data_ptr() + 2), dict(t=0, g=g.data_ptr() + 1),
                                        dict(out=out.data_ptr() + 1), dict(ws=ws.data_ptr() + 8), dict(bytes=size - 1), dict(steps=0),
                                        dict(steps=65), dict(eps=-1.0), dict(scale=float("nan")), dict(g=base), dict(out=base), dict(ws=base)])


@pytest.mark.parametrize("M,N,K", [(5, 24, 40), (300, 264, 520)])
def test_a_residual_in_place_of_another_type_or_stride_is_refused(M, N, K):
    x, w, out = _filled(M, K), _filled(N, K), _filled(M, 2 * N, dtype=F32)
    ok = dict(x=x.data_ptr(), M=M, K=K, ldx=K, w=w.data_ptr(), N=N, ldw=K, bias=None, tb=0, act=0, r=out.data_ptr(), tr=1, ldr=N, pre=None,
              ldp=0, out=out.data_ptr(), to=1, ldo=N, ws=None, n=api.linear_workspace_bytes(M, N, K), flags=None, stream=None)
    assert ok["n"] == 0
    assert _entry("acrl_linear", ok) == _abi.OK and bool((out.view(-1)[: M * N] == K + 1).all())
    assert _entry("acrl_linear", ok, M=1, ldr=N + 8) == _abi.OK          # of one row no stride is used
    for bad in (dict(tr=0), dict(to=0), dict(ldr=N + 8), dict(ldo=N + 8)):
        assert _entry("acrl_linear", ok, **bad) == _abi.ERR_INVALID_ARG, bad


def _unit(n):
    """n roundings to 24 bits, of half a step each."""
    return n * 2.0 ** -24


def _tail(act, u):
    """In 64 bits: f and f', and how far fp32 may be off, each a sum of relative errors times the terms that they are errors of.
    Of 2^-24 each: an exponent z, a product of a few roundings (2.5 for gelu's u^2 / 2 with its constant, 5 for the tanh form's,
    1.25 for silu's with its constant), comes back as that many times |z|; an exponential and its square 10; a reciprocal and what
    it is of 5; gelu's polynomial 8 and the reciprocal in it again 5; the products a few.  Results below fp32's normal numbers to a
    few of its least steps."""
    u = u.double()
    if act == "gelu":
        p, q, bell = torch.erfc(-u / 2 ** 0.5) / 2, torch.erfc(u / 2 ** 0.5) / 2, torch.exp(-u * u / 2) / (2 * math.pi) ** 0.5
        each, slope = _unit(32) + _unit(2.5) * u * u / 2, p + u * bell
        # beyond 0 Phi is 1 less its tail
        off_p = each * torch.where(u < 0, p, q) + _unit(2) * p
        off_f, off_s = u.abs() * off_p + _unit(2) * (u * p).abs(), off_p + (each + _unit(4)) * u.abs() * bell
    else:
        if act == "silu":
            z, dz, n = u, torch.ones_like(u), 1.25
        else:
            k = (8 / math.pi) ** 0.5
            z, dz, n = k * (u + 0.044715 * u ** 3), k * (1 + 3 * 0.044715 * u * u), 5
        p, q = torch.sigmoid(z), torch.sigmoid(-z)
        each = _unit(16) + _unit(n) * z.abs()
        slope = p + u * p * q * dz
        off_p = each * p * torch.where(z < 0, torch.ones_like(z), q) + _unit(6) * p
        off_f = u.abs() * off_p + _unit(2) * (u * p).abs()
        off_s = off_p + (2 * each + _unit(12)) * u.abs() * p * q * dz.abs()
    least = 2.0 ** -149 * 4
    return u * p, slope, off_f + least * (4 + u.abs()), off_s + least * (4 + u.abs() ** 3)


def _within(got, exact, off, what):
    """Rounding is monotone: `got` lies between the roundings of the ends of exact +- off."""
    lo, hi = (exact - off).to(got.dtype), (exact + off).to(got.dtype)
    bad = ~((got >= lo) & (got <= hi))
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), exact[bad][:4].tolist())


@pytest.mark.parametrize("act,least", [("gelu", -14.5), ("gelu_tanh", -10.5), ("silu", -110.0)])
@pytest.mark.parametrize("M", [2, 40, 300])
def test_activations_keep_their_digits_in_the_tail(act, least, M):
    """f with an error relative to itself, as far down as fp32 goes, in each of the layer's kernels: u is the bias, of an empty
    row's sum and of one of zeros."""
    N = 16384
    u = torch.cat([torch.linspace(least, 0, N // 2), torch.linspace(0, -least, N // 4), -torch.logspace(-30, 1, N // 8),
                   torch.logspace(-30, 1, N // 8)]).to(DEV)
    y, _, off, _ = _tail(act, u)
    for K in (0, 8, 520):
        x, w = torch.zeros((M, K), dtype=BF, device=DEV), torch.zeros((N, K), dtype=BF, device=DEV)
        for dtype in (F32, BF):
            out = acrl.linear(x, w, u, act=act, out_dtype=dtype)
            assert bool((out == out[:1]).all())
            _within(out[0], y, off, (K, dtype))


@pytest.mark.parametrize("act,least", [("gelu", -14.5), ("gelu_tanh", -10.5), ("silu", -110.0)])
def test_slopes_keep_their_digits_in_the_tail(act, least):
    """f' likewise: by dbias in fp32, and rounded to bf16 on its way through a product with the identity."""
    u = torch.cat([torch.linspace(least, -least, 3900), torch.logspace(-30, 1, 98), -torch.logspace(-30, 1, 98)]).to(DEV).to(BF)
    _, slope, _, off = _tail(act, u)
    N = len(u)
    one = torch.ones((1, N), dtype=BF, device=DEV)
    none = torch.empty((N, 0), dtype=BF, device=DEV)
    _, _, db = acrl.linear_backward(one, none[:1], none, act=act, pre=u[None], bias=True, need_dx=False, need_dw=False)
    _within(db, slope, off, "dbias")
    rows, eye = u.view(-1, 64), torch.eye(64, device=DEV).to(BF)
    dx, _, _ = acrl.linear_backward(torch.ones_like(rows), torch.zeros_like(rows), eye, act=act, pre=rows, dx_dtype=F32, need_dw=False)
    normal = slope.view(-1, 64).abs() >= 2.0 ** -120       # the tensor cores' products of smaller numbers are not at issue
    _within(dx.to(BF)[normal], slope.view(-1, 64)[normal], off.view(-1, 64)[normal], "dx")


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activations_of_the_largest_numbers(act):
    """f and f' where an exponential over- or underflows, and of NaN."""
    inf, nan = float("inf"), float("nan")
    u = torch.tensor([-3e38, -1e30, -1e4, -300.0, 300.0, 1e4, 1e30, 3e38, inf, nan], device=DEV)
    for M in (1, 300):
        for dtype in (F32, BF):
            y = acrl.linear(torch.zeros((M, 8), dtype=BF, device=DEV), torch.zeros((len(u), 8), dtype=BF, device=DEV), u, act=act, out_dtype=dtype)
            assert bool((y[:, :4] == 0).all()) and torch.equal(y[:, 4:9], u[4:9].to(dtype).expand(M, 5)) and bool(y[:, 9].isnan().all())
    u[8] = 200.0    # f' at infinity is not a limit that the formulas take
    pre = u.to(BF)[None]
    none = torch.empty((len(u), 0), dtype=BF, device=DEV)
    slope = acrl.linear_backward(torch.ones_like(pre), none[:1], none, act=act, pre=pre, bias=True, need_dx=False, need_dw=False)[2]
    assert slope[:9].tolist() == [0.0] * 4 + [1.0] * 5 and bool(slope[9].isnan())
