"""The bf16 layer, its gradients and the update at the edges of what their entry points accept."""

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
