"""acrl_linear, acrl_linear_backward and acrl_orthogonalize refuse bad arguments on the host, before anything is launched.
CPU only."""

import ctypes
import shutil

import pytest

from paper_2607_24062_gb300 import _abi, build

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and not build.up_to_date(),
                                reason="needs nvcc to build the library")
E, OK = _abi.ERR_INVALID_ARG, _abi.OK
FAKE = 0x1000   # never dereferenced
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    build.build()
    return _abi.lib()


def _call(fn, args, **changed):
    assert not set(changed) - set(args)
    return fn(*{**args, **changed}.values())


def test_linear(L):
    for bad in ((-1, 4, 4), (4, -1, 4), (4, 4, -1)):
        assert L.acrl_linear_workspace_bytes(*bad) == -1
    ok = dict(x=FAKE, M=5, K=40, ldx=40, w=FAKE, N=24, ldw=48, bias=FAKE + 2, tb=0, act=2, r=FAKE, tr=1, ldr=24, pre=FAKE, ldp=24,
              out=FAKE, to=0, ldo=24, ws=FAKE, n=BIG, flags=None, stream=None)
    # a host address (FAKE) is refused as well: every operand is device memory
    for bad in ({}, dict(x=None), dict(w=None), dict(out=None), dict(M=-1), dict(N=-1), dict(K=-1), dict(M=1 << 31), dict(N=1 << 31),
                dict(K=1 << 31, ldx=1 << 32, ldw=1 << 32), dict(ldx=32), dict(ldx=44), dict(ldw=36), dict(ldo=16), dict(ldo=28),
                dict(ldr=20), dict(ldp=20), dict(x=FAKE + 8), dict(w=FAKE + 2), dict(out=FAKE + 8), dict(r=FAKE + 4),
                dict(pre=FAKE + 2), dict(act=5), dict(act=-1), dict(to=2), dict(tb=2), dict(tr=-1), dict(n=-1)):
        assert _call(L.acrl_linear, ok, **bad) == E, bad
    assert _call(L.acrl_linear, ok, M=0) == OK
    assert _call(L.acrl_linear, ok, N=0, ldw=40) == OK


def test_linear_workspace(L):
    """What a call needs is what the size function says, and an unaligned or missing workspace is refused where one is needed."""
    ok = dict(x=FAKE, M=16, K=65536, ldx=65536, w=FAKE, N=24, ldw=65536, bias=None, tb=0, act=0, r=None, tr=0, ldr=0, pre=None,
              ldp=0, out=FAKE, to=0, ldo=24, ws=FAKE, n=0, flags=None, stream=None)
    n = L.acrl_linear_workspace_bytes(16, 24, 65536)
    assert n >= 0
    if n > 0:
        for bad in (dict(n=n - 1), dict(n=n, ws=None), dict(n=n, ws=FAKE + 8)):
            assert _call(L.acrl_linear, ok, **bad) == E, bad


def test_linear_backward(L):
    assert L.acrl_linear_backward_workspace_bytes(-1, 1, 1) == -1
    n = L.acrl_linear_backward_workspace_bytes(5, 24, 40)
    assert n >= 5 * 24 * 2
    ok = dict(dy=FAKE, M=5, N=24, lddy=24, x=FAKE, K=40, ldx=40, w=FAKE, ldw=40, act=1, pre=FAKE, ldp=24, dx=FAKE, tx=0, lddx=40,
              dw=FAKE, tw=1, lddw=40, db=FAKE, ws=FAKE, n=n, flags=None, stream=None)
    for bad in ({}, dict(dy=None), dict(x=None), dict(w=None), dict(pre=None), dict(ws=None), dict(n=n - 1), dict(M=-1), dict(N=-1),
                dict(K=-1), dict(M=1 << 31), dict(lddy=20), dict(ldx=36), dict(ldw=32), dict(ldp=28), dict(lddx=32), dict(lddw=44),
                dict(act=5), dict(act=0), dict(tx=2), dict(tw=-1), dict(dy=FAKE + 2), dict(x=FAKE + 8), dict(w=FAKE + 4),
                dict(pre=FAKE + 8), dict(dx=FAKE + 4), dict(dw=FAKE + 2), dict(ws=FAKE + 8)):
        assert _call(L.acrl_linear_backward, ok, **bad) == E, bad
    assert _call(L.acrl_linear_backward, ok, dx=None, dw=None, db=None) == OK    # nothing is asked for
    assert _call(L.acrl_linear_backward, ok, dx=None, dw=None, N=0, lddy=0, ldp=0) == OK


def test_orthogonalize(L):
    for bad in ((-1, 4, 4), (4, -1, 4), (4, 4, -1)):
        assert L.acrl_orthogonalize_workspace_bytes(*bad) == -1
    assert L.acrl_orthogonalize_workspace_bytes(0, 4, 4) == 0
    n = L.acrl_orthogonalize_workspace_bytes(2, 24, 40)
    assert n >= 2 * 2 * 24 * 40 * 2
    of = lambda *v: (ctypes.c_float * len(v))(*v)   # noqa: E731
    ok = dict(g=FAKE, t=1, B=2, m=24, n=40, ldg=40, gs=24 * 40, c=of(*[3.4445, -4.775, 2.0315] * 5), steps=5, eps=1e-7, scale=1.0,
              out=FAKE, ldo=40, os=24 * 40, ws=FAKE, bytes=n, flags=None, stream=None)
    for bad in ({}, dict(g=None), dict(out=None), dict(ws=None), dict(c=None), dict(t=2), dict(B=-1), dict(m=-1), dict(n=-1),
                dict(m=1 << 31), dict(n=1 << 31), dict(ldg=36), dict(gs=24 * 40 - 4), dict(ldo=32), dict(os=24 * 40 - 8),
                dict(g=FAKE + 2), dict(t=0, g=FAKE + 1), dict(out=FAKE + 1), dict(ws=FAKE + 8), dict(bytes=n - 1), dict(steps=0), dict(steps=65), dict(eps=-1.0),
                dict(eps=float("inf")), dict(scale=float("nan")), dict(c=of(*[3.4445, -4.775, float("inf")] * 5))):
        assert _call(L.acrl_orthogonalize, ok, **bad) == E, bad
    for none in (dict(B=0), dict(m=0), dict(n=0)):
        assert _call(L.acrl_orthogonalize, ok, **none) == OK
