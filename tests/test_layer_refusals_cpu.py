"""acrl_linear, acrl_linear_backward and acrl_orthogonalize refuse bad arguments on the host: each list begins with a call that is
accepted, so that what is changed in it is what is refused.  CPU only."""

import ctypes
import shutil

import pytest

from paper_2607_24062_gb300 import _abi, build

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and not build.up_to_date(),
                                reason="needs nvcc to build the library")
E, OK = _abi.ERR_INVALID_ARG, _abi.OK
FAKE = 0x1000   # a host address, never dereferenced
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    build.build()
    return _abi.lib()


def _call(fn, args, **changed):
    assert not set(changed) - set(args)
    return fn(*{**args, **changed}.values())


def test_outputs_of_empty_sums_are_looked_at(L):
    """Without columns to add up the results are still written: into device memory only.  (Where no device is present, a call that
    came as far as its launch would return another error.)"""
    linear = dict(x=None, M=5, K=0, ldx=0, w=None, N=24, ldw=0, bias=None, tb=0, act=0, r=None, tr=0, ldr=0, pre=None, ldp=0,
                  out=FAKE, to=0, ldo=24, ws=None, n=0, flags=None, stream=None)
    assert _call(L.acrl_linear, linear, M=0) == OK
    assert _call(L.acrl_linear, linear) == E
    back = dict(dy=None, M=0, N=24, lddy=24, x=None, K=40, ldx=40, w=None, ldw=40, act=0, pre=None, ldp=0, dx=None, tx=0, lddx=0,
                dw=None, tw=1, lddw=40, db=None, ws=None, n=BIG, flags=None, stream=None)
    assert _call(L.acrl_linear_backward, back) == OK
    assert _call(L.acrl_linear_backward, back, dw=FAKE) == E
    assert _call(L.acrl_linear_backward, back, db=FAKE) == E
    assert _call(L.acrl_linear_backward, back, M=5, N=0, lddy=0, ldx=40, dx=FAKE, lddx=40) == E


MOST = 2 ** 31 - 8193


def test_sizes_of_matrices_that_no_gpu_holds(L):
    """The workspace of the largest sizes is counted within 64 bits, or the sizes are refused: never a number below zero."""
    for M in (1, 5, 300, 2 ** 17, 2 ** 24, MOST):
        for N in (1, 40, 2 ** 17, 2 ** 24, 2 ** 31 - 8200, MOST):
            for K in (0, 1, 40, 2 ** 17, 2 ** 24, MOST):
                held = max(M * N, M * K, N * K) < 2 ** 48
                n = L.acrl_linear_backward_workspace_bytes(M, N, K)
                assert (n >= M * N * 2 and n < 2 ** 60) if held else n == 0
                assert 0 <= L.acrl_linear_workspace_bytes(M, N, K) < 2 ** 60
    # nothing is asked for, so that the sizes alone are refused
    back = dict(dy=FAKE, M=5, N=24, lddy=2 ** 31, x=None, K=40, ldx=0, w=None, ldw=0, act=0, pre=None, ldp=0, dx=None, tx=0, lddx=0,
                dw=None, tw=1, lddw=0, db=None, ws=None, n=2 ** 62, flags=None, stream=None)
    for fine in (dict(), dict(M=MOST), dict(N=MOST), dict(K=MOST), dict(M=2 ** 24, N=2 ** 24 - 1)):
        assert _call(L.acrl_linear_backward, back, **fine) == OK, fine
    for bad in (dict(M=MOST, N=MOST), dict(M=MOST, K=MOST), dict(N=MOST, K=MOST), dict(M=2 ** 24, N=2 ** 24), dict(M=MOST + 1),
                dict(N=MOST + 1), dict(K=MOST + 1)):
        assert _call(L.acrl_linear_backward, back, **bad) == E, bad


def _refused(fn, ok, bad):
    """`ok` is accepted, and with each of the changes refused."""
    assert _call(fn, ok) == OK
    for changed in bad:
        assert _call(fn, ok, **changed) == E, changed


def test_linear_of_no_rows(L):
    """Without rows nothing is launched, and what does not depend on them is looked at all the same."""
    ok = dict(x=None, M=0, K=40, ldx=40, w=None, N=24, ldw=40, bias=FAKE, tb=0, act=2, r=FAKE, tr=1, ldr=24, pre=None, ldp=0, out=None,
              to=0, ldo=24, ws=None, n=0, flags=None, stream=None)
    _refused(L.acrl_linear, ok, [dict(M=-1), dict(N=-1), dict(K=-1), dict(M=MOST + 1), dict(N=MOST + 1), dict(K=MOST + 1), dict(N=MOST, K=MOST),
                                 dict(act=5), dict(act=-1), dict(to=2), dict(to=-1), dict(tb=2), dict(tr=-1), dict(n=-1)])
    # the types of what is not there do not matter
    assert _call(L.acrl_linear, ok, bias=None, tb=7, r=None, tr=7) == OK
    assert _call(L.acrl_linear, ok, N=0) == OK


def test_linear_workspaces(L):
    """A sum that is split needs one, for its size alone; few rows, whole sums and empty ones do not."""
    for M, N, K in ((48, 4096, 16384), (129, 256, 8192), (100, 1024, 32768)):
        n = L.acrl_linear_workspace_bytes(M, N, K)
        assert n > 0 and n % 4 == 0 and n >= 2 * 4 * M * N // 8
    for M, N, K in ((1, 4096, 16384), (16, 24, 65536), (4096, 4096, 16384), (0, 4096, 16384), (48, 0, 16384), (48, 4096, 0)):
        assert L.acrl_linear_workspace_bytes(M, N, K) == 0
    for bad in ((-1, 4, 4), (4, -1, 4), (4, 4, -1)):
        assert L.acrl_linear_workspace_bytes(*bad) == -1 and L.acrl_linear_backward_workspace_bytes(*bad) == -1


def test_backward_of_nothing(L):
    """With no gradient asked for nothing is launched; what every gradient is made of is looked at."""
    n = L.acrl_linear_backward_workspace_bytes(5, 24, 40)
    assert n > 0
    ok = dict(dy=FAKE, M=5, N=24, lddy=24, x=None, K=40, ldx=0, w=None, ldw=0, act=1, pre=FAKE, ldp=24, dx=None, tx=0, lddx=0,
              dw=None, tw=1, lddw=0, db=None, ws=None, n=n, flags=None, stream=None)
    _refused(L.acrl_linear_backward, ok, [dict(n=n - 1), dict(n=-1), dict(M=-1), dict(N=-1), dict(K=-1), dict(act=5), dict(act=-1), dict(act=0),
                                          dict(dy=None), dict(dy=FAKE + 2), dict(lddy=20), dict(lddy=16), dict(pre=None), dict(pre=FAKE + 8),
                                          dict(ldp=28), dict(ldp=16)])
    assert _call(L.acrl_linear_backward, ok, act=0, pre=None) == OK
    # without rows, those of a gradient of zeros
    ok = dict(ok, M=0, dy=None, pre=None, act=0)
    _refused(L.acrl_linear_backward, ok, [dict(dw=FAKE, lddw=40, tw=2), dict(dw=FAKE, lddw=32), dict(dw=FAKE, lddw=44), dict(dw=FAKE + 4, lddw=40)])


def test_update_of_no_matrices(L):
    of = lambda *v: (ctypes.c_float * len(v))(*v)   # noqa: E731
    three = [3.4445, -4.775, 2.0315]
    ok = dict(g=None, t=1, B=0, m=24, n=40, ldg=40, gs=24 * 40, c=of(*three * 5), steps=5, eps=1e-7, scale=1.0, out=None, ldo=40,
              os=24 * 40, ws=None, bytes=0, flags=None, stream=None)
    bad = [dict(t=2), dict(t=-1), dict(B=-1), dict(m=-1), dict(n=-1), dict(m=MOST + 1), dict(n=MOST + 1), dict(c=None), dict(steps=0),
           dict(steps=-1), dict(steps=65, c=of(*three * 65)), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")),
           dict(scale=float("nan")), dict(scale=float("-inf")), dict(bytes=-1)]
    bad += [dict(c=of(*three * 4, *[v if j != i else x for j, v in enumerate(three)])) for i in range(3) for x in (float("inf"), float("nan"))]
    _refused(L.acrl_orthogonalize, ok, bad)
    assert _call(L.acrl_orthogonalize, ok, steps=64, c=of(*three * 64)) == OK
    assert _call(L.acrl_orthogonalize, ok, B=2, m=0) == OK and _call(L.acrl_orthogonalize, ok, B=2, n=0) == OK
    n = L.acrl_orthogonalize_workspace_bytes(2, 24, 40)
    assert n > 2 * 2 * 24 * 40 * 2
