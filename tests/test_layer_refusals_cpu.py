"""acrl_linear, acrl_linear_backward and acrl_orthogonalize refuse bad arguments on the host: each list begins with a call that is
accepted, so that what is changed in it is what is refused.  CPU only."""

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
