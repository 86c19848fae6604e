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
