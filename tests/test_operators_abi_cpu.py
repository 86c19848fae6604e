"""The entry points of the 8-bit matrices and of the reference-policy losses refuse bad arguments on the host, before
anything is launched.  CPU only."""

import shutil

import pytest

from paper_2607_24062_gb300 import _abi, build

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and not build.up_to_date(),
                                reason="needs nvcc to build the library")
E, OK = _abi.ERR_INVALID_ARG, _abi.OK
FAKE = 0x1000   # never dereferenced


@pytest.fixture(scope="module")
def L():
    build.build()
    return _abi.lib()


def _call(fn, args, **changed):
    return fn(*{**args, **changed}.values())


def test_quantize(L):
    ok = dict(x=FAKE, dtype=0, R=4, C=40, ldx=40, fmt=0, block=0, transpose=0, q=FAKE, ldq=48, scale=FAKE, lds=1,
              flags=FAKE, stream=None)
    for bad in (dict(x=None), dict(q=None), dict(scale=None), dict(dtype=2), dict(fmt=2), dict(block=2),
                dict(R=-1), dict(C=-1), dict(ldx=32), dict(ldx=44), dict(ldq=32), dict(ldq=40), dict(lds=0),
                dict(x=FAKE + 8), dict(q=FAKE + 8), dict(dtype=1, ldx=42), dict(C=200, ldx=200, ldq=208),
                dict(transpose=1, R=200, ldq=208), dict(R=1 << 32)):
        assert _call(L.acrl_fp8_quantize, ok, **bad) == E, bad
    assert _call(L.acrl_fp8_quantize, ok, R=0) == OK
    assert _call(L.acrl_fp8_quantize, ok, C=0, ldq=0, lds=0) == OK


def test_matmul(L):
    ok = dict(a=FAKE, M=5, K=40, lda=48, fa=0, sa=FAKE, ldas=1, ba=0, b=FAKE, N=24, ldb=48, fb=0, sb=FAKE, ldbs=1, bb=1,
              out=FAKE, dtype=0, ldo=24, flags=FAKE, stream=None)
    # a host address (FAKE) is refused as well: every operand is device memory
    for bad in ({}, dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(out=None), dict(M=-1),
                dict(N=-1), dict(K=-1), dict(lda=32), dict(lda=40), dict(ldb=44), dict(ldas=0), dict(ldbs=0), dict(fa=2),
                dict(fb=-1), dict(ba=2), dict(bb=2), dict(dtype=2), dict(ldo=16), dict(ldo=28), dict(out=FAKE + 8),
                dict(a=FAKE + 8), dict(b=FAKE + 4), dict(M=1 << 31), dict(K=1 << 31, lda=1 << 32, ldb=1 << 32)):
        assert _call(L.acrl_fp8_matmul, ok, **bad) == E, bad
    assert _call(L.acrl_fp8_matmul, ok, M=0) == OK
    assert _call(L.acrl_fp8_matmul, ok, N=0) == OK


def test_linear(L):
    assert L.acrl_fp8_linear_workspace_bytes(-1, 4, 4) == -1 and L.acrl_fp8_linear_workspace_bytes(4, 4, -1) == -1
    assert L.acrl_fp8_linear_workspace_bytes(1, 4096, 4096) == 0   # one row is quantised in the product's kernel
    n = L.acrl_fp8_linear_workspace_bytes(5, 24, 40)
    assert n >= 5 * (48 + 1)
    ok = dict(x=FAKE, M=5, K=40, ldx=40, fx=0, w=FAKE, N=24, ldw=48, fw=0, sw=FAKE, ldws=1, bw=1, out=FAKE, dtype=0, ldo=24,
              ws=FAKE, n=n, flags=FAKE, stream=None)
    for bad in ({}, dict(x=None), dict(w=None), dict(sw=None), dict(out=None), dict(ws=None), dict(ws=FAKE + 8), dict(n=n - 1),
                dict(ldx=32), dict(ldw=40), dict(ldo=20), dict(fx=2), dict(fw=2), dict(bw=2), dict(M=-1), dict(M=1, n=0, ws=None, x=None),
                dict(M=1, n=0, ws=None, ldx=44)):
        assert _call(L.acrl_fp8_linear, ok, **bad) == E, bad
    assert _call(L.acrl_fp8_linear, ok, N=0) == OK


def test_linear_backward(L):
    assert L.acrl_fp8_linear_backward_workspace_bytes(-1, 1, 1) == -1
    n = L.acrl_fp8_linear_backward_workspace_bytes(5, 24, 40)
    assert n >= 5 * 24 + 24 * 5 + 40 * 5
    ok = dict(dy=FAKE, M=5, N=24, lddy=24, fy=0, x=FAKE, K=40, ldx=40, fx=0, wt=FAKE, ldwt=32, fw=0, swt=FAKE, ldwts=1, bw=1,
              dx=FAKE, tx=0, lddx=40, dw=FAKE, tw=1, lddw=40, ws=FAKE, n=n, flags=None, stream=None)
    for bad in ({}, dict(dy=None), dict(x=None), dict(wt=None), dict(swt=None), dict(dx=None), dict(dw=None), dict(ws=None),
                dict(n=n - 1), dict(M=-1), dict(N=-1), dict(K=-1), dict(lddy=20), dict(ldx=36), dict(ldwt=24), dict(lddx=32),
                dict(lddw=44), dict(fy=2), dict(fx=2), dict(fw=2), dict(bw=2), dict(tx=2), dict(tw=-1), dict(dy=FAKE + 2),
                dict(x=FAKE + 8), dict(dx=FAKE + 4), dict(ws=FAKE + 8)):
        assert _call(L.acrl_fp8_linear_backward, ok, **bad) == E, bad


def test_policy_loss(L):
    ok = dict(z=FAKE, T=4, V=16, ld=16, ids=FAKE, mask=None, old=None, coef=FAKE, low=0.2, high=0.2, dual=0.0, kl=0,
              kl_coef=None, x=None, ldx=0, ref=None, grad=FAKE, logp=FAKE, kl_out=None, tl=FAKE, loss=FAKE, flags=None,
              stream=None)
    for bad in (dict(z=None), dict(ids=None), dict(grad=None), dict(logp=None), dict(tl=None), dict(loss=None), dict(T=-1),
                dict(V=0), dict(ld=8), dict(ld=20), dict(z=FAKE + 2), dict(grad=FAKE + 8), dict(low=-0.1), dict(low=1.0),
                dict(high=-0.1), dict(high=float("nan")), dict(dual=1.0), dict(dual=-2.0), dict(kl=6), dict(kl=-1),
                dict(kl_coef=FAKE), dict(kl_out=FAKE), dict(kl=1), dict(kl=3), dict(kl=4), dict(kl=4, x=FAKE),
                dict(kl=4, x=FAKE, ldx=20), dict(kl=5, x=FAKE + 8, ldx=16), dict(V=(1 << 30) + 8, ld=(1 << 30) + 8)):
        assert _call(L.acrl_policy_loss_grad_logits, ok, **bad) == E, bad


def test_preference_loss(L):
    assert L.acrl_preference_workspace_bytes(-1, 1) == -1 and L.acrl_preference_workspace_bytes(1, -1) == -1
    n = L.acrl_preference_workspace_bytes(4, 2)
    ok = dict(logp=FAKE, ref=None, mask=None, T=9, rewards=FAKE, so=FAKE, S=4, go=FAKE, Gn=2, form=0, beta=0.1, margin=0.0,
              smooth=0.0, mean=0, ratio=FAKE, coef=FAKE, loss=FAKE, ws=FAKE, n=n, flags=None, stream=None)
    for bad in (dict(logp=None), dict(rewards=None), dict(so=None), dict(go=None), dict(ratio=None), dict(coef=None),
                dict(loss=None), dict(ws=None), dict(ws=FAKE + 8), dict(n=n - 1), dict(T=-1), dict(S=-1), dict(Gn=-1),
                dict(Gn=0), dict(S=0), dict(form=3), dict(form=-1), dict(beta=0.0), dict(beta=float("inf")),
                dict(margin=float("nan")), dict(smooth=0.5), dict(smooth=-0.1)):
        assert _call(L.acrl_preference_loss, ok, **bad) == E, bad


def test_preference_step(L):
    assert L.acrl_preference_step_workspace_bytes(-1, 1, 1) == -1
    n = L.acrl_preference_step_workspace_bytes(9, 4, 2)
    ok = dict(z=FAKE, T=9, V=16, ld=16, ids=FAKE, mask=None, ref=None, rewards=FAKE, so=FAKE, S=4, go=FAKE, Gn=2, form=0,
              beta=0.1, margin=0.0, smooth=0.0, mean=0, lse=FAKE, logp=FAKE, ratio=FAKE, coef=FAKE, grad=FAKE, loss=FAKE,
              ws=FAKE, n=n, flags=FAKE, stream=None)
    for bad in (dict(z=None), dict(ids=None), dict(rewards=None), dict(so=None), dict(go=None), dict(lse=None), dict(logp=None),
                dict(ratio=None), dict(coef=None), dict(grad=None), dict(loss=None), dict(ws=None), dict(flags=None),
                dict(n=n - 1), dict(ws=FAKE + 4), dict(z=FAKE + 2), dict(grad=FAKE + 8), dict(T=-1), dict(V=0), dict(ld=8),
                dict(ld=20), dict(S=-1), dict(S=0), dict(Gn=0), dict(form=3), dict(beta=-1.0), dict(smooth=0.5)):
        assert _call(L.acrl_preference_step, ok, **bad) == E, bad


def test_token_logp(L):
    ok = dict(z=FAKE, T=9, V=16, ld=16, ids=FAKE, mask=None, lse=FAKE, logp=FAKE, flags=None, stream=None)
    for bad in (dict(z=None), dict(ids=None), dict(lse=None), dict(logp=None), dict(z=FAKE + 2), dict(T=-1), dict(V=0), dict(ld=8),
                dict(ld=20), dict(V=(1 << 30) + 8, ld=(1 << 30) + 8)):
        assert _call(L.acrl_token_logp, ok, **bad) == E, bad
    assert _call(L.acrl_token_logp, ok, T=0, z=None, ids=None) == OK
