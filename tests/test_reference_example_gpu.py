"""Fp8Head against its formula, and the example that runs the 8-bit products, the policy loss and the preference step
together."""

import os
import sys

import pytest
import torch

import paper_2607_24062_gb300 as acrl

pytestmark = pytest.mark.gpu


def _values(t):
    """The float64 matrix that an 8-bit one stands for."""
    rows = 128 if t.scale.shape[0] < t.shape[0] else 1
    s = torch.exp2(t.scale.double() - 127).repeat_interleave(rows, 0).repeat_interleave(128, 1)
    return t.q.float().double() * s[: t.shape[0], : t.shape[1]]


@pytest.mark.parametrize("T,V,K", [(1, 1000, 64), (37, 4099, 200), (130, 515, 129)])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_fp8_head(T, V, K, fmt):
    g = torch.Generator().manual_seed(T + V)
    w = torch.randn(V, K, generator=g).bfloat16().cuda()
    h = torch.zeros(T, (K + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")[:, :K]
    h.copy_(torch.randn(T, K, generator=g))
    wp = torch.zeros(V, (K + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")[:, :K]
    wp.copy_(w)
    head = acrl.Fp8Head(wp, fmt=fmt)
    z = head.logits(h)
    assert z.shape == (T, V) and z.stride(0) == (V + 7) // 8 * 8
    a, b = _values(acrl.fp8_quantize(h)), _values(head.weight)
    exact, size = a @ b.t(), a.abs() @ b.abs().t()
    # the accumulation in fp32 over K terms, then one rounding to bf16
    assert bool(((z.double() - exact).abs() <= K * 2.0 ** -22 * size + 2.0 ** -8 * exact.abs()).all())
    ids = torch.randint(0, V, (T,), generator=g).int().cuda()
    mask = (torch.arange(T) % 5 != 3).to(torch.uint8).cuda()
    lp = torch.log_softmax(z.double(), -1).gather(1, ids.long()[:, None])[:, 0] * mask
    # token_stats' bound for its log-probs: a rounding of a sum of V terms and of the difference of two logits
    got = head.logp(h, ids, mask)
    assert bool(((got.double() - lp).abs() <= 1e-5 * (1 + lp.abs())).all()) and float(got[mask == 0].abs().sum()) == 0


def test_example_trains():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
    try:
        import reference_kl
    finally:
        sys.path.pop(0)
    log = reference_kl.train(steps=6)
    assert [kind for kind, *_ in log] == ["policy"] * 3 + ["preference"] * 3
    assert all(abs(loss) < 10 and abs(other) < 10 for _, loss, other in log)
    # before any update the policy is the reference but for the rounding of the 8-bit head: a KL well under that of
    # logits with an error of 2^-4 of their size (their spread is about 1), and above 0
    assert 0 < log[0][2] < 0.01
    assert log[2][2] != log[0][2]


def test_head_log_probs_add_up():
    """A response's log-probs by the head, summed: their errors are the step's, below 4e-6 + 2e-7 |logp| each with signs that mix
    (6 standard deviations of 1,500 errors of fp32's spacing at 16); a bias of 1.5e-7 would make 2.2e-4."""
    T, V, K = 1500, 32000, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    head = acrl.Fp8Head((0.25 * torch.randn((V, K), generator=g, device="cuda")).bfloat16())
    h = torch.randn((T, K), generator=g, device="cuda").bfloat16()
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    lp = torch.log_softmax(head.logits(h).double(), -1).gather(1, ids.long()[:, None])[:, 0]
    got = head.logp(h, ids).double()
    assert bool(((got - lp).abs() <= 4e-6 + 2e-7 * lp.abs()).all())
    assert abs(float((got - lp).sum())) <= 6 * 1e-6 * T ** 0.5 / 2
