"""The preference loss over the responses of a prompt against its definition in 64 bits."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2607_24062_gb300 as acrl  # noqa: E402
from paper_2607_24062_gb300 import api  # noqa: E402

DEV = "cuda"


def _batch(sizes, lengths, seed, masked=0.1, levels=3):
    """Prompts of `sizes` responses with the given lengths (cycled)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    S = sum(sizes)
    n = [lengths[i % len(lengths)] for i in range(S)]
    T = sum(n)
    so = torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=torch.int64, device=DEV)
    go = torch.tensor([0] + list(torch.tensor(sizes).cumsum(0)), dtype=torch.int32, device=DEV)
    logp = -torch.rand(T, generator=g, device=DEV) * 3
    return dict(logp=logp, ref=logp + 0.3 * torch.randn(T, generator=g, device=DEV),
                mask=(torch.rand(T, generator=g, device=DEV) >= masked).to(torch.uint8),
                rewards=torch.randint(0, levels, (S,), generator=g, device=DEV).float(), so=so, go=go)


def _plain(b, beta=0.1, form="sigmoid", margin=0.0, label_smoothing=0.0, length_norm=False):
    """Loss, D and dL/dlogp by autograd in float64."""
    logp = b["logp"].double().cpu().requires_grad_()
    ref = torch.zeros_like(logp) if b["ref"] is None else b["ref"].double().cpu()
    mask = torch.ones(logp.numel(), dtype=torch.bool) if b["mask"] is None else b["mask"].bool().cpu()
    so, go, R = b["so"].tolist(), b["go"].tolist(), b["rewards"].tolist()
    D, n = [], []
    for i in range(len(so) - 1):
        m = mask[so[i]: so[i + 1]]
        d = (logp - ref)[so[i]: so[i + 1]][m]
        n.append(int(m.sum()))
        D.append(d.sum() / (max(1, n[-1]) if length_norm else 1))
    per = []
    for g in range(len(go) - 1):
        f = []
        for i in range(go[g], go[g + 1]):
            for j in range(go[g], go[g + 1]):
                if R[i] > R[j] and n[i] and n[j]:
                    h = beta * (D[i] - D[j]) - margin
                    f.append((1 - label_smoothing) * torch.nn.functional.softplus(-h) +
                             label_smoothing * torch.nn.functional.softplus(h) if form == "sigmoid" else
                             torch.relu(1 - h) if form == "hinge" else ((h - 0.5) / beta) ** 2)
        if f:
            per.append(torch.stack(f).mean())
    loss = torch.stack(per).mean() if per else (logp * 0).sum()
    grad = torch.autograd.grad(loss, logp)[0]
    return float(loss), torch.stack(D).detach() if D else torch.zeros(0), grad


def _check(b, o, **kw):
    """fp64 sums of fp32 log-probs, h and its functions in fp32: relative errors of a few 2^-24, h absolutely 2^-24 |h|."""
    loss, D, grad = _plain(b, **kw)
    assert torch.allclose(o.ratio.double().cpu(), D, rtol=2e-7, atol=1e-12)
    assert abs(float(o.loss) - loss) <= 4e-6 * abs(loss) + 1e-12
    got = o.coef.double().cpu()
    assert bool(((got + grad).abs() <= 4e-6 * grad.abs() + 2e-6 * grad.abs().max()).all())
    if b["mask"] is not None:
        assert not bool(o.coef[b["mask"] == 0].any())


def _run(b, **kw):
    return acrl.preference_loss(b["logp"], b["ref"], b["mask"], b["rewards"], b["so"], b["go"], **kw)


@pytest.mark.parametrize("form", ["sigmoid", "hinge", "ipo"])
@pytest.mark.parametrize("length_norm", [False, True])
@pytest.mark.parametrize("sizes,lengths", [([2], [1]), ([2, 2, 2], [5, 40]), ([1, 8, 3, 4], [0, 7, 300, 1025]),
                                           ([130, 2], [3, 9, 1]), ([8] * 40, [17, 64, 2, 0, 90])])
def test_preference(form, length_norm, sizes, lengths):
    b = _batch(sizes, lengths, len(sizes) + lengths[-1])
    kw = dict(form=form, length_norm=length_norm, beta=0.2 if form == "sigmoid" else 0.5)
    flags = api.new_flags()
    _check(b, _run(b, flags=flags, **kw), **kw)
    assert acrl.read_flags(flags) == 0


def test_options():
    b = _batch([4, 6, 2], [9, 20], 3)
    for kw in (dict(label_smoothing=0.2), dict(margin=0.7), dict(beta=3.0, margin=-0.2), dict(form="hinge", margin=0.3),
               dict(form="ipo", margin=0.1, beta=0.05)):
        _check(b, _run(b, **kw), **kw)
    for part in ("mask", "ref"):
        c = dict(b, **{part: None})
        _check(c, _run(c))


def test_no_pairs():
    """Equal rewards, single responses and prompts whose other side is masked make no pair; they count for nothing."""
    b = _batch([2, 1, 3, 2], [4, 6], 4, masked=0.0)
    b["rewards"][:] = torch.tensor([1, 1, 0, 1, 0, 0, 1, 0.0], device=DEV)
    b["mask"][int(b["so"][7]): int(b["so"][8])] = 0            # the last prompt's rejected answer has no valid token
    _check(b, _run(b))
    b["rewards"][:] = 0.5
    o = _run(b)
    assert float(o.loss) == 0 and not bool(o.coef.any())
    b["mask"][:] = 0
    b["rewards"][::2] = 1
    o = _run(b)
    assert float(o.loss) == 0 and not bool(o.coef.any()) and not bool(o.ratio.any())


def test_far_apart():
    """Log ratios of thousands: the sigmoid's tails, with no overflow."""
    b = _batch([2, 2], [50], 5, masked=0.0)
    b["ref"][: 50] -= 300.0
    b["ref"][150:] -= 300.0
    b["rewards"][:] = torch.tensor([1, 0, 1, 0.0], device=DEV)
    _check(b, _run(b))


def test_undefined():
    b = _batch([2, 2], [5], 6, masked=0.0)
    b["rewards"][:] = torch.tensor([1, 0, 0, 1.0], device=DEV)
    b["logp"][2] = math.nan
    flags = api.new_flags()
    o = _run(b, flags=flags)
    assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE
    assert bool(o.loss.isnan()) and bool(o.coef[:10].isnan().all()) and bool(o.coef[10:].isfinite().all())
    b["mask"][2] = 0                                            # the same token masked
    flags = api.new_flags()
    _check(b, _run(b, flags=flags))
    assert acrl.read_flags(flags) == 0
    b["rewards"][1] = math.nan
    flags = api.new_flags()
    assert bool(_run(b, flags=flags).loss.isfinite())
    assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE


def test_offsets_that_break_the_rules():
    b = _batch([2, 2], [5], 7, masked=0.0)
    for so, go in (([0, 5, 3, 15, 20], None), ([0, 5, 10, 15, 21], None), ([1, 5, 10, 15, 20], None), ([0, 5, 10, 15, 19], None),
                   (None, [0, 3, 2]), (None, [0, 2, 5]), (None, [1, 2, 4]), (None, [0, 2, 3])):
        c = dict(b)
        if so:
            c["so"] = torch.tensor(so, dtype=torch.int64, device=DEV)
        if go:
            c["go"] = torch.tensor(go, dtype=torch.int32, device=DEV)
        flags = api.new_flags()
        _run(c, flags=flags)
        assert acrl.read_flags(flags) & acrl.FLAG_BAD_OFFSETS


def test_step_from_logits():
    sizes, lengths, V = [2, 3], [6, 11, 4], 777
    b = _batch(sizes, lengths, 8)
    T = b["logp"].numel()
    g = torch.Generator(device=DEV).manual_seed(1)
    z = (2 * torch.randn((T, 784), generator=g, device=DEV)).to(torch.bfloat16)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    x = z[:, :V].double().requires_grad_()
    logp = torch.log_softmax(x, 1).gather(1, ids.long()[:, None])[:, 0]
    step = acrl.PreferenceStep(T, V, 784, sum(sizes), len(sizes), beta=0.3)
    step.run(z, ids, b["mask"], b["ref"], b["rewards"], b["so"], b["go"])
    c = dict(b, logp=torch.where(b["mask"].bool(), logp.detach(), torch.zeros_like(logp)).float())
    loss, D, grad = _plain(c, beta=0.3)
    (logp * grad.to(DEV)).sum().backward()
    # log-probs within 4e-6 + 2^-23 |logp|: up to 12 of them in a ratio, beta and the pairs' mean below 1
    assert abs(float(step.loss) - loss) <= 1e-4 * abs(loss)
    assert bool(((step.grad[:, :V].double() - x.grad).abs() <= 2.0 ** -8 * 1.02 * x.grad.abs() + 1e-5 * grad.abs().max()).all())
    assert acrl.read_flags(step.flags) == 0
    # and its scalar as an autograd node
    y = z.clone().requires_grad_()
    node = acrl.pairs_loss(step, y[:, :V], ids, b["mask"], b["ref"], b["rewards"], b["so"], b["go"])
    (2.0 * node).backward()
    assert torch.allclose(y.grad[:, :V].float(), 2.0 * step.grad[:, :V].float(), rtol=2.0 ** -8)


@pytest.mark.parametrize("V,gap", [(1, 0), (7, 8), (64, 0), (4096, 0), (5003, 8), (20011, 0), (70001, 0), (151936, 0)])
def test_log_probs_of_the_step(V, gap):
    """lse and logp of the step's rows: fp32 sums (4e-6 + 2e-7 of the number, as for the policy loss), masked rows and bad ids,
    undefined rows; and no bias that a response's tokens would add up."""
    T = 96 if V < 60000 else 40
    g = torch.Generator(device=DEV).manual_seed(V)
    ld = (V + 7) // 8 * 8 + gap
    z = (2 * torch.randn((T, ld), generator=g, device=DEV)).to(torch.bfloat16)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    mask[::5] = 0
    z[5] = math.nan                                 # masked: not looked at
    ids[1] = V
    z[2, 0] = math.nan
    z[3, :V] = -math.inf
    if V > 1:
        z[4, V - 1] = -math.inf                     # a column taken out
        ids[4] = 0
        z[6, :V] = -3.3895313892515355e38           # all but one
        z[6, 0], ids[6] = 1.0, 0
    step = acrl.PreferenceStep(T, V, ld, 2, 1)
    so, go = torch.tensor([0, T // 2, T], device=DEV), torch.tensor([0, 2], dtype=torch.int32, device=DEV)
    step.run(z, ids, mask, None, torch.tensor([1.0, 0.0], device=DEV), so, go)
    assert acrl.read_flags(step.flags) == acrl.FLAG_BAD_ID | acrl.FLAG_NONFINITE
    lse = torch.logsumexp(z[:, :V].double(), 1)
    lp = z[:, :V].gather(1, ids.clamp(max=V - 1).long()[:, None])[:, 0].double() - lse
    live = mask.bool()
    assert not bool(step.logp[~live].any()) and not bool(step.lse[~live].any()) and float(step.logp[1]) == 0
    assert bool(step.logp[[2, 3]].isnan().all()) and bool(step.lse[[2, 3]].isnan().all())
    live[[1, 2, 3]] = False
    for got, want in ((step.lse, lse), (step.logp, lp)):
        assert bool(((got - want).abs() <= 4e-6 + 2e-7 * want.abs())[live].all())


def test_sums_of_many_tokens():
    """The log ratio of 1,500 tokens against a reference that is the policy itself, rounded to fp32: what is left are the
    log-probs' own errors.  Each is below 4e-6 + 2e-7 |logp| in size and their signs mix; a bias of 1e-7 would make 1.5e-4."""
    T, V = 1500, 32000
    g = torch.Generator(device=DEV).manual_seed(4)
    z = (2 * torch.randn((T, V), generator=g, device=DEV)).to(torch.bfloat16)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    lp = torch.log_softmax(z.double(), 1).gather(1, ids.long()[:, None])[:, 0]
    step = acrl.PreferenceStep(T, V, V, 1, 1)
    step.run(z, ids, None, lp.float(), torch.ones(1, device=DEV), torch.tensor([0, T], device=DEV),
             torch.tensor([0, 1], dtype=torch.int32, device=DEV))
    # 6 standard deviations of 1,500 errors of 1e-6 (fp32's spacing at 16), the reference's own rounding among them
    assert abs(float(step.ratio)) <= 6 * 1e-6 * math.sqrt(T) / 2


def test_refusals():
    b = _batch([2, 2], [5], 9)
    for change in (dict(logp=b["logp"].double()), dict(ref=b["ref"][:3]), dict(mask=b["mask"].bool()),
                   dict(rewards=b["rewards"][:2]), dict(so=b["so"].int()), dict(go=b["go"].long()), dict(so=b["so"][:0])):
        with pytest.raises(acrl.AcrlError):
            _run(dict(b, **change))
    for kw in (dict(beta=0.0), dict(form="dpo"), dict(label_smoothing=0.6), dict(margin=math.inf), dict(coef=b["logp"][:1]),
               dict(workspace=torch.empty(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(acrl.AcrlError):
            _run(b, **kw)
    step = acrl.PreferenceStep(20, 64, 64, 4, 2)
    with pytest.raises(acrl.AcrlError):
        step.run(torch.zeros((19, 64), dtype=torch.bfloat16, device=DEV), None, None, None, b["rewards"], b["so"], b["go"])


@pytest.mark.parametrize("V", [1000, 4096, 20011, 70001, 151936])
@pytest.mark.parametrize("shape", ["head", "blocks", "peaks"])
def test_log_probs_of_columns_far_below_the_others(V, shape):
    """As test_log_probs_of_the_step, with columns 60 to 110 below the row's largest: a head of the row, blocks of 256 columns, or
    all but a few."""
    T = 51
    g = torch.Generator(device=DEV).manual_seed(V)
    ld = (V + 7) // 8 * 8
    if shape == "head":
        down = (torch.arange(V, device=DEV) < V // 4 + 1)[None].repeat(T, 1)
    elif shape == "blocks":
        down = (torch.rand((T, V // 256 + 1), generator=g, device=DEV) < 0.5).repeat_interleave(256, 1)[:, :V]
        down[:, :256] = True
    else:
        down = torch.rand((T, V), generator=g, device=DEV) >= 4.0 / V
    down[:, V - 1] = False
    z = torch.zeros((T, ld), device=DEV)
    z[:, :V] = 0.25 * torch.randn((T, V), generator=g, device=DEV) - down * (60.0 + torch.arange(T, device=DEV))[:, None]
    z = z.to(torch.bfloat16)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    ids[::2] = V - 1
    step = acrl.PreferenceStep(T, V, ld, 2, 1)
    so, go = torch.tensor([0, 20, T], device=DEV), torch.tensor([0, 2], dtype=torch.int32, device=DEV)
    step.run(z, ids, None, None, torch.tensor([1.0, 0.0], device=DEV), so, go)
    assert acrl.read_flags(step.flags) == 0
    lse = torch.logsumexp(z[:, :V].double(), 1)
    lp = z[:, :V].gather(1, ids.long()[:, None])[:, 0].double() - lse
    for got, want in ((step.lse, lse), (step.logp, lp)):
        assert bool(((got - want).abs() <= 4e-6 + 2e-7 * want.abs()).all())


def test_token_logp():
    """The step's lse and log-probs by themselves, to the last bit, on any stream; nothing for no rows."""
    T, V = 40, 5003
    g = torch.Generator(device=DEV).manual_seed(6)
    z = (2 * torch.randn((T, 5008), generator=g, device=DEV)).to(torch.bfloat16)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    mask = (torch.arange(T, device=DEV) % 4 > 0).to(torch.uint8)
    step = acrl.PreferenceStep(T, V, 5008, 2, 1)
    step.run(z, ids, mask, None, torch.tensor([1.0, 0.0], device=DEV), torch.tensor([0, 9, T], device=DEV),
             torch.tensor([0, 2], dtype=torch.int32, device=DEV))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for lse, logp in (api.token_logp(z, ids, mask, V=V), api.token_logp(z, ids, mask, V=V, stream=side)):
        torch.cuda.synchronize()
        assert torch.equal(lse, step.lse) and torch.equal(logp, step.logp)
    assert [t.numel() for t in api.token_logp(z[:0], ids[:0], V=V)] == [0, 0]
    flags = api.new_flags()
    ids[3], z[5, 7] = V, math.nan
    logp = api.token_logp(z, ids, mask, V=V, flags=flags)[1]
    assert acrl.read_flags(flags) == acrl.FLAG_BAD_ID | acrl.FLAG_NONFINITE
    assert float(logp[3]) == 0 and bool(logp[5].isnan())
    for bad in (dict(ids=ids.long()), dict(ids=ids[:3]), dict(mask=mask.bool()), dict(logits=z.float()), dict(V=5009), dict(logp=ids)):
        with pytest.raises(acrl.AcrlError):
            api.token_logp(**{**dict(logits=z, ids=ids, mask=mask, V=V), **bad})


@pytest.mark.parametrize("T,V", [(2000, 4096), (1500, 32000), (300, 151936)])
@pytest.mark.parametrize("rest", [0.1, 1e-2, 1e-3, 1e-5])
def test_log_probs_of_likely_tokens(T, V, rest):
    """Rows whose sampled column has nearly all of the probability, as for the policy loss: a spread of up to 5e-7, and in common
    the exponential's mean error (5e-8) and the sums' roundings, 1.5e-7 together."""
    g = torch.Generator(device=DEV).manual_seed(8)
    z = 2.5 * torch.randn((T, V), generator=g, device=DEV)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    z[torch.arange(T), ids.long()] = torch.logsumexp(z, 1) - math.log(rest) + torch.rand(T, generator=g, device=DEV)
    z = z.to(torch.bfloat16)
    lse = torch.cat([torch.logsumexp(part.double(), 1) for part in z.split(100)])
    lp = z.gather(1, ids.long()[:, None])[:, 0].double() - lse
    got = api.token_logp(z, ids)
    for a, b in zip(got, (lse, lp)):
        assert bool(((a - b).abs() <= 4e-6 + 2e-7 * b.abs()).all())
    assert abs(float((got[1] - lp).mean())) <= 1.5e-7 + 6 * 5e-7 / math.sqrt(T)
