"""The policy loss with a KL term, from logits to gradient, against its definition in 64 bits."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2607_24062_gb300 as acrl  # noqa: E402
from paper_2607_24062_gb300 import api  # noqa: E402

DEV = "cuda"
KINDS = [None, "k1", "k2", "k3", "exact", "reverse"]


def _inputs(T, V, seed, kl="exact", gap=0, spread=2.0, apart=0.4):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ld = (V + 7) // 8 * 8 + gap
    z = (torch.randn((T, ld), generator=g, device=DEV) * spread).to(torch.bfloat16)
    x = (z.float() + apart * torch.randn((T, ld), generator=g, device=DEV)).to(torch.bfloat16)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    lp = torch.log_softmax(z[:, :V].double(), 1).gather(1, ids.long()[:, None])[:, 0]
    rnd = lambda s: s * torch.randn(T, generator=g, device=DEV)   # noqa: E731
    full = kl in ("exact", "reverse")
    return dict(z=z, ids=ids, mask=(torch.rand(T, generator=g, device=DEV) < 0.8).to(torch.uint8), coef=rnd(0.5),
                kl_coef=None if kl is None else rnd(0.1).abs(), old=(lp + rnd(0.3)).float(),
                ref_logits=x if full else None, ref_logp=None if full or kl is None else (lp + rnd(0.4)).float(), V=V, kl=kl)


def _run(i, **kw):
    return acrl.policy_loss_grad_logits(i["z"], i["ids"], i["mask"], i["coef"], V=i["V"], old_logp=i["old"], kl=i["kl"],
                                        kl_coef=i["kl_coef"], ref_logits=i["ref_logits"], ref_logp=i["ref_logp"], **kw)


def _plain_loss(i, z, low, high, dual):
    """Per-token loss, logp and KL of float64 logits, differentiable in them."""
    lp = torch.log_softmax(z, 1)
    ids = i["ids"].long()[:, None]
    logp = lp.gather(1, ids)[:, 0]
    T = z.shape[0]
    c = torch.zeros(T, device=DEV, dtype=torch.float64) if i["coef"] is None else i["coef"].double()
    r = torch.ones_like(logp) + 0 * logp if i["old"] is None else torch.exp(logp - i["old"].double())
    if i["old"] is None:
        r = torch.exp(logp - logp.detach())
    up = torch.minimum(r, torch.full_like(r, 1 + high))
    down = torch.maximum(r, torch.full_like(r, 1 - low))
    if dual:
        down = torch.minimum(down, torch.full_like(r, dual))
    loss = -c * torch.where(c >= 0, up, down)
    kl = torch.zeros_like(logp)
    if i["kl"] in ("exact", "reverse"):
        lq = torch.log_softmax(i["ref_logits"][:, : i["V"]].double(), 1)
        p, q = lp.exp(), lq.exp()
        term = p * (lp - lq) if i["kl"] == "exact" else q * (lq - lp)
        w = p if i["kl"] == "exact" else q
        kl = torch.where(w > 0, term, torch.zeros_like(term)).sum(1)
    elif i["kl"]:
        d = logp - i["ref_logp"].double()
        kl = {"k1": d, "k2": d * d / 2, "k3": torch.exp(-d) - 1 + d}[i["kl"]]
    k = torch.zeros(T, device=DEV, dtype=torch.float64) if i["kl_coef"] is None else i["kl_coef"].double()
    return loss + k * kl, logp, kl


def _check(i, o, low=0.2, high=0.2, dual=0.0):
    """fp32 statistics: an exponential's exponent of up to ~20 is rounded at 2^-24 of it and the exponential itself at
    2^-22, so lse, and with it every p relatively, is off by at most 4e-6; KL sums p d with |d| up to what the rows hold.
    The gradient adds one rounding to bf16."""
    V, z = i["V"], i["z"][:, : i["V"]].double().requires_grad_()
    loss, logp, kl = _plain_loss(i, z, low, high, dual)
    m = torch.ones_like(logp) if i["mask"] is None else i["mask"].double()
    (loss * m).sum().backward()
    lp = torch.log_softmax(z.detach(), 1)
    m = m.bool()
    zero = torch.zeros_like(logp)
    e_logp = 4e-6 + 2e-7 * logp.abs()
    assert bool(((o.logp - torch.where(m, logp, zero)).abs() <= torch.where(m, e_logp, zero)).all())
    size = torch.zeros_like(lp)
    e_kl = zero
    if i["kl"] in ("exact", "reverse"):
        lq = torch.log_softmax(i["ref_logits"][:, :V].double(), 1)
        a = (lp - lq).abs()
        w = lp.exp() if i["kl"] == "exact" else lq.exp()
        d = (i["z"][:, :V].double() - i["ref_logits"][:, :V].double()).abs()
        e_kl = 8e-6 * (1 + torch.where(w > 0, w * (a + d), torch.zeros_like(w)).sum(1))
        size = torch.where(w > 0, lp.exp() * (a + kl[:, None].abs() + e_kl[:, None]) + lq.exp(), torch.zeros_like(w))
    elif i["kl"]:
        d = logp - i["ref_logp"].double()
        e_kl = e_logp * (2 + d.abs() + torch.exp(-d)) + 1e-6 * kl.abs()
    if o.kl is not None:
        assert bool(((o.kl - torch.where(m, kl, zero)).abs() <= torch.where(m, e_kl, zero)).all())
    k = zero if i["kl_coef"] is None else i["kl_coef"].double()
    c = zero if i["coef"] is None else i["coef"].double().abs()
    r = torch.ones_like(logp) if i["old"] is None else torch.exp(logp - i["old"].double())
    # rows whose ratio is within its error of an edge of the clip may fall on either side
    edge = torch.zeros_like(m)
    if i["old"] is not None:
        for b in (1 - low, 1 + high, dual or math.inf):
            edge |= (r - b).abs() <= 4 * e_logp * b
    cap = r.clamp(max=max(1 + high, dual or math.inf))
    e_loss = c * cap.clamp(max=1e6) * 4 * e_logp + k * e_kl + 2e-7 * loss.abs()
    assert bool(((o.token_loss - torch.where(m, loss, zero)).abs() <= torch.where(m, e_loss, zero)).all())
    total = torch.where(m, loss, zero)
    assert abs(float(o.loss) - float(total.sum())) <= float(torch.where(m, e_loss, zero).sum()) + 1e-6 * float(total.abs().sum()) + 1e-30
    g, got = z.grad, o.grad[:, :V].double()
    # of the one-hot term: c r and the estimators' slopes, each with its error
    slope = c * r.clamp(max=1e6) + (k * (2 + (logp - i["ref_logp"].double()).abs() + torch.exp(i["ref_logp"].double() - logp))
                                    if i["ref_logp"] is not None else 0)
    p = lp.exp()
    near = 8e-6 * (slope[:, None] * p + k[:, None] * size) + (k * e_kl)[:, None] * p
    near.scatter_add_(1, i["ids"].long()[:, None], (8e-6 * slope + 4 * slope * e_logp)[:, None])
    bound = 2.0 ** -8 * 1.001 * g.abs() + near + 2.0 ** -125
    ok = ((got - g).abs() <= bound) | edge[:, None]
    assert bool(ok.all()), ((~ok).nonzero()[:4].tolist(), got[~ok][:4], g[~ok][:4])


@pytest.mark.parametrize("kl", KINDS)
@pytest.mark.parametrize("T,V,gap", [(1, 1, 0), (3, 7, 8), (5, 8, 0), (6, 63, 16), (4, 1000, 0), (7, 4096, 8), (3, 20011, 0),
                                     (2, 65544, 0), (2, 151936, 8), (1, 400003, 0)])
def test_policy_loss(kl, T, V, gap):
    i = _inputs(T, V, 100 * T + V, kl, gap)
    flags = api.new_flags()
    if gap:
        grad = torch.full_like(i["z"], 3.0)
        o = _run(i, flags=flags, grad=grad)
        assert bool((grad[:, V:] == 3).all())
    else:
        o = _run(i, flags=flags)
    assert acrl.read_flags(flags) == 0
    _check(i, o)


@pytest.mark.parametrize("kl", ["exact", "k3"])
@pytest.mark.parametrize("low,high,dual,old", [(0.0, 0.0, 0.0, True), (0.2, 0.28, 3.0, True), (0.9, 2.0, 1.5, True),
                                               (0.1, 0.1, 0.0, False)])
def test_clip(kl, low, high, dual, old):
    i = _inputs(64, 333, 5, kl)
    i["old"] = i["old"] - 1.2 * (torch.arange(64, device=DEV) % 3 - 1) if old else None
    _check(i, _run(i, clip_low=low, clip_high=high, dual_clip=dual), low, high, dual)


@pytest.mark.parametrize("kl", ["exact", "reverse", "k2"])
def test_parts_left_out(kl):
    i = _inputs(9, 500, 6, kl)
    i["mask"] = None
    _check(i, _run(i))
    _check(dict(i, coef=None), _run(dict(i, coef=None)))            # distillation: the KL term alone
    free = dict(i, kl_coef=None)                                     # the KL as a figure only
    o = _run(free)
    _check(free, o)
    none = dict(i, kl=None, kl_coef=None, ref_logits=None, ref_logp=None)
    if kl == "k2":                                                   # without its term, the gradient of the loss alone
        assert torch.equal(o.grad[:, :500], _run(none).grad[:, :500])


@pytest.mark.parametrize("kl", ["exact", "reverse"])
@pytest.mark.parametrize("V", [9, 1000, 40000])
@pytest.mark.parametrize("value", [-math.inf, -3.3895313892515355e38])
def test_columns_taken_out(kl, V, value):
    """Columns that a mask took out of the policy, of both, or (where it puts no weight on them) of the reference."""
    i = _inputs(6, V, 7, kl)
    cut = torch.rand((6, V), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) < 0.3
    cut[torch.arange(6), i["ids"].long()] = False
    cut[3] = True                                   # all but the sampled column
    cut[3, int(i["ids"][3])] = False
    one, both = cut.clone(), cut.clone()
    one[::2], both[1::2] = False, False
    z, x = i["z"][:, :V], i["ref_logits"][:, :V]
    (z if kl == "exact" else x)[one] = value
    z[both], x[both] = value, value
    flags = api.new_flags()
    i["mask"] = None
    o = _run(i, flags=flags)
    assert acrl.read_flags(flags) == 0
    _check(i, o)


@pytest.mark.parametrize("kl", ["exact", "reverse", "k3", None])
def test_undefined_rows(kl):
    i = _inputs(12, 300, 8, kl)
    i["mask"] = torch.ones(12, dtype=torch.uint8, device=DEV)
    i["coef"] = torch.full((12,), 0.3, device=DEV)
    i["ids"][:] = 17
    clean = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in i.items()}
    z = i["z"]
    z[0, 5] = math.nan
    z[1, 5] = math.inf
    z[2, :300] = -math.inf
    z[3, 17] = -math.inf                            # the sampled column
    i["old"][4] = math.nan
    i["mask"][5] = 0
    z[5, 3] = math.nan                              # masked: not looked at
    i["ids"][6], i["ids"][7] = 300, -1
    i["coef"][8] = 0.0
    if i["kl_coef"] is not None:
        i["kl_coef"][8] = 0.0
    z[8, 5] = math.nan                              # no coefficient: a zero gradient, the figures undefined
    undefined, valued = [0, 1, 2, 3, 4], [10, 11]
    if kl in ("exact", "reverse"):
        # weight where the other side has none: an infinite KL
        (i["ref_logits"] if kl == "exact" else z)[9, 40] = -math.inf
        undefined.append(9)
    elif kl == "k3":
        i["ref_logp"][9] = math.nan
        undefined.append(9)
    else:
        valued.append(9)
    flags = api.new_flags()
    o = _run(i, flags=flags)
    assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE | acrl.FLAG_BAD_ID
    assert bool(o.grad[undefined, :300].isnan().all()) and bool(o.token_loss[undefined].isnan().all())
    assert bool(o.loss.isnan())
    for r in (5, 6, 7):
        assert not bool(o.grad[r, :300].any()) and float(o.logp[r]) == 0 and float(o.token_loss[r]) == 0
        assert o.kl is None or float(o.kl[r]) == 0
    assert not bool(o.grad[8, :300].any()) and float(o.token_loss[8]) == 0 and math.isnan(float(o.logp[8]))
    want = _run(clean)
    assert torch.equal(o.grad[valued, :300], want.grad[valued, :300])
    assert torch.equal(o.logp[valued], want.logp[valued])


def test_against_differences():
    """dL/dz_j as a central difference of the call's own loss.  Steps of 2^-5 on logits of multiples of 2^-6 below 2 are
    exact; the third derivative of these losses is below 8 (c r + k (1 + |a|)) < 16, so the difference is off by at most
    16 h^2 / 6 = 3e-3, and the loss's own rounding by 4e-6 / h."""
    g = torch.Generator(device=DEV).manual_seed(3)
    V, h = 24, 2.0 ** -5
    base = torch.randint(-60, 60, (V,), generator=g, device=DEV) / 64.0
    for kl in ("exact", "reverse", "k3"):
        ref = (torch.randint(-60, 60, (V,), generator=g, device=DEV) / 64.0).to(torch.bfloat16)
        z = base.repeat(2 * V + 1, 1)
        z[torch.arange(V), torch.arange(V)] += h
        z[V + torch.arange(V), torch.arange(V)] -= h
        z = z.to(torch.bfloat16)
        assert torch.equal(z[-1].float(), base)
        T = 2 * V + 1
        full = kl != "k3"
        o = acrl.policy_loss_grad_logits(
            z, torch.full((T,), 4, dtype=torch.int32, device=DEV), None, torch.full((T,), 0.7, device=DEV),
            old_logp=torch.full((T,), -3.2, device=DEV), clip_high=9.0, kl=kl, kl_coef=torch.full((T,), 0.5, device=DEV),
            ref_logits=ref.repeat(T, 1) if full else None, ref_logp=None if full else torch.full((T,), -2.9, device=DEV))
        diff = (o.token_loss[:V] - o.token_loss[V: 2 * V]) / (2 * h)
        assert bool(((diff - o.grad[-1].float()).abs() <= 3.2e-3 + 2.0 ** -8 * diff.abs()).all())


def test_nothing_and_other_stream():
    i = _inputs(5, 40, 9)
    empty = {k: v[:0] if isinstance(v, torch.Tensor) else v for k, v in i.items()}
    assert float(_run(empty).loss) == 0
    want = _run(i)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = _run(i, stream=s)
    s.synchronize()
    assert torch.equal(got.grad, want.grad) and torch.equal(got.loss, want.loss)


def test_same_bits_again():
    i = _inputs(6, 50001, 10)
    a, b = _run(i), _run(i)
    assert torch.equal(a.grad[:, :50001], b.grad[:, :50001]) and torch.equal(a.kl, b.kl) and torch.equal(a.loss, b.loss)


def test_autograd_node():
    i = _inputs(5, 77, 11)
    want = _run(i)
    y = i["z"].clone().requires_grad_()
    logp = torch.empty(5, device=DEV)
    loss = acrl.policy_loss(y[:, :77], i["ids"], i["mask"], i["coef"], old_logp=i["old"], kl="exact", kl_coef=i["kl_coef"],
                            ref_logits=i["ref_logits"], logp=logp)
    assert torch.equal(loss.detach().reshape(1), want.loss) and torch.equal(logp, want.logp)
    loss.backward()
    assert torch.equal(y.grad[:, :77], want.grad[:, :77]) and not bool(y.grad[:, 77:].any())


def test_refusals():
    i = _inputs(4, 64, 1)
    for change in (dict(kl="k4"), dict(kl="k1"), dict(kl=None), dict(ref_logits=None), dict(ids=i["ids"].long()),
                   dict(coef=i["coef"].double()), dict(coef=i["coef"][:2]), dict(z=i["z"].float()), dict(z=i["z"].t()),
                   dict(ref_logits=i["ref_logits"][:3]), dict(ref_logits=i["ref_logits"][:, :32]), dict(V=65)):
        with pytest.raises(acrl.AcrlError):
            _run(dict(i, **change))
    for kw in (dict(clip_low=1.0), dict(clip_high=-0.1), dict(dual_clip=0.5), dict(grad=i["z"][:2]),
               dict(grad=i["z"].float()), dict(logp=i["coef"][:1])):
        with pytest.raises(acrl.AcrlError):
            _run(i, **kw)


def _heights(T, V, shape, seed, low=60, step=1):
    """Logits of rows whose columns stand at one of two heights, the lower one `low` + `step` t below in row t: a head of the row
    below the rest ("head"), blocks of 256 columns at either height by chance ("blocks"), or single columns above ("peaks")."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    ld, col = (V + 7) // 8 * 8, torch.arange(V, device=DEV)
    if shape == "head":
        down = (col < V // 4 + 1)[None].repeat(T, 1)
    elif shape == "blocks":
        down = (torch.rand((T, V // 256 + 1), generator=g, device=DEV) < 0.5).repeat_interleave(256, 1)[:, :V]
        down[:, :256] = True
    else:
        down = torch.rand((T, V), generator=g, device=DEV) >= 4.0 / V
    down[:, V - 1] = False
    drop = low + step * torch.arange(T, device=DEV, dtype=torch.float32)
    z = torch.zeros((T, ld), device=DEV)
    z[:, :V] = 0.25 * torch.randn((T, V), generator=g, device=DEV) - down * drop[:, None]
    return z.to(torch.bfloat16)


# rows of one warp, of several, and of a cluster of two and of eight CTAs, with what fits in shared memory and more
@pytest.mark.parametrize("kl", ["exact", "reverse", "k3", None])
@pytest.mark.parametrize("shape", ["head", "blocks", "peaks"])
@pytest.mark.parametrize("T,V,step", [(51, 1000, 1), (51, 4096, 1), (51, 20011, 1), (156, 20011, 0.3125), (17, 65544, 3),
                                      (156, 65544, 0.3125), (160, 151936, 0.3125)])
def test_columns_far_below_the_others(kl, shape, T, V, step):
    """Columns that lie 60 to 110 below the row's largest, and where a warp meets them before those: every number of such a row
    is an ordinary one."""
    i = _inputs(T, V, 200 + V, kl)
    i["z"] = _heights(T, V, shape, V, step=step)
    i["mask"] = None
    i["ids"] = torch.where(torch.arange(T, device=DEV) % 3 > 0, V - 1, i["ids"]).to(torch.int32)
    lp = torch.log_softmax(i["z"][:, :V].double(), 1).gather(1, i["ids"].long()[:, None])[:, 0]
    g = torch.Generator(device=DEV).manual_seed(1)
    i["old"] = (lp + 0.3 * torch.randn(T, generator=g, device=DEV)).float()
    if i["ref_logits"] is not None:     # near the policy's logits, or with heights of its own
        x, other = i["z"].float(), _heights(T, V, shape, V + 1, step=step).float()
        x[::2] = other[::2]
        i["ref_logits"] = (x + 0.25 * torch.randn(x.shape, generator=g, device=DEV)).to(torch.bfloat16)
    elif kl:
        i["ref_logp"] = (lp + 0.3 * torch.randn(T, generator=g, device=DEV)).float()
    flags = api.new_flags()
    o = _run(i, flags=flags)
    assert acrl.read_flags(flags) == 0
    _check(i, o)


@pytest.mark.parametrize("kl", ["exact", "reverse", "k2", None])
@pytest.mark.parametrize("gap", [79.0, 81.0, 83.0, 85.0, 87.0, 95.0])
def test_leading_columns_of_one_height(kl, gap):
    """The first 256 of 4,096 columns at -gap, the others at 0: lse = log 3,840 to the last bits."""
    i = _inputs(8, 4096, 3, kl)
    i["z"][:, :256], i["z"][:, 256:] = -gap, 0.0
    i["mask"] = None
    i["ids"] = torch.full((8,), 4000, dtype=torch.int32, device=DEV)
    i["old"] = None
    if kl == "k2":
        i["ref_logp"] = torch.full((8,), -8.0, device=DEV)
    flags = api.new_flags()
    o = _run(i, flags=flags)
    assert acrl.read_flags(flags) == 0
    assert bool(((o.logp.double() + math.log(3840.0)).abs() <= 4e-6).all())
    _check(i, o)


def test_autograd_node_on_another_stream():
    """What a call on a busy stream writes is there when the node's own stream reads it, forwards and backwards."""
    i = _inputs(40, 5000, 12)
    want = _run(i)
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=DEV)
    grad, loss_of = torch.full_like(i["z"], 7.0), torch.full((1,), 7.0, device=DEV)
    y = i["z"].clone().requires_grad_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):                       # tens of milliseconds
            big = torch.tanh(big @ big)
    loss = acrl.policy_loss(y[:, :5000], i["ids"], i["mask"], i["coef"], old_logp=i["old"], kl="exact", kl_coef=i["kl_coef"],
                            ref_logits=i["ref_logits"], stream=side, grad=grad, loss=loss_of)
    loss.backward()
    got = y.grad.clone()
    torch.cuda.synchronize()
    assert torch.equal(loss.detach().reshape(1), want.loss)
    assert torch.equal(got[:, :5000], want.grad[:, :5000])
    # and the other way round: logits that the current stream is still to write
    z = i["z"].clone()
    late = torch.full_like(z, 3.0)
    torch.cuda.synchronize()
    for _ in range(20):
        big = torch.tanh(big @ big)
    late.copy_(z)
    loss = acrl.policy_loss(late[:, :5000], i["ids"], i["mask"], i["coef"], old_logp=i["old"], kl="exact", kl_coef=i["kl_coef"],
                            ref_logits=i["ref_logits"], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(loss.reshape(1), want.loss)


def test_numbers_that_overflow():
    """A ratio beyond fp32 that nothing clips, or a coefficient that is no number: the row is undefined and says so."""
    T, V = 6, 300
    z = (2 * torch.randn((T, 304), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)).to(torch.bfloat16)
    ids = torch.full((T,), 9, dtype=torch.int32, device=DEV)
    lp = torch.log_softmax(z[:, :V].double(), 1)[:, 9].float()
    coef = torch.tensor([-0.5, 0.5, -0.5, -0.5, 0.0, -0.5], device=DEV)
    old = lp - torch.tensor([100.0, 100.0, 1.0, 0.0, 100.0, math.inf], device=DEV)
    for dual in (0.0, 3.0):
        flags = api.new_flags()
        o = acrl.policy_loss_grad_logits(z, ids, None, coef, V=V, old_logp=old, dual_clip=dual, flags=flags)
        bad = [0, 5] if dual == 0.0 else []          # a dual clip bounds them; a positive coefficient's are bounded anyway
        good = [t for t in range(T) if t not in bad]
        assert acrl.read_flags(flags) == (acrl.FLAG_NONFINITE if bad else 0)
        assert bool(o.grad[bad, :V].isnan().all()) and bool(o.token_loss[bad].isnan().all())
        assert bool(o.grad[good, :V].isfinite().all()) and bool(o.token_loss[good].isfinite().all())
        assert bool(o.logp.isfinite().all()) and bool(o.loss.isnan()) == bool(bad)
    # coefficients that are no numbers
    flags = api.new_flags()
    o = acrl.policy_loss_grad_logits(z, ids, None, torch.tensor([math.nan, 1, math.inf, 1, 1, 1], device=DEV), V=V, kl="k1",
                                     kl_coef=torch.tensor([0, math.nan, 0, 0, 0, 0], device=DEV), ref_logp=lp, flags=flags)
    assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE
    assert bool(o.grad[:3, :V].isnan().all()) and bool(o.token_loss[:3].isnan().all())
    assert bool(o.grad[3:, :V].isfinite().all()) and bool(o.token_loss[3:].isfinite().all())


def test_estimates_that_overflow():
    """An infinite estimate of the KL is undefined as a figure, and in the loss where it has a factor there."""
    T, V = 6, 300
    z = (2 * torch.randn((T, 304), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)).to(torch.bfloat16)
    ids = torch.full((T,), 9, dtype=torch.int32, device=DEV)
    lp = torch.log_softmax(z[:, :V].double(), 1)[:, 9].float()
    coef = torch.tensor([-0.5, 0.5, -0.5, -0.5, 0.0, -0.5], device=DEV)
    ref = lp + torch.tensor([100.0, 1e30, 0.1, 0.0, 100.0, math.inf], device=DEV)
    k = torch.tensor([0.1, 0.1, 0.1, 0.1, 0.0, 0.0], device=DEV)
    for kl, undefined in (("k3", [0, 1, 4, 5]), ("k2", [1, 5])):
        for kl_coef in (k, None):
            flags = api.new_flags()
            o = acrl.policy_loss_grad_logits(z, ids, None, coef, V=V, kl=kl, kl_coef=kl_coef, ref_logp=ref, flags=flags)
            assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE
            assert o.kl.isnan().nonzero()[:, 0].tolist() == undefined and bool(o.logp.isfinite().all())
            bad = [t for t in undefined if kl_coef is not None and float(k[t]) != 0]
            good = [t for t in range(T) if t not in bad]
            assert bool(o.grad[bad, :V].isnan().all()) and bool(o.token_loss[bad].isnan().all())
            assert bool(o.grad[good, :V].isfinite().all()) and bool(o.token_loss[good].isfinite().all())


@pytest.mark.parametrize("kl", ["exact", "reverse"])
def test_log_prob_beside_an_infinite_kl(kl):
    """Where only the KL is infinite the log-prob is a number, and is given."""
    i = _inputs(4, 300, 8, kl)
    i["mask"] = None
    (i["ref_logits"] if kl == "exact" else i["z"])[1, 40] = -math.inf
    i["ids"][:] = 17
    flags = api.new_flags()
    o = _run(i, flags=flags)
    assert acrl.read_flags(flags) == acrl.FLAG_NONFINITE
    assert o.kl.isnan().nonzero()[:, 0].tolist() == [1]
    want = torch.log_softmax(i["z"][:, :300].double(), 1)[:, 17]
    assert bool(((o.logp - want).abs() <= 4e-6 + 2e-7 * want.abs()).all())


def test_autograd_node_again_and_again():
    """A graph that is kept gives the same gradient each time, whatever was done to the leaf's in between."""
    i = _inputs(5, 80, 11)
    y = i["z"].clone().requires_grad_()
    loss = acrl.policy_loss(y, i["ids"], i["mask"], i["coef"], old_logp=i["old"], kl="exact", kl_coef=i["kl_coef"],
                            ref_logits=i["ref_logits"])
    loss.backward(retain_graph=True)
    first = y.grad.clone()
    y.grad.mul_(3.0)                # as a clipped gradient norm does
    y.grad = None
    loss.backward(retain_graph=True)
    assert torch.equal(y.grad, first)
    loss.backward()                 # and added up
    assert torch.equal(y.grad, first + first)
    loss_again = _run(dict(i, z=y.detach(), V=80)).grad
    assert torch.equal(first, loss_again)


@pytest.mark.parametrize("kl", ["exact", "reverse", "k3", None])
@pytest.mark.parametrize("height", [0.0, 20.0, -20.0])
def test_log_probs_add_up(kl, height):
    """The log-probs' errors, below 4e-6 + 2e-7 |logp| each, have signs that mix: 6 standard deviations of a sum of 2,000 errors of
    fp32's spacing at 16, wherever the logits stand.  (A common part of 1e-7 would make 2.0e-4.)"""
    T, V = 2000, 4096
    i = _inputs(T, V, 21, kl)
    z = i["z"].float() + height
    z[:, ::61] += 4.0
    i["z"], i["mask"] = z.to(torch.bfloat16), None
    lp = torch.log_softmax(i["z"].double(), 1).gather(1, i["ids"].long()[:, None])[:, 0]
    i["old"] = lp.float()
    if i["ref_logits"] is not None:
        i["ref_logits"] = (i["z"].float() + 0.4 * torch.randn(z.shape, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)).to(torch.bfloat16)
    error = _run(i).logp.double() - lp
    assert bool((error.abs() <= 4e-6 + 2e-7 * lp.abs()).all())
    assert abs(float(error.sum())) <= 6 * 1e-6 * math.sqrt(T) / 2


@pytest.mark.parametrize("kl", ["exact", "reverse", "k3", None])
@pytest.mark.parametrize("T,V", [(2000, 4096), (1500, 32000), (300, 151936)])
@pytest.mark.parametrize("rest", [0.1, 1e-2, 1e-3, 1e-5])
def test_log_probs_of_likely_tokens(kl, T, V, rest):
    """Rows whose sampled column has nearly all of the probability.  The log-probs' errors have a spread of up to 5e-7 (the largest
    column's exponent, of up to 32, is rounded at 2^-24 of it: 1e-6 / sqrt(3) / 2 and the sums'), of which 6 standard deviations of
    the mean are allowed; in common they have what the exponential's have (ex2.approx: 5e-8 on average) and the sums'
    roundings, 1.5e-7 together."""
    i = _inputs(T, V, 22, kl)
    g = torch.Generator(device=DEV).manual_seed(7)
    z = 2.5 * torch.randn((T, V), generator=g, device=DEV)
    z[torch.arange(T), i["ids"].long()] = torch.logsumexp(z, 1) - math.log(rest) + torch.rand(T, generator=g, device=DEV)
    i["z"], i["mask"] = z.to(torch.bfloat16), None
    lp = torch.cat([torch.log_softmax(part.double(), 1).gather(1, ids.long()[:, None])[:, 0]
                    for part, ids in zip(i["z"].split(100), i["ids"].split(100))])
    i["old"] = lp.float()
    if i["ref_logits"] is not None:
        i["ref_logits"] = (i["z"].float() + 0.4 * torch.randn(z.shape, generator=g, device=DEV)).to(torch.bfloat16)
    error = _run(i).logp.double() - lp
    assert bool((error.abs() <= 4e-6 + 2e-7 * lp.abs()).all())
    assert abs(float(error.mean())) <= 1.5e-7 + 6 * 5e-7 / math.sqrt(T)
