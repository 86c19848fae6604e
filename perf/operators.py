"""The operators around a reference policy, as they are timed: 8-bit matrices with a scale for each block of 128 and
their products, the clipped policy loss with a KL term, and the preference loss over the responses of a prompt.

`kind` of a case:

  quantize     fp8_quantize: a matrix to 8-bit floating point, one scale per row and 128 columns ("row") or per
               128 x 128 ("tile"), of the matrix or of its transpose;
  linear       fp8_linear: activations quantised in the call, times a weight quantised beforehand (tiles);
  linear_grad  fp8_linear_backward: the gradients of that product with respect to both operands;
  policy       policy_loss_grad_logits: log-probs, the clipped loss, its KL term and dL/dlogits in one call; `kl` is
               "exact" / "reverse" (over the vocabulary, against the reference's logits) or "k1" / "k2" / "k3" (from
               the reference's log-probs of the sampled tokens);
  preference   PreferenceStep.run: statistics of the logits, the pairs of each prompt, loss and dL/dlogits; with
               V = 0 preference_loss alone, from log-probs.

Sizes are those of the repository's workloads (4 x 256 tokens at V = 4,096; V = 32,000 and 20,011; 64 x 8 responses of
up to 2,048 tokens; V = 151,936 with a hidden size of 4,096 or 2,048) and generic ones between them.  Lengths, masks
and rewards follow from the case alone; every other value is drawn from the seed."""

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
FORMATS = {"e4m3": (torch.float8_e4m3fn, 448.0, 3, -6), "e5m2": (torch.float8_e5m2, 57344.0, 2, -14)}
MOST_ELEMS = 622_000_000     # elements of the largest matrix or batch of logits
MOST_FLOPS = 5.0e12          # of a drawn product
CLIP_LOW, CLIP_HIGH, DUAL = 0.2, 0.28, 3.0
BETA = 0.1


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------

def _quantize(R, C, **more):
    return {"kind": "quantize", "R": R, "C": C, "block": "row", "fmt": "e4m3", "transpose": False, "dtype": "bf16", **more}


def _policy(prompts, group, lo, hi, V, kl, **more):
    return {"kind": "policy", "prompts": prompts, "group": group, "lo": lo, "hi": hi, "V": V, "kl": kl, "old": True,
            "pad": 0, **more}


def _preference(prompts, group, lo, hi, V, **more):
    return {"kind": "preference", "prompts": prompts, "group": group, "lo": lo, "hi": hi, "V": V, "form": "sigmoid",
            "mean": False, "smooth": 0.0, "ref": True, "pad": 0, **more}


def listed():
    return [
        # the activations of a micro-batch of 4,096 tokens, before a linear layer
        dict(_quantize(4096, 4096), name="quantize_activations"),
        # the LM-head weight of a large-vocabulary model, as it is loaded or after an optimiser step
        dict(_quantize(151936, 4096, block="tile"), name="quantize_head"),
        # an odd number of token gradients, transposed for the weight-gradient product, with the wider exponent
        dict(_quantize(5003, 2056, transpose=True, fmt="e5m2"), name="quantize_grad_t"),
        # one token through a square layer: latency
        {"kind": "linear", "M": 1, "K": 4096, "N": 4096, "name": "linear_token"},
        # scoring a handful of tokens with a large-vocabulary head: the weight's bytes
        {"kind": "linear", "M": 48, "K": 4096, "N": 151936, "name": "linear_decode"},
        # the reference logits of a micro-batch of 4,096 tokens
        {"kind": "linear", "M": 4096, "K": 4096, "N": 151936, "name": "linear_large"},
        # a layer's backward pass at ragged sizes: both gradients
        {"kind": "linear_grad", "M": 2507, "K": 2048, "N": 8200, "fmt": "e4m3", "name": "linear_grad_ragged"},
        # the smallest batch: four responses of 256 tokens, a small vocabulary, KL over the vocabulary
        dict(_policy(4, 1, 256, 256, 4096, "exact"), name="policy_tiny"),
        # a micro-batch at a large vocabulary, KL over the vocabulary against the reference's logits
        dict(_policy(2, 4, 256, 700, 151936, "exact"), name="policy_exact_large"),
        # the same vocabulary, KL estimated from the reference's log-probs of the sampled tokens, padded responses
        dict(_policy(2, 8, 64, 400, 151936, "k3", pad=16), name="policy_sampled"),
        # pairs from cached log-probs alone: 64 prompts x 8 responses of up to 2,048 tokens
        dict(_preference(64, 8, 1, 2048, 0), name="preference_tokens"),
        # the whole preference step on chosen and rejected answers at a large vocabulary
        dict(_preference(8, 2, 64, 384, 151936), name="preference_step"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _some_rows(rng, V, most):
    rows = _log_int(rng, 1, max(1, min(most, 400_000_000 // max(V, 1))))
    group = rng.choice([2, 4, 8])
    prompts = _log_int(rng, 1, max(1, min(64, rows // (4 * group))))
    hi = max(1, rows // (prompts * group))
    return prompts, group, rng.randint(max(1, hi // 8), hi), hi, rng.choice([0, 0, 16]) if hi >= 64 else 0


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "linear_grad", "policy", "policy", "preference"])
    if kind == "quantize":
        R = _log_int(rng, 1, 151936)
        return _quantize(R, _log_int(rng, 64, max(64, min(16384, MOST_ELEMS // R))), block=rng.choice(["row", "tile"]),
                         fmt=rng.choice(["e4m3", "e5m2"]), transpose=rng.choice([False, True]),
                         dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "linear":
        K, N = 8 * _log_int(rng, 64, 1024), _log_int(rng, 512, 151936)
        N = min(N, MOST_ELEMS // K)
        return {"kind": kind, "M": _log_int(rng, 1, max(1, min(8192, int(MOST_FLOPS / (2 * K * N))))), "K": K, "N": N}
    if kind == "linear_grad":
        return {"kind": kind, "M": _log_int(rng, 64, 4096), "K": 8 * _log_int(rng, 64, 512), "N": 8 * _log_int(rng, 64, 2048),
                "fmt": rng.choice(["e4m3", "e5m2"])}
    V = _log_int(rng, 2048, 151936)
    if rng.random() < 0.5:
        V = V // 8 * 8
    if kind == "policy":
        prompts, group, lo, hi, pad = _some_rows(rng, V, 4096)
        return _policy(prompts, group, lo, hi, V, rng.choice(["exact", "exact", "reverse", "k1", "k2", "k3"]), pad=pad,
                       old=rng.random() < 0.7)
    V = rng.choice([0, V])
    prompts, group, lo, hi, pad = _some_rows(rng, V, 4096 if V else 400_000)
    return _preference(prompts, group, lo, hi, V, pad=pad, form=rng.choice(["sigmoid", "sigmoid", "hinge", "ipo"]),
                       mean=rng.random() < 0.3, smooth=rng.choice([0.0, 0.1]), ref=rng.random() < 0.8)


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _matrix(R, C, gen, dtype=torch.bfloat16, std=1.0):
    """Activations, weights or gradients: normal values whose rows differ in size, a few columns (outliers) larger."""
    ld = (C + 7) // 8 * 8
    x = torch.empty((R, ld), device=DEV).normal_(0.0, std, generator=gen)
    x.mul_(torch.exp(0.5 * torch.randn((R, 1), generator=gen, device=DEV)))
    x[:, :: 97].mul_(8.0)
    x = x.to(dtype)
    x[:, C:] = 0
    return x[:, :C]


def _structure(case):
    """Row offsets, mask and rewards of a batch of responses: from the case alone."""
    rng = random.Random("%(prompts)s %(group)s %(lo)s %(hi)s" % case)
    S, pad = case["prompts"] * case["group"], case["pad"] or 1
    n = [rng.randint(case["lo"], case["hi"]) for _ in range(S)]
    rows = [(k + pad - 1) // pad * pad for k in n]
    off = [0]
    for r in rows:
        off.append(off[-1] + r)
    T = off[-1]
    seq = torch.tensor(off, dtype=torch.int64, device=DEV)
    length = torch.tensor(n, dtype=torch.int64, device=DEV)
    row = torch.arange(T, device=DEV)
    resp = torch.searchsorted(seq, row, right=True) - 1
    mask = (row - seq[resp] < length[resp]).to(torch.uint8)
    grp = torch.arange(0, S + 1, case["group"], dtype=torch.int32, device=DEV)
    rewards = torch.tensor([float(rng.random() < 0.4) for _ in range(S)], device=DEV)
    rewards[:: case["group"]] = 1.0      # a prompt's first answer is a good one, and its second is not
    rewards[1:: case["group"]] = 0.0
    return SimpleNamespace(T=T, S=S, G=case["prompts"], seq=seq, grp=grp, resp=resp, mask=mask, rewards=rewards,
                           length=length)


def _rows_of(case):
    """T and the valid rows of a batch, without a GPU."""
    rng = random.Random("%(prompts)s %(group)s %(lo)s %(hi)s" % case)
    pad = case["pad"] or 1
    n = [rng.randint(case["lo"], case["hi"]) for _ in range(case["prompts"] * case["group"])]
    return sum((k + pad - 1) // pad * pad for k in n), sum(n)


def _logits(T, V, gen):
    ld = (V + 7) // 8 * 8
    z = torch.empty((T, ld), device=DEV).normal_(0.0, 2.0, generator=gen)
    z[:, :: 61].add_(4.0)
    z = z.to(torch.bfloat16)
    z[:, V:] = 0
    return z


def _sampled(z, V, gen):
    """Token ids drawn from softmax(z), and their log-probs."""
    x = z[:, :V].float()
    lse = x.max(1, keepdim=True).values
    lse = lse + torch.log(torch.exp(x - lse).sum(1, keepdim=True))
    noise = torch.empty_like(x).exponential_(generator=gen).log_()
    ids = (x - noise).argmax(1)
    return ids.to(torch.int32), x.gather(1, ids[:, None])[:, 0] - lse[:, 0]


def prepare(case, seed):
    kind, gen = case["kind"], _gen(seed)
    s = SimpleNamespace(case=case, kind=kind)
    if kind == "quantize":
        s.x = _matrix(case["R"], case["C"], gen, torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        return s
    if kind in ("linear", "linear_grad"):
        M, K, N = case["M"], case["K"], case["N"]
        s.x = _matrix(M, K, gen)
        w = _matrix(N, K, gen, std=0.02)
        q, scale = _plain_quantize(w, "tile", "e4m3", False)
        if kind == "linear":
            s.w, s.w_scale = q, scale
            s.out = torch.empty((M, (N + 7) // 8 * 8), dtype=torch.bfloat16, device=DEV)
        else:   # the transposed weight, laid out with the weight itself
            s.wt, s.wt_scale = _padded(q.view(torch.uint8).t(), 16).view(q.dtype), scale.t().contiguous()
            s.dy = _matrix(M, N, gen, std=1e-3)
        return s
    b = _structure(case)
    s.b, T, V = b, b.T, case["V"]
    if kind == "preference" and V == 0:
        s.logp = -torch.empty(T, device=DEV).exponential_(1.0, generator=gen)
        s.ref = s.logp + 0.2 * torch.randn(T, generator=gen, device=DEV) if case["ref"] else None
        return s
    s.z = _logits(T, V, gen)
    s.ids, logp = _sampled(s.z, V, gen)
    s.grad = torch.zeros_like(s.z)
    if kind == "preference":
        s.ref = logp + 0.2 * torch.randn(T, generator=gen, device=DEV) if case["ref"] else None
        return s
    adv = torch.randn(b.S, generator=gen, device=DEV)
    n = b.length[b.resp].float()
    w = torch.exp(0.3 * torch.randn(T, generator=gen, device=DEV)).clamp(max=3.0)
    s.coef = b.mask * adv[b.resp] * w / (b.S * n)
    s.kl_coef = 0.05 * b.mask / (b.S * n)
    s.old = logp + 0.1 * torch.randn(T, generator=gen, device=DEV) if case["old"] else None
    s.r = s.ref = None
    if case["kl"] in ("exact", "reverse"):
        s.r = (s.z.float() + torch.empty(s.z.shape, device=DEV).normal_(0.0, 0.4, generator=gen)).to(torch.bfloat16)
        s.r[:, V:] = 0
    else:
        s.ref = logp + 0.3 * torch.randn(T, generator=gen, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------

def _padded(x, to):
    """x with its rows at a stride that is a multiple of `to`."""
    ld = (x.shape[1] + to - 1) // to * to
    p = torch.zeros((x.shape[0], ld), dtype=x.dtype, device=x.device)
    p[:, : x.shape[1]] = x
    return p[:, : x.shape[1]]


def _power(e):
    """2^e in 32 bits, e a tensor of whole numbers from -127 to 127."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22)).view(torch.float32)


def _plain_quantize(x, block, fmt, transpose):
    """q in the 8-bit format (as such a tensor) and the scales' biased exponents (uint8)."""
    dtype, top, _, _ = FORMATS[fmt]
    x = x.float()
    if transpose:
        x = x.t()
    R, C = x.shape
    high = 128 if block == "tile" else 1
    KB, RB = (C + 127) // 128, (R + high - 1) // high
    p = torch.zeros((RB * high, KB * 128), device=x.device)
    p[:R, :C] = x
    p = p.view(RB, high, KB, 128)
    a = p.abs().amax((1, 3))
    m, e = torch.frexp(a)                                     # a = m 2^e, 1/2 <= m < 1; the format's largest is 7/8 of a power of two
    e = e - round(math.log2(top / 0.875)) + (m > 0.875).int()
    e = torch.where(a > 0, e, torch.zeros_like(e)).clamp(-127, 127)
    q = (p * _power(-e)[:, None, :, None]).reshape(RB * high, KB * 128)[:R, :C].to(dtype)
    return _padded(q.view(torch.uint8), 16).view(dtype), (e + 127).to(torch.uint8)


def _plain_values(q, scale):
    """The values that q and its scales stand for, in 32 bits."""
    R, C = q.shape
    s = _power(scale.to(torch.int32) - 127)
    if scale.shape[0] != R:
        s = s.repeat_interleave(128, 0)[:R]
    return q.float() * s.repeat_interleave(128, 1)[:, :C]


def _plain_logprobs(z):
    x = z.float()
    x = x - x.max(1, keepdim=True).values
    return x - torch.log(torch.exp(x).sum(1, keepdim=True))


def _plain_policy(s):
    case, b, V = s.case, s.b, s.case["V"]
    valid = b.mask.bool()
    lp = _plain_logprobs(s.z[:, :V])
    ids = s.ids.long()[:, None]
    logp = lp.gather(1, ids)[:, 0]
    c = s.coef
    r = torch.ones_like(logp) if s.old is None else torch.exp(logp - s.old)
    up = torch.clamp(r, max=1 + CLIP_HIGH)
    down = torch.clamp(torch.clamp(r, min=1 - CLIP_LOW), max=DUAL)
    loss = -c * torch.where(c >= 0, up, down)
    live = torch.where(c >= 0, r <= 1 + CLIP_HIGH, (r >= 1 - CLIP_LOW) & (r <= DUAL))
    toward = torch.where(live, c * r, torch.zeros_like(c))     # -dL/dlogp of the clipped term
    k, p = s.kl_coef, torch.exp(lp)
    if s.r is not None:
        a = lp - _plain_logprobs(s.r[:, :V])                   # log p - log q
        if case["kl"] == "exact":
            kl = (p * (a + torch.expm1(-a))).sum(1)            # the terms' sum is that of p a, and none is negative
            over = p * (a - kl[:, None])
        else:
            q = torch.exp(lp - a)
            kl = (q * (torch.expm1(a) - a)).sum(1)
            over = p - q
    else:
        d = logp - s.ref
        if case["kl"] == "k1":
            kl, slope = d, torch.ones_like(d)
        elif case["kl"] == "k2":
            kl, slope = 0.5 * d * d, d
        else:
            kl, slope = torch.expm1(-d) + d, -torch.expm1(-d)
        toward, over = toward - k * slope, None
    grad = toward[:, None] * p
    if over is not None:
        grad += k[:, None] * over
    grad.scatter_add_(1, ids, -toward[:, None])
    zero = torch.zeros_like(logp)
    grad = torch.where(valid[:, None], grad, torch.zeros((), device=grad.device)).to(torch.bfloat16)
    loss = torch.where(valid, loss + k * kl, zero)
    return {"grad": grad, "logp": torch.where(valid, logp, zero), "kl": torch.where(valid, kl, zero), "token_loss": loss,
            "loss": loss.sum().reshape(1)}


def _plain_pairs(s, logp):
    """loss, -dL/dlogp per token and the responses' log ratios."""
    case, b, G = s.case, s.b, s.case["group"]
    d = logp if s.ref is None else logp - s.ref
    valid = b.mask.bool()
    # sums of a hundred or more terms: in 64 bits, rounded once
    D = torch.zeros(b.S, dtype=torch.float64, device=DEV).index_add_(0, b.resp, torch.where(valid, d, torch.zeros_like(d)).double())
    n = b.length.double()
    if case["mean"]:
        D = D / n
    D = D.float()
    h = BETA * (D.view(-1, G, 1) - D.view(-1, 1, G))
    R = b.rewards.view(-1, G)
    pair = R[:, :, None] > R[:, None, :]
    e = case["smooth"]
    soft = torch.log1p(torch.exp(-h.abs()))
    if case["form"] == "sigmoid":
        each = (1 - e) * (soft + torch.relu(-h)) + e * (soft + torch.relu(h))
        slope = -(1 - e) * torch.sigmoid(-h) + e * torch.sigmoid(h)
    elif case["form"] == "hinge":
        each, slope = torch.relu(1 - h), -(h < 1).float()
    else:
        each, slope = ((h - 0.5) / BETA) ** 2, 2 * (h - 0.5) / BETA ** 2
    count = pair.sum((1, 2)).float()
    some = count > 0
    Q = some.sum().clamp(min=1).float()
    weight = torch.where(some, 1 / (count.clamp(min=1) * Q), torch.zeros_like(count))[:, None, None] * pair
    loss = (weight * each).sum()
    slope = weight * slope
    g = (BETA * (slope.sum(2) - slope.sum(1))).reshape(-1)     # dL/dD
    if case["mean"]:
        g = g / b.length.float()
    return loss.reshape(1), torch.where(valid, -g[b.resp], torch.zeros_like(d)), D


def _plain_preference(s):
    if s.case["V"] == 0:
        loss, coef, D = _plain_pairs(s, s.logp)
        return {"loss": loss, "coef": coef, "ratio": D}
    lp = _plain_logprobs(s.z[:, : s.case["V"]])
    ids = s.ids.long()[:, None]
    logp = torch.where(s.b.mask.bool(), lp.gather(1, ids)[:, 0], torch.zeros_like(lp[:, 0]))
    loss, coef, D = _plain_pairs(s, logp)
    grad = coef[:, None] * torch.exp(lp)
    grad.scatter_add_(1, ids, -coef[:, None])
    return {"loss": loss, "coef": coef, "ratio": D, "logp": logp, "grad": grad.to(torch.bfloat16)}


def _plain(s):
    case = s.case
    if s.kind == "quantize":
        q, scale = _plain_quantize(s.x, case["block"], case["fmt"], case["transpose"])
        return {"q": q, "scale": scale.view(torch.float8_e8m0fnu)}
    if s.kind == "linear":
        x = _plain_values(*_plain_quantize(s.x, "row", "e4m3", False))
        return {"out": (x @ _plain_values(s.w, s.w_scale).t()).to(torch.bfloat16)}
    if s.kind == "linear_grad":
        dy = _plain_values(*_plain_quantize(s.dy, "row", case["fmt"], False))
        dyt = _plain_values(*_plain_quantize(s.dy, "row", case["fmt"], True))
        xt = _plain_values(*_plain_quantize(s.x, "row", "e4m3", True))
        return {"dx": (dy @ _plain_values(s.wt, s.wt_scale).t()).to(torch.bfloat16), "dw": dyt @ xt.t()}
    return _plain_policy(s) if s.kind == "policy" else _plain_preference(s)


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def _framework(s):
    import paper_2607_24062_gb300 as acrl

    case = s.case
    if s.kind == "quantize":
        t = acrl.fp8_quantize(s.x, block=case["block"], fmt=case["fmt"], transpose=case["transpose"])
        return {"q": t.q, "scale": t.scale.view(torch.float8_e8m0fnu)}
    if s.kind == "linear":
        return {"out": acrl.fp8_linear(s.x, acrl.Fp8Tensor(s.w, s.w_scale), out=s.out)}
    if s.kind == "linear_grad":
        dx, dw = acrl.fp8_linear_backward(s.dy, s.x, acrl.Fp8Tensor(s.wt, s.wt_scale), fmt=case["fmt"],
                                          dw_dtype=torch.float32)
        return {"dx": dx, "dw": dw}
    b, V = s.b, case["V"]
    if s.kind == "policy":
        o = acrl.policy_loss_grad_logits(s.z, s.ids, b.mask, s.coef, V=V, old_logp=s.old, clip_low=CLIP_LOW,
                                         clip_high=CLIP_HIGH, dual_clip=DUAL, kl=case["kl"], kl_coef=s.kl_coef,
                                         ref_logits=s.r, ref_logp=s.ref, grad=s.grad)
        return {"grad": o.grad[:, :V], "logp": o.logp, "kl": o.kl, "token_loss": o.token_loss, "loss": o.loss}
    how = dict(beta=BETA, form=case["form"], label_smoothing=case["smooth"], length_norm=case["mean"])
    if V == 0:
        o = acrl.preference_loss(s.logp, s.ref, b.mask, b.rewards, b.seq, b.grp, **how)
        return {"loss": o.loss, "coef": o.coef, "ratio": o.ratio}
    step = getattr(s, "step", None)
    if step is None:                                            # a training program keeps it from step to step
        step = s.step = acrl.PreferenceStep(b.T, V, s.z.shape[1], b.S, b.G, device=DEV, grad=s.grad, **how)
    step.run(s.z, s.ids, b.mask, s.ref, b.rewards, b.seq, b.grp)
    return {"loss": step.loss, "coef": step.coef, "ratio": step.ratio, "logp": step.logp, "grad": step.grad[:, :V]}


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------
# work
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    blocks = lambda n: (n + 127) // 128   # noqa: E731
    if kind == "quantize":
        R, C = (case["C"], case["R"]) if case["transpose"] else (case["R"], case["C"])
        scales = (blocks(R) if case["block"] == "tile" else R) * blocks(C)
        return {"bytes": R * C * ((2 if case["dtype"] == "bf16" else 4) + 1) + scales, "flops": 2 * R * C}
    if kind in ("linear", "linear_grad"):
        M, K, N = case["M"], case["K"], case["N"]
        w = N * K + blocks(N) * blocks(K)
        if kind == "linear":
            return {"bytes": 2 * M * K + w + 2 * M * N, "flops": 2 * M * N * K}
        return {"bytes": 2 * M * N + 2 * M * K + w + 2 * M * K + 4 * N * K, "flops": 4 * M * N * K}
    T, n = _rows_of(case)
    V = case["V"]
    if kind == "policy":
        full = case["kl"] in ("exact", "reverse")
        return {"bytes": n * V * (4 if full else 2) + 2 * T * V + T * 33, "flops": n * V * (12 if full else 6)}
    if V == 0:
        return {"bytes": T * 13, "flops": 4 * T}
    # the logits are needed before the pairs are known and again after: twice where they do not fit the second-level cache
    return {"bytes": n * V * (2 if 2 * n * V < 100_000_000 else 4) + 2 * T * V + T * 25, "flops": n * V * 6}


# ---------------------------------------------------------------------------------------------------------------
# 64 bits, from the definitions
# ---------------------------------------------------------------------------------------------------------------

def _exact_power(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_quantize(x, block, fmt):
    """Values of q and of the scales of a float64 matrix."""
    _, top, bits, low = FORMATS[fmt]
    R, C = x.shape
    tall = 128 if block == "tile" else 1
    full = torch.nn.functional.pad(x.abs(), (0, -C % 128, 0, -R % tall))
    a = full.unflatten(0, (-1, tall)).unflatten(2, (-1, 128)).amax(3).amax(1)
    # the smallest power of two whose product with `top` reaches a: from a guess, corrected by comparison
    guess = torch.floor(torch.log2(torch.where(a > 0, a / top, torch.ones_like(a))))
    scale = _exact_power(guess - 1)
    scale = torch.where(scale * top < a, 2 * scale, scale)
    scale = torch.where(scale * top < a, 2 * scale, scale)
    scale = torch.where(scale * top < a, 2 * scale, scale)
    scale = torch.where(a > 0, scale, torch.ones_like(a)).clamp(min=2.0 ** -127)
    each = scale.repeat_interleave(tall, 0)[:R].repeat_interleave(128, 1)[:, :C]
    y = x / each
    at = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** low))).clamp(min=low)
    step = _exact_power(at - bits)
    return torch.round(y / step) * step, scale, each


def _exact_policy(case, s):
    b, V = s.b, case["V"]
    rows = max(1, (1 << 27) // V)
    outs = []
    for i in range(0, b.T, rows):
        z = s.z[i: i + rows, :V].double()
        lp = z - torch.logsumexp(z, 1, keepdim=True)
        p, ids = lp.exp(), s.ids[i: i + rows].long()[:, None]
        logp = lp.gather(1, ids)[:, 0]
        c, k = s.coef[i: i + rows].double(), s.kl_coef[i: i + rows].double()
        ratio = torch.ones_like(logp) if s.old is None else (logp - s.old[i: i + rows].double()).exp()
        # minus the surrogate objective as a function of log p, and its derivative piece by piece
        value = torch.where(c >= 0, torch.minimum(ratio, torch.full_like(ratio, 1 + CLIP_HIGH)),
                            ratio.clamp(1 - CLIP_LOW, DUAL))
        flat = torch.where(c >= 0, ratio > 1 + CLIP_HIGH, (ratio < 1 - CLIP_LOW) | (ratio > DUAL))
        slope = torch.where(flat, torch.zeros_like(c), -c * ratio)
        g = torch.zeros_like(p)
        if s.r is not None:
            x = s.r[i: i + rows, :V].double()
            lq = x - torch.logsumexp(x, 1, keepdim=True)
            if case["kl"] == "exact":
                kl = (p * (lp - lq)).sum(1)
                g += k[:, None] * p * (lp - lq - kl[:, None])
            else:
                kl = (lq.exp() * (lq - lp)).sum(1)
                g += k[:, None] * (p - lq.exp())
        else:
            d = logp - s.ref[i: i + rows].double()
            kl = {"k1": d, "k2": d ** 2 / 2, "k3": (-d).exp() - 1 + d}[case["kl"]]
            slope = slope + k * {"k1": torch.ones_like(d), "k2": d, "k3": 1 - (-d).exp()}[case["kl"]]
        g -= slope[:, None] * p
        g.scatter_add_(1, ids, slope[:, None])
        m = b.mask[i: i + rows].double()
        outs.append((g * m[:, None], logp * m, kl * m, (-c * value + k * kl) * m))
    grad, logp, kl, loss = (torch.cat(o) for o in zip(*outs))
    return {"grad": grad, "logp": logp, "kl": kl, "token_loss": loss, "loss": loss.sum().reshape(1)}


def _exact_pairs(case, b, logp, ref, rewards):
    d = logp if ref is None else logp - ref.double()
    off, mask, R = b.seq.tolist(), b.mask.bool(), rewards.tolist()
    D, n = [], []
    for i in range(b.S):
        part = d[off[i]: off[i + 1]][mask[off[i]: off[i + 1]]]
        n.append(part.numel())
        D.append(float(part.sum()) / (n[-1] if case["mean"] else 1))
    G, e, total, g = case["group"], case["smooth"], 0.0, [0.0] * b.S
    found = [[(i, j) for i in range(q, q + G) for j in range(q, q + G) if R[i] > R[j]] for q in range(0, b.S, G)]
    Q = sum(bool(f) for f in found)
    soft = lambda v: max(v, 0.0) + math.log1p(math.exp(-abs(v)))   # noqa: E731
    sig = lambda v: 1 / (1 + math.exp(-v)) if v >= 0 else math.exp(v) / (1 + math.exp(v))   # noqa: E731
    for f in found:
        for i, j in f:
            h = BETA * (D[i] - D[j])
            if case["form"] == "sigmoid":
                each, slope = (1 - e) * soft(-h) + e * soft(h), -(1 - e) * sig(-h) + e * sig(h)
            elif case["form"] == "hinge":
                each, slope = max(0.0, 1 - h), -1.0 if h < 1 else 0.0
            else:
                each, slope = (h / BETA - 1 / (2 * BETA)) ** 2, 2 * (h / BETA - 1 / (2 * BETA)) / BETA
            total += each / (len(f) * Q)
            g[i] += BETA * slope / (len(f) * Q)
            g[j] -= BETA * slope / (len(f) * Q)
    per = torch.tensor([-x / (k if case["mean"] else 1) for x, k in zip(g, n)], dtype=torch.float64, device=DEV)
    coef = per[b.resp] * b.mask
    return torch.tensor([total], dtype=torch.float64), coef, torch.tensor(D, dtype=torch.float64)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "quantize":
        x = s.x.double()
        q, scale, _ = _exact_quantize(x.t() if case["transpose"] else x, case["block"], case["fmt"])
        return {"q": q, "scale": scale}
    if kind == "linear":
        if 2.0 * case["M"] * case["N"] * case["K"] > 6e12:
            return None
        q, _, each = _exact_quantize(s.x.double(), "row", "e4m3")
        scale = _exact_power(s.w_scale.int() - 127).repeat_interleave(128, 0)[: case["N"]]
        w = s.w.double() * scale.repeat_interleave(128, 1)[:, : case["K"]]
        return {"out": (q * each) @ w.t()}
    if kind == "linear_grad":
        fmt, N = case["fmt"], case["N"]
        q, _, each = _exact_quantize(s.dy.double(), "row", fmt)
        qt, _, eacht = _exact_quantize(s.dy.double().t().contiguous(), "row", fmt)
        xt, _, eachx = _exact_quantize(s.x.double().t().contiguous(), "row", "e4m3")
        scale = _exact_power(s.wt_scale.int() - 127).repeat_interleave(128, 0)[: case["K"]]
        wt = s.wt.double() * scale.repeat_interleave(128, 1)[:, :N]
        return {"dx": (q * each) @ wt.t(), "dw": (qt * eacht) @ (xt * eachx).t()}
    if kind == "policy":
        return _exact_policy(case, s)
    b, V = s.b, case["V"]
    if V == 0:
        loss, coef, D = _exact_pairs(case, b, s.logp.double(), s.ref, b.rewards)
        return {"loss": loss, "coef": coef, "ratio": D}
    rows = max(1, (1 << 27) // V)
    ids = s.ids.long()[:, None]
    lse = torch.cat([torch.logsumexp(s.z[i: i + rows, :V].double(), 1) for i in range(0, b.T, rows)])
    logp = (s.z[:, :V].gather(1, ids)[:, 0].double() - lse) * b.mask
    loss, coef, D = _exact_pairs(case, b, logp, s.ref, b.rewards)
    grad = torch.empty((b.T, V), dtype=torch.float64, device=DEV)
    for i in range(0, b.T, rows):
        g = coef[i: i + rows, None] * (s.z[i: i + rows, :V].double() - lse[i: i + rows, None]).exp()
        grad[i: i + rows] = g.scatter_add_(1, ids[i: i + rows], -coef[i: i + rows, None])
    return {"loss": loss, "coef": coef, "ratio": D, "logp": logp, "grad": grad}
