"""A policy trained against a frozen reference, on synthetic hidden states: an 8-bit layer and a bf16 LM head, an
8-bit copy of the head as the rollout engine, and the starting head in 8 bits as the reference.

    python examples/reference_kl.py [--steps 8]

Each policy step samples from the rollout, weights its tokens for the discrepancy between rollout and policy, and takes
the clipped loss with the exact KL to the reference; the second half takes preference steps on the responses' rewards.
Prints one line per step."""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2607_24062_gb300 as acrl  # noqa: E402


def batch(gen, prompts, responses, longest, dev):
    """Offsets of `prompts` prompts with `responses` responses of 1 to `longest` tokens."""
    n = torch.randint(1, longest + 1, (prompts * responses,), generator=gen)
    seq = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)])
    grp = torch.arange(0, prompts * responses + 1, responses, dtype=torch.int32)
    return seq.to(dev), grp.to(dev), n


def train(steps=8, V=4099, K=256, H=384, prompts=8, responses=4, longest=48, kl_beta=0.05, lr=0.2, seed=0):
    """Returns a list of (kind, loss, mean KL to the reference or mean log-ratio of the responses) per step."""
    dev = torch.device("cuda")
    torch.manual_seed(seed)
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, generator=gen).to(dev)  # noqa: E731
    layer_w, head_w = rnd(H, K) * K ** -0.5, rnd(V, H) * H ** -0.5     # fp32; bf16 copies are trained
    seq, grp, n = batch(gen, prompts, responses, longest, dev)
    T, S, Gn, ld = int(n.sum()), prompts * responses, prompts, (V + 7) // 8 * 8
    x = rnd(T, K).bfloat16()
    mask = torch.ones(T, dtype=torch.uint8, device=dev)
    ref = acrl.Fp8Head(head_w.bfloat16())                              # frozen: quantised once
    ref_hidden = acrl.fp8_layer(x, layer_w.bfloat16())
    ref_logits = ref.logits(ref_hidden)
    params = acrl.Params()
    state = acrl.controller_init(params)
    kl_coef = torch.full((T,), kl_beta / T, device=dev)
    preference = acrl.PreferenceStep(T, V, ld, S, Gn, beta=0.1)
    log = []
    for step in range(steps):
        layer, head = (w.bfloat16().requires_grad_() for w in (layer_w, head_w))
        hidden = acrl.fp8_layer(x, layer)
        logits = torch.nn.functional.pad(hidden @ head.t(), (0, ld - V))[:, :V]   # rows that start on 16 bytes
        if step <= steps // 2:                           # a rollout by the current head in 8 bits; the preference steps
            z_mu = acrl.Fp8Head(head.detach()).logits(hidden.detach()).float()   # stay with their first
            ids = torch.distributions.Categorical(logits=z_mu).sample().int()
            logp_mu = torch.log_softmax(z_mu, -1).gather(1, ids.long()[:, None])[:, 0]
            reward = torch.stack([(ids[a:b] % 2 == 0).float().mean() for a, b in zip(seq[:-1], seq[1:])])
        if step < steps // 2:
            old = acrl.token_stats(logits.detach(), ids, mask, V=V)[1]
            w = acrl.importance_weights(state, params, old, logp_mu, mask, reward, seq, grp)
            kl = torch.empty(T, device=dev)
            loss = acrl.policy_loss(logits, ids, mask, w.coef, old_logp=old, kl="exact", kl_coef=kl_coef,
                                    ref_logits=ref_logits, kl_out=kl)
            log.append(("policy", float(loss.detach()), float(kl.mean())))
        else:
            ref_logp = ref.logp(ref_hidden, ids, mask)
            loss = acrl.pairs_loss(preference, logits, ids, mask, ref_logp, reward, seq, grp)
            log.append(("preference", float(loss.detach()), float(preference.ratio.mean())))
        loss.backward()
        with torch.no_grad():
            layer_w -= lr * layer.grad.float()
            head_w -= lr * head.grad.float()
    return log


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=8)
    for kind, loss, other in train(ap.parse_args().steps):
        print(f"{kind:10s}  loss {loss:+.5f}  {'KL' if kind == 'policy' else 'mean log-ratio'} {other:+.5f}")
