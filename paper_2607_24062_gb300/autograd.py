"""The on-policy ACRL loss as a torch.autograd function.

    loss = acrl_loss(step, logits, ids, mask, logp_mu, rewards, seq_offsets, group_offsets)
    loss.backward()      # dL/dlogits flows into whatever produced the logits

The forward runs the whole pass of `AcrlStep` (statistics, discrepancy,
advantages, controller, then the gradient kernel, which writes dL/dlogits in
bf16 while it computes the loss), so the backward needs no second pass over
the logits: it hands back that buffer, or a contiguous copy scaled by the
incoming gradient when that is not 1.  The gradient is the one of Eq. ACRL on the on-policy step
(theta = theta_old, so r = 1), with the importance weights treated as
constants, as the paper's rho is built from theta_old.

The returned gradient is a view of `step.grad`: it stays valid until the same
step object runs again.

The losses with a reference policy work alike: `policy_loss` (the clipped loss
with a KL term) and `pairs_loss` (a PreferenceStep) write dL/dlogits in their
forward.  `fp8_layer` is a linear layer on 8-bit matrices, whose backward makes
both gradients on 8-bit matrices too; `linear_layer` one in bf16 with bias,
activation and residual.
"""

from __future__ import annotations

from typing import Callable

import torch
from torch.autograd.function import once_differentiable

from . import api
from .pipeline import AcrlStep, PreferenceStep


def _scaled(g: torch.Tensor, grad_out: torch.Tensor) -> torch.Tensor:
    """The forward's gradient, or a contiguous copy scaled by the incoming one where that is not 1."""
    if float(grad_out) != 1.0:  # one scalar read; the common loss.backward() passes 1
        if torch.is_grad_enabled() or grad_out.dtype != torch.float32 or grad_out.device != g.device:
            g = g * grad_out.to(g.dtype)  # a graph of the backward itself, or no scalar the kernel reads
        else:
            g = api.scale_grad(g, grad_out, out=torch.empty(g.shape, dtype=g.dtype, device=g.device))
    return g


class _AcrlLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, step, ids, mask, logp_mu, rewards, seq_offsets, group_offsets, exchange):
        step.run(logits, ids, mask, logp_mu, rewards, seq_offsets, group_offsets, exchange=exchange)
        ctx.step = step
        ctx.rows, ctx.cols = logits.shape
        return step.loss.reshape(()).clone()

    @staticmethod
    def backward(ctx, grad_out):
        return _scaled(ctx.step.grad[: ctx.rows, : ctx.cols], grad_out), None, None, None, None, None, None, None, None


def acrl_loss(step: AcrlStep, logits: torch.Tensor, ids, mask, logp_mu, rewards, seq_offsets, group_offsets,
              exchange: Callable[[torch.Tensor], None] | None = None) -> torch.Tensor:
    """The step's scalar loss (fp32, 0-d) with dL/dlogits attached for
    autograd.  `logits` is the bf16 [T, V] tensor `step` was built for (row
    stride `step.ld`); the other arguments are those of `AcrlStep.run`."""
    if logits.shape != (step.T, step.V) or logits.stride(0) != step.ld:
        raise ValueError(f"logits: expected shape ({step.T}, {step.V}) with row stride {step.ld}")
    return _AcrlLoss.apply(logits, step, ids, mask, logp_mu, rewards, seq_offsets, group_offsets, exchange)


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids, mask, coef, kw):
        stream = kw.get("stream")
        if stream is not None:    # the logits and the rest of the graph are the current stream's
            here = torch.cuda.current_stream(stream.device)
            stream.wait_stream(here)
        out = api.policy_loss_grad_logits(logits.detach(), ids, mask, coef, **kw)
        if stream is not None:
            here.wait_stream(stream)
            for t in (out.grad, out.loss):    # of `stream`, and read here
                t.record_stream(here)
        # the very tensor that the backward returns: a leaf takes a gradient that nobody else holds as its .grad, and what is
        # done to that would be done to the next backward's too
        ctx.grad = out.grad[: logits.shape[0], : logits.shape[1]]
        return out.loss.reshape(()).clone()

    @staticmethod
    def backward(ctx, grad_out):
        return _scaled(ctx.grad, grad_out), None, None, None, None


def policy_loss(logits: torch.Tensor, ids, mask, coef, **kw) -> torch.Tensor:
    """The scalar loss of policy_loss_grad_logits (same arguments; fp32, 0-d) with dL/dlogits attached for autograd.
    `logits` is bf16 [T, V] with a row stride that is a multiple of eight; outputs given by keyword (logp, kl_out,
    token_loss) are filled.  With `stream` the kernels run there, after what the current stream holds and before what it gets
    next."""
    if kw.get("V") not in (None, logits.shape[1]):
        raise ValueError("logits: pass the view [T, V] itself")
    kw["V"] = logits.shape[1]
    return _PolicyLoss.apply(logits, ids, mask, coef, kw)


class _PairsLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, step, ids, mask, ref_logp, rewards, seq_offsets, group_offsets):
        step.run(logits.detach(), ids, mask, ref_logp, rewards, seq_offsets, group_offsets)
        ctx.step, ctx.shape = step, logits.shape
        return step.loss.reshape(()).clone()

    @staticmethod
    def backward(ctx, grad_out):
        g = _scaled(ctx.step.grad[: ctx.shape[0], : ctx.shape[1]], grad_out)
        return g, None, None, None, None, None, None, None


def pairs_loss(step: PreferenceStep, logits: torch.Tensor, ids, mask, ref_logp, rewards, seq_offsets,
               group_offsets) -> torch.Tensor:
    """A PreferenceStep's scalar loss (fp32, 0-d) with dL/dlogits attached for autograd; as acrl_loss, the gradient is a
    view of `step.grad`."""
    if logits.shape != (step.T, step.V) or logits.stride(0) != step.ld:
        raise ValueError(f"logits: expected shape ({step.T}, {step.V}) with row stride {step.ld}")
    return _PairsLoss.apply(logits, step, ids, mask, ref_logp, rewards, seq_offsets, group_offsets)


def _rows_of_eight(x: torch.Tensor) -> torch.Tensor:
    """x, or a copy of it whose rows start on 16 bytes."""
    if x.stride(1) == 1 and x.stride(0) % 8 == 0 and x.stride(0) >= x.shape[1] and x.data_ptr() % 16 == 0:
        return x
    pad = torch.empty((x.shape[0], (x.shape[1] + 7) // 8 * 8), dtype=x.dtype, device=x.device)[:, : x.shape[1]]
    return pad.copy_(x)


class _Fp8Layer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, grad_fmt):
        w = _rows_of_eight(weight.detach())
        x = _rows_of_eight(x.detach())
        y = api.fp8_linear(x, api.fp8_quantize(w, block="tile"))
        ctx.save_for_backward(x, w)
        ctx.grad_fmt = grad_fmt
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        dx, dw = api.fp8_linear_backward(_rows_of_eight(dy), x, api.fp8_quantize(w, block="tile", transpose=True),
                                         fmt=ctx.grad_fmt, dw_dtype=torch.float32)
        return dx, dw.to(w.dtype), None


def fp8_layer(x: torch.Tensor, weight: torch.Tensor, grad_fmt: str = "e4m3") -> torch.Tensor:
    """x [M, K] times the transpose of weight [N, K] (both bf16), computed on 8-bit matrices; the backward's two products
    are on 8-bit matrices as well, the incoming gradient in `grad_fmt`.  They have no derivative of their own."""
    return _Fp8Layer.apply(x, weight, grad_fmt)


class _LinearLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act):
        w, x = _rows_of_eight(weight.detach()), _rows_of_eight(x.detach())
        pre = None
        if act is not None and any(ctx.needs_input_grad[:3]):
            pre = api._padded((x.shape[0], w.shape[0]), 8, torch.bfloat16, x.device)
        r = None if residual is None else _rows_of_eight(residual.detach())
        y = api.linear(x, w, None if bias is None else bias.detach().contiguous(), act=act, residual=r, pre_out=pre)
        ctx.save_for_backward(x, w, pre)
        ctx.act = act
        ctx.bias_dtype = None if bias is None else bias.dtype
        ctx.residual_dtype = None if residual is None else residual.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w, pre = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dw = dbias = None
        if any(need[:3]):
            dx, dw, dbias = api.linear_backward(_rows_of_eight(dy), x, w, act=ctx.act, pre=pre, bias=need[2], need_dx=need[0],
                                                need_dw=need[1], dw_dtype=torch.bfloat16)
        return dx, dw, None if dbias is None else dbias.to(ctx.bias_dtype), dy.to(ctx.residual_dtype) if need[3] else None, None


def linear_layer(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, act: str | None = None,
                 residual: torch.Tensor | None = None) -> torch.Tensor:
    """act(x W^T + bias) + residual for autograd: x [M, K] and weight [N, K] bf16, bias [N] and residual [M, N] bf16 or
    float32; bf16 [M, N].  With an activation the pre-activation is kept in bf16 for the backward.  The gradients have no
    derivative of their own.  To capture a backward into a graph, run it once before on another stream, and
    keep no eager result of the same leaves alive meanwhile: torch would join that result's stream to the capture, and end the
    process."""
    return _LinearLayer.apply(x, weight, bias, residual, act)
