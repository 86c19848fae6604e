"""Python binding of the ACRL C ABI: one function per entry point, same names
without the `acrl_` prefix.  Arguments are torch tensors on the current CUDA
device; this layer only checks dtypes/shapes, passes raw pointers and the
current stream, allocates outputs the caller did not provide, and turns a
non-OK status into an exception.  Every step of the computation runs in the
library's kernels."""

from __future__ import annotations

import ctypes
import functools
from dataclasses import dataclass

import numpy as np
import torch

from . import _abi
from ._abi import BATCH_DTYPE, GRP_DTYPE, SEQ_DTYPE, STATE_DTYPE, AcrlError, Params, check, lib  # noqa: F401


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def _one_device(tensors) -> torch.device:
    """The GPU every buffer of one call lives on (they must agree)."""
    first, index = None, -1
    for t in tensors:
        if t is None:
            continue
        at = t.get_device()    # the index alone: comparing torch.device objects costs a short call several microseconds
        if first is None:
            first, index = t, at
        elif at != index or (at < 0 and t.device != first.device):
            raise AcrlError(f"buffers on {first.device} and {t.device}: every buffer of a call must be on one GPU")
    if first is None or index < 0 or not first.is_cuda:
        raise AcrlError("expected CUDA tensors")
    return first.device


_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_ENTRY = {}    # the library's functions by name, as looked up


def _call(name: str, tensors, stream, *args) -> None:
    """Call entry point `name` with `args` followed by the stream, on the GPU
    that holds `tensors` (the stream defaults to that GPU's current stream)."""
    index = -1
    for t in tensors:
        if t is not None:
            at = t.get_device()
            if at != index:
                if index >= 0 or at < 0 or not t.is_cuda:
                    _one_device(tensors)    # says what is wrong
                index = at
    if index < 0:
        _one_device(tensors)
    if stream is not None and stream.device.index != index:
        raise AcrlError(f"{name}: stream on {stream.device}, buffers on cuda:{index}")
    fn = _ENTRY.get(name)
    if fn is None:
        fn = _ENTRY[name] = getattr(lib(), name)
    if index == _current_device():
        # the current stream's handle without a Stream object around it
        st = fn(*args, torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(index):
            st = fn(*args, torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream)
    if st:
        check(st, name)


def _on_stream(f, name: str, t, stream, *args, **kw):
    """f(*args, **kw) with `stream` the current one: what it allocates then belongs to the stream that uses it.  (Memory of
    the current stream could still be in use there, or be handed out again while `stream` has yet to read it.)"""
    if stream.device.index != t.get_device():
        raise AcrlError(f"{name}: stream on {stream.device}, buffers on {t.device}")
    with torch.cuda.stream(stream):
        return f(*args, **kw)


def _flags(flags, dev):
    return new_flags(dev) if flags is None else _need(flags, torch.int32, 1, "flags")


def _need(t: torch.Tensor, dtype, n: int | None, name: str):
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous() and \
            (n is None or t.numel() >= n):
        return t
    if not isinstance(t, torch.Tensor):
        raise AcrlError(f"{name}: expected a torch tensor")
    if t.dtype != dtype:
        raise AcrlError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if not t.is_cuda:
        raise AcrlError(f"{name}: must be a CUDA tensor")
    if not t.is_contiguous():
        raise AcrlError(f"{name}: must be contiguous")
    if n is not None and t.numel() < n:
        raise AcrlError(f"{name}: has {t.numel()} elements, needs {n}")
    return t


def _opt(t, dtype, n, name):
    return None if t is None else _need(t, dtype, n, name)


def _rows(x: torch.Tensor, name: str):
    if x.dtype != torch.bfloat16 or x.dim() != 2:
        raise AcrlError(f"{name}: expected a 2-D bfloat16 tensor")
    if not x.is_cuda or x.stride(1) != 1:
        raise AcrlError(f"{name}: must be a CUDA tensor with unit column stride")
    return x.shape[0], x.stride(0)


def struct_buffer(dtype: np.dtype, n: int, device=None) -> torch.Tensor:
    """Device bytes for n ABI structs."""
    return torch.zeros(max(1, n) * dtype.itemsize, dtype=torch.uint8, device=device or "cuda")


def read_structs(buf: torch.Tensor, dtype: np.dtype, n: int) -> np.ndarray:
    return buf[: n * dtype.itemsize].cpu().numpy().view(dtype)


def new_flags(device=None) -> torch.Tensor:
    return torch.zeros(1, dtype=torch.int32, device=device or "cuda")


def token_stats(logits, ids, mask=None, *, V=None, lse=None, logp=None, entropy=None, flags=None, stream=None):
    """acrl_token_stats.  Returns (lse, logp, entropy) float32 [T]."""
    T, ld = _rows(logits, "logits")
    V = ld if V is None else V
    dev = logits.device
    _need(ids, torch.int32, T, "ids")
    _opt(mask, torch.uint8, T, "mask")
    lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else _need(lse, torch.float32, T, "lse")
    logp = torch.empty(T, dtype=torch.float32, device=dev) if logp is None else _need(logp, torch.float32, T, "logp")
    entropy = torch.empty(T, dtype=torch.float32, device=dev) if entropy is None else \
        _need(entropy, torch.float32, T, "entropy")
    flags = _flags(flags, dev)
    _call("acrl_token_stats", (logits, ids, mask, lse, logp, entropy, flags), stream, _ptr(logits), T, V, ld,
          _ptr(ids), _ptr(mask), _ptr(lse), _ptr(logp), _ptr(entropy), _ptr(flags))
    return lse, logp, entropy


@dataclass
class Discrepancy:
    lr: torch.Tensor
    d: torch.Tensor
    seq: torch.Tensor    # device bytes of acrl_seq_stats[S]
    grp: torch.Tensor    # device bytes of acrl_group_stats[Gn]
    batch: torch.Tensor  # device bytes of acrl_batch_stats
    S: int
    Gn: int

    def seq_host(self):
        return read_structs(self.seq, SEQ_DTYPE, self.S)

    def grp_host(self):
        return read_structs(self.grp, GRP_DTYPE, self.Gn)

    def batch_host(self):
        return read_structs(self.batch, BATCH_DTYPE, 1)[0]


def seq_discrepancy(logp_pi, logp_mu, mask, seq_offsets, group_offsets, entropy=None, *, out: Discrepancy | None = None,
                    flags=None, stream=None) -> Discrepancy:
    """acrl_seq_discrepancy."""
    T = logp_pi.numel()
    S = seq_offsets.numel() - 1
    Gn = group_offsets.numel() - 1
    dev = logp_pi.device
    _need(logp_pi, torch.float32, T, "logp_pi")
    _need(logp_mu, torch.float32, T, "logp_mu")
    _opt(mask, torch.uint8, T, "mask")
    _need(seq_offsets, torch.int64, S + 1, "seq_offsets")
    _need(group_offsets, torch.int32, Gn + 1, "group_offsets")
    _opt(entropy, torch.float32, T, "entropy")
    if out is None:
        out = Discrepancy(torch.empty(T, dtype=torch.float32, device=dev), torch.empty(T, dtype=torch.float32, device=dev),
                          struct_buffer(SEQ_DTYPE, S, dev), struct_buffer(GRP_DTYPE, Gn, dev),
                          struct_buffer(BATCH_DTYPE, 1, dev), S, Gn)
    flags = _flags(flags, dev)
    _call("acrl_seq_discrepancy", (logp_pi, logp_mu, mask, seq_offsets, group_offsets, entropy, out.lr, out.d,
                                   out.seq, out.grp, out.batch, flags), stream,
          _ptr(logp_pi), _ptr(logp_mu), _ptr(mask), T, _ptr(seq_offsets), S, _ptr(group_offsets), Gn, _ptr(entropy),
          _ptr(out.lr), _ptr(out.d), _ptr(out.seq), _ptr(out.grp), _ptr(out.batch), _ptr(flags))
    return out


def grpo_advantage(rewards, group_offsets, params: Params, *, adv=None, flags=None, stream=None):
    """acrl_grpo_advantage.  Returns adv float32 [S]."""
    S = rewards.numel()
    Gn = group_offsets.numel() - 1
    _need(rewards, torch.float32, S, "rewards")
    _need(group_offsets, torch.int32, Gn + 1, "group_offsets")
    adv = torch.empty(S, dtype=torch.float32, device=rewards.device) if adv is None else _need(adv, torch.float32, S, "adv")
    flags = _flags(flags, rewards.device)
    _call("acrl_grpo_advantage", (rewards, group_offsets, adv, flags), stream, _ptr(rewards), _ptr(group_offsets), Gn,
          S, ctypes.byref(params), _ptr(adv), _ptr(flags))
    return adv


def controller_init(params: Params, state=None, device=None, stream=None) -> torch.Tensor:
    """acrl_controller_init; allocates the 48-byte device state if not given."""
    state = struct_buffer(STATE_DTYPE, 1, device) if state is None else state
    _need(state, torch.uint8, STATE_DTYPE.itemsize, "state")
    _call("acrl_controller_init", (state,), stream, _ptr(state), ctypes.byref(params))
    return state


def read_state(state: torch.Tensor) -> np.void:
    return read_structs(state, STATE_DTYPE, 1)[0]


def save_state(state: torch.Tensor, stream=None) -> bytes:
    """acrl_controller_save: the controller state's 48 bytes, for a checkpoint
    (the state is plain data)."""
    _need(state, torch.uint8, STATE_DTYPE.itemsize, "state")
    buf = ctypes.create_string_buffer(STATE_DTYPE.itemsize)
    _call("acrl_controller_save", (state,), stream, _ptr(state), ctypes.addressof(buf))
    return buf.raw


def load_state(blob: bytes, state: torch.Tensor | None = None, device=None, stream=None) -> torch.Tensor:
    """acrl_controller_load: restore a state saved by save_state; resuming
    from it is bit-exact."""
    if len(blob) != STATE_DTYPE.itemsize:
        raise AcrlError("controller state: wrong size")
    state = struct_buffer(STATE_DTYPE, 1, device) if state is None else \
        _need(state, torch.uint8, STATE_DTYPE.itemsize, "state")
    buf = ctypes.create_string_buffer(bytes(blob), STATE_DTYPE.itemsize)
    _call("acrl_controller_load", (state,), stream, _ptr(state), ctypes.addressof(buf))
    return state


def controller_step(state, params: Params, disc: Discrepancy, mask, seq_offsets, group_offsets, adv, *, weight=None,
                    coef=None, alpha=None, ent_coef=None, flags=None, stream=None):
    """acrl_controller_step.  Returns (weight [T], coef [T], alpha [S]); the
    entropy-bonus factors go to `ent_coef` [T] when given."""
    T = disc.lr.numel()
    dev = disc.lr.device
    weight = torch.empty(T, dtype=torch.float32, device=dev) if weight is None else _need(weight, torch.float32, T, "weight")
    coef = torch.empty(T, dtype=torch.float32, device=dev) if coef is None else _need(coef, torch.float32, T, "coef")
    alpha = torch.empty(disc.S, dtype=torch.float32, device=dev) if alpha is None else \
        _need(alpha, torch.float32, disc.S, "alpha")
    _need(adv, torch.float32, disc.S, "adv")
    _opt(mask, torch.uint8, T, "mask")
    _opt(ent_coef, torch.float32, T, "ent_coef")
    _need(state, torch.uint8, STATE_DTYPE.itemsize, "state")
    flags = _flags(flags, dev)
    _call("acrl_controller_step", (state, disc.lr, mask, seq_offsets, group_offsets, disc.seq, disc.grp, disc.batch,
                                   adv, weight, coef, alpha, ent_coef, flags), stream,
          _ptr(state), ctypes.byref(params), _ptr(disc.lr), _ptr(mask), T, _ptr(seq_offsets), disc.S,
          _ptr(group_offsets), disc.Gn, _ptr(disc.seq), _ptr(disc.grp), _ptr(disc.batch), _ptr(adv), _ptr(weight),
          _ptr(coef), _ptr(alpha), _ptr(ent_coef), _ptr(flags))
    return weight, coef, alpha


def importance_weights(state, params: Params, logp_pi, logp_mu, mask, rewards, seq_offsets, group_offsets,
                       entropy=None, *, out: Discrepancy, adv, weight, coef, alpha=None, ent_coef=None, flags,
                       stream=None) -> None:
    """acrl_importance_weights: seq_discrepancy, grpo_advantage and controller_step in one call, into the caller's
    buffers."""
    T, S, Gn = logp_pi.numel(), seq_offsets.numel() - 1, group_offsets.numel() - 1
    f32 = torch.float32
    _need(state, torch.uint8, STATE_DTYPE.itemsize, "state")
    _need(logp_pi, f32, T, "logp_pi")
    _need(logp_mu, f32, T, "logp_mu")
    _opt(mask, torch.uint8, T, "mask")
    _need(rewards, f32, S, "rewards")
    _need(seq_offsets, torch.int64, S + 1, "seq_offsets")
    _need(group_offsets, torch.int32, Gn + 1, "group_offsets")
    _opt(entropy, f32, T, "entropy")
    _need(out.lr, f32, T, "lr")
    _need(out.d, f32, T, "d")
    _need(out.seq, torch.uint8, S * SEQ_DTYPE.itemsize, "seq")
    _need(out.grp, torch.uint8, Gn * GRP_DTYPE.itemsize, "grp")
    _need(out.batch, torch.uint8, BATCH_DTYPE.itemsize, "batch")
    _need(adv, f32, S, "adv")
    _need(weight, f32, T, "weight")
    _need(coef, f32, T, "coef")
    _opt(alpha, f32, S, "alpha")
    _opt(ent_coef, f32, T, "ent_coef")
    _need(flags, torch.int32, 1, "flags")
    _call("acrl_importance_weights",
          (state, logp_pi, logp_mu, mask, rewards, seq_offsets, group_offsets, entropy, out.lr, out.d, out.seq, out.grp,
           out.batch, adv, weight, coef, alpha, ent_coef, flags), stream,
          _ptr(state), ctypes.byref(params), _ptr(logp_pi), _ptr(logp_mu), _ptr(mask), T, _ptr(rewards),
          _ptr(seq_offsets), S, _ptr(group_offsets), Gn, _ptr(entropy), _ptr(out.lr), _ptr(out.d), _ptr(out.seq),
          _ptr(out.grp), _ptr(out.batch), _ptr(adv), _ptr(weight), _ptr(coef), _ptr(alpha), _ptr(ent_coef), _ptr(flags))


def loss_grad_logits(logits, ids, mask, lse, old_logp, coef, clip_eps: float, *, V=None, entropy=None, ent_coef=None,
                     grad=None, token_loss=None, loss=None, flags=None, stream=None):
    """acrl_loss_grad_logits.  Returns (grad bf16 [T, ld], token_loss [T], loss [1]).
    `entropy` and `ent_coef` (both or neither) add the entropy bonus."""
    T, ld = _rows(logits, "logits")
    V = ld if V is None else V
    dev = logits.device
    _need(ids, torch.int32, T, "ids")
    _opt(mask, torch.uint8, T, "mask")
    _opt(lse, torch.float32, T, "lse")
    _opt(old_logp, torch.float32, T, "old_logp")
    _need(coef, torch.float32, T, "coef")
    _opt(entropy, torch.float32, T, "entropy")
    _opt(ent_coef, torch.float32, T, "ent_coef")
    if grad is None:
        grad = torch.empty((T, ld), dtype=torch.bfloat16, device=dev)
    elif grad.dtype != torch.bfloat16 or grad.dim() != 2 or grad.stride(0) != ld or grad.stride(1) != 1 or \
            grad.shape[0] < T:
        raise AcrlError("grad: expected a bf16 [T, ld] tensor with the logits' row stride")
    token_loss = torch.empty(T, dtype=torch.float32, device=dev) if token_loss is None else \
        _need(token_loss, torch.float32, T, "token_loss")
    loss = torch.empty(1, dtype=torch.float32, device=dev) if loss is None else _need(loss, torch.float32, 1, "loss")
    flags = _flags(flags, dev)
    _call("acrl_loss_grad_logits", (logits, ids, mask, lse, old_logp, coef, entropy, ent_coef, grad, token_loss, loss,
                                    flags), stream,
          _ptr(logits), T, V, ld, _ptr(ids), _ptr(mask), _ptr(lse), _ptr(old_logp), _ptr(coef), _ptr(entropy),
          _ptr(ent_coef), float(clip_eps), _ptr(grad), _ptr(token_loss), _ptr(loss), _ptr(flags))
    return grad, token_loss, loss


def step(state, params: Params, logits, ids, mask, logp_mu, rewards, seq_offsets, group_offsets, *, V, lse, logp,
         entropy, out: Discrepancy, adv, weight, coef, alpha=None, ent_coef=None, grad, token_loss, loss, flags,
         stream=None) -> None:
    """acrl_step: token_stats, importance_weights and loss_grad_logits in one call, into the caller's buffers."""
    T, ld = _rows(logits, "logits")
    S, Gn = seq_offsets.numel() - 1, group_offsets.numel() - 1
    f32 = torch.float32
    _need(state, torch.uint8, STATE_DTYPE.itemsize, "state")
    _need(ids, torch.int32, T, "ids")
    _opt(mask, torch.uint8, T, "mask")
    _need(logp_mu, f32, T, "logp_mu")
    _need(rewards, f32, S, "rewards")
    _need(seq_offsets, torch.int64, S + 1, "seq_offsets")
    _need(group_offsets, torch.int32, Gn + 1, "group_offsets")
    for name, t in (("lse", lse), ("logp", logp), ("entropy", entropy), ("lr", out.lr), ("d", out.d),
                    ("weight", weight), ("coef", coef), ("token_loss", token_loss)):
        _need(t, f32, T, name)
    _need(out.seq, torch.uint8, S * SEQ_DTYPE.itemsize, "seq")
    _need(out.grp, torch.uint8, Gn * GRP_DTYPE.itemsize, "grp")
    _need(out.batch, torch.uint8, BATCH_DTYPE.itemsize, "batch")
    _need(adv, f32, S, "adv")
    _opt(alpha, f32, S, "alpha")
    _opt(ent_coef, f32, T, "ent_coef")
    if grad.dtype != torch.bfloat16 or grad.dim() != 2 or grad.stride(0) != ld or grad.stride(1) != 1 or \
            grad.shape[0] < T:
        raise AcrlError("grad: expected a bf16 [T, ld] tensor with the logits' row stride")
    _need(loss, f32, 1, "loss")
    _need(flags, torch.int32, 1, "flags")
    bufs = (lse, logp, entropy, out.lr, out.d, out.seq, out.grp, out.batch, adv, weight, coef, alpha, ent_coef, grad,
            token_loss, loss, flags)
    _call("acrl_step", (state, logits, ids, mask, logp_mu, rewards, seq_offsets, group_offsets) + bufs, stream,
          _ptr(state), ctypes.byref(params), _ptr(logits), T, V, ld, _ptr(ids), _ptr(mask), _ptr(logp_mu),
          _ptr(rewards), _ptr(seq_offsets), S, _ptr(group_offsets), Gn, *[_ptr(t) for t in bufs])


def reduce_loss(token_loss, *, loss=None, stream=None):
    """acrl_reduce_loss."""
    T = token_loss.numel()
    _need(token_loss, torch.float32, T, "token_loss")
    loss = torch.empty(1, dtype=torch.float32, device=token_loss.device) if loss is None else \
        _need(loss, torch.float32, 1, "loss")
    _call("acrl_reduce_loss", (token_loss, loss), stream, _ptr(token_loss), T, _ptr(loss))
    return loss


def scale_grad(grad, scale, *, V=None, out=None, stream=None):
    """acrl_scale_grad: grad (bf16 [T, ld]) times the float32 scalar on the device.  Returns `out` (row stride V, or a
    multiple of eight), by default bf16 [T, ldo] with V rounded up to a multiple of eight; its contents are undefined
    where the scalar is exactly 1."""
    T, ld = _rows(grad, "grad")
    V = grad.shape[1] if V is None else V
    if V > ld:
        raise AcrlError(f"V = {V} is more than the row stride {ld}")
    _need(scale, torch.float32, 1, "scale")
    ldo = (V + 7) // 8 * 8
    if out is None:
        out = torch.empty((T, ldo), dtype=torch.bfloat16, device=grad.device)
    else:
        To, ldo = _rows(out, "out")
        if To < T or out.shape[1] < V:
            raise AcrlError(f"out: shape {tuple(out.shape)}, needs {(T, V)}")
    _call("acrl_scale_grad", (grad, scale, out), stream, _ptr(grad), T, V, ld, _ptr(scale), _ptr(out), ldo)
    return out


def lmhead_workspace_bytes(M: int, N: int) -> int:
    return int(lib().acrl_lmhead_workspace_bytes(M, N))


def lmhead_logits_stats(hidden, weight, *, N=None, logits=None, partials=None, flags=None, stream=None):
    """acrl_lmhead_logits_stats.  hidden bf16 [M, K], weight bf16 [N, K].
    Returns (logits bf16 [M, ldl], partials workspace)."""
    M, ldh = _rows(hidden, "hidden")
    Nw, ldw = _rows(weight, "weight")
    N = Nw if N is None else N
    K = hidden.shape[1]
    if weight.shape[1] != K:
        raise AcrlError("hidden and weight disagree on K")
    dev = hidden.device
    ldl = ((N + 7) // 8) * 8
    if logits is None:
        logits = torch.empty((M, ldl), dtype=torch.bfloat16, device=dev)
    else:
        _, ldl = _rows(logits, "logits")
    nbytes = lmhead_workspace_bytes(M, N)
    if partials is None:
        partials = torch.empty(max(1, nbytes // 4), dtype=torch.float32, device=dev)
    else:
        _need(partials, torch.float32, (nbytes + 3) // 4, "partials")
    flags = _flags(flags, dev)
    _call("acrl_lmhead_logits_stats", (hidden, weight, logits, partials, flags), stream, _ptr(hidden), M, K, ldh,
          _ptr(weight), N, ldw, _ptr(logits), ldl, _ptr(partials), _ptr(flags))
    return logits, partials


def lmhead_merge(partials, logits, ids, mask=None, *, N=None, lse=None, logp=None, entropy=None, flags=None,
                 stream=None):
    """acrl_lmhead_merge.  Returns (lse, logp, entropy)."""
    M, ldl = _rows(logits, "logits")
    N = ldl if N is None else N
    dev = logits.device
    _need(ids, torch.int32, M, "ids")
    _opt(mask, torch.uint8, M, "mask")
    lse = torch.empty(M, dtype=torch.float32, device=dev) if lse is None else _need(lse, torch.float32, M, "lse")
    logp = torch.empty(M, dtype=torch.float32, device=dev) if logp is None else _need(logp, torch.float32, M, "logp")
    entropy = torch.empty(M, dtype=torch.float32, device=dev) if entropy is None else \
        _need(entropy, torch.float32, M, "entropy")
    _need(partials, torch.float32, (lmhead_workspace_bytes(M, N) + 3) // 4, "partials")
    flags = _flags(flags, dev)
    _call("acrl_lmhead_merge", (partials, logits, ids, mask, lse, logp, entropy, flags), stream, _ptr(partials),
          _ptr(logits), M, N, ldl, _ptr(ids), _ptr(mask), _ptr(lse), _ptr(logp), _ptr(entropy), _ptr(flags))
    return lse, logp, entropy


def lmhead_stats_noalloc(hidden, weight, ids, mask=None, *, N=None, logits=None, lse=None, logp=None, entropy=None,
                         flags=None, stream=None):
    """acrl_lmhead_stats_noalloc (GEMM + merge with the library's fixed scratch).
    Returns (logits, lse, logp, entropy)."""
    M, ldh = _rows(hidden, "hidden")
    Nw, ldw = _rows(weight, "weight")
    N = Nw if N is None else N
    K = hidden.shape[1]
    if weight.shape[1] != K:
        raise AcrlError("hidden and weight disagree on K")
    dev = hidden.device
    if logits is None:
        logits = torch.empty((M, ((N + 7) // 8) * 8), dtype=torch.bfloat16, device=dev)
    _, ldl = _rows(logits, "logits")
    _need(ids, torch.int32, M, "ids")
    _opt(mask, torch.uint8, M, "mask")
    f32 = dict(dtype=torch.float32, device=dev)
    lse = torch.empty(M, **f32) if lse is None else _need(lse, torch.float32, M, "lse")
    logp = torch.empty(M, **f32) if logp is None else _need(logp, torch.float32, M, "logp")
    entropy = torch.empty(M, **f32) if entropy is None else _need(entropy, torch.float32, M, "entropy")
    flags = _flags(flags, dev)
    _call("acrl_lmhead_stats_noalloc", (hidden, weight, logits, ids, mask, lse, logp, entropy, flags), stream,
          _ptr(hidden), M, K, ldh, _ptr(weight), N, ldw, _ptr(logits), ldl, _ptr(ids), _ptr(mask), _ptr(lse),
          _ptr(logp), _ptr(entropy), _ptr(flags))
    return logits, lse, logp, entropy


# ---------------------------------------------------------------------------
# 8-bit matrices
# ---------------------------------------------------------------------------

_FP8 = {"e4m3": (_abi.FP8_E4M3, torch.float8_e4m3fn), "e5m2": (_abi.FP8_E5M2, torch.float8_e5m2)}
_FP8_FORMAT = {dtype: code for code, dtype in _FP8.values()}
_FP8_BLOCK = {"row": _abi.FP8_ROW, "tile": _abi.FP8_TILE}
_OUT_DTYPE = {torch.bfloat16: _abi.BF16, torch.float32: _abi.F32}


@dataclass(frozen=True)
class Fp8Tensor:
    """An 8-bit matrix [rows, cols]: q (torch.float8_e4m3fn or float8_e5m2, rows at a stride of 16 bytes) and the
    scales of its blocks, uint8 [rows or ceil(rows / 128), ceil(cols / 128)], byte s standing for 2^(s - 127)."""

    q: torch.Tensor
    scale: torch.Tensor

    def __post_init__(self):
        q, s = self.q, self.scale
        if q.dtype not in _FP8_FORMAT or q.dim() != 2 or not q.is_cuda:
            raise AcrlError("q: expected a 2-D float8_e4m3fn or float8_e5m2 CUDA tensor")
        if s.dtype != torch.uint8 or s.dim() != 2 or not s.is_cuda:
            raise AcrlError("scale: expected a 2-D uint8 CUDA tensor")
        (R, C), (SR, SC) = q.shape, s.shape
        (ldq, cq), (lds, cs) = q.stride(), s.stride()
        if (cq != 1 and C > 1) or (cs != 1 and SC > 1):
            raise AcrlError("q and scale: expected unit column strides")
        if SC < (C + 127) // 128 or (SR != R and SR != (R + 127) // 128):
            raise AcrlError(f"scale: shape {(SR, SC)} fits neither the rows nor the 128 x 128 tiles of {(R, C)}")
        # one row is one tile of one row: the same scales either way
        block = "row" if SR == R else "tile"
        # of a single row, or with nothing in a row, the stride says nothing, and any that the library accepts will do
        self._known(block, R, ldq if R > 1 and C > 0 else (C + 15) // 16 * 16, _FP8_FORMAT[q.dtype],
                    lds if SR > 1 and SC > 0 else SC)

    def _known(self, block: str, rows: int, ldq: int, code: int, lds: int) -> None:
        self.__dict__.update(block=block, _layout=(rows, ldq, code, lds, _FP8_BLOCK[block]))

    @property
    def _args(self):
        """Address, rows, row stride, format, scales' address, their row stride, block: as the library takes a matrix."""
        rows, ldq, code, lds, block = self._layout
        return self.q.data_ptr(), rows, ldq, code, self.scale.data_ptr(), lds, block

    @classmethod
    def _made(cls, q, scale, *known):
        """One whose parts need no check."""
        t = object.__new__(cls)
        t.__dict__.update(q=q, scale=scale)
        t._known(*known)
        return t

    @property
    def shape(self):
        return self.q.shape

    def values(self) -> torch.Tensor:
        """The float32 matrix that the bytes stand for (for inspection)."""
        R, C = self.q.shape
        e = self.scale[:, : (C + 127) // 128].to(torch.int32)
        s = torch.where(e > 0, e << 23, 1 << 22).view(torch.float32)    # 2^(s - 127); 2^-127 has no leading one
        s = torch.where(e == 255, torch.nan, s)
        if self.block == "tile":
            s = s.repeat_interleave(128, 0)[:R]
        return self.q.to(torch.float32) * s.repeat_interleave(128, 1)[:, :C]


def _ld(t: torch.Tensor) -> int:
    """The row stride of a matrix; where there is at most one row, or nothing in a row, any that a kernel accepts."""
    return t.stride(0) if t.shape[0] > 1 and t.shape[1] > 0 else (t.shape[1] + 15) // 16 * 16


def _fp8_args(t: Fp8Tensor, name: str):
    if not isinstance(t, Fp8Tensor):
        raise AcrlError(f"{name}: expected an Fp8Tensor")
    return t._args


def _fp8_format(fmt: str) -> int:
    if fmt not in _FP8:
        raise AcrlError(f"fmt: {fmt!r}, expected one of {sorted(_FP8)}")
    return _FP8[fmt][0]


def _padded(shape, to: int, dtype, dev) -> torch.Tensor:
    """A new matrix with its rows, the last one too, at a stride that is a multiple of `to`."""
    ld = (shape[1] + to - 1) // to * to
    x = torch.empty((shape[0], ld), dtype=dtype, device=dev)
    return x if ld == shape[1] else x[:, : shape[1]]


def fp8_quantize(x, *, block="row", fmt="e4m3", transpose=False, out: Fp8Tensor | None = None, flags=None,
                 stream=None) -> Fp8Tensor:
    """acrl_fp8_quantize: x (bf16 or float32 [R, C]) or its transpose as an 8-bit matrix with power-of-two scales per
    128 columns of a row (block="row") or per 128 x 128 ("tile")."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or not x.is_cuda:
        raise AcrlError("x: expected a 2-D CUDA tensor")
    if stream is not None:
        return _on_stream(fp8_quantize, "acrl_fp8_quantize", x, stream, x, block=block, fmt=fmt, transpose=transpose, out=out,
                          flags=flags)
    xt = _OUT_DTYPE.get(x.dtype)
    (R, C), (ldx, cs) = x.shape, x.stride()
    if xt is None or (cs != 1 and C > 1):
        raise AcrlError("x: expected bfloat16 or float32 with unit column stride")
    kind = _FP8_BLOCK.get(block)
    if kind is None or fmt not in _FP8:
        raise AcrlError(f"block {block!r}, fmt {fmt!r}: expected one of {sorted(_FP8_BLOCK)} and one of {sorted(_FP8)}")
    code, dtype = _FP8[fmt]
    rows, cols = (C, R) if transpose else (R, C)
    srows, kb = (rows if kind == _abi.FP8_ROW else (rows + 127) // 128), (cols + 127) // 128
    if out is None:
        ldq, lds = (cols + 15) // 16 * 16, (kb + 3) // 4 * 4
        out = Fp8Tensor._made(torch.empty_strided((rows, cols), (ldq, 1), dtype=dtype, device=x.device),
                              torch.empty_strided((srows, kb), (lds, 1), dtype=torch.uint8, device=x.device),
                              "row" if srows == rows else "tile", rows, ldq, code, lds)
    elif tuple(out.q.shape) != (rows, cols) or out.q.dtype != dtype or out.scale.shape[0] != srows:
        raise AcrlError(f"out: an 8-bit matrix of another shape, format or block than {(rows, cols)} {fmt} {block}")
    if flags is not None:
        _need(flags, torch.int32, 1, "flags")
    ptr, _, ldq, _, sptr, lds, _ = out._args
    _call("acrl_fp8_quantize", (x, out.q, out.scale, flags), None, x.data_ptr(), xt, R, C,
          ldx if R > 1 and C > 0 else (C + 15) // 16 * 16, code, kind, 1 if transpose else 0, ptr, ldq, sptr, lds,
          None if flags is None else flags.data_ptr())
    return out


def _product_out(out, M: int, N: int, dtype, dev):
    """(`out` as [M, N], its row stride)."""
    if out is None:
        ldo = (N + 7) // 8 * 8
        return _padded((M, N), 8, dtype, dev), ldo
    if not isinstance(out, torch.Tensor) or out.dtype not in _OUT_DTYPE or out.dim() != 2 or not out.is_cuda or \
            (out.shape[1] > 1 and out.stride(1) != 1) or out.shape[0] != M or out.shape[1] < N:
        raise AcrlError(f"out: expected a bfloat16 or float32 CUDA matrix of {(M, N)} with unit column stride")
    return out if out.shape[1] == N else out[:, :N], out.stride(0) if M > 1 and N > 0 else (N + 7) // 8 * 8


def fp8_matmul(a: Fp8Tensor, b: Fp8Tensor, *, out_dtype=torch.bfloat16, out=None, flags=None, stream=None):
    """acrl_fp8_matmul: a [M, K] times the transpose of b [N, K], as `out_dtype` [M, N]."""
    aa, bb = _fp8_args(a, "a"), _fp8_args(b, "b")
    if stream is not None:
        return _on_stream(fp8_matmul, "acrl_fp8_matmul", a.q, stream, a, b, out_dtype=out_dtype, out=out, flags=flags)
    M, N, K = a.shape[0], b.shape[0], a.shape[1]
    if b.shape[1] != K:
        raise AcrlError(f"a and b disagree on K: {K} and {b.shape[1]}")
    if out_dtype not in _OUT_DTYPE:
        raise AcrlError(f"out_dtype: {out_dtype}, expected bfloat16 or float32")
    out, ldo = _product_out(out, M, N, out_dtype, a.q.device)
    _opt(flags, torch.int32, 1, "flags")
    _call("acrl_fp8_matmul", (a.q, a.scale, b.q, b.scale, out, flags), None, aa[0], M, K, *aa[2:], bb[0], N, *bb[2:],
          _ptr(out), _OUT_DTYPE[out.dtype], ldo, _ptr(flags))
    return out


def fp8_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    """acrl_fp8_linear_workspace_bytes."""
    return int(lib().acrl_fp8_linear_workspace_bytes(M, N, K))


def fp8_linear(x, weight: Fp8Tensor, *, fmt="e4m3", out_dtype=torch.bfloat16, out=None, workspace=None, flags=None,
               stream=None):
    """acrl_fp8_linear: x (bf16 [M, K]) quantised by rows, times the transpose of `weight` [N, K]; [M, N]."""
    M, K = _bf16_rows(x, "x")
    w = _fp8_args(weight, "weight")
    if stream is not None:
        return _on_stream(fp8_linear, "acrl_fp8_linear", x, stream, x, weight, fmt=fmt, out_dtype=out_dtype, out=out,
                          workspace=workspace, flags=flags)
    N = w[1]
    if weight.shape[1] != K:
        raise AcrlError(f"x and weight disagree on K: {K} and {weight.shape[1]}")
    if out_dtype not in _OUT_DTYPE:
        raise AcrlError(f"out_dtype: {out_dtype}, expected bfloat16 or float32")
    out, ldo = _product_out(out, M, N, out_dtype, x.device)
    n = lib().acrl_fp8_linear_workspace_bytes(M, N, K)
    if workspace is not None:
        _need(workspace, torch.uint8, n, "workspace")
    elif n > 0:
        workspace = torch.empty(n, dtype=torch.uint8, device=x.device)
    _opt(flags, torch.int32, 1, "flags")
    _call("acrl_fp8_linear", (x, weight.q, weight.scale, out, workspace, flags), None, x.data_ptr(), M, K, _ld(x),
          _fp8_format(fmt), w[0], N, *w[2:], out.data_ptr(), _OUT_DTYPE[out.dtype], ldo, _ptr(workspace), n, _ptr(flags))
    return out


def fp8_linear_backward_workspace_bytes(M: int, N: int, K: int) -> int:
    """acrl_fp8_linear_backward_workspace_bytes."""
    return int(lib().acrl_fp8_linear_backward_workspace_bytes(M, N, K))


def _bf16_rows(x, name: str):
    if not isinstance(x, torch.Tensor) or x.dtype != torch.bfloat16 or x.dim() != 2 or not x.is_cuda or \
            (x.shape[1] > 1 and x.stride(1) != 1):
        raise AcrlError(f"{name}: expected a 2-D bfloat16 CUDA tensor with unit column stride")
    return x.shape


def fp8_linear_backward(dy, x, weight_t: Fp8Tensor, *, fmt="e4m3", x_fmt="e4m3", dx_dtype=torch.bfloat16,
                        dw_dtype=torch.float32, dx=None, dw=None, workspace=None, flags=None, stream=None):
    """acrl_fp8_linear_backward, the gradients of y = x W^T: dx = Q(dy) W and dw = Q(dy^T) Q(x^T)^T, products of 8-bit
    matrices over N and over the rows.  dy [M, N] and x [M, K] bf16; `weight_t` is the 8-bit W^T [K, N]
    (fp8_quantize(w, block="tile", transpose=True)); `fmt` and `x_fmt` are dy's and x's formats.  Returns (dx [M, K],
    dw [N, K])."""
    (M, N), (Mx, K) = _bf16_rows(dy, "dy"), _bf16_rows(x, "x")
    w = _fp8_args(weight_t, "weight_t")
    if stream is not None:
        return _on_stream(fp8_linear_backward, "acrl_fp8_linear_backward", dy, stream, dy, x, weight_t, fmt=fmt, x_fmt=x_fmt,
                          dx_dtype=dx_dtype, dw_dtype=dw_dtype, dx=dx, dw=dw, workspace=workspace, flags=flags)
    if Mx != M or tuple(weight_t.shape) != (K, N):
        raise AcrlError(f"dy {(M, N)}, x {(Mx, K)} and weight_t {tuple(weight_t.shape)} do not belong together")
    if dx_dtype not in _OUT_DTYPE or dw_dtype not in _OUT_DTYPE:
        raise AcrlError("dx_dtype, dw_dtype: expected bfloat16 or float32")
    dx, lddx = _product_out(dx, M, K, dx_dtype, dy.device)
    dw, lddw = _product_out(dw, N, K, dw_dtype, dy.device)
    n = lib().acrl_fp8_linear_backward_workspace_bytes(M, N, K)
    workspace = torch.empty(n, dtype=torch.uint8, device=dy.device) if workspace is None else \
        _need(workspace, torch.uint8, n, "workspace")
    _opt(flags, torch.int32, 1, "flags")
    _call("acrl_fp8_linear_backward", (dy, x, weight_t.q, weight_t.scale, dx, dw, workspace, flags), None, dy.data_ptr(), M, N,
          _ld(dy), _fp8_format(fmt), x.data_ptr(), K, _ld(x), _fp8_format(x_fmt), w[0], *w[2:], dx.data_ptr(),
          _OUT_DTYPE[dx.dtype], lddx, dw.data_ptr(), _OUT_DTYPE[dw.dtype], lddw, workspace.data_ptr(), n, _ptr(flags))
    return dx, dw


# ---------------------------------------------------------------------------
# a layer in bf16, its gradients and the update of its weight
# ---------------------------------------------------------------------------

_ACT = {None: _abi.ACT_NONE, "relu": _abi.ACT_RELU, "gelu": _abi.ACT_GELU, "gelu_tanh": _abi.ACT_GELU_TANH, "silu": _abi.ACT_SILU}


def _act(act) -> int:
    code = _ACT.get(act)
    if code is None:
        raise AcrlError(f"act: {act!r}, expected one of {list(_ACT)}")
    return code


def _operand(t, name: str):
    """(rows, columns, row stride) of a 2-D bf16 CUDA tensor; these calls are short, and each look at a tensor costs."""
    if isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.is_cuda:
        shape = t.shape
        if len(shape) == 2:
            R, C = shape
            ld, cs = t.stride()
            if cs == 1 or C <= 1:
                return R, C, ld if R > 1 and C > 0 else (C + 7) // 8 * 8
    raise AcrlError(f"{name}: expected a 2-D bfloat16 CUDA tensor with unit column stride")


_BF16_ONLY, _BF16_F32 = (torch.bfloat16,), (torch.bfloat16, torch.float32)


def _given(t, M: int, N: int, dtypes, name: str):
    """The row stride of a matrix [M, N] that the caller gives."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.dim() != 2 or not t.is_cuda or \
            (N > 1 and t.stride(1) != 1) or t.shape[0] != M or t.shape[1] != N:
        raise AcrlError(f"{name}: expected a CUDA matrix of {(M, N)}, {' or '.join(str(d) for d in dtypes)}, with unit column stride")
    return t.stride(0) if M > 1 and N > 0 else (N + 7) // 8 * 8


def _result(out, M: int, N: int, dtype, dev):
    """_product_out, a new matrix without the view that cuts its padding off: the last row ends with its columns."""
    if out is not None:
        return _product_out(out, M, N, dtype, dev)
    ld = (N + 7) // 8 * 8
    return torch.empty_strided((M, N), (ld, 1), dtype=dtype, device=dev), ld


@functools.lru_cache(maxsize=256)
def _size_of(name: str, *sizes: int) -> int:
    """What a *_workspace_bytes entry point says, by its sizes alone."""
    return int(getattr(lib(), name)(*sizes))


def _workspace(workspace, n: int, dev):
    if workspace is not None:
        return _need(workspace, torch.uint8, n, "workspace")
    return torch.empty(n, dtype=torch.uint8, device=dev) if n > 0 else None


def linear_workspace_bytes(M: int, N: int, K: int) -> int:
    """acrl_linear_workspace_bytes."""
    return int(lib().acrl_linear_workspace_bytes(M, N, K))


def linear(x, weight, bias=None, *, act=None, residual=None, pre_out=None, out_dtype=torch.bfloat16, out=None, workspace=None,
           flags=None, stream=None):
    """acrl_linear: act(x W^T + bias) + residual as `out_dtype` [M, N].  x bf16 [M, K], weight bf16 [N, K]; bias float32 or
    bfloat16 [N]; `act` is None, "relu", "gelu", "gelu_tanh" or "silu"; residual bfloat16 or float32 [M, N] (`out` itself is
    allowed); `pre_out` bf16 [M, N] takes x W^T + bias, for linear_backward."""
    M, K, ldx = _operand(x, "x")
    N, Kw, ldw = _operand(weight, "weight")
    if stream is not None:
        return _on_stream(linear, "acrl_linear", x, stream, x, weight, bias, act=act, residual=residual, pre_out=pre_out,
                          out_dtype=out_dtype, out=out, workspace=workspace, flags=flags)
    if Kw != K:
        raise AcrlError(f"x and weight disagree on K: {K} and {Kw}")
    if out_dtype not in _OUT_DTYPE:
        raise AcrlError(f"out_dtype: {out_dtype}, expected bfloat16 or float32")
    code = _act(act)
    pb = pr = pp = None
    tb = tr = ldr = ldp = 0
    if bias is not None:
        if not isinstance(bias, torch.Tensor) or bias.dtype not in _OUT_DTYPE or tuple(bias.shape) != (N,) or \
                not bias.is_cuda or not bias.is_contiguous():
            raise AcrlError(f"bias: expected a contiguous float32 or bfloat16 CUDA vector of {N}")
        pb, tb = bias.data_ptr(), _OUT_DTYPE[bias.dtype]
    if residual is not None:
        ldr = _given(residual, M, N, _BF16_F32, "residual")
        pr, tr = residual.data_ptr(), _OUT_DTYPE[residual.dtype]
    if pre_out is not None:
        ldp = _given(pre_out, M, N, _BF16_ONLY, "pre_out")
        pp = pre_out.data_ptr()
    out, ldo = _result(out, M, N, out_dtype, x.device)
    n = _size_of("acrl_linear_workspace_bytes", M, N, K)
    if n > 0 or workspace is not None:
        workspace = _workspace(workspace, n, x.device)
    if flags is not None:
        _need(flags, torch.int32, 1, "flags")
    _call("acrl_linear", (x, weight, bias, residual, pre_out, out, workspace, flags), None, x.data_ptr(), M, K, ldx,
          weight.data_ptr(), N, ldw, pb, tb, code, pr, tr, ldr, pp, ldp, out.data_ptr(), _OUT_DTYPE[out.dtype], ldo,
          None if workspace is None else workspace.data_ptr(), n, None if flags is None else flags.data_ptr())
    return out


def linear_backward_workspace_bytes(M: int, N: int, K: int) -> int:
    """acrl_linear_backward_workspace_bytes."""
    return int(lib().acrl_linear_backward_workspace_bytes(M, N, K))


def linear_backward(dy, x, weight, *, act=None, pre=None, bias=False, need_dx=True, need_dw=True, dx_dtype=torch.bfloat16,
                    dw_dtype=torch.float32, dx=None, dw=None, dbias=None, workspace=None, flags=None, stream=None):
    """acrl_linear_backward, the gradients of linear: with g = dy act'(pre), dx = g W, dw = g^T x and, with `bias`,
    dbias = sum of g over the rows.  dy bf16 [M, N], x bf16 [M, K], weight bf16 [N, K], `pre` the bf16 [M, N] that linear
    wrote.  Returns (dx [M, K], dw [N, K], dbias float32 [N]), None where not asked for; the gradient of the residual is dy.  After
    an activation g is rounded to bf16 for both products, whatever type dx and dw have."""
    M, N, lddy = _operand(dy, "dy")
    Mx, K, ldx = _operand(x, "x")
    Nw, Kw, ldw = _operand(weight, "weight")
    if stream is not None:
        return _on_stream(linear_backward, "acrl_linear_backward", dy, stream, dy, x, weight, act=act, pre=pre, bias=bias,
                          need_dx=need_dx, need_dw=need_dw, dx_dtype=dx_dtype, dw_dtype=dw_dtype, dx=dx, dw=dw, dbias=dbias,
                          workspace=workspace, flags=flags)
    if Mx != M or Nw != N or Kw != K:
        raise AcrlError(f"dy {(M, N)}, x {(Mx, K)} and weight {(Nw, Kw)} do not belong together")
    if dx_dtype not in _OUT_DTYPE or dw_dtype not in _OUT_DTYPE:
        raise AcrlError("dx_dtype, dw_dtype: expected bfloat16 or float32")
    code = _act(act)
    if (act is None) != (pre is None):
        raise AcrlError(f"act={act!r} takes " + ("no pre" if act is None else "pre, the pre-activation that linear wrote"))
    if (dx is not None and not need_dx) or (dw is not None and not need_dw) or (dbias is not None and not bias):
        raise AcrlError("dx, dw, dbias: an output that is not asked for")
    ldp = 0 if pre is None else _given(pre, M, N, _BF16_ONLY, "pre")
    dev = dy.device
    px = pw = pb = None
    tx = tw = lddx = lddw = 0
    if need_dx:
        dx, lddx = _result(dx, M, K, dx_dtype, dev)
        px, tx = dx.data_ptr(), _OUT_DTYPE[dx.dtype]
    if need_dw:
        dw, lddw = _result(dw, N, K, dw_dtype, dev)
        pw, tw = dw.data_ptr(), _OUT_DTYPE[dw.dtype]
    if bias:
        dbias = _vec(dbias, torch.float32, N, "dbias", dev)
        pb = dbias.data_ptr()
    n = _size_of("acrl_linear_backward_workspace_bytes", M, N, K)
    workspace = _workspace(workspace, n, dev)
    if flags is not None:
        _need(flags, torch.int32, 1, "flags")
    _call("acrl_linear_backward", (dy, x, weight, pre, dx, dw, dbias, workspace, flags), None, dy.data_ptr(), M, N, lddy,
          x.data_ptr(), K, ldx, weight.data_ptr(), ldw, code, _ptr(pre), ldp, px, tx, lddx, pw, tw, lddw, pb, _ptr(workspace), n,
          _ptr(flags))
    return dx, dw, dbias


def orthogonalize_workspace_bytes(batch: int, m: int, n: int) -> int:
    """acrl_orthogonalize_workspace_bytes."""
    return int(lib().acrl_orthogonalize_workspace_bytes(batch, m, n))


def _matrices(t, name: str):
    """(batch, m, n, row stride, matrix stride) of one matrix or a batch of them, padded strides where a size is one."""
    to = 8 if t.dtype == torch.bfloat16 else 4
    B, (m, n) = (t.shape[0] if t.dim() == 3 else 1), t.shape[-2:]
    if n > 1 and t.stride(-1) != 1:
        raise AcrlError(f"{name}: expected unit column stride")
    ld = t.stride(-2) if m > 1 and n > 0 else (n + to - 1) // to * to
    return B, m, n, ld, t.stride(0) if t.dim() == 3 and B > 1 else m * ld


def _step_coeffs(coeffs, steps) -> list[float]:
    """Three numbers for each step, from one triple or from as many as there are steps."""
    try:
        c = np.asarray(coeffs, dtype=np.float32)
        if isinstance(steps, int) and steps >= 1 and c.shape in ((3,), (steps, 3)):
            return np.broadcast_to(c, (steps, 3)).ravel().tolist()
    except (TypeError, ValueError):
        pass
    raise AcrlError("steps, coeffs: expected a number of steps, and three numbers, or three for each of them")


def orthogonalize(g, *, steps=5, coeffs=(3.4445, -4.7750, 2.0315), eps=1e-7, scale=1.0, out=None, workspace=None, flags=None,
                  stream=None):
    """acrl_orthogonalize: an update, bf16 or float32 [m, n] or a batch [B, m, n] of them, with its singular values brought
    near one by `steps` Newton-Schulz steps, times `scale`; bf16 of the same shape.  `coeffs` is (a, b, c), or one such triple
    for each step.  `out` may be g."""
    if not isinstance(g, torch.Tensor) or g.dtype not in _OUT_DTYPE or g.dim() not in (2, 3) or not g.is_cuda:
        raise AcrlError("g: expected a bfloat16 or float32 CUDA matrix, or a batch of them")
    if stream is not None:
        return _on_stream(orthogonalize, "acrl_orthogonalize", g, stream, g, steps=steps, coeffs=coeffs, eps=eps, scale=scale,
                          out=out, workspace=workspace, flags=flags)
    B, m, n, ldg, stride = _matrices(g, "g")
    flat = _step_coeffs(coeffs, steps)
    if out is None:
        ld = (n + 7) // 8 * 8
        out = torch.empty_strided(g.shape, ((ld, 1) if g.dim() == 2 else (m * ld, ld, 1)), dtype=torch.bfloat16, device=g.device)
    elif not isinstance(out, torch.Tensor) or out.dtype != torch.bfloat16 or out.shape != g.shape or not out.is_cuda:
        raise AcrlError(f"out: expected a bfloat16 CUDA tensor of {tuple(g.shape)}")
    _, _, _, ldo, out_stride = _matrices(out, "out")
    nbytes = _size_of("acrl_orthogonalize_workspace_bytes", B, m, n)
    workspace = _workspace(workspace, nbytes, g.device)
    if flags is not None:
        _need(flags, torch.int32, 1, "flags")
    _call("acrl_orthogonalize", (g, out, workspace, flags), None, g.data_ptr(), _OUT_DTYPE[g.dtype], B, m, n, ldg, stride,
          (ctypes.c_float * len(flat))(*flat), steps, eps, scale, out.data_ptr(), ldo, out_stride, _ptr(workspace), nbytes,
          _ptr(flags))
    return out


# ---------------------------------------------------------------------------
# losses with a reference policy
# ---------------------------------------------------------------------------

_KL = {None: _abi.KL_NONE, "k1": _abi.KL_K1, "k2": _abi.KL_K2, "k3": _abi.KL_K3, "exact": _abi.KL_EXACT,
       "reverse": _abi.KL_REVERSE}
_PREF = {"sigmoid": _abi.PREF_SIGMOID, "hinge": _abi.PREF_HINGE, "ipo": _abi.PREF_IPO}


@dataclass
class PolicyLoss:
    grad: torch.Tensor          # bf16 [T, ld] dL/dlogits
    logp: torch.Tensor          # float32 [T] log-prob of the sampled token
    kl: torch.Tensor | None     # float32 [T] the KL term per token (None without one)
    token_loss: torch.Tensor    # float32 [T]
    loss: torch.Tensor          # float32 [1]


def _vec(t, dtype, n, name, dev):
    return torch.empty(n, dtype=dtype, device=dev) if t is None else _need(t, dtype, n, name)


def policy_loss_grad_logits(logits, ids, mask, coef, *, V=None, old_logp=None, clip_low=0.2, clip_high=0.2, dual_clip=0.0,
                            kl=None, kl_coef=None, ref_logits=None, ref_logp=None, grad=None, logp=None, kl_out=None,
                            token_loss=None, loss=None, flags=None, stream=None) -> PolicyLoss:
    """acrl_policy_loss_grad_logits.  `kl` is None, "exact" or "reverse" (with `ref_logits`, bf16 [T, ld_ref]), or "k1",
    "k2" or "k3" (with `ref_logp`, float32 [T]); `kl_coef` float32 [T] its factor per token."""
    T, ld = _rows(logits, "logits")
    if stream is not None:
        return _on_stream(policy_loss_grad_logits, "acrl_policy_loss_grad_logits", logits, stream, logits, ids, mask, coef, V=V,
                          old_logp=old_logp, clip_low=clip_low, clip_high=clip_high, dual_clip=dual_clip, kl=kl,
                          kl_coef=kl_coef, ref_logits=ref_logits, ref_logp=ref_logp, grad=grad, logp=logp, kl_out=kl_out,
                          token_loss=token_loss, loss=loss, flags=flags)
    V = ld if V is None else V
    dev = logits.device
    if kl not in _KL:
        raise AcrlError(f"kl: {kl!r}, expected one of {list(_KL)}")
    full = kl in ("exact", "reverse")
    if full != (ref_logits is not None) or (kl is not None and not full) != (ref_logp is not None):
        raise AcrlError(f"kl={kl!r} takes " + ("ref_logits" if full else "neither ref_logits nor ref_logp" if kl is None
                                                else "ref_logp") + " and no other")
    ldr = 0
    if full:
        Tr, ldr = _rows(ref_logits, "ref_logits")
        if Tr < T or ref_logits.shape[1] < V:
            raise AcrlError(f"ref_logits: shape {tuple(ref_logits.shape)}, needs {(T, V)}")
    _need(ids, torch.int32, T, "ids")
    f32 = torch.float32
    if mask is not None:
        _need(mask, torch.uint8, T, "mask")
    if coef is not None:
        _need(coef, f32, T, "coef")
    if kl_coef is not None:
        _need(kl_coef, f32, T, "kl_coef")
    if old_logp is not None:
        _need(old_logp, f32, T, "old_logp")
    if ref_logp is not None:
        _need(ref_logp, f32, T, "ref_logp")
    if grad is None:
        grad = torch.empty((T, ld), dtype=torch.bfloat16, device=dev)
    elif grad.dtype != torch.bfloat16 or grad.dim() != 2 or grad.stride(0) != ld or grad.stride(1) != 1 or \
            grad.shape[0] < T:
        raise AcrlError("grad: expected a bf16 [T, ld] tensor with the logits' row stride")
    logp, token_loss = _vec(logp, f32, T, "logp", dev), _vec(token_loss, f32, T, "token_loss", dev)
    kl_out = None if kl is None else _vec(kl_out, f32, T, "kl_out", dev)
    loss = _vec(loss, f32, 1, "loss", dev)
    if flags is not None:
        _need(flags, torch.int32, 1, "flags")
    _call("acrl_policy_loss_grad_logits",
          (logits, ids, mask, old_logp, coef, kl_coef, ref_logits, ref_logp, grad, logp, kl_out, token_loss, loss, flags),
          None, logits.data_ptr(), T, V, ld, ids.data_ptr(), None if mask is None else mask.data_ptr(),
          None if old_logp is None else old_logp.data_ptr(), None if coef is None else coef.data_ptr(), clip_low, clip_high,
          dual_clip, _KL[kl], None if kl_coef is None else kl_coef.data_ptr(),
          None if ref_logits is None else ref_logits.data_ptr(), ldr, None if ref_logp is None else ref_logp.data_ptr(),
          grad.data_ptr(), logp.data_ptr(), None if kl_out is None else kl_out.data_ptr(), token_loss.data_ptr(),
          loss.data_ptr(), None if flags is None else flags.data_ptr())
    return PolicyLoss(grad, logp, kl_out, token_loss, loss)


def token_logp(logits, ids, mask=None, *, V=None, lse=None, logp=None, flags=None, stream=None):
    """acrl_token_logp.  Returns (lse, logp) float32 [T]."""
    T, ld = _rows(logits, "logits")
    if stream is not None:
        return _on_stream(token_logp, "acrl_token_logp", logits, stream, logits, ids, mask, V=V, lse=lse, logp=logp, flags=flags)
    V = ld if V is None else V
    _need(ids, torch.int32, T, "ids")
    _opt(mask, torch.uint8, T, "mask")
    lse, logp = (_vec(t, torch.float32, T, name, logits.device) for t, name in ((lse, "lse"), (logp, "logp")))
    _opt(flags, torch.int32, 1, "flags")
    _call("acrl_token_logp", (logits, ids, mask, lse, logp, flags), None, _ptr(logits), T, V, ld, _ptr(ids), _ptr(mask),
          _ptr(lse), _ptr(logp), _ptr(flags))
    return lse, logp


@dataclass
class Preference:
    loss: torch.Tensor     # float32 [1]
    coef: torch.Tensor     # float32 [T] -dL/dlogp
    ratio: torch.Tensor    # float32 [S] log-ratio of each response


def preference_workspace_bytes(S: int, Gn: int) -> int:
    """acrl_preference_workspace_bytes."""
    return int(lib().acrl_preference_workspace_bytes(S, Gn))


def preference_loss(logp, ref_logp, mask, rewards, seq_offsets, group_offsets, *, beta=0.1, form="sigmoid", margin=0.0,
                    label_smoothing=0.0, length_norm=False, ratio=None, coef=None, loss=None, workspace=None, flags=None,
                    stream=None) -> Preference:
    """acrl_preference_loss: pairs of a prompt's responses by their rewards; `form` "sigmoid", "hinge" or "ipo"."""
    T, S, Gn = logp.numel(), seq_offsets.numel() - 1, group_offsets.numel() - 1
    f32, dev = torch.float32, logp.device
    if stream is not None:
        return _on_stream(preference_loss, "acrl_preference_loss", logp, stream, logp, ref_logp, mask, rewards, seq_offsets,
                          group_offsets, beta=beta, form=form, margin=margin, label_smoothing=label_smoothing,
                          length_norm=length_norm, ratio=ratio, coef=coef, loss=loss, workspace=workspace, flags=flags)
    if form not in _PREF:
        raise AcrlError(f"form: {form!r}, expected one of {list(_PREF)}")
    if S < 0 or Gn < 0:
        raise AcrlError("seq_offsets / group_offsets: empty")
    _need(logp, f32, T, "logp")
    _opt(ref_logp, f32, T, "ref_logp")
    _opt(mask, torch.uint8, T, "mask")
    _need(rewards, f32, S, "rewards")
    _need(seq_offsets, torch.int64, S + 1, "seq_offsets")
    _need(group_offsets, torch.int32, Gn + 1, "group_offsets")
    ratio, coef, loss = _vec(ratio, f32, S, "ratio", dev), _vec(coef, f32, T, "coef", dev), _vec(loss, f32, 1, "loss", dev)
    n = lib().acrl_preference_workspace_bytes(S, Gn)
    workspace = _vec(workspace, torch.uint8, n, "workspace", dev)
    if flags is not None:
        _need(flags, torch.int32, 1, "flags")
    _call("acrl_preference_loss",
          (logp, ref_logp, mask, rewards, seq_offsets, group_offsets, ratio, coef, loss, workspace, flags), None,
          logp.data_ptr(), None if ref_logp is None else ref_logp.data_ptr(), None if mask is None else mask.data_ptr(), T,
          rewards.data_ptr(), seq_offsets.data_ptr(), S, group_offsets.data_ptr(), Gn, _PREF[form], beta, margin,
          label_smoothing, int(length_norm), ratio.data_ptr(), coef.data_ptr(), loss.data_ptr(), workspace.data_ptr(), n,
          None if flags is None else flags.data_ptr())
    return Preference(loss, coef, ratio)


def preference_step_workspace_bytes(T: int, S: int, Gn: int) -> int:
    """acrl_preference_step_workspace_bytes."""
    return int(lib().acrl_preference_step_workspace_bytes(T, S, Gn))


def preference_step(logits, ids, mask, ref_logp, rewards, seq_offsets, group_offsets, *, V, lse, logp, ratio, coef, grad, loss,
                    workspace, flags, beta=0.1, form="sigmoid", margin=0.0, label_smoothing=0.0, length_norm=False,
                    stream=None) -> None:
    """acrl_preference_step, into the caller's buffers."""
    T, ld = _rows(logits, "logits")
    S, Gn = seq_offsets.numel() - 1, group_offsets.numel() - 1
    f32 = torch.float32
    if form not in _PREF:
        raise AcrlError(f"form: {form!r}, expected one of {list(_PREF)}")
    _need(ids, torch.int32, T, "ids")
    if mask is not None:
        _need(mask, torch.uint8, T, "mask")
    if ref_logp is not None:
        _need(ref_logp, f32, T, "ref_logp")
    _need(rewards, f32, S, "rewards")
    _need(seq_offsets, torch.int64, S + 1, "seq_offsets")
    _need(group_offsets, torch.int32, Gn + 1, "group_offsets")
    for name, t, n in (("lse", lse, T), ("logp", logp, T), ("ratio", ratio, S), ("coef", coef, T), ("loss", loss, 1)):
        _need(t, f32, n, name)
    if grad.dtype != torch.bfloat16 or grad.dim() != 2 or grad.stride(0) != ld or grad.stride(1) != 1 or grad.shape[0] < T:
        raise AcrlError("grad: expected a bf16 [T, ld] tensor with the logits' row stride")
    _need(flags, torch.int32, 1, "flags")
    _need(workspace, torch.uint8, None, "workspace")
    _call("acrl_preference_step", (logits, ids, mask, ref_logp, rewards, seq_offsets, group_offsets, lse, logp, ratio, coef, grad,
                                   loss, workspace, flags), stream,
          logits.data_ptr(), T, V, ld, ids.data_ptr(), None if mask is None else mask.data_ptr(),
          None if ref_logp is None else ref_logp.data_ptr(), rewards.data_ptr(), seq_offsets.data_ptr(), S,
          group_offsets.data_ptr(), Gn, _PREF[form], beta, margin, label_smoothing, int(length_norm), lse.data_ptr(),
          logp.data_ptr(), ratio.data_ptr(), coef.data_ptr(), grad.data_ptr(), loss.data_ptr(), workspace.data_ptr(),
          workspace.numel(), flags.data_ptr())


def selftest_wait_timeout(flags, limit_ns: int, stream=None) -> None:
    """acrl_selftest_wait_timeout: a bounded wait on a barrier nothing arrives on."""
    _need(flags, torch.int32, 1, "flags")
    _call("acrl_selftest_wait_timeout", (flags,), stream, _ptr(flags), int(limit_ns))


def controller_save(state: torch.Tensor, stream=None) -> bytes:
    """acrl_controller_save (the same as save_state)."""
    return save_state(state, stream)


def controller_load(blob: bytes, state: torch.Tensor | None = None, device=None, stream=None) -> torch.Tensor:
    """acrl_controller_load (the same as load_state)."""
    return load_state(blob, state, device, stream)


# The host-buffer pipeline at the level of its handle (pipeline.HostPipeline wraps these).
def host_pipeline_workspace_bytes(T: int, ld: int, S: int, Gn: int, chunks: int) -> int:
    """acrl_host_pipeline_workspace_bytes (-1 for an invalid shape)."""
    return int(lib().acrl_host_pipeline_workspace_bytes(T, ld, S, Gn, chunks))


def host_pipeline_create(T: int, V: int, ld: int, S: int, Gn: int, chunks: int, workspace: torch.Tensor):
    """acrl_host_pipeline_create on a device workspace tensor (on its device).  Returns the handle."""
    _need(workspace, torch.uint8, max(0, host_pipeline_workspace_bytes(T, ld, S, Gn, chunks)), "workspace")
    handle = ctypes.c_void_p()
    with torch.cuda.device(_one_device((workspace,))):
        check(lib().acrl_host_pipeline_create(ctypes.byref(handle), T, V, ld, S, Gn, chunks, workspace.data_ptr(),
                                              workspace.numel()), "acrl_host_pipeline_create")
    return handle


def host_pipeline_step(handle, params: Params, state, logits, ids, mask, logp_mu, rewards, seq_offsets, group_offsets,
                       grad, loss, flags, stream) -> None:
    """acrl_host_pipeline_step; host arrays as raw addresses (int), device ones as tensors."""
    check(lib().acrl_host_pipeline_step(handle, ctypes.byref(params), _ptr(state), logits, ids, mask, logp_mu,
                                        rewards, seq_offsets, group_offsets, grad, loss, _ptr(flags),
                                        stream.cuda_stream), "acrl_host_pipeline_step")


def host_pipeline_begin(handle, logits, ids, mask, logp_mu, rewards, seq_offsets, group_offsets, flags,
                        stream) -> None:
    """acrl_host_pipeline_begin; host arrays as raw addresses (int)."""
    check(lib().acrl_host_pipeline_begin(handle, logits, ids, mask, logp_mu, rewards, seq_offsets, group_offsets,
                                         _ptr(flags), stream.cuda_stream), "acrl_host_pipeline_begin")


def host_pipeline_finish(handle, params: Params, state, grad, loss, flags, stream) -> None:
    """acrl_host_pipeline_finish; the host gradient and loss as raw addresses (int)."""
    check(lib().acrl_host_pipeline_finish(handle, ctypes.byref(params), _ptr(state), grad, loss, _ptr(flags),
                                          stream.cuda_stream), "acrl_host_pipeline_finish")


def host_pipeline_batch_stats(handle) -> int:
    """acrl_host_pipeline_batch_stats: the device address of the pipeline's batch statistics."""
    return int(lib().acrl_host_pipeline_batch_stats(handle) or 0)


def host_pipeline_destroy(handle) -> None:
    """acrl_host_pipeline_destroy."""
    check(lib().acrl_host_pipeline_destroy(handle), "acrl_host_pipeline_destroy")


def abi_version() -> int:
    """acrl_abi_version."""
    return int(lib().acrl_abi_version())


def status_string(status: int) -> str:
    """acrl_status_string."""
    return lib().acrl_status_string(status).decode()


def struct_size(which: int) -> int:
    """acrl_struct_size."""
    return int(lib().acrl_struct_size(which))


def read_flags(flags, stream=None) -> int:
    """acrl_read_flags (synchronises the stream)."""
    host = ctypes.c_int32(0)
    _need(flags, torch.int32, 1, "flags")
    _call("acrl_read_flags", (flags,), stream, _ptr(flags), ctypes.byref(host))
    return int(host.value)


def check_flags(flags, stream=None) -> None:
    """acrl_check_flags: synchronises the stream and raises AcrlError (naming
    the bits) if any device flag is set."""
    _need(flags, torch.int32, 1, "flags")
    dev = _one_device((flags,))
    with torch.cuda.device(dev):
        s = torch.cuda.current_stream(dev) if stream is None else stream
        st = lib().acrl_check_flags(_ptr(flags), s.cuda_stream)
    if st == _abi.ERR_DEVICE_FLAGS:
        raise AcrlError(f"device flags raised: 0x{read_flags(flags, stream):x}")
    check(st, "acrl_check_flags")


__all__ = ["Params", "AcrlError", "token_stats", "seq_discrepancy", "grpo_advantage", "controller_init",
           "controller_step", "importance_weights", "step", "loss_grad_logits", "reduce_loss", "scale_grad",
           "read_flags", "check_flags", "read_state", "Discrepancy",
           "PolicyLoss", "policy_loss_grad_logits", "token_logp", "Preference", "preference_loss", "preference_workspace_bytes",
           "preference_step", "preference_step_workspace_bytes",
           "Fp8Tensor", "fp8_quantize", "fp8_matmul", "fp8_linear", "fp8_linear_backward", "fp8_linear_workspace_bytes",
           "fp8_linear_backward_workspace_bytes",
           "lmhead_logits_stats", "lmhead_merge", "lmhead_workspace_bytes", "lmhead_stats_noalloc", "save_state",
           "load_state", "controller_save", "controller_load", "selftest_wait_timeout",
           "host_pipeline_workspace_bytes", "host_pipeline_create", "host_pipeline_step", "host_pipeline_begin",
           "host_pipeline_finish", "host_pipeline_batch_stats", "host_pipeline_destroy", "abi_version",
           "status_string", "struct_size", "struct_buffer", "read_structs", "new_flags", "_abi"]
