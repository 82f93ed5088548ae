"""Torch plumbing for the head of the sequence tower: the norm of the residual stream, log probabilities of given items under a softmax over
the catalogue, and the loss against a larger tower's best items.  As in `sequence`, nothing here computes anything on its own: every step is a
call into libmtrains_b200.so on torch's current stream of the tensors' device.  First derivatives only (torch raises where others are asked for).
Calls may be captured into CUDA graphs; a backward pass is captured while no autograd graph of an eager pass over the same leaves is alive, as torch
wants it."""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as mb
from .sequence import KIND, _kind, _rows, _same_device, _stride


def _matrix(t: torch.Tensor, what: str) -> int:
    if t.dim() != 2:
        raise ValueError(f"{what} {tuple(t.shape)}: two dimensions")
    return _kind(t, what)


def _vector(t: Optional[torch.Tensor], n: int, dtype: torch.dtype, device: torch.device, what: str) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if t.dtype != dtype or tuple(t.shape) != (n,):
        raise ValueError(f"{what}: {dtype} {(n,)}, not {t.dtype} {tuple(t.shape)}")
    _same_device(t, device, what)
    return t.contiguous()


# ---------------------------------------------------------------------------- norm
def _check_norm(x, weight, residual):
    _matrix(x, "x")
    if weight.dim() != 1 or weight.shape[0] != x.shape[1]:
        raise ValueError(f"weight {tuple(weight.shape)}: one for each of {x.shape[1]} columns")
    _kind(weight, "weight")
    _same_device(weight, x.device, "weight")
    if residual is not None:
        if residual.shape != x.shape or residual.dtype != x.dtype:
            raise ValueError(f"x {tuple(x.shape)} {x.dtype} and residual {tuple(residual.shape)} {residual.dtype} must be alike, [N, D]")
        _same_device(residual, x.device, "residual")


class _RMSNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        _check_norm(x, weight, residual)
        x, weight, residual = _rows(x), weight.contiguous(), None if residual is None else _rows(residual)
        (N, D), kind = x.shape, KIND[x.dtype]
        out = torch.empty(N, D, dtype=x.dtype, device=x.device)
        total = None if residual is None else torch.empty_like(out)
        inv = torch.empty(N, dtype=torch.float32, device=x.device) if any(ctx.needs_input_grad) else None
        with torch.cuda.device(x.device):
            mb.rms_norm_forward(x, _stride(x), residual, 0 if residual is None else _stride(residual), weight, KIND[weight.dtype], kind, N, D, eps,
                                total, D, out, D, inv, torch.cuda.current_stream(x.device))
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x if total is None else total, weight, inv)
        return out if total is None else (out, total)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad, grad_total=None):
        x, weight, inv = ctx.saved_tensors
        if grad is None:                     # the norm's output is not used: what reaches the sum goes on as it is
            has_residual = ctx.needs_input_grad[2]
            return grad_total, None, grad_total if has_residual else None, None
        grad, grad_total = _rows(grad), None if grad_total is None else _rows(grad_total)
        (N, D), kind = x.shape, KIND[x.dtype]
        dx = torch.empty(N, D, dtype=x.dtype, device=x.device)
        dw = torch.empty(D, dtype=torch.float32, device=x.device) if ctx.needs_input_grad[1] else None
        ws = None if dw is None else torch.empty(mb.rms_norm_workspace_bytes(N, D), dtype=torch.uint8, device=x.device)
        with torch.cuda.device(x.device):
            mb.rms_norm_backward(x, _stride(x), weight, KIND[weight.dtype], kind, N, D, inv, grad, _stride(grad), grad_total,
                                 0 if grad_total is None else _stride(grad_total), dx, D, dw, ws, 0 if ws is None else ws.numel(),
                                 torch.cuda.current_stream(x.device))
        return (dx if ctx.needs_input_grad[0] else None, None if dw is None else dw.to(weight.dtype), dx if ctx.needs_input_grad[2] else None,
                None)


def rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6):
    """x / sqrt(mean x^2 + eps) * weight over the rows of [N, D]; with a residual (norm of x + residual, x + residual): the sum is the stream
    that goes on to the next layer, rounded to the tensors' type before it is normalised."""
    return _RMSNorm.apply(x, weight, residual, eps)


def rms_norm_8bit(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6, group: int = 0):
    """The same with the norm in 8 bits: (codes float8_e4m3fn [N, D], scales fp32 [N, groups][, x + residual]); `group` columns (32, 64, 128,
    256; 0: the row) share a scale, and codes * scales are the values.  For serving: no gradient, and inputs that ask for one are refused."""
    _check_norm(x, weight, residual)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, residual)):
        raise ValueError("the norm in 8 bits has no gradient: call it under torch.no_grad(), or rms_norm")
    x, weight, residual = _rows(x), weight.contiguous(), None if residual is None else _rows(residual)
    (N, D), kind = x.shape, KIND[x.dtype]
    codes = torch.empty(N, D, dtype=torch.float8_e4m3fn, device=x.device)
    scales = torch.empty(N, -(-D // group) if group > 0 else 1, dtype=torch.float32, device=x.device)
    total = None if residual is None else torch.empty(N, D, dtype=x.dtype, device=x.device)
    with torch.cuda.device(x.device):
        mb.rms_norm_forward_8bit(x, _stride(x), residual, 0 if residual is None else _stride(residual), weight, KIND[weight.dtype], kind, N, D, eps,
                                 total, D, codes, D, scales, group, None, torch.cuda.current_stream(x.device))
    return (codes, scales) if total is None else (codes, scales, total)


def rows_from_8bit(codes: torch.Tensor, scales: torch.Tensor, group: int = 0, dtype: torch.dtype = torch.bfloat16):
    """The values of codes and scales of rms_norm_8bit, [N, D] of `dtype`."""
    if codes.dtype != torch.float8_e4m3fn or codes.dim() != 2 or not codes.is_cuda:
        raise ValueError(f"codes: float8_e4m3fn [N, D] on the GPU, not {codes.dtype} {tuple(codes.shape)}")
    if dtype not in KIND:
        raise TypeError(f"values: {dtype} (fp32, fp16 or bf16)")
    N, D = codes.shape
    want = (N, -(-D // group) if group > 0 else 1)
    if scales.dtype != torch.float32 or tuple(scales.shape) != want:
        raise ValueError(f"scales: fp32 {want}, not {scales.dtype} {tuple(scales.shape)}")
    _same_device(scales, codes.device, "scales")
    codes, scales = _rows(codes), scales.contiguous()
    out = torch.empty(N, D, dtype=dtype, device=codes.device)
    with torch.cuda.device(codes.device):
        mb.rows_from_8bit(codes, _stride(codes), scales, group, N, D, out, KIND[dtype], D, torch.cuda.current_stream(codes.device))
    return out


# ---------------------------------------------------------------------------- log probabilities
class LogProbs(NamedTuple):
    logp: Optional[torch.Tensor]          # fp32 [N], None without targets
    entropy: torch.Tensor                 # fp32 [N]
    top_index: Optional[torch.Tensor]     # int64 [N, top_k], None where top_k is 0
    top_logp: Optional[torch.Tensor]      # fp32 [N, top_k], without a gradient


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, top_k, scale):
        kind, (N, V), dev = _matrix(logits, "logits"), logits.shape, logits.device
        targets = _vector(targets, N, torch.int64, dev, "targets")
        logits = _rows(logits)
        new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device=dev)  # noqa: E731
        logp = None if targets is None else new(N)
        entropy, stats = new(N), new(N, 2) if ctx.needs_input_grad[0] else None
        top_index, top_logp = (new(N, top_k, dtype=torch.int64), new(N, top_k)) if top_k > 0 else (None, None)
        with torch.cuda.device(dev):
            mb.logprobs_forward(logits, _stride(logits), kind, N, V, scale, targets, top_k, logp, entropy, stats, top_index, top_logp,
                                torch.cuda.current_stream(dev))
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, targets, stats, entropy)
        if top_k > 0:
            ctx.mark_non_differentiable(top_index, top_logp)
        return logp, entropy, top_index, top_logp

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_logp, grad_entropy, *_):
        logits, targets, stats, entropy = ctx.saved_tensors
        if grad_logp is None and grad_entropy is None:
            return None, None, None, None
        (N, V), dev = logits.shape, logits.device
        grad_logp, grad_entropy = (None if g is None else g.contiguous() for g in (grad_logp, grad_entropy))
        out = torch.empty(N, V, dtype=logits.dtype, device=dev)
        with torch.cuda.device(dev):
            mb.logprobs_backward(logits, _stride(logits), KIND[logits.dtype], N, V, ctx.scale, targets, stats, entropy, grad_logp, grad_entropy,
                                 out, V, torch.cuda.current_stream(dev))
        return out, None, None, None


def log_probs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, top_k: int = 0, scale: float = 1.0) -> LogProbs:
    """Under softmax(scale * logits) over the rows of [N, V]: log probability of targets (int64 [N]; negative: none, 0), entropy, the top_k
    best items (lowest index first among equals) and their log probabilities.  Differentiable in logits through logp and entropy.  Items are ruled out
    by -infinity.  Targets are on the GPU and are not looked at: one that is >= V gives NaN."""
    return LogProbs(*_LogProbs.apply(logits, targets, top_k, scale))


# ---------------------------------------------------------------------------- distillation
def _distill(logits, index, teacher_logits, rest, weights, scale, loss, grad):
    (N, V), dev = logits.shape, logits.device
    with torch.cuda.device(dev):
        mb.distill_loss(logits, _stride(logits), KIND[logits.dtype], N, V, scale, index, teacher_logits, KIND[teacher_logits.dtype], index.shape[1],
                        rest, weights, loss, grad, V, torch.cuda.current_stream(dev))


def _check_teacher(logits, index, teacher_logits, rest):
    _matrix(logits, "logits")
    N, dev = logits.shape[0], logits.device
    if index.dtype != torch.int64 or index.dim() != 2 or index.shape[0] != N:
        raise ValueError(f"index: int64 [{N}, K], not {index.dtype} {tuple(index.shape)}")
    _matrix(teacher_logits, "teacher_logits")
    if teacher_logits.shape != index.shape:
        raise ValueError(f"teacher_logits {tuple(teacher_logits.shape)}: as many as index {tuple(index.shape)}")
    _same_device(index, dev, "index")
    _same_device(teacher_logits, dev, "teacher_logits")
    if any(t is not None and t.requires_grad for t in (teacher_logits, rest)):
        raise ValueError("the teacher's scores get no gradient: detach them")
    return _rows(logits), index.contiguous(), teacher_logits.contiguous(), _vector(rest, N, torch.float32, dev, "rest")


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, index, teacher_logits, rest, scale):
        logits, index, teacher_logits, rest = _check_teacher(logits, index, teacher_logits, rest)
        loss = torch.empty(logits.shape[0], dtype=torch.float32, device=logits.device)
        _distill(logits, index, teacher_logits, rest, None, scale, loss, None)
        ctx.scale = scale
        ctx.save_for_backward(logits, index, teacher_logits, rest)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        logits, index, teacher_logits, rest = ctx.saved_tensors
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        _distill(logits, index, teacher_logits, rest, grad.contiguous(), ctx.scale, None, out)
        return out, None, None, None, None


def distill_loss(logits: torch.Tensor, index: torch.Tensor, teacher_logits: torch.Tensor, rest: Optional[torch.Tensor] = None, scale: float = 1.0):
    """Loss fp32 [N] of a student's scores [N, V] against the best K items of a teacher (index int64, teacher_logits [N, K]; negative index: place
    not used): the Kullback-Leibler divergence of softmax(scale * logits) from the teacher's distribution over those items, and over one more place for
    all others where `rest` (fp32 [N], log of the sum of exp(scale * t) over them) is given.  No factor 1 / scale^2.  Indices are on the GPU and are not
    looked at: one that is >= V gives NaN."""
    return _DistillLoss.apply(logits, index, teacher_logits, rest, scale)


@torch.no_grad()
def distill_loss_and_grad(logits: torch.Tensor, index: torch.Tensor, teacher_logits: torch.Tensor, rest: Optional[torch.Tensor] = None,
                          weights: Optional[torch.Tensor] = None, scale: float = 1.0):
    """(loss fp32 [N], gradient of sum(weights * loss) in logits) in one pass over the scores, where distill_loss reads them once for the loss and
    once more for its gradient.  For `hidden @ items` use it as `loss, g = distill_loss_and_grad(scores.detach(), ...); scores.backward(g)`."""
    logits, index, teacher_logits, rest = _check_teacher(logits, index, teacher_logits, rest)
    weights = _vector(weights, logits.shape[0], torch.float32, logits.device, "weights")
    loss = torch.empty(logits.shape[0], dtype=torch.float32, device=logits.device)
    grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _distill(logits, index, teacher_logits, rest, weights, scale, loss, grad)
    return loss, grad
