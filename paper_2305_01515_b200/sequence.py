"""Torch plumbing for the sequence tower beside the tables: the gated recurrence and the relative position bias as
differentiable functions, AdamW over a list of parameters.  Nothing here computes anything on its own; every step is a call into
libmtrains_b200.so on torch's current stream of the tensors' device."""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch
from torch.autograd.function import once_differentiable

from . import binding as mb

KIND = {torch.float32: mb.DTYPE_FP32, torch.float16: mb.DTYPE_FP16, torch.bfloat16: mb.DTYPE_BF16}


def _kind(t: torch.Tensor, what: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if t.dtype not in KIND:
        raise TypeError(f"{what}: {t.dtype} (fp32, fp16 or bf16)")
    return KIND[t.dtype]


def _same_device(t: torch.Tensor, device: torch.device, what: str) -> None:
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, not on {device}")


def _rows(t: torch.Tensor) -> torch.Tensor:
    """An [N, D] tensor whose channels are contiguous and whose rows do not overlap (a column range of a wider one is)."""
    return t if t.stride(1) == 1 and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]) else t.contiguous()


def _stride(t: torch.Tensor) -> int:
    return max(t.stride(0), t.shape[1])


def _check_status(workspace: torch.Tensor) -> None:
    """Waits for the call that used this workspace; offsets out of order or range raise, a wait that ran out does in the binding."""
    with torch.cuda.device(workspace.device):
        if mb.recurrence_status(workspace, torch.cuda.current_stream(workspace.device)):
            raise ValueError("offsets do not run from 0 to N in order: the rows that they leave out hold nothing")


class _GatedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, value, offsets, h0, check):
        if gate.dim() != 2 or gate.shape != value.shape or gate.dtype != value.dtype:
            raise ValueError(f"gate {tuple(gate.shape)} {gate.dtype} and value {tuple(value.shape)} {value.dtype} must be alike, [N, D]")
        if offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_cuda or not offsets.is_contiguous():
            raise ValueError("offsets: contiguous int64 [S + 1] on the GPU")
        N, D, S = gate.shape[0], gate.shape[1], offsets.numel() - 1
        kind = _kind(gate, "gate")
        for t, what in ((value, "value"), (offsets, "offsets"), (h0, "h0")):
            if t is not None:
                _same_device(t, gate.device, what)
        if h0 is not None and (h0.dtype != torch.float32 or tuple(h0.shape) != (S, D)):
            raise ValueError(f"h0: fp32 {(S, D)}, not {h0.dtype} {tuple(h0.shape)}")
        gate, value, h0 = _rows(gate), _rows(value), None if h0 is None else h0.contiguous()
        out = torch.empty(N, D, dtype=gate.dtype, device=gate.device)
        final = torch.empty(S, D, dtype=torch.float32, device=gate.device)
        need = any(ctx.needs_input_grad)
        entry = torch.empty(mb.recurrence_chunks(N, D, kind), D, dtype=torch.float32, device=gate.device) if need else None
        ws = torch.empty(mb.recurrence_workspace_bytes(N, S, D, kind), dtype=torch.uint8, device=gate.device)
        with torch.cuda.device(gate.device):
            mb.recurrence_forward(gate, _stride(gate), value, _stride(value), kind, N, D, offsets, S, h0, out, D, final, entry, ws,
                                  ws.numel(), torch.cuda.current_stream(gate.device))
        if check:
            _check_status(ws)
        ctx.check = check
        ctx.save_for_backward(gate, value, offsets, h0, entry)
        return out, final

    @staticmethod
    @once_differentiable                     # a second derivative has no kernel: torch raises where one is asked for
    def backward(ctx, grad_out, grad_final):
        gate, value, offsets, h0, entry = ctx.saved_tensors
        N, D, S, kind = gate.shape[0], gate.shape[1], offsets.numel() - 1, KIND[gate.dtype]
        grad_out, grad_final = _rows(grad_out), grad_final.contiguous()
        d_gate, d_value = (torch.empty(N, D, dtype=gate.dtype, device=gate.device) for _ in range(2))
        d_h0 = torch.empty(S, D, dtype=torch.float32, device=gate.device) if h0 is not None else None
        ws = torch.empty(mb.recurrence_workspace_bytes(N, S, D, kind), dtype=torch.uint8, device=gate.device)
        with torch.cuda.device(gate.device):
            mb.recurrence_backward(gate, _stride(gate), value, _stride(value), kind, N, D, offsets, S, h0, entry, grad_out, _stride(grad_out),
                                   grad_final, d_gate, D, d_value, D, d_h0, ws, ws.numel(), torch.cuda.current_stream(gate.device))
        if ctx.check:
            _check_status(ws)
        return d_gate, d_value, None, d_h0, None


def gated_recurrence(gate: torch.Tensor, value: torch.Tensor, offsets: torch.Tensor, h0: Optional[torch.Tensor] = None, check: bool = False):
    """h_t = h_{t-1} + sigmoid(gate_t) (value_t - h_{t-1}) over packed sequences: (h [N, D], state after each sequence fp32 [S, D]).
    First derivatives only.  The offsets are on the GPU and are trusted: they have to run from 0 to N in order, else rows of the results are
    undefined.  check: wait for the call, and for its backward, and raise where they do not."""
    return _GatedRecurrence.apply(gate, value, offsets, h0, check)


def log_bucket_starts(n: int, far: int) -> List[int]:
    """First distances of n buckets: half of them hold one distance each, the others grow evenly in the logarithm, the last begins at
    `far`.  In whole numbers, so that no rounded logarithm moves a border.  A spacing of its own: the common formula, which cuts the
    logarithm up to `far` into n / 2 parts, has its last bucket begin before `far` (32 buckets up to 128: 16, 19, 21, 24, 27, 31, ..., 99, 113, here
    16, 19, 22, 25, 28, 32, ..., 112, 128).  A table trained with other buckets needs their starts, which RelposBuckets takes as they are."""
    exact = max(n // 2, 1)
    if far < exact:
        raise ValueError(f"the last of {n} buckets cannot begin at {far}")
    starts, p = list(range(exact)), max(n - exact - 1, 1)
    for k in range(n - exact):               # the smallest d with (d / exact)^p >= (far / exact)^k
        lo, hi = exact, far
        while lo < hi:
            mid = (lo + hi) // 2
            lo, hi = (lo, mid) if mid ** p * exact ** k >= far ** k * exact ** p else (mid + 1, hi)
        starts.append(lo)
    return starts


def _bias(table, buckets, Lq, Lk, q_offset, dtype):
    kind = _kind(table, "table")
    if dtype not in KIND:
        raise TypeError(f"bias: {dtype} (fp32, fp16 or bf16)")
    if table.dim() != 2 or table.shape[0] != buckets.rows:
        raise ValueError(f"table {tuple(table.shape)}: one row for each of {buckets.rows} buckets")
    table, H = table.contiguous(), table.shape[1]
    out = torch.empty(H, Lq, Lk, dtype=dtype, device=table.device)
    with torch.cuda.device(table.device):
        mb.relpos_bias_forward(buckets, table, kind, H, Lq, Lk, q_offset, out, KIND[dtype], Lq * Lk, Lk, torch.cuda.current_stream(table.device))
    return out


def _table_gradient(buckets, grad, q_offset):
    grad = grad if grad.stride(3) == 1 and min(grad.stride()) >= 0 else grad.contiguous()
    B, H, Lq, Lk = grad.shape
    out = torch.empty(buckets.rows, H, dtype=torch.float32, device=grad.device)
    ws = torch.empty(mb.relpos_bias_workspace_bytes(buckets, H), dtype=torch.uint8, device=grad.device)
    with torch.cuda.device(grad.device):
        mb.relpos_bias_backward(buckets, grad, _kind(grad, "gradient"), B, H, Lq, Lk, q_offset, *grad.stride()[:3], out, ws, ws.numel(),
                                torch.cuda.current_stream(grad.device))
    return out


class _RelposBias(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, buckets, Lq, Lk, q_offset, dtype):
        ctx.args = (buckets, q_offset, table.dtype)
        return _bias(table, buckets, Lq, Lk, q_offset, dtype)

    @staticmethod
    def backward(ctx, grad):
        buckets, q_offset, dtype = ctx.args
        return _gradient_of_table(grad.unsqueeze(0), buckets, q_offset).to(dtype), None, None, None, None, None


class _TableGradient(torch.autograd.Function):
    """Linear in the gradient of the scores, so that its own derivative is the bias again, with 0 where keys are masked."""

    @staticmethod
    def forward(ctx, grad, buckets, q_offset):
        ctx.args = (buckets, q_offset, grad.shape, grad.dtype)
        return _table_gradient(buckets, grad, q_offset)

    @staticmethod
    def backward(ctx, way):
        buckets, q_offset, shape, dtype = ctx.args
        bias = _RelposBias.apply(way, buckets.without_mask(), shape[2], shape[3], q_offset, dtype)
        return (bias.tril(q_offset) if buckets.desc.causal else bias).expand(shape), None, None


def _gradient_of_table(grad, buckets, q_offset):
    """With a graph of its own only where a second derivative may be asked for: the graph's node costs 10 us a call."""
    return _TableGradient.apply(grad, buckets, q_offset) if torch.is_grad_enabled() else _table_gradient(buckets, grad, q_offset)


def relpos_bias(table: torch.Tensor, buckets: mb.RelposBuckets, Lq: int, Lk: int, q_offset: int = 0, dtype: torch.dtype = torch.float32):
    """The bias [H, Lq, Lk] of attention scores from a table [buckets.rows, H]."""
    return _RelposBias.apply(table, buckets, Lq, Lk, q_offset, dtype)


class _AddRelposBias(torch.autograd.Function):
    @staticmethod
    def forward(ctx, scores, table, buckets, q_offset):
        if scores.dim() != 4:
            raise ValueError(f"scores {tuple(scores.shape)}: [B, H, Lq, Lk]")
        _same_device(scores, table.device, "scores")
        ctx.args = (buckets, q_offset, table.dtype)
        return scores + _bias(table, buckets, scores.shape[2], scores.shape[3], q_offset, scores.dtype)

    @staticmethod
    def backward(ctx, grad):
        buckets, q_offset, dtype = ctx.args
        return grad, _gradient_of_table(grad, buckets, q_offset).to(dtype), None, None


def add_relpos_bias(scores: torch.Tensor, table: torch.Tensor, buckets: mb.RelposBuckets, q_offset: int = 0):
    """scores [B, H, Lq, Lk] + the bias that the batch shares; the table's gradient is summed over the batch in one pass over the scores'."""
    return _AddRelposBias.apply(scores, table, buckets, q_offset)


class AdamW:
    """AdamW over a list of parameters in one launch a step; the gradients are p.grad at the time of the step.  state_bits: 32 or 8; masters:
    keep fp32 copies of 16-bit parameters.  Tensors of one dimension (biases, scales) take no weight decay.  A parameter whose storage was
    replaced by another of its size and type (p.data = ..., module.to(...)) is found at the next step and updated where it is then."""

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 state_bits: int = 32, masters: bool = False):
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        self._kind, self._dtype, self._device = _kind(self.params[0], "parameters"), self.params[0].dtype, self.params[0].device
        self._sizes, self._state_bits = [p.numel() for p in self.params], state_bits
        self._check_params()
        self.lr, self.betas, self.eps, self.weight_decay, self.steps = lr, betas, eps, weight_decay, 0
        for p in self.params:
            if p.grad is None:
                p.grad = torch.zeros_like(p)
        self.masters = [p.detach().float() for p in self.params] if masters else None
        self._make_handle([p.grad for p in self.params])
        self.state = torch.zeros(self.handle.state_bytes, dtype=torch.uint8, device=self._device)

    def _check_params(self) -> None:
        for k, (p, n) in enumerate(zip(self.params, self._sizes)):
            if p.dtype is not self._dtype or p.numel() != n or not p.is_contiguous():
                raise ValueError(f"parameter {k}: parameters are contiguous, of one type, and keep their sizes")
            _same_device(p, self._device, f"parameter {k}")
        spans = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()) for p in self.params if p.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("a parameter is given twice, or two of them share memory")

    def _make_handle(self, grads: List[torch.Tensor]) -> None:
        with torch.cuda.device(self._device):
            self.handle = mb.AdamW(self._sizes, self._kind, self._kind, self._state_bits, [p.detach() for p in self.params], grads, self.masters,
                                   decays=[p.dim() > 1 for p in self.params])
        self._grads = grads                                 # the handle holds their addresses: they stay until it has others
        self._param_at, self._grad_at = [p.data_ptr() for p in self.params], [g.data_ptr() for g in grads]

    @torch.no_grad()
    def refresh_masters(self) -> None:
        """After new values were written into the parameters (loaded weights): a master that does not round to its parameter takes its value."""
        for p, m in zip(self.params, self.masters or []):
            m.copy_(torch.where(m.to(p.dtype) == p, m, p.float()))

    @torch.no_grad()
    def step(self, grad_scale: Optional[torch.Tensor] = None) -> None:
        grads = [p.grad for p in self.params]
        for g, n in zip(grads, self._sizes):
            if g is None or g.dtype is not self._dtype or g.numel() != n or not g.is_contiguous():
                raise ValueError("every parameter needs a contiguous gradient of its own type")
        # the handle holds addresses: what lies elsewhere now is looked at and handed over
        param_at, grad_at = [p.data_ptr() for p in self.params], [g.data_ptr() for g in grads]
        moved, renewed = param_at != self._param_at, grad_at != self._grad_at
        if moved:
            self._check_params()
        if renewed and {g.get_device() for g in grads} != {self._device.index}:
            raise ValueError(f"a gradient is not on {self._device}")
        if grad_scale is not None:
            if grad_scale.dtype != torch.float32 or grad_scale.numel() != 1:
                raise ValueError(f"grad_scale: one fp32 number, not {grad_scale.dtype} {tuple(grad_scale.shape)}")
            _same_device(grad_scale, self._device, "grad_scale")
        stream = torch.cuda.current_stream(self._device)
        if moved:
            torch.cuda.synchronize(self._device)            # steps that still use the old description
            self.refresh_masters()
            self._make_handle(grads)
        with torch.cuda.device(self._device):
            if renewed:
                mb.adamw_set_grads(self.handle, grad_at, stream)
            self._grads, self._grad_at = grads, grad_at
            mb.adamw_step(self.handle, self.state, self.lr, *self.betas, self.eps, self.weight_decay, self.steps + 1, grad_scale, self.steps + 1, stream)
        self.steps += 1

    def zero_grad(self) -> None:
        for p in self.params:
            if p.grad is not None:
                p.grad.zero_()
