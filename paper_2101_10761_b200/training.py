"""A linear layer whose three products are 4-bit, and the optimiser step on the averaged gradient.

Thin ``torch`` plumbing around :mod:`binding` (buffers, autograd bookkeeping); all arithmetic on matrices runs in the
library's kernels.
"""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import binding as B

Quantized = Tuple[torch.Tensor, torch.Tensor]


def _buffers(rows: int, cols: int, device) -> Quantized:
    return (torch.empty(B.sidco_mx4_code_bytes(rows, cols), dtype=torch.uint8, device=device),
            torch.empty(B.sidco_mx4_scale_bytes(rows, cols), dtype=torch.uint8, device=device))


def quantize(x: torch.Tensor, rowwise: bool = True, transposed: bool = True
             ) -> Tuple[Optional[Quantized], Optional[Quantized]]:
    """(row form, transposed form) of a matrix, each (codes, scales) or None; both from one read of x."""
    if x.dim() != 2:
        raise ValueError(f"a matrix is wanted, got {x.dim()} dimensions")
    rows, cols = x.shape
    if x.numel() and (x.stride(1) != 1 or x.stride(0) < cols):      # (rows may lie apart, elements may not)
        x = x.contiguous()
    ld = max(x.stride(0), cols) if rows > 1 else cols
    with torch.cuda.device(x.device):
        r = _buffers(rows, cols, x.device) if rowwise else None
        t = _buffers(cols, rows, x.device) if transposed else None
        B.sidco_mx4_quantize(x, rows, cols, ld, *(r or (None, None)), *(t or (None, None)))
    return r, t


def _check(name: str, form: Quantized, rows: int, cols: int, device) -> None:
    """The buffers of a quantised [rows, cols] lie on `device` and are as large as the kernels read."""
    for what, t, least in zip(("codes", "scales"), form, (B.sidco_mx4_code_bytes(rows, cols),
                                                          B.sidco_mx4_scale_bytes(rows, cols))):
        if t.device != device or t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() < least:
            raise ValueError(f"the {what} of {name} must be {least} contiguous bytes on {device} for [{rows}, {cols}], got "
                             f"{tuple(t.shape)} of {t.dtype} on {t.device}")


def matmul(a: Quantized, b: Quantized, m: int, n: int, k: int, dtype: torch.dtype = torch.bfloat16,
           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """A [m, k] B [n, k]^T of quantised matrices as a new [m, n], or added to `out`."""
    _check("a", a, m, k, a[0].device)
    _check("b", b, n, k, a[0].device)
    if out is not None and out.device != a[0].device:
        raise ValueError(f"out is on {out.device}, the operands on {a[0].device}")
    with torch.cuda.device(a[0].device):
        if out is None:
            c = torch.empty(m, n, dtype=dtype, device=a[0].device)
            B.sidco_mx4_matmul(*a, *b, m, n, k, c, n)
            return c
        if out.shape != (m, n) or (n > 1 and out.stride(1) != 1) or (m > 1 and out.stride(0) < n):
            raise ValueError(f"out must be [{m}, {n}] with contiguous rows")
        B.sidco_mx4_matmul(*a, *b, m, n, k, out, max(out.stride(0), n), add=True)
        return out


class _Linear(torch.autograd.Function):
    """Y = X W^T of operands quantised along their rows, the axis of the sums.

    The gradients pass straight through the rounding: dX = dY W and dW = dY^T X, with all three quantised along the axis of
    these sums, so X and W by their columns.  They differ from the derivatives of the computed Y by the two roundings.  There
    are no second derivatives: a graph through the backward pass raises."""

    @staticmethod
    def forward(ctx, x, weight):
        m, k, n = x.shape[0], x.shape[1], weight.shape[0]
        need_x, need_w = ctx.needs_input_grad
        x_row, x_t = quantize(x, True, need_w)
        w_row, w_t = quantize(weight, True, need_x)
        ctx.sizes, ctx.types = (m, n, k), (x.dtype, weight.dtype)
        ctx.save_for_backward(*(x_t or ()), *(w_t or ()))
        ctx.has = (x_t is not None, w_t is not None)
        return matmul(x_row, w_row, m, n, k, x.dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        m, n, k = ctx.sizes
        saved = list(ctx.saved_tensors)
        x_t = (saved.pop(0), saved.pop(0)) if ctx.has[0] else None
        w_t = (saved.pop(0), saved.pop(0)) if ctx.has[1] else None
        dy_row, dy_t = quantize(dy, w_t is not None, x_t is not None) if w_t or x_t else (None, None)
        dx = matmul(dy_row, w_t, m, k, n, ctx.types[0]) if w_t else None
        dw = matmul(dy_t, x_t, n, k, m, ctx.types[1]) if x_t else None
        return dx, dw


def mx4_linear(x: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """x [..., k] times weight [n, k]^T with 4-bit operands in the forward and both backward products."""
    if x.shape[-1] != weight.shape[1]:
        raise ValueError(f"x has {x.shape[-1]} columns, weight {weight.shape[1]}")
    y = _Linear.apply(x.reshape(x.shape[:-1].numel(), x.shape[-1]), weight)
    return y.reshape(*x.shape[:-1], weight.shape[0])


class OrthogonalizedUpdate:
    """Momentum and orthogonalised update of the matrices of a flat parameter vector.

    `shapes` are the matrices in the order of the flat vector; `offsets` default to one directly behind the other.  The
    momentum, the update and the workspace are allocated once."""

    def __init__(self, shapes: Sequence[Tuple[int, int]], device="cuda", offsets: Optional[Sequence[int]] = None,
                 mu: float = 0.95, nesterov: bool = True, steps: int = 5):
        self.rows, self.cols = [int(r) for r, _ in shapes], [int(c) for _, c in shapes]
        sizes = [r * c for r, c in zip(self.rows, self.cols)]
        self.offsets: List[int] = [sum(sizes[:i]) for i in range(len(sizes))] if offsets is None else list(offsets)
        d = max((o + n for o, n in zip(self.offsets, sizes)), default=0)
        self.mu, self.nesterov, self.steps = mu, nesterov, steps
        self.momentum = torch.zeros(d, dtype=torch.float32, device=device)
        self.update = torch.zeros(d, dtype=torch.bfloat16, device=device)
        self.workspace = torch.empty(B.sidco_orthogonalize_workspace_bytes(self.rows, self.cols), dtype=torch.uint8,
                                     device=device)

    def step(self, grad: torch.Tensor) -> torch.Tensor:
        """The update (bf16, flat) for a flat gradient; the caller scales and subtracts it."""
        if grad.numel() < self.momentum.numel() or not grad.is_contiguous():
            raise ValueError("the gradient must be a contiguous flat vector over all matrices")
        if grad.device != self.momentum.device:
            raise ValueError(f"the gradient is on {grad.device}, the momentum on {self.momentum.device}")
        with torch.cuda.device(self.momentum.device):
            B.sidco_orthogonalize(grad, self.momentum, self.mu, self.nesterov, self.offsets, self.rows, self.cols,
                                  self.steps, self.update, self.workspace, self.workspace.numel())
        return self.update
