"""What a training step calls around the exchange of gradients: a linear layer whose three products are 4-bit, the lookup of
tokens, dropout, the cross entropy of the output projection, and the optimiser step on the averaged gradient.

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


def _rows(x: torch.Tensor) -> Tuple[torch.Tensor, int]:
    """A matrix whose elements of a row are neighbours, and the distance of its rows."""
    rows, cols = x.shape
    if x.numel() and ((cols > 1 and x.stride(1) != 1) or (rows > 1 and x.stride(0) < cols)):
        x = x.contiguous()
    return x, max(x.stride(0), cols) if rows > 1 else cols


def _check_random(p: float, step: Optional[torch.Tensor], device) -> None:
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"p must lie in [0, 1], got {p}")
    if step is not None and (step.dtype not in (torch.int64, torch.uint64) or step.numel() != 1 or step.device != device):
        raise ValueError(f"step must be one 64-bit integer on {device}")


def _check_status(status: Optional[torch.Tensor], device) -> None:
    if status is not None and (status.dtype != torch.int32 or status.numel() != 1 or status.device != device):
        raise ValueError(f"status must be one int32 on {device}")


_WORDS = 1 << 64


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, scale, p, seed, call, step, dtype, status):
        vocab, cols = table.shape
        n = tokens.numel()
        rows, ld = _rows(table)
        flat = tokens.reshape(-1).contiguous()
        out = torch.empty(n, cols, dtype=dtype, device=table.device)
        with torch.cuda.device(table.device):
            B.sidco_embedding(rows, vocab, cols, ld, flat, n, scale, out, cols, p=p, seed=seed, call=call, step=step,
                              status=status)
        ctx.save_for_backward(flat, step)
        ctx.args, ctx.sizes, ctx.type = (scale, p, seed, call), (n, vocab, cols), table.dtype
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        (flat, step), (n, vocab, cols) = ctx.saved_tensors, ctx.sizes
        scale, p, seed, call = ctx.args
        dy, ld = _rows(dy)
        need = B.sidco_embedding_grad_workspace_bytes(n, vocab, cols)
        with torch.cuda.device(dy.device):
            dtable = torch.empty(vocab, cols, dtype=ctx.type, device=dy.device)
            workspace = torch.empty(need, dtype=torch.uint8, device=dy.device)
            B.sidco_embedding_grad(dy, ld, flat, n, vocab, cols, scale, dtable, cols, workspace, need, p=p, seed=seed,
                                   call=call, step=step)
        return dtable, None, None, None, None, None, None, None, None


def embedding(tokens: torch.Tensor, table: torch.Tensor, scale: float = 1.0, p: float = 0.0, seed: int = 0, call: int = 0,
              step: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None,
              status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * dropout(table[tokens]), [..., cols] in `dtype` (that of the table by default).

    A negative token is padding: its row is zero and it has no gradient, as a token beyond the table.  The latter is
    reported in `status`, one int32 on the device that is set to 0 or to ``binding.EMBEDDING_ST_TOKEN``.  The mask is a
    function of (seed, call + step, position), see :func:`dropout`.  The gradient is dense, in the table's type."""
    if table.dim() != 2:
        raise ValueError(f"the table must be a matrix, got {table.dim()} dimensions")
    if tokens.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"tokens must be int32 or int64, got {tokens.dtype}")
    if tokens.device != table.device:
        raise ValueError(f"the tokens are on {tokens.device}, the table on {table.device}")
    _check_random(p, step, table.device)
    _check_status(status, table.device)
    y = _Embedding.apply(table, tokens, float(scale), float(p), seed % _WORDS, call % _WORDS, step, dtype or table.dtype, status)
    return y.reshape(*tokens.shape, table.shape[1])


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, call, step, residual):
        x = x.contiguous()
        out = torch.empty_like(x)
        with torch.cuda.device(x.device):
            B.sidco_dropout(x, x.numel(), p, seed, call, out, residual=None if residual is None else residual.contiguous(),
                            step=step)
        ctx.save_for_backward(step)
        ctx.args = (p, seed, call)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        (step,), dx = ctx.saved_tensors, None
        if ctx.needs_input_grad[0]:
            dy = dy.contiguous()
            dx = torch.empty_like(dy)
            with torch.cuda.device(dy.device):
                B.sidco_dropout(dy, dy.numel(), *ctx.args, dx, step=step)
        return dx, None, None, None, None, dy if ctx.needs_input_grad[5] else None


def dropout(x: torch.Tensor, p: float, seed: int, call: int = 0, step: Optional[torch.Tensor] = None,
            residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dropout(x) (+ residual) with a mask that is never stored: it is a function of the element's index, `seed` and the
    number of the call, call + step.  Give each use in a step its own `call`; `step`, one 64-bit integer on the device, is
    read when the kernels run, so that a captured step draws new masks (count it up behind the backward pass, which draws
    the same mask again)."""
    if residual is not None and (residual.shape != x.shape or residual.dtype != x.dtype or residual.device != x.device):
        raise ValueError(f"the residual must be {tuple(x.shape)} of {x.dtype} on {x.device}, as x")
    _check_random(p, step, x.device)
    return _Dropout.apply(x, float(p), seed % _WORDS, call % _WORDS, step, residual)


class _LinearCrossEntropy(torch.autograd.Function):
    """The gradients come from the forward pass, where the logits are; the backward pass multiplies them by the factor in
    front of the loss, in place, and hands them out, once.  Those in fp16 wait in fp32 for the factor, which is the scale of a
    scaled loss: the gradients of a mean over thousands of rows lie below that type's range without it."""

    @staticmethod
    def forward(ctx, x, weight, labels, row_weights, scale, piece_rows, status, wanted):
        (rows, hidden), vocab = x.shape, weight.shape[0]
        need_x, need_w, _, need_c = (wanted and need for need in ctx.needs_input_grad[:4])
        x, ldx = _rows(x)
        w, ldw = _rows(weight)
        loss = torch.empty((), dtype=torch.float32, device=x.device)
        wide = {torch.float16: torch.float32}
        dx = torch.empty(rows, hidden, dtype=wide.get(x.dtype, x.dtype), device=x.device) if need_x else None
        dw = torch.empty(vocab, hidden, dtype=wide.get(weight.dtype, weight.dtype), device=x.device) if need_w else None
        dc = torch.empty(rows, dtype=torch.float32, device=x.device) if need_c else None     # (the rows' losses)
        need = B.sidco_linear_cross_entropy_workspace_bytes(x, w, ldw, rows, vocab, hidden, need_x + 2 * need_w, piece_rows)
        with torch.cuda.device(x.device):
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
            B.sidco_linear_cross_entropy(x, ldx, w, ldw, labels, rows, vocab, hidden, dc, loss, dx, hidden, dw, hidden,
                                         workspace, need, row_weights=row_weights, scale=scale, piece_rows=piece_rows,
                                         status=status)
        ctx.grads, ctx.types = (dx, dw, dc), (x.dtype, weight.dtype, torch.float32)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        if ctx.grads is None:
            raise RuntimeError("the gradients of linear_cross_entropy are handed out once; call it again")
        grads, ctx.grads = ctx.grads, None
        dloss = dloss.float()
        with torch.cuda.device(dloss.device):
            dx, dw, dc = (_scaled(g, t, dloss) for g, t in zip(grads, ctx.types))
        return dx, dw, None, dc, None, None, None, None


def _scaled(g: Optional[torch.Tensor], dtype: torch.dtype, factor: torch.Tensor) -> Optional[torch.Tensor]:
    """g times a number on the device: in place, or from fp32 to another type with one rounding."""
    if g is None or g.dtype == dtype:
        if g is not None:
            B.sidco_scale_gradient(g, g.numel(), factor)
        return g
    out = torch.empty_like(g, dtype=dtype)
    B.sidco_round_gradient(g, g.numel(), factor, out)
    return out


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, labels: torch.Tensor,
                         row_weights: Optional[torch.Tensor] = None, scale: float = 1.0, piece_rows: int = 0,
                         status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Softmax cross entropy of scale * x weight^T against `labels`.  The logits are not stored; where gradients are wanted,
    their exponentials are held in 16 bits for `piece_rows` rows at a time, by default as many as fit into 512 MB or what the
    gradient of weight takes in 32 bits, whichever is more.

    x [..., hidden] in bf16 or fp16, weight [vocab, hidden] in the same type or fp32 (a master copy: rounded for the
    products, its gradient in fp32), labels [...] int32 or int64.  Rows with a negative label do not count, nor do those with
    a label beyond the vocabulary, which is reported in `status`, one int32 on the device that is set to 0 or to
    ``binding.CROSS_ENTROPY_ST_LABEL``.  The result is the mean over the others, or with row_weights [...] (fp32) the sum of the
    rows' losses times these, which may require a gradient themselves.

    The gradients are computed with the loss and handed out once: a second backward pass raises.  Those in fp16 are held in
    fp32 until then and rounded behind the factor in front of the loss.  Under ``torch.no_grad()`` the loss alone is computed,
    with a third of the operations."""
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"x must be bf16 or fp16, got {x.dtype}")
    if weight.dim() != 2 or x.dim() < 1 or x.shape[-1] != weight.shape[1] or not weight.numel():
        raise ValueError(f"x {tuple(x.shape)} and weight {tuple(weight.shape)} do not fit")
    if weight.dtype not in (x.dtype, torch.float32):
        raise ValueError(f"weight must be {x.dtype} or fp32, got {weight.dtype}")
    if labels.shape != x.shape[:-1] or labels.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"labels must be {tuple(x.shape[:-1])} of int32 or int64, got {tuple(labels.shape)} of {labels.dtype}")
    if row_weights is not None and (row_weights.shape != labels.shape or row_weights.dtype != torch.float32):
        raise ValueError(f"row_weights must be {tuple(labels.shape)} of fp32, got {tuple(row_weights.shape)} of "
                         f"{row_weights.dtype}")
    for t in (weight, labels, row_weights):
        if t is not None and t.device != x.device:
            raise ValueError(f"all arguments must be on {x.device}, got one on {t.device}")
    _check_status(status, x.device)
    rows = labels.numel()
    # (inside the function gradients look switched off always, and a parameter needs one even where they are)
    return _LinearCrossEntropy.apply(x.reshape(rows, x.shape[-1]), weight, labels.reshape(-1).contiguous(),
                                     None if row_weights is None else row_weights.reshape(-1).contiguous(), float(scale),
                                     int(piece_rows), status, torch.is_grad_enabled())


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
