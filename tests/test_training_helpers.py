"""What the layer and the optimiser object refuse, on the CPU."""
import contextlib

import pytest
import torch

from paper_2101_10761_b200 import training as T


def test_a_penalty_on_the_gradient_raises_instead_of_counting_nothing(monkeypatch):
    """With exact products in place of the kernels, so that the layer runs here."""
    monkeypatch.setattr(T, "quantize", lambda x, rowwise=True, transposed=True: ((x, x) if rowwise else None,
                                                                                  (x.T, x.T) if transposed else None))
    monkeypatch.setattr(T, "matmul", lambda a, b, m, n, k, dtype=None, out=None: a[0] @ b[0].T)
    x, w = torch.randn(5, 7), torch.randn(3, 7, requires_grad=True)
    x.requires_grad_()
    y = T.mx4_linear(x, w).square().sum()
    dx, dw = torch.autograd.grad(y, (x, w), create_graph=True)
    assert torch.allclose(dx, 2 * (x @ w.T) @ w) and torch.allclose(dw, 2 * (x @ w.T).T @ x)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dx.square().sum().backward()


def form(rows, cols, device="meta"):
    from paper_2101_10761_b200 import binding as B
    return (torch.empty(B.sidco_mx4_code_bytes(rows, cols), dtype=torch.uint8, device=device),
            torch.empty(B.sidco_mx4_scale_bytes(rows, cols), dtype=torch.uint8, device=device))


@pytest.mark.parametrize("m, n, k", [(41, 20, 33), (40, 21, 33), (40, 20, 65), (200, 20, 33), (40, 200, 33)])
def test_product_refuses_sizes_that_its_operands_do_not_have(m, n, k):
    """Operands of [40, 33] and [20, 33] (on the meta device: nothing may be launched)."""
    with pytest.raises(ValueError, match="contiguous bytes"):
        T.matmul(form(40, 33), form(20, 33), m, n, k)


def test_product_refuses_other_buffers():
    a, b = form(40, 33), form(20, 33)
    with pytest.raises(ValueError, match="scales of b"):
        T.matmul(a, (b[0], b[1][:-1]), 40, 20, 33)
    with pytest.raises(ValueError, match="codes of a"):
        T.matmul((a[0].float(), a[1]), b, 40, 20, 33)
    with pytest.raises(ValueError, match="codes of a"):
        T.matmul((torch.empty(2 * a[0].numel(), dtype=torch.uint8, device="meta")[::2], a[1]), b, 40, 20, 33)
    with pytest.raises(ValueError, match="codes of b"):
        T.matmul(a, form(20, 33, "cpu"), 40, 20, 33)
    with pytest.raises(ValueError, match="out is on"):
        T.matmul(a, b, 40, 20, 33, out=torch.zeros(40, 20))


def test_optimizer_object_refuses_a_gradient_from_elsewhere():
    opt = T.OrthogonalizedUpdate([(4, 5)], device="meta")
    with pytest.raises(ValueError, match="momentum on meta"):
        opt.step(torch.zeros(20))


def test_product_takes_a_single_column_whatever_its_second_stride(monkeypatch):
    """(m, 1) with strides (1, m), as the transpose of a row has: its rows have one element each."""
    seen = []
    monkeypatch.setattr(T.B, "sidco_mx4_matmul", lambda *a, **k: seen.append(a[8]))
    monkeypatch.setattr(T.torch.cuda, "device", lambda d: contextlib.nullcontext())
    out = torch.zeros(1, 40, device="meta").T
    assert out.stride() == (1, 40)
    assert T.matmul(form(40, 33), form(1, 33), 40, 1, 33, out=out) is out and seen == [1]
    with pytest.raises(ValueError, match="contiguous rows"):
        T.matmul(form(40, 33), form(2, 33), 40, 2, 33, out=torch.zeros(2, 40, device="meta").T)
