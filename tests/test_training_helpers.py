"""What the layer and the optimiser object refuse, on the CPU."""
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
