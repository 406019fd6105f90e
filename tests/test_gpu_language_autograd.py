"""The autograd functions of a language model's training step on the GPU: what they allocate and what their gradients keep."""
import pytest

pytestmark = pytest.mark.gpu


def T_():
    import torch

    from paper_2101_10761_b200 import training
    return torch, training


def test_evaluation_with_parameters_takes_no_room_for_gradients():
    """The gradient of W alone would take 41 MB, the exponentials of a training call 20 MB; what the loss needs is below 1 MB."""
    torch, T = T_()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(256, 512, generator=g, device="cuda").bfloat16()
    w = torch.nn.Parameter((torch.randn(40000, 512, generator=g, device="cuda") / 16).bfloat16())
    y = torch.randint(0, 40000, (256,), generator=g, device="cuda")
    loss = T.linear_cross_entropy(x, w, y)
    assert loss.requires_grad
    want = loss.item()
    del loss
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    with torch.no_grad():
        loss = T.linear_cross_entropy(x, w, y)
    assert not loss.requires_grad and loss.item() == want
    assert torch.cuda.max_memory_allocated() - before < 4 << 20


@pytest.mark.parametrize("only", [False, True])
def test_gradient_of_the_row_weights(only):
    """The rows' losses times the factor, against 64 bits: fp32 logits of 24 products of about 1, sums and logarithm (2^-18),
    and the rounding of the product."""
    torch, T = T_()
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(5, 9, 24, generator=g, device="cuda").bfloat16().requires_grad_(not only)
    w = (torch.randn(70, 24, generator=g, device="cuda") / 4).bfloat16().requires_grad_(not only)
    y = torch.randint(-9, 70, (5, 9), generator=g, device="cuda")
    c = torch.rand(5, 9, generator=g, device="cuda").requires_grad_()
    (T.linear_cross_entropy(x, w, y, c) * 3).backward()
    z = x.detach().double() @ w.detach().double().T
    want = 3 * torch.nn.functional.cross_entropy(z.view(45, 70), y.view(45).clamp(min=-1), ignore_index=-1, reduction="none").view(5, 9)
    size = (x.detach().double().abs() @ w.detach().double().abs().T).max()
    off = 3 * (2 * (24 / 16 + 3) * 2.0 ** -22 * size + 2.0 ** -18) + 2.0 ** -24 * want.max()
    assert (c.grad.double() - want).abs().max() <= off and bool((c.grad[y < 0] == 0).all())
    assert only or (x.grad is not None and w.grad is not None)
