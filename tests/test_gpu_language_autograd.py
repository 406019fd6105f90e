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
