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


@pytest.mark.parametrize("master", [False, True])
def test_fp16_gradients_keep_their_bits_under_a_scaled_loss(master):
    """The mean over 4096 rows: a gradient of x is near 2^-12 times 0.02, at the end of fp16's range, and those of the words that
    are no labels far below it.  The factor brings them back: off by what the roundings of the gradient of the logits and of the
    result leave, 2^-11 (1 + 2^-3) of the norm (as in the tests of the call), and hardly an element is zero."""
    torch, T = T_()
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, vocab, hidden, factor = 4096, 6000, 200, 2.0 ** 14
    x = torch.randn(rows, hidden, generator=g, device="cuda").half().requires_grad_()
    w = torch.randn(vocab, hidden, generator=g, device="cuda") * 0.02
    w = (w if master else w.half()).requires_grad_()
    y = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    (T.linear_cross_entropy(x, w, y) * factor).backward()
    hx, hw = x.detach().double(), w.detach().half().double()
    d = torch.softmax(hx @ hw.T, 1)
    d[torch.arange(rows, device="cuda"), y] -= 1
    d *= factor / rows
    for got, want, t in ((x.grad, d @ hw, x), (w.grad, d.T @ hx, w)):
        assert got.dtype == t.dtype
        assert (got.double() - want).norm() <= 2.0 ** -11 * (1 + 2.0 ** -3) * want.norm()
        assert (got == 0).double().mean() <= 1e-3


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("shift", [0, 1])
def test_round_gradient(dtype, shift):
    torch, T = T_()
    dtype = getattr(torch, dtype)
    x = torch.randn(100010, device="cuda") * 1e-6
    f = torch.tensor(65536.0 * 3, device="cuda")
    for n in (1, 3, 4, 1023, 100003):
        out = torch.full((100010,), 7.0, device="cuda", dtype=dtype)
        T.B.sidco_round_gradient(x[shift:], n, f, out[shift:])
        want = torch.full_like(out, 7.0)
        want[shift:n + shift] = (x[shift:n + shift] * f).to(dtype)
        assert torch.equal(out, want)
    out = torch.full((100010,), 7.0, device="cuda", dtype=dtype)
    T.B.sidco_round_gradient(x, 100003, f, out[shift:])
    assert torch.equal(out[shift:100003 + shift], (x[:100003] * f).to(dtype))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("lddx,shift", [(130, 0), (131, 1), (132, 0), (136, 0)])
def test_dx_in_32_bits(dtype, lddx, shift):
    """Rounded, dX in 32 bits is dX in 16 bits; rows without a label are zero, what lies between the rows is left."""
    torch, T = T_()
    B, rows, vocab, hidden = T.B, 700, 1500, 130
    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(rows, hidden, generator=g, device="cuda").to(dtype)
    w = (torch.randn(vocab, hidden, generator=g, device="cuda") / 4).to(dtype)
    y = torch.randint(-300, vocab, (rows,), generator=g, device="cuda")
    for grads in (1, 3):
        need = B.sidco_linear_cross_entropy_workspace_bytes(x, w, hidden, rows, vocab, hidden, grads)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        got = []
        for t in (dtype, torch.float32):
            store = torch.full((rows * lddx + 8,), float("nan"), dtype=t, device="cuda")
            dw = torch.empty(vocab, hidden, dtype=dtype, device="cuda")
            B.sidco_linear_cross_entropy(x, hidden, w, hidden, y, rows, vocab, hidden, None, None, store[shift:], lddx,
                                         dw if grads & 2 else None, hidden, ws, need)
            inside = store[shift:shift + rows * lddx].view(rows, lddx)
            got.append(inside[:, :hidden].clone())
            inside[:, :hidden] = float("nan")
            assert bool(torch.isnan(store).all())
        assert torch.equal(got[1].to(dtype), got[0]) and bool((got[1][y < 0] == 0).all()) and bool(got[1].any())


def test_labels_and_tokens_outside_the_vocabulary_are_reported():
    torch, T = T_()
    x, w = torch.randn(4, 5, 16, device="cuda").bfloat16(), torch.randn(30, 16, device="cuda").bfloat16().requires_grad_()
    y = torch.randint(-1, 30, (4, 5), device="cuda")
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    T.linear_cross_entropy(x, w, y, status=status).backward()
    assert status.item() == 0
    T.embedding(y, w, status=status.fill_(7))
    assert status.item() == 0
    y[1, 2] = 30
    T.linear_cross_entropy(x, w, y, status=status)
    assert status.item() == T.B.CROSS_ENTROPY_ST_LABEL
    rows = T.embedding(y, w, status=status.zero_())
    assert status.item() == T.B.EMBEDDING_ST_TOKEN and not bool(rows[1, 2].any())
    rows.float().sum().backward()


def test_fp16_step_with_weighted_rows_in_a_graph():
    """Captured and replayed with other inputs and another factor: the gradients of the eager step, bit for bit."""
    torch, T = T_()
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(300, 72, generator=g, device="cuda").half().requires_grad_()
    w = (torch.randn(500, 72, generator=g, device="cuda") / 4).half().requires_grad_()
    c = torch.rand(300, generator=g, device="cuda").requires_grad_()
    y = torch.randint(-20, 500, (300,), generator=g, device="cuda")
    factor = torch.tensor(64.0, device="cuda")

    def step():
        return torch.autograd.grad(T.linear_cross_entropy(x, w, y, c) * factor, (x, w, c))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(3):
        with torch.no_grad():
            x.normal_(generator=g)
            y.random_(-20, 500, generator=g)
            factor.fill_(1.0 if k == 0 else 1000.0 * k)
        graph.replay()
        for got, want, t in zip(captured, step(), (x, w, c)):
            assert got.dtype == t.dtype and got.shape == t.shape and torch.equal(got, want) and bool(torch.isfinite(got).all())
