"""The lookup, dropout and cross entropy as a training step calls them: through autograd, together, in a captured step."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import language_oracle as L

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def T_():
    import torch

    from paper_2101_10761_b200 import training
    return torch, training


def test_embedding_gradients_and_shapes():
    torch, T = T_()
    r = np.random.Generator(np.random.PCG64(1))
    table = torch.tensor(r.standard_normal((50, 18)), dtype=torch.float32, device="cuda", requires_grad=True)
    tokens = torch.tensor(r.integers(-1, 50, (3, 4, 5)), device="cuda")
    y = T.embedding(tokens, table, scale=2.0, p=0.3, seed=-5, call=2 ** 64 + 3, dtype=torch.bfloat16)
    assert y.shape == (3, 4, 5, 18) and y.dtype == torch.bfloat16
    held, flat = table.detach().double().cpu().numpy(), tokens.reshape(-1).cpu().numpy()
    want = L.embedding(held, flat, 2.0, 0.3, 2 ** 64 - 5, 3)
    assert np.abs(y.detach().double().cpu().numpy().reshape(-1, 18) - want).max() <= 2.0 ** -8 * np.abs(want).max()
    dy = torch.tensor(r.standard_normal((60, 18)), device="cuda").bfloat16().view(3, 4, 5, 18)
    y.backward(dy.transpose(0, 1).contiguous().transpose(0, 1))                       # strides of its own
    want = L.embedding_grad(dy.double().cpu().numpy().reshape(-1, 18), flat, 50, 2.0, 0.3, 2 ** 64 - 5, 3)
    assert table.grad.dtype == torch.float32 and np.allclose(table.grad.cpu().numpy(), want, rtol=1e-5, atol=1e-5)
    wide = torch.randn(50, 36, device="cuda").half()
    assert torch.equal(T.embedding(tokens, wide[:, ::2]), T.embedding(tokens, wide[:, ::2].contiguous()))
    assert T.embedding(tokens[:0], table).shape == (0, 4, 5, 18)


def test_dropout_gradients():
    torch, T = T_()
    x = torch.randn(7, 33, device="cuda").half().requires_grad_()
    res = torch.randn(7, 33, device="cuda").half().requires_grad_()
    y = T.dropout(x, 0.25, seed=9, call=1, residual=res)
    dy = torch.randn_like(y)
    y.backward(dy)
    f = torch.from_numpy(L.factors(7 * 33, 0.25, 9, 1)).view(7, 33).cuda()
    assert torch.allclose(y.double(), x.double() * f + res.double(), atol=2e-2) and torch.equal(res.grad, dy)
    assert torch.allclose(x.grad.double(), dy.double() * f, rtol=2.0 ** -10) and torch.equal(x.grad == 0, (f == 0) | (dy == 0))
    z = T.dropout(x.detach().T, 0.25, seed=9)                                         # strided
    assert torch.equal(z, T.dropout(x.detach().T.contiguous(), 0.25, seed=9))


@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
def test_cross_entropy_gradients(weighted, master):
    torch, T = T_()
    r = np.random.Generator(np.random.PCG64(2))
    x = torch.tensor(r.standard_normal((6, 11, 40)), device="cuda").bfloat16().requires_grad_()
    w = torch.tensor(r.standard_normal((70, 40)) / 4, device="cuda")
    w = (w.float() if master else w.bfloat16()).requires_grad_()
    labels = torch.tensor(r.integers(-30, 70, (6, 11)), device="cuda")
    c = torch.tensor(r.random((6, 11)), device="cuda").float() if weighted else None
    loss = T.linear_cross_entropy(x, w, labels, c, scale=0.8)
    (loss * 3).backward(retain_graph=True)
    hw = w.detach().bfloat16().double().cpu().numpy()
    _, want, dx, dw = L.linear_cross_entropy(x.detach().double().cpu().numpy().reshape(66, 40), hw, labels.cpu().numpy().reshape(-1),
                                             None if c is None else c.double().cpu().numpy().reshape(-1), float(np.float32(0.8)))
    assert loss.dtype == torch.float32 and abs(loss.item() - want) < 1e-4 * abs(want)
    for got, d, t in ((x.grad.reshape(66, 40), dx, x), (w.grad, dw, w)):
        assert got.dtype == t.dtype
        assert np.linalg.norm(got.double().cpu().numpy() - 3 * d) <= 2.0 ** -7 * np.linalg.norm(3 * d)
    with pytest.raises(RuntimeError, match="handed out once"):
        loss.backward()


def test_cross_entropy_gradient_against_differences():
    """A step h along the gradient itself changes the loss by h |grad|^2, up to the rounding of x (2^-8 of |h grad x|-like
    terms do not enter: x is taken as it is rounded)."""
    torch, T = T_()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(64, 48, generator=g, device="cuda").half().requires_grad_()
    w = (torch.randn(90, 48, generator=g, device="cuda") / 5).half().requires_grad_()
    y = torch.randint(0, 90, (64,), generator=g, device="cuda")
    T.linear_cross_entropy(x, w, y).backward()
    with torch.no_grad():
        for t, other in ((x, w), (w, x)):
            d = t.grad.float() / t.grad.float().norm()
            up, down = (t + 0.5 * d).half(), (t - 0.5 * d).half()                       # the points as they are held
            want = (t.grad.double() * (up.double() - down.double())).sum().item()
            a, b = ((T.linear_cross_entropy(p, w, y) if t is x else T.linear_cross_entropy(x, p, y)).item() for p in (up, down))
            assert abs((a - b) - want) < 0.02 * abs(want), (a - b, want)               # (third-order terms of the loss)


def test_no_gradient_wanted():
    torch, T = T_()
    x, w = torch.randn(30, 16, device="cuda").half(), torch.randn(20, 16, device="cuda").half()
    y = torch.randint(0, 20, (30,), device="cuda")
    plain = T.linear_cross_entropy(x, w, y)
    assert not plain.requires_grad
    only_x = x.clone().requires_grad_()
    loss = T.linear_cross_entropy(only_x, w, y, piece_rows=1)
    loss.backward()
    assert only_x.grad is not None and loss.item() == pytest.approx(plain.item(), rel=1e-6)


@pytest.mark.parametrize("factor", [1.0, -2.5])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_scale_gradient(dtype, factor):
    torch, T = T_()
    x = torch.randn(100003, device="cuda").to(getattr(torch, dtype))
    f = torch.tensor(factor, device="cuda")
    for shift in (0, 1):
        y = x.clone()
        T.B.sidco_scale_gradient(y[shift:], 100000, f)
        want = x.clone()
        want[shift:100000 + shift] = (x[shift:100000 + shift].float() * factor).to(x.dtype)
        assert torch.equal(y, want)


def example():
    spec = importlib.util.spec_from_file_location("language_model_training",
                                                  os.path.join(ROOT, "examples", "language_model_training.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("tied", [False, True])
def test_whole_step_has_the_gradients_of_its_parts(tied):
    """Lookup, dropout onto the residual and cross entropy together, the two layers between at their own gradients: against
    the same step in 64 bits with the masks of the oracle and exact products in place of the 4-bit ones.

    The sides that the rectifier takes are the step's: its argument is off by three roundings of bf16 in x, w and the product,
    together up to 2^-8 of its size in the mean square, so that about arctan(2^-8) / pi = 0.12 % of the 36 x 64 arguments, three,
    change sign, and each takes a gradient with it whose share of the norm no bound on roundings limits."""
    torch, T = T_()
    m = example()
    model = m.Model(60, 32, 64, tied, 0.2, "cuda")
    tokens = torch.randint(-1, 60, (4, 9), device="cuda")
    labels = torch.randint(-1, 60, (4, 9), device="cuda")
    products = []

    def exact(x, w):
        products.append(x @ w.to(x.dtype).T)
        return products[-1]

    kept, m.mx4_linear = m.mx4_linear, exact
    try:
        loss = model.loss(tokens, labels)
    finally:
        m.mx4_linear = kept
    loss.backward()
    flat = model.flat.detach().double().requires_grad_()
    w = [v.view(s) for v, s in zip(flat.split(model.sizes), model.shapes)]
    f1, f2 = (torch.from_numpy(L.factors(36 * 32, 0.2, seed, 0)).view(36, 32).cuda() for seed in (1, 2))
    t = tokens.view(-1)
    x = torch.where((t >= 0)[:, None], w[0][t.clamp(min=0)], 0.0) * 32 ** 0.5 * f1
    x = x @ w[1].T * (products[0].detach().view(36, 64) > 0) @ w[2].T * f2 + x
    want = torch.nn.functional.cross_entropy(x @ (w[0] if tied else w[3]).T * 32 ** -0.5, labels.view(-1), ignore_index=-1)
    want.backward()
    assert abs(loss.item() - want.item()) < 2e-2 * want.item()
    # twelve roundings at most on any way through the step, each 2^-8 / sqrt(3) at most in the mean square: 2^-7, and a quarter more
    assert (model.flat.grad - flat.grad).norm() < 1.25 * 2 ** -7 * flat.grad.norm()


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("tied", [False, True])
def test_example_runs(tied, graph):
    torch, _ = T_()
    losses = example().train(steps=4, tied=tied, graph=graph, vocab=301, width=96, hidden=160, sequences=5, length=12)
    assert len(losses) == 4 and all(np.isfinite(losses))


def test_captured_step_draws_the_masks_of_the_eager_one():
    m = example()
    kw = dict(steps=4, vocab=301, width=96, hidden=160, sequences=5, length=12, p=0.4)
    assert m.train(graph=False, **kw) == m.train(graph=True, **kw)
