"""The oracle of dropout, embedding and cross entropy against published vectors, a framework and differences (CPU)."""
import numpy as np
import torch

from oracle import language_oracle as L


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def test_generator_gives_the_published_words():
    """The first two known answers of the generator's authors: all bits clear, all bits set."""
    full = 0xffffffff
    got = L.philox(np.zeros((1, 4), np.int64), 0)[0].tolist()
    assert got == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    got = L.philox(np.full((1, 4), full, np.int64), (full << 32) | full)[0].tolist()
    assert got == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


def test_generator_drops_the_share_it_is_asked_for():
    """200000 independent draws: the share is within five standard deviations, also among neighbours of equal draws."""
    n = 200000
    for p in (0.1, 0.5, 0.65):
        dropped = L.factors(n, p, 12345, 7) == 0
        assert abs(dropped.mean() - p) < 5 * (p * (1 - p) / n) ** 0.5
        both = (dropped[1:] & dropped[:-1]).mean()
        assert abs(both - p * p) < 5 * (p * p * (1 - p * p) / n) ** 0.5 * 2
    assert not np.array_equal(L.factors(n, .5, 1, 0), L.factors(n, .5, 1, 1))
    assert not np.array_equal(L.factors(n, .5, 1, 0), L.factors(n, .5, 2, 0))
    assert (L.factors(9, 0.0, 1, 1) == 1).all() and (L.factors(9, 1.0, 1, 1) == 0).all()


def test_embedding_and_gradient_against_the_framework():
    r = rng(1)
    table, tokens = r.standard_normal((11, 6)), r.integers(0, 11, 40)
    dy = r.standard_normal((40, 6))
    t = torch.tensor(table, requires_grad=True)
    y = torch.nn.functional.embedding(torch.tensor(tokens), t) * 1.5
    y.backward(torch.tensor(dy))
    assert np.allclose(L.embedding(table, tokens, 1.5), y.detach().numpy(), rtol=1e-14)
    assert np.allclose(L.embedding_grad(dy, tokens, 11, 1.5), t.grad.numpy(), rtol=1e-13, atol=1e-14)


def test_cross_entropy_against_the_framework():
    r = rng(2)
    x, w = r.standard_normal((9, 5)), r.standard_normal((13, 5))
    labels = r.integers(0, 13, 9)
    labels[[2, 5]] = -100
    weights = r.random(9)
    for c in (None, weights):
        tx, tw = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
        each = torch.nn.functional.cross_entropy(tx @ tw.T * 0.7, torch.tensor(labels), reduction="none")
        total = each.sum() / 7 if c is None else (each * torch.tensor(c)).sum()
        total.backward()
        got = L.linear_cross_entropy(x, w, labels, c, 0.7)
        for a, b in zip(got, (each.detach(), total.detach(), tx.grad, tw.grad)):
            assert np.allclose(a, b.numpy(), rtol=1e-12, atol=1e-14)


def test_cross_entropy_gradient_against_differences():
    r = rng(3)
    x, w, labels = r.standard_normal((3, 4)), r.standard_normal((6, 4)), np.array([5, -1, 0])
    _, _, dx, dw = L.linear_cross_entropy(x, w, labels, None, 1.3)
    h = 1e-6
    for m, d in ((x, dx), (w, dw)):
        for i in np.ndindex(m.shape):
            old = m[i]
            m[i] = old + h
            up = L.linear_cross_entropy(x, w, labels, None, 1.3)[1]
            m[i] = old - h
            down = L.linear_cross_entropy(x, w, labels, None, 1.3)[1]
            m[i] = old
            assert abs((up - down) / (2 * h) - d[i]) < 1e-8
