"""What the autograd functions of a training step ask the library for, on the CPU: the calls are recorded, not made."""
import contextlib

import pytest
import torch

from paper_2101_10761_b200 import training as T


@pytest.fixture
def asked(monkeypatch):
    """[(gradients that workspace is asked for, whether dx and dw are given)] of the calls of the cross entropy."""
    calls, grads = [], []

    def workspace_bytes(x, w, ldw, rows, vocab, hidden, grads_, piece_rows=0, **kw):
        grads.append(int(grads_))
        return 0

    def call(x, ldx, w, ldw, labels, rows, vocab, hidden, row_losses, loss, dx, lddx, dw, lddw, *a, **kw):
        calls.append((grads.pop(), dx is not None, dw is not None))
    monkeypatch.setattr(T.B, "sidco_linear_cross_entropy_workspace_bytes", workspace_bytes)
    monkeypatch.setattr(T.B, "sidco_linear_cross_entropy", call)
    monkeypatch.setattr(T.torch.cuda, "device", lambda d: contextlib.nullcontext())
    return calls


def arguments(x_needs=False):
    x = torch.zeros(2, 3, 8, device="meta").bfloat16().requires_grad_(x_needs)
    return x, torch.nn.Parameter(torch.zeros(9, 8, device="meta")), torch.zeros(2, 3, dtype=torch.int64, device="meta")


@pytest.mark.parametrize("off", [torch.no_grad, torch.inference_mode])
def test_evaluation_asks_for_no_gradients(asked, off):
    """A parameter's requires_grad stays set under no_grad: the loss alone is wanted all the same."""
    x, w, y = arguments()
    with off():
        assert not T.linear_cross_entropy(x, w, y).requires_grad
    assert asked == [(0, False, False)]


def test_training_asks_for_the_gradients_that_are_needed(asked):
    x, w, y = arguments()
    assert T.linear_cross_entropy(x, w, y).requires_grad
    T.linear_cross_entropy(*arguments(True))
    T.linear_cross_entropy(arguments(True)[0], w.detach(), y)
    with torch.no_grad(), torch.enable_grad():
        T.linear_cross_entropy(x, w, y)
    assert asked == [(2, False, True), (3, True, True), (1, True, False), (2, False, True)]


def test_weights_of_the_rows_get_their_gradient(asked, monkeypatch):
    """It is the rows' losses times the factor in front of the loss; the losses are asked for only then."""
    rows_asked = []
    plain = T.B.sidco_linear_cross_entropy

    def call(*a, **kw):
        rows_asked.append(a[8] is not None)
        plain(*a, **kw)
    scaled = []
    monkeypatch.setattr(T.B, "sidco_linear_cross_entropy", call)
    monkeypatch.setattr(T.B, "sidco_scale_gradient", lambda g, n, f: scaled.append((g.shape, n)))
    x, w, y = arguments()
    c = torch.zeros(2, 3, device="meta", requires_grad=True)
    T.linear_cross_entropy(x, w.detach(), y, c).backward()
    assert c.grad.shape == (2, 3) and scaled == [((6,), 6)] and asked == [(0, False, False)]
    T.linear_cross_entropy(x, w, y, c.detach())
    with torch.no_grad():
        T.linear_cross_entropy(x, w, y, c)
    assert rows_asked == [True, False, False]


def test_status_is_handed_on_and_checked(asked, monkeypatch):
    """Labels and tokens outside the vocabulary can be told apart from padding."""
    seen = []
    plain = T.B.sidco_linear_cross_entropy

    def call(*a, **kw):
        seen.append(kw["status"])
        plain(*a, **kw)
    monkeypatch.setattr(T.B, "sidco_linear_cross_entropy", call)
    monkeypatch.setattr(T.B, "sidco_embedding", lambda *a, **kw: seen.append(kw["status"]))
    x, w, y = arguments()
    status = torch.zeros(1, dtype=torch.int32, device="meta")
    T.linear_cross_entropy(x, w, y, status=status)
    T.embedding(y, w, status=status)
    assert len(seen) == 2 and all(s is status for s in seen)
    for bad in (torch.zeros(2, dtype=torch.int32, device="meta"), torch.zeros(1, device="meta"), torch.zeros(1, dtype=torch.int32)):
        with pytest.raises(ValueError, match="status must be"):
            T.linear_cross_entropy(x, w, y, status=bad)
        with pytest.raises(ValueError, match="status must be"):
            T.embedding(y, w, status=bad)
