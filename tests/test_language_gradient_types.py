"""Types of the cross entropy's gradients: what the calls refuse, and what the autograd function asks for, on the CPU."""
import contextlib

import pytest
import torch

P, Q, R, F = 0x100000, 0x4000000, 0x8000000, 0xc000000        # never dereferenced: every call fails validation first


@pytest.fixture(scope="module")
def B():
    from paper_2101_10761_b200 import binding, build
    build.build()
    return binding


def code(call, *args, **kw):
    from paper_2101_10761_b200 import binding
    with pytest.raises(binding.SidcoError) as e:
        call(*args, stream=0, **kw)
    return e.value.code


def test_round_gradient_refuses(B):
    f = B.sidco_round_gradient
    assert code(f, P, -1, F, Q, out_type=2) == -10 and code(f, P, (1 << 40) + 1, F, Q, out_type=2) == -10
    assert code(f, P, 8, F, Q, out_type=3) == -13 and code(f, P, 8, F, Q) == -13
    for args in ((None, F, Q), (P, None, Q), (P, F, None)):
        assert code(f, args[0], 8, args[1], args[2], out_type=2) == -1
    assert code(f, P + 2, 8, F, Q, out_type=2) == -14 and code(f, P, 8, F + 2, Q, out_type=2) == -14
    assert code(f, P, 8, F, Q + 1, out_type=2) == -14 and code(f, P, 8, F, Q + 2, out_type=0) == -14
    assert code(f, P, 8, F, P, out_type=2) == -9 and code(f, P + 14, 8, P + 12, P, out_type=2) == -14
    assert code(f, P, 8, F, P + 28, out_type=2) == -9 and code(f, Q, 8, P + 12, P, out_type=2) == -9
    f(None, 0, None, None, out_type=2, stream=0)                  # nothing to do


def test_room_for_the_gradient_of_the_logits(B):
    """512 MB, or what dw takes in 32 bits where there is one: rows of a piece of 128000 words at hidden 4096."""
    def need(grads, piece_rows):
        return B.sidco_linear_cross_entropy_workspace_bytes(0, P, 4096, 16384, 128000, 4096, grads, piece_rows, x_type=1, w_type=1)
    assert need(1, 0) == need(1, 2048) < need(1, 2049)
    assert need(2, 0) == need(2, 8192) < need(2, 8193) and need(3, 0) == need(3, 8192)


def test_cross_entropy_refuses_types_of_dx(B):
    f = B.sidco_linear_cross_entropy
    x, w, y, dx, dw, ws = (0x10000000 * (i + 1) for i in range(6))
    need = B.sidco_linear_cross_entropy_workspace_bytes(0, w, 8, 4, 9, 8, x_type=1, w_type=1)

    def refused(dx=dx, lddx=8, **kw):
        return code(f, x, 8, w, 8, y, 4, 9, 8, None, None, dx, lddx, dw, 8, ws, need, x_type=1, w_type=1, label_type=4, dw_type=1, **kw)
    assert refused(dx_type=2) == -13 and refused(dx_type=3) == -13
    assert refused(dx_type=0, dx=dx + 2) == -14 and refused(dx_type=1, dx=dx + 1) == -14
    assert refused(dx_type=0, dx=dw - 124) == -9                  # (its last element)
    assert refused(dx_type=0, dx=dx, lddx=7) == -6
    assert refused(dx_type=0, dx=ws - 100) == -9


def test_gradients_in_16_bits_wait_for_their_factor(monkeypatch):
    """fp16 in fp32, rounded once behind the factor; bf16, whose range is that of fp32, in its own type."""
    from paper_2101_10761_b200 import training as T
    made, rounded, scaled = [], [], []
    monkeypatch.setattr(T.B, "sidco_linear_cross_entropy_workspace_bytes", lambda *a, **kw: 0)
    monkeypatch.setattr(T.B, "sidco_linear_cross_entropy", lambda *a, **kw: made.append((a[10].dtype, a[12].dtype)))
    monkeypatch.setattr(T.B, "sidco_round_gradient", lambda x, n, f, out: rounded.append((x.dtype, n, f.dtype, out.dtype)))
    monkeypatch.setattr(T.B, "sidco_scale_gradient", lambda x, n, f: scaled.append((x.dtype, n, f.dtype)))
    monkeypatch.setattr(T.torch.cuda, "device", lambda d: contextlib.nullcontext())
    h, b, s = torch.float16, torch.bfloat16, torch.float32

    def step(x_type, w_type):
        x = torch.zeros(2, 3, 8, device="meta", dtype=x_type, requires_grad=True)
        w = torch.zeros(9, 8, device="meta", dtype=w_type, requires_grad=True)
        T.linear_cross_entropy(x, w, torch.zeros(2, 3, dtype=torch.int64, device="meta")).backward()
        assert x.grad.dtype == x_type and w.grad.dtype == w_type and x.grad.shape == x.shape
    step(h, h)
    assert made.pop() == (s, s) and rounded == [(s, 48, s, h), (s, 72, s, h)] and not scaled
    rounded.clear()
    step(h, s)
    assert made.pop() == (s, s) and rounded == [(s, 48, s, h)] and scaled == [(s, 72, s)]
    rounded.clear(), scaled.clear()
    step(b, b)
    assert made.pop() == (b, b) and scaled == [(b, 48, s), (b, 72, s)] and not rounded
