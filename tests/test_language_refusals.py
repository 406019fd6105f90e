"""Argument errors of dropout, embedding and cross entropy, found on the host before any CUDA call (no GPU)."""
import numpy as np
import pytest

P = 0x100000                                   # never dereferenced: every call below fails validation first
Q = 0x4000000
BIG = 1 << 31
NAN = float("nan")


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


def test_dropout_refuses(B):
    d = B.sidco_dropout
    assert code(d, P, -1, .5, 0, 0, Q, x_type=0) == -10
    assert code(d, P, (1 << 40) + 1, .5, 0, 0, Q, x_type=0) == -10
    assert code(d, P, 8, .5, 0, 0, Q, x_type=3) == -13
    assert code(d, P, 8, .5, 0, 0, Q) == -13                       # a raw address without a type
    for p in (-.1, 1.001, NAN, float("inf")):
        assert code(d, P, 8, p, 0, 0, Q, x_type=1) == -6
    assert code(d, None, 8, .5, 0, 0, Q, x_type=0) == -1
    assert code(d, P, 8, .5, 0, 0, None, x_type=0) == -1
    assert code(d, P + 2, 8, .5, 0, 0, Q, x_type=0) == -14
    assert code(d, P, 8, .5, 0, 0, Q + 1, x_type=1) == -14
    assert code(d, P, 8, .5, 0, 0, Q, residual=P + 1, x_type=1) == -14
    assert code(d, P, 8, .5, 0, 0, Q, step=P + 4, x_type=1) == -14
    assert code(d, P, 8, .5, 0, 0, P + 4, x_type=0) == -9
    assert code(d, Q, 8, .5, 0, 0, P + 4, residual=P, x_type=0) == -9
    d(None, 0, .5, 0, 0, None, x_type=0, stream=0)                 # nothing to do


def test_embedding_refuses(B):
    e = B.sidco_embedding
    kw = dict(table_type=0, token_type=4, out_type=1)

    def with_(**k):
        return {**kw, **k}
    assert code(e, P, BIG, 8, 8, P, 4, 1., Q, 8, **kw) == -10
    assert code(e, P, 9, (1 << 24) + 1, BIG, P, 4, 1., Q, BIG, **kw) == -10
    assert code(e, P, 9, 8, 8, P, -1, 1., Q, 8, **kw) == -10
    assert code(e, P, 9, 8, 8, P, 4, 1., Q, 8, **with_(table_type=3)) == -13
    assert code(e, P, 9, 8, 8, P, 4, 1., Q, 8, **with_(out_type=-1)) == -13
    assert code(e, P, 9, 8, 8, P, 4, 1., Q, 8, **with_(token_type=0)) == -13
    assert code(e, P, 9, 8, 8, np.zeros(4, np.float32), 4, 1., Q, 8, table_type=0, out_type=0) == -13
    assert code(e, P, 9, 8, 7, P, 4, 1., Q, 8, **kw) == -6
    assert code(e, P, 9, 8, 8, P, 4, 1., Q, 7, **kw) == -6
    assert code(e, P, 9, 8, 8, P, 4, 1., Q, 8, p=NAN, **kw) == -6
    assert code(e, P, 9, 8, 8, P, 4, 1., Q, 8, p=.5, step=P + 1, **kw) == -14
    for args in ((None, P, Q), (P, None, Q), (P, P, None)):
        assert code(e, args[0], 9, 8, 8, args[1], 4, 1., args[2], 8, **kw) == -1
    assert code(e, P + 2, 9, 8, 8, P, 4, 1., Q, 8, **kw) == -14
    assert code(e, P, 9, 8, 8, P + 4, 4, 1., Q, 8, **kw) == -14
    assert code(e, P, 9, 8, 8, P, 4, 1., Q + 1, 8, **kw) == -14
    assert code(e, P, 9, 8, 8, P, 4, 1., Q, 8, status=P + 2, **kw) == -14
    assert code(e, P, 9, 8, 8, Q, 4, 1., P + 9 * 32 - 4, 8, **kw) == -9       # the last element of the table
    assert code(e, P, 9, 8, 8, Q, 4, 1., Q + 24, 8, **kw) == -9


def test_embedding_grad_refuses(B):
    g = B.sidco_embedding_grad
    W = 0x8000000
    N = 4000                                   # (up to 2048 tokens need no workspace)
    kw = dict(dy_type=1, token_type=3, dtable_type=0)
    need = B.sidco_embedding_grad_workspace_bytes(N, 9, 8)

    def with_(**k):
        return {**kw, **k}
    assert need > 0 and B.sidco_embedding_grad_workspace_bytes(2048, 9, 8) == 0
    with pytest.raises(B.SidcoError) as err:
        B.sidco_embedding_grad_workspace_bytes(BIG, 9, 8)
    assert err.value.code == -10
    assert code(g, P, 8, P, N, BIG, 8, 1., Q, 8, W, need, **kw) == -10
    assert code(g, P, 8, P, N, 9, 8, 1., Q, 8, W, need, **with_(dy_type=7)) == -13
    assert code(g, P, 8, P, N, 9, 8, 1., Q, 8, W, need, **with_(dtable_type=7)) == -13
    assert code(g, P, 8, P, N, 9, 8, 1., Q, 8, W, need, **with_(token_type=2)) == -13
    assert code(g, P, 7, P, N, 9, 8, 1., Q, 8, W, need, **kw) == -6
    assert code(g, P, 8, P, N, 9, 8, 1., Q, 7, W, need, **kw) == -6
    assert code(g, P, 8, P, N, 9, 8, 1., Q, 8, W, need, p=2., **kw) == -6
    for args in ((None, P, Q), (P, None, Q), (P, P, None)):
        assert code(g, args[0], 8, args[1], N, 9, 8, 1., args[2], 8, W, need, **kw) == -1
    assert code(g, P + 1, 8, P, N, 9, 8, 1., Q, 8, W, need, **kw) == -14
    assert code(g, P, 8, P + 2, N, 9, 8, 1., Q, 8, W, need, **kw) == -14
    assert code(g, P, 8, P, N, 9, 8, 1., Q + 2, 8, W, need, **kw) == -14
    assert code(g, P, 8, P, N, 9, 8, 1., Q, 8, None, need, **kw) == -8
    assert code(g, P, 8, P, N, 9, 8, 1., Q, 8, W, need - 1, **kw) == -8
    assert code(g, P, 8, P, N, 9, 8, 1., Q, 8, W + 128, need, **kw) == -8
    assert code(g, P, 8, W, N, 9, 8, 1., P + 60, 8, Q, need, **kw) == -9
    assert code(g, P, 8, Q + 4, N, 9, 8, 1., Q, 8, W, need, **kw) == -9
    assert code(g, W, 8, P, N, 9, 8, 1., Q, 8, W, need, **kw) == -9
    assert code(g, P, 8, W + 256, N, 9, 8, 1., Q, 8, W, need, **kw) == -9
    assert code(g, P, 8, P, N, 9, 8, 1., W, 8, W, need, **kw) == -9


def test_cross_entropy_refuses(B):
    f = B.sidco_linear_cross_entropy
    x, w, y, each, loss, dx, dw, ws, c = (0x10000000 * (i + 1) for i in range(9))
    kw = dict(x_type=1, w_type=1, label_type=4, dw_type=1)
    need = B.sidco_linear_cross_entropy_workspace_bytes(0, w, 8, 4, 9, 8, x_type=1, w_type=1)

    def args(**k):
        a = dict(x=x, ldx=8, w=w, ldw=8, labels=y, rows=4, vocab=9, hidden=8, each=each, loss=loss, dx=dx, lddx=8, dw=dw,
                 lddw=8, ws=ws, need=need)
        a.update({n: v for n, v in k.items() if n in a})
        return list(a.values()), {**kw, **{n: v for n, v in k.items() if n not in a}}

    def refused(**k):
        a, b = args(**k)
        return code(f, *a, **b)
    for n in ("rows", "vocab", "hidden"):
        assert refused(**{n: -1}) == -10
    assert refused(rows=(1 << 28) + 1) == -10 and refused(vocab=(1 << 28) + 1) == -10 and refused(piece_rows=-1) == -10
    assert refused(hidden=(1 << 20) + 1, ldx=1 << 21) == -10
    assert refused(vocab=0) == -10 and refused(hidden=0) == -10
    assert refused(vocab=1 << 28, hidden=1 << 20, ldx=1 << 20, ldw=1 << 20, lddx=1 << 20, lddw=1 << 20) == -10      # too many tiles
    for t in (0, 3, -1):
        assert refused(x_type=t) == -13
    assert refused(w_type=2) == -13 and refused(dw_type=2) == -13 and refused(label_type=0) == -13
    assert refused(x_type=2, w_type=0, dw_type=1) == -13
    for n in ("ldx", "ldw", "lddx", "lddw"):
        assert refused(**{n: 7}) == -6
    for s in (NAN, float("inf")):
        assert refused(scale=s) == -6
    for n in ("x", "w", "labels"):
        assert refused(**{n: None}) == -1
    for n, v in (("x", x), ("w", w), ("dx", dx), ("dw", dw), ("labels", y), ("each", each), ("loss", loss)):
        assert refused(**{n: v + 1}) == -14
    assert refused(labels=y + 4) == -14 and refused(row_weights=c + 2) == -14 and refused(status=c + 2) == -14
    assert refused(w=w + 2, w_type=0) == -14
    assert refused(ws=None) == -8 and refused(need=need - 1) == -8 and refused(ws=ws + 128) == -8
    assert refused(w=w + 8) == -8                                  # its copy does not fit
    assert refused(dx=x) == -9 and refused(dw=w) == -9 and refused(each=dw + 9 * 16 - 4) == -9
    assert refused(ws=x) == -9 and refused(loss=each + 12) == -9 and refused(row_weights=each) == -9
    assert refused(dx=ws + 256) == -9 and refused(status=loss) == -9 and refused(labels=dx + 56) == -9

    size = B.sidco_linear_cross_entropy_workspace_bytes
    plain = size(0, 0, 1504, 700, 10000, 1500, x_type=1, w_type=1)
    assert 700 * 10000 * 2 < plain < 80 << 20
    assert size(0, 0, 1500, 700, 10000, 1500, x_type=1, w_type=1) >= plain + 10000 * 1500 * 2      # W is copied
    assert size(0, 0, 1504, 700, 10000, 1500, x_type=1, w_type=0) >= plain + 10000 * 1500 * 2
    assert size(0, 0, 1504, 700, 10000, 1500, grads=False, x_type=1, w_type=1) < 6 << 20
    # e never takes more than 512 MB or the gradient of w in 32 bits
    assert size(0, 0, 64, 1 << 20, 50000, 64, x_type=1, w_type=1) < (1 << 29) + (1 << 20) * 64 * 2 + 50000 * 64 * 4 + (400 << 20)
    for bad in (dict(rows=-1), dict(vocab=-1), dict(piece_rows=-1), dict(rows=1 << 29)):
        a = dict(ldw=8, rows=4, vocab=9, hidden=8)
        a.update(bad)
        with pytest.raises(B.SidcoError) as e:
            size(0, 0, x_type=1, w_type=1, **a)
        assert e.value.code == -10
    for bad, want in ((dict(x_type=0, w_type=1), -13), (dict(x_type=1, w_type=2), -13), (dict(x_type=1, w_type=1, grads=4), -6)):
        with pytest.raises(B.SidcoError) as e:
            size(0, 0, 8, 4, 9, 8, **bad)
        assert e.value.code == want
    assert size(0, 0, 8, 0, 9, 8, x_type=1, w_type=1) == 0


def test_scale_gradient_refuses(B):
    f = B.sidco_scale_gradient
    assert code(f, P, -1, Q, x_type=0) == -10 and code(f, P, (1 << 40) + 1, Q, x_type=0) == -10
    assert code(f, P, 4, Q, x_type=5) == -13
    assert code(f, None, 4, Q, x_type=0) == -1 and code(f, P, 4, None, x_type=0) == -1
    assert code(f, P + 2, 4, Q, x_type=0) == -14 and code(f, P, 4, Q + 2, x_type=0) == -14
    assert code(f, P, 4, P + 12, x_type=0) == -9
    f(None, 0, None, x_type=0, stream=0)
