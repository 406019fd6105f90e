"""Accuracy of the cross entropy's logits at the ends of its range."""
import pytest

pytestmark = pytest.mark.gpu


def T_():
    import torch

    from paper_2101_10761_b200 import training
    return torch, training


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("hidden", [4096, 65536, 1 << 20])
@pytest.mark.parametrize("products", [1, 64])
def test_logits_of_few_products_keep_their_bits(products, hidden, dtype):
    """Rows with one or 64 products that are not zero: their sums are exact or off by 64 cuts of 2^-23 at most, and what is put
    back for long sums adds 0.27 / 16 x 2^-24 for each of hidden, of 16384 at most.  The losses are -s, with s from -20 to -40."""
    torch, T = T_()
    B, rows = T.B, 64
    g = torch.Generator(device="cuda").manual_seed(hidden + products)
    x = torch.zeros(rows, hidden, device="cuda")
    at = torch.randperm(hidden, generator=g, device="cuda")[:products]
    x[:, at] = (1 + torch.rand(rows, products, generator=g, device="cuda")) * -20 / products
    x = x.to(getattr(torch, dtype))
    w = torch.zeros(2, hidden, device="cuda", dtype=x.dtype)
    w[0] = 1.0
    y = torch.zeros(rows, dtype=torch.int64, device="cuda")
    need = B.sidco_linear_cross_entropy_workspace_bytes(x, w, hidden, rows, 2, hidden, 0)
    ws, each = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")
    B.sidco_linear_cross_entropy(x, hidden, w, hidden, y, rows, 2, hidden, each, None, None, hidden, None, hidden, ws, need)
    s = x.double().sum(1)
    want = torch.log1p(torch.exp(s)) - s
    off = (0.27 / 16 * 2.0 ** -24 * min(hidden, 16384) + products * 2.0 ** -23 + 2.0 ** -22) * s.abs() + 2.0 ** -18
    assert ((each.double() - want).abs() <= off).all(), ((each.double() - want) / off).abs().max()


@pytest.mark.parametrize("hidden", [20000, 1 << 17])
def test_sums_far_longer_than_what_is_put_back(hidden):
    """Dense rows against 64 bits, within the bound that the sums have: (hidden / 16 + 2) 2^-22 of the magnitudes, twice."""
    torch, T = T_()
    B, rows, vocab = T.B, 40, 70
    g = torch.Generator(device="cuda").manual_seed(hidden)
    x = torch.randn(rows, hidden, generator=g, device="cuda").bfloat16()
    w = (torch.randn(vocab, hidden, generator=g, device="cuda") * 2 * hidden ** -0.5).bfloat16()
    y = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    need = B.sidco_linear_cross_entropy_workspace_bytes(x, w, hidden, rows, vocab, hidden, 0)
    ws, each = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")
    B.sidco_linear_cross_entropy(x, hidden, w, hidden, y, rows, vocab, hidden, each, None, None, hidden, None, hidden, ws, need)
    z = x.double() @ w.double().T
    want = torch.nn.functional.cross_entropy(z, y, reduction="none")
    size = (x.double().abs() @ w.double().abs().T).amax(1)
    off = 2 * ((hidden / 16 + 2) * 2.0 ** -22 + 2.0 ** -22) * size + 2.0 ** -18
    assert ((each.double() - want).abs() <= off).all()


@pytest.mark.parametrize("ldw", [64, 72, 1 << 39])
def test_a_single_word_at_any_distance_of_rows(ldw):
    """ldw of a matrix of one row means nothing.  Losses and gradients are zero up to what the statistics round: with s a logit in
    powers of two, base = s - 14 and log2 of the sum plus s are off by half a step each, 2^-24 (|s| + 14), the difference from
    the base by 14 x 2^-24, and exponential and logarithm by two steps of 2^-23 each: below 2^-23 (|s| + 14) + 2^-21 of one
    in all.  That is the loss (ln 2 of it), and the logit's gradient times the row's weight."""
    torch, T = T_()
    B, rows, hidden = T.B, 70, 64
    x, w = torch.randn(rows, hidden, device="cuda").bfloat16(), torch.randn(1, hidden, device="cuda").bfloat16()
    y = torch.zeros(rows, dtype=torch.int32, device="cuda")
    need = B.sidco_linear_cross_entropy_workspace_bytes(x, w, ldw, rows, 1, hidden)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = [torch.full(s, 7.0, device="cuda", dtype=t) for s, t in (((rows,), torch.float32), ((), torch.float32),
                                                                    ((rows, hidden), x.dtype), ((1, hidden), x.dtype))]
    B.sidco_linear_cross_entropy(x, hidden, w, ldw, y, rows, 1, hidden, out[0], out[1], out[2], hidden, out[3], hidden, ws, need)
    s = (x.double() @ w[0].double()).abs() * 1.4427
    off = 2.0 ** -23 * (s + 14) + 2.0 ** -21
    each, loss, dx, dw = (t.double() for t in out)
    assert (each.abs() <= off).all() and loss.abs() <= off.mean() * (1 + 2.0 ** -20)
    assert (dx.abs() <= (off / rows)[:, None] * w.double().abs() * (1 + 2.0 ** -7)).all()
    assert (dw[0].abs() <= (off / rows) @ x.double().abs() * (1 + 2.0 ** -6)).all()
