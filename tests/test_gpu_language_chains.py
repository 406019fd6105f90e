"""Calls directly behind the calls that write what they read: the kernels start under one another, and the results are those of
calls that wait for the device in between, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu


def T_():
    import torch

    from paper_2101_10761_b200 import binding
    return torch, binding


@pytest.mark.parametrize("tokens,cols", [(900, 96), (5000, 130), (3000, 64)])
@pytest.mark.parametrize("add", [False, True])
def test_dropout_then_gradient_of_the_table(tokens, cols, add):
    torch, B = T_()
    g = torch.Generator(device="cuda").manual_seed(tokens)
    vocab = 700
    dy = torch.randn(20, tokens, cols, generator=g, device="cuda").bfloat16()
    t = torch.randint(-50, vocab, (tokens,), generator=g, device="cuda")
    need = B.sidco_embedding_grad_workspace_bytes(tokens, vocab, cols)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def run(wait):
        out, dx = [], torch.zeros(tokens, cols, dtype=torch.bfloat16, device="cuda")
        table = torch.zeros(vocab, cols, device="cuda")
        for i in range(20):
            B.sidco_dropout(dy[i], dy[i].numel(), 0.3, 5, i, dx)
            wait()
            B.sidco_embedding_grad(dx, cols, t, tokens, vocab, cols, 1.5, table, cols, ws, need, add=add)
            wait()
            out.append(table.clone())
        return torch.stack(out)
    assert torch.equal(run(lambda: None), run(torch.cuda.synchronize))


@pytest.mark.parametrize("cols,dtype", [(96, "float32"), (130, "bfloat16"), (131, "float32")])
def test_update_of_the_table_then_lookup(cols, dtype):
    """The table is scaled in place by a kernel of the library; tokens and rows are read by the next."""
    torch, B = T_()
    g = torch.Generator(device="cuda").manual_seed(cols)
    vocab, n = 4000, 3000
    first = torch.randn(vocab, cols, generator=g, device="cuda").to(getattr(torch, dtype))
    t = torch.randint(-5, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    factor = torch.tensor(-0.75, device="cuda")

    def run(wait):
        table, out = first.clone(), torch.empty(20, n, cols, device="cuda")
        for i in range(20):
            B.sidco_scale_gradient(table, table.numel(), factor)
            wait()
            B.sidco_embedding(table, vocab, cols, cols, t, n, 2.0, out[i], cols, p=0.1 * (i % 2), seed=3, call=i)
            wait()
        return out
    assert torch.equal(run(lambda: None), run(torch.cuda.synchronize))
