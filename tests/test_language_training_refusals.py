"""What the lookup, dropout and cross entropy of a training step refuse, on the CPU."""
import pytest
import torch

from paper_2101_10761_b200 import training as T


def test_embedding_refuses():
    table, tokens = torch.zeros(5, 4, device="meta"), torch.zeros(3, dtype=torch.int64, device="meta")
    with pytest.raises(ValueError, match="matrix"):
        T.embedding(tokens, table[0])
    with pytest.raises(ValueError, match="int32 or int64"):
        T.embedding(tokens.float(), table)
    with pytest.raises(ValueError, match="tokens are on cpu"):
        T.embedding(torch.zeros(3, dtype=torch.int64), table)
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(ValueError, match="p must lie"):
            T.embedding(tokens, table, p=p)
    for step in (torch.zeros(2, dtype=torch.int64, device="meta"), torch.zeros(1, device="meta"), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(ValueError, match="step must be"):
            T.embedding(tokens, table, p=0.5, step=step)


def test_dropout_refuses():
    x = torch.zeros(5, 4, device="meta")
    with pytest.raises(ValueError, match="p must lie"):
        T.dropout(x, 2.0, 1)
    for res in (torch.zeros(4, 5, device="meta"), x.half(), torch.zeros(5, 4)):
        with pytest.raises(ValueError, match="residual must be"):
            T.dropout(x, 0.5, 1, residual=res)


def test_cross_entropy_refuses():
    x, w = torch.zeros(2, 3, 8, device="meta").half(), torch.zeros(9, 8, device="meta").half()
    y = torch.zeros(2, 3, dtype=torch.int64, device="meta")
    with pytest.raises(ValueError, match="bf16 or fp16"):
        T.linear_cross_entropy(x.float(), w, y)
    for bad in (w[:, :7], w[0], w[:0]):
        with pytest.raises(ValueError, match="do not fit"):
            T.linear_cross_entropy(x, bad, y)
    with pytest.raises(ValueError, match="or fp32"):
        T.linear_cross_entropy(x, w.bfloat16(), y)
    for bad in (y[0], y.float()):
        with pytest.raises(ValueError, match="labels must be"):
            T.linear_cross_entropy(x, w, bad)
    with pytest.raises(ValueError, match="row_weights must be"):
        T.linear_cross_entropy(x, w, y, y.double())
    with pytest.raises(ValueError, match="all arguments"):
        T.linear_cross_entropy(x, w, torch.zeros(2, 3, dtype=torch.int64))
