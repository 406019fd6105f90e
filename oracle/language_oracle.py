"""Dropout, embedding and cross entropy of the output projection in 64 bits, from their definitions (test infrastructure)."""
import numpy as np


def philox(counters, seed):
    """Philox4x32-10 (Salmon et al. 2011): [n, 4] 32-bit counters and a 64-bit key to [n, 4] words."""
    c = [np.asarray(counters)[:, i].astype(np.uint64) for i in range(4)]
    low = np.uint64(0xffffffff)
    k0, k1 = seed & 0xffffffff, seed >> 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return np.stack(c, 1)


def factors(n, p, seed, call):
    """What dropout multiplies n elements by; p as its 32-bit value."""
    p = float(np.float32(p))
    block = np.arange(-(-n // 4), dtype=np.uint64)
    call &= (1 << 64) - 1
    counters = np.stack([block & np.uint64(0xffffffff), block >> np.uint64(32),
                         np.full_like(block, call & 0xffffffff), np.full_like(block, call >> 32)], 1)
    words = philox(counters, seed).reshape(-1)[:n]
    keep = words >= np.uint64(int(np.floor(p * 2.0 ** 32 + 0.5)))
    return np.where(keep, 1 / (1 - p) if p < 1 else 0.0, 0.0)


def dropout(x, p, seed, call):
    """x of any shape; what is dropped becomes zero whatever it was."""
    f = factors(x.size, p, seed, call).reshape(x.shape)
    return np.where(f == 0, 0.0, x * f)


def embedding(table, tokens, scale=1.0, p=0.0, seed=0, call=0):
    vocab, cols = table.shape
    known = (tokens >= 0) & (tokens < vocab)
    y = np.zeros((len(tokens), cols))
    y[known] = table[tokens[known]] * scale
    return dropout(y, p, seed, call) if p else y


def embedding_grad(dy, tokens, vocab, scale=1.0, p=0.0, seed=0, call=0):
    known = (tokens >= 0) & (tokens < vocab)
    d = dropout(dy, p, seed, call) if p else dy
    out = np.zeros((vocab, dy.shape[1]))
    np.add.at(out, tokens[known], d[known] * scale)
    return out


def linear_cross_entropy(x, w, labels, weights=None, scale=1.0):
    """(loss of every row, total, dx, dw); weights None: the mean over the rows that have a label."""
    rows, vocab = x.shape[0], w.shape[0]
    counted = (labels >= 0) & (labels < vocab)
    c = np.full(rows, 1 / max(1, counted.sum())) if weights is None else weights
    each, dx, dw = np.zeros(rows), np.zeros_like(x), np.zeros_like(w)
    if counted.any():
        y = labels[counted]
        z = x[counted] @ w.T * scale
        top = z.max(1, keepdims=True)
        e = np.exp(z - top)
        total = e.sum(1, keepdims=True)
        at = np.arange(len(y))
        each[counted] = np.log(total[:, 0]) + top[:, 0] - z[at, y]
        d = e / total
        d[at, y] -= 1
        d *= scale * c[counted][:, None]
        dx[counted] = d @ w
        dw = d.T @ x[counted]
    return each, float((each[counted] * c[counted]).sum()), dx, dw
