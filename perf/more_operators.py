"""Timed cases of the embedding, the dropout and the cross entropy of the output projection, with their plain forms.

Every operator is computed in two ways: in elementary torch operations in 32 bits (``own`` false) and by the calls a
user makes of ``paper_2101_10761_b200.binding`` (``own`` true).  ``prepare`` gives both the same inputs.

Dropout: element i of a tensor is dropped if word i % 4 of Philox4x32-10 is below round(p 2^32); the generator's key is the
seed, its counter i / 4 in the low and the number of the call in the high 64 bits.
"""
import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
MOST = 4096 * 128000 * 4096           # rows x vocabulary x hidden of the largest loss


def listed():
    return [
        # input of the LSTM language model: 20 sequences of 35 tokens, fp32 master table, dropout of the large model
        {"name": "lookup 700x1500", "op": "lookup", "n": 700, "vocab": 10000, "cols": 1500, "table": "fp32", "type": "bf16",
         "p": 0.65, "padding": 0.0},
        # input of a large model: 16 sequences of 2048 tokens, some of them padded, no dropout
        {"name": "lookup 32768x4096", "op": "lookup", "n": 32768, "vocab": 128000, "cols": 4096, "table": "bf16",
         "type": "bf16", "p": 0.0, "padding": 0.1},
        # the LSTM's embedding gradient, dense in the flat fp32 gradient: 99 % of its rows are zero
        {"name": "table gradient 700 of 10000x1500", "op": "table gradient", "n": 700, "vocab": 10000, "cols": 1500,
         "type": "bf16", "table": "fp32", "p": 0.65, "padding": 0.0, "add": False},
        # many tokens of few words: long sums, added to the gradient that a tied output projection has left
        {"name": "table gradient 65536 of 5003x1030 add", "op": "table gradient", "n": 65536, "vocab": 5003, "cols": 1030,
         "type": "fp16", "table": "fp32", "p": 0.1, "padding": 0.1, "add": True},
        # large model
        {"name": "table gradient 32768 of 128000x2048", "op": "table gradient", "n": 32768, "vocab": 128000, "cols": 2048,
         "type": "bf16", "table": "bf16", "p": 0.0, "padding": 0.0, "add": False},
        # between the LSTM's layers: forward and backward
        {"name": "dropout 700x1500", "op": "dropout", "n": 700 * 1500, "type": "bf16", "p": 0.65, "residual": False},
        # behind a block of a large model, added to its residual stream
        {"name": "dropout 8192x8192 residual", "op": "dropout", "n": 8192 * 8192, "type": "bf16", "p": 0.1,
         "residual": True},
        # an odd count in 32 bits
        {"name": "dropout 9999999 fp32", "op": "dropout", "n": 9999999, "type": "fp32", "p": 0.5, "residual": False},
        # the LSTM's output projection and loss, a training step and an evaluation
        {"name": "loss 700x10000x1500", "op": "loss", "rows": 700, "vocab": 10000, "hidden": 1500, "type": "bf16",
         "ignored": 0.0, "weighted": False, "add": False, "grads": True},
        {"name": "loss 700x10000x1500 evaluation", "op": "loss", "rows": 700, "vocab": 10000, "hidden": 1500,
         "type": "bf16", "ignored": 0.0, "weighted": False, "add": False, "grads": False},
        # answers behind prompts: half of the labels are ignored, the others weighted, sizes without alignment
        {"name": "loss 3001x32003x1031 masked", "op": "loss", "rows": 3001, "vocab": 32003, "hidden": 1031, "type": "fp16",
         "ignored": 0.5, "weighted": True, "add": True, "grads": True},
        # a large model
        {"name": "loss 4096x128000x4096", "op": "loss", "rows": 4096, "vocab": 128000, "hidden": 4096, "type": "bf16",
         "ignored": 0.0, "weighted": False, "add": False, "grads": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["lookup", "table gradient", "dropout", "loss", "loss"])
    if op == "dropout":
        return {"op": op, "n": _log(rng, 1000, 8192 * 8192), "type": rng.choice(list(TYPES)),
                "p": rng.choice([0.05, 0.1, 0.3, 0.5, 0.65]), "residual": rng.random() < 0.5}
    if op == "loss":
        rows = _log(rng, 1, 8192)
        vocab = _log(rng, 200, min(131072, 4096 * 131072 / rows))
        return {"op": op, "rows": rows, "vocab": vocab, "hidden": _log(rng, 64, min(8192, MOST / rows / vocab)),
                "type": rng.choice(["bf16", "fp16"]), "ignored": rng.choice([0.0, 0.0, 0.1, 0.6]),
                "weighted": rng.random() < 0.3, "add": rng.random() < 0.3, "grads": rng.random() < 0.8}
    n = _log(rng, 1, 65536)
    cols = _log(rng, 32, min(8192, 32768 * 4096 / n))
    case = {"op": op, "n": n, "vocab": _log(rng, 100, min(131072, 2.6e8 / cols)), "cols": cols,
            "type": rng.choice(list(TYPES)), "table": rng.choice(list(TYPES)), "p": rng.choice([0.0, 0.0, 0.1, 0.65]),
            "padding": rng.choice([0.0, 0.1])}
    return case if op == "lookup" else {**case, "add": rng.random() < 0.4}


# ---------------------------------------------------------------------------------------------- inputs


def _zipf(vocab, device):
    """How often the words of a text occur, by rank."""
    return 1.0 / (torch.arange(vocab, device=device, dtype=torch.float64) + 2.7)


def _words(n, vocab, g):
    """Tokens of a Zipf law over a shuffled vocabulary."""
    edges = torch.cumsum(_zipf(vocab, "cuda"), 0)
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * edges[-1]
    rank = torch.searchsorted(edges, u).clamp(max=vocab - 1)
    return torch.randperm(vocab, generator=g, device="cuda")[rank]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    s = {"case": case, "seed": random.Random(seed).getrandbits(63), "call": seed % 1000}
    if case["op"] == "dropout":
        s["x"], s["dy"] = (normal(case["n"]).to(TYPES[case["type"]]) for _ in range(2))
        s["residual"] = normal(case["n"], scale=3.0).to(TYPES[case["type"]]) if case["residual"] else None
    elif case["op"] == "loss":
        rows, vocab, hidden, dtype = case["rows"], case["vocab"], case["hidden"], TYPES[case["type"]]
        labels = _words(rows, vocab, g)
        w = normal(vocab, hidden, scale=2 * hidden ** -0.5)
        # some rows know their label, some do not
        x = normal(rows, hidden) + torch.rand(rows, 1, generator=g, device="cuda") * 2 * w[labels]
        if case["ignored"]:
            labels = torch.where(torch.rand(rows, generator=g, device="cuda") < case["ignored"], -100, labels)
        s["x"], s["w"], s["labels"] = x.to(dtype), w.to(dtype), labels
        # (with the factor by which training in 16 bits keeps its gradients above the smallest numbers)
        s["weights"] = torch.rand(rows, generator=g, device="cuda") * (1024 / rows) if case["weighted"] else None
        if case["grads"]:                              # what earlier steps have left, or nothing
            s["dw"] = (normal(vocab, hidden, scale=1e-3) if case["add"] else torch.zeros_like(w)).to(dtype)
    else:
        n, vocab, cols = case["n"], case["vocab"], case["cols"]
        tokens = _words(n, vocab, g)
        if case["padding"]:
            tokens = torch.where(torch.rand(n, generator=g, device="cuda") < case["padding"], -1, tokens)
        s["tokens"], s["scale"] = tokens, cols ** 0.5
        if case["op"] == "lookup":
            s["table"] = normal(vocab, cols, scale=cols ** -0.5).to(TYPES[case["table"]])
        else:
            s["dy"] = normal(n, cols, scale=1e-3).to(TYPES[case["type"]])
            s["dtable"] = normal(vocab, cols, scale=1e-3 if case["add"] else 0.0).to(TYPES[case["table"]])
    return s


# ---------------------------------------------------------------------------------------------- plain forms


def _threshold(p):
    """(draws below it drop, the factor of the others) for p as a 32-bit number."""
    p = torch.tensor(p, dtype=torch.float32).double().item()
    return int(math.floor(p * 2 ** 32 + 0.5)), 1 / (1 - p)


def _keep(n, p, seed, call):
    """Truth values of n elements."""
    low = 0xffffffff
    i = torch.arange(-(-n // 4), device="cuda", dtype=torch.int64)
    c = [i & low, i >> 32, torch.full_like(i, call & low), torch.full_like(i, call >> 32)]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57       # (products wrap; their 64 bits are right)
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return (torch.stack(c, 1).view(-1)[:n]) >= _threshold(p)[0]


def _dropped(x, s):
    p = s["case"]["p"]
    if p == 0:
        return x
    keep = _keep(x.numel(), p, s["seed"], s["call"]).view(x.shape)
    return torch.where(keep, x * _threshold(p)[1], 0.0)


def _plain(s):
    case = s["case"]
    if case["op"] == "dropout":
        y = _dropped(s["x"].float(), s)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(s["x"].dtype), "dx": _dropped(s["dy"].float(), s).to(s["x"].dtype)}
    if case["op"] == "lookup":
        t = s["tokens"]
        y = torch.where((t >= 0)[:, None], s["table"][t.clamp(min=0)].float() * s["scale"], 0.0)
        return _dropped(y, s).to(TYPES[case["type"]])
    if case["op"] == "table gradient":
        t = s["tokens"]
        dy = _dropped(s["dy"].float(), s) * s["scale"]
        sums = torch.zeros(case["vocab"], case["cols"], device="cuda")
        sums.index_add_(0, t.clamp(min=0), torch.where((t >= 0)[:, None], dy, 0.0))
        s["dtable"].copy_(sums + s["dtable"].float() if case["add"] else sums)
        return s["dtable"]
    labels, x, w = s["labels"], s["x"].float(), s["w"].float()
    rows = torch.arange(case["rows"], device="cuda")
    counted = labels >= 0
    safe = labels.clamp(min=0)
    c = s["weights"] if s["weights"] is not None else 1.0 / counted.sum().clamp(min=1).float()
    c = torch.where(counted, c, 0.0)
    logits = x @ w.T
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    each = torch.where(counted, (torch.log(total) + top)[:, 0] - logits[rows, safe], 0.0)
    out = {"rows": each, "loss": (each * c).sum()}
    if case["grads"]:
        d = e / total
        d[rows, safe] -= 1.0
        d *= c[:, None]
        out["dx"] = (d @ w).to(s["x"].dtype)
        dw = d.T @ x
        s["dw"].copy_(dw + s["dw"].float() if case["add"] else dw)
        out["dw"] = s["dw"]
    return out


# ---------------------------------------------------------------------------------------------- the framework's calls


def _kept(s, name, make):
    """A buffer that the caller keeps from one call to the next."""
    if name not in s:
        s[name] = make()
    return s[name]


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def _framework(s):
    from paper_2101_10761_b200 import binding as K
    case = s["case"]
    if case["op"] == "dropout":
        y, dx = _kept(s, "out", lambda: (torch.empty_like(s["x"]), torch.empty_like(s["dy"])))
        K.sidco_dropout(s["x"], case["n"], case["p"], s["seed"], s["call"], y, residual=s["residual"])
        K.sidco_dropout(s["dy"], case["n"], case["p"], s["seed"], s["call"], dx)
        return {"y": y, "dx": dx}
    if case["op"] == "lookup":
        n, vocab, cols = case["n"], case["vocab"], case["cols"]
        out = _kept(s, "out", lambda: torch.empty(n, cols, dtype=TYPES[case["type"]], device="cuda"))
        K.sidco_embedding(s["table"], vocab, cols, cols, s["tokens"], n, s["scale"], out, cols, p=case["p"],
                          seed=s["seed"], call=s["call"])
        return out
    if case["op"] == "table gradient":
        n, vocab, cols = case["n"], case["vocab"], case["cols"]
        need = _kept(s, "need", lambda: K.sidco_embedding_grad_workspace_bytes(n, vocab, cols))
        K.sidco_embedding_grad(s["dy"], cols, s["tokens"], n, vocab, cols, s["scale"], s["dtable"], cols,
                               _kept(s, "workspace", lambda: _bytes(need)), need, add=case["add"], p=case["p"],
                               seed=s["seed"], call=s["call"])
        return s["dtable"]
    rows, vocab, hidden = case["rows"], case["vocab"], case["hidden"]
    each, loss = _kept(s, "out", lambda: (torch.empty(rows, device="cuda"), torch.empty((), device="cuda")))
    out = {"rows": each, "loss": loss}
    if case["grads"]:
        out["dx"] = _kept(s, "dx", lambda: torch.empty_like(s["x"]))
        out["dw"] = s["dw"]
    need = _kept(s, "need", lambda: K.sidco_linear_cross_entropy_workspace_bytes(s["x"], s["w"], hidden, rows, vocab, hidden,
                                                                                 grads=case["grads"]))
    K.sidco_linear_cross_entropy(s["x"], hidden, s["w"], hidden, s["labels"], rows, vocab, hidden, each, loss,
                                 out.get("dx"), hidden, out.get("dw"), hidden,
                                 _kept(s, "workspace", lambda: _bytes(need)), need, row_weights=s["weights"],
                                 add=case["add"])
    return out


def run(state):
    return _framework(state) if own else _plain(state)


def _different(case):
    """How many different words are to be expected among the tokens."""
    q = _zipf(case["vocab"], "cpu")
    return int((1 - (1 - q / q.sum()) ** (case["n"] * (1 - case["padding"]))).sum())


def work(case):
    if case["op"] == "dropout":
        return {"bytes": case["n"] * SIZE[case["type"]] * (5 if case["residual"] else 4), "flops": 0}
    if case["op"] == "lookup":
        return {"bytes": case["cols"] * (_different(case) * SIZE[case["table"]] + case["n"] * SIZE[case["type"]])
                + 8 * case["n"], "flops": 0}
    if case["op"] == "table gradient":
        rows = 2 * _different(case) if case["add"] else case["vocab"]
        read = case["n"] * (1 - case["padding"])
        return {"bytes": case["cols"] * (rows * SIZE[case["table"]] + read * SIZE[case["type"]]) + 8 * case["n"],
                "flops": 0}
    rows, vocab, hidden, size = case["rows"], case["vocab"], case["hidden"], SIZE[case["type"]]
    counted = rows * (1 - case["ignored"])
    grads = 1 if case["grads"] else 0
    return {"bytes": size * hidden * (rows + vocab) * (1 + grads) + (size * hidden * vocab if case["add"] and grads else 0)
            + 12 * rows, "flops": 2 * counted * vocab * hidden * (1 + 2 * grads)}


# ---------------------------------------------------------------------------------------------- from the definition


def _exact_keep(n, p, seed, call):
    """The generator once more, with products of 16-bit halves."""
    def times(a, b):                                       # (high, low) 32 bits of a product of two 32-bit numbers
        a0, a1, b0, b1 = a % 65536, a // 65536, b % 65536, b // 65536
        low, mid1, mid2 = a0 * b0, a1 * b0, a0 * b1
        mid = low // 65536 + mid1 % 65536 + mid2 % 65536
        return a1 * b1 + mid1 // 65536 + mid2 // 65536 + mid // 65536, mid % 65536 * 65536 + low % 65536

    keep = torch.empty(n, dtype=torch.bool, device="cuda")
    whole = 2 ** 32
    for at in range(0, n, 1 << 24):
        blocks = torch.arange(at // 4, -(-min(n, at + (1 << 24)) // 4), device="cuda")
        x0, x1 = blocks % whole, blocks // whole
        x2, x3 = torch.full_like(blocks, call % whole), torch.full_like(blocks, call // whole)
        for r in range(10):
            h0, l0 = times(x0, 0xD2511F53)
            h2, l2 = times(x2, 0xCD9E8D57)
            x0, x1, x2, x3 = (h2 ^ x1 ^ ((seed % whole + r * 0x9E3779B9) % whole), l2,
                              h0 ^ x3 ^ ((seed // whole + r * 0xBB67AE85) % whole), l0)
        part = torch.stack((x0, x1, x2, x3), -1).flatten().double() / whole
        end = min(n, at + (1 << 24))
        keep[at:end] = part[:end - at] * whole >= _threshold(p)[0]
    return keep


def exact(case, seed):
    s = prepare(case, seed)
    p = case.get("p", 0.0)

    def factor(*shape):
        if not p:
            return torch.ones((), dtype=torch.float64, device="cuda")
        return _exact_keep(math.prod(shape), p, s["seed"], s["call"]).view(shape) * _threshold(p)[1]

    if case["op"] == "dropout":
        f = factor(case["n"])
        y = s["x"].double() * f
        return {"y": y if s["residual"] is None else y + s["residual"].double(), "dx": s["dy"].double() * f}
    if case["op"] == "lookup":
        rows = torch.cat((s["table"].double(), torch.zeros(1, case["cols"], dtype=torch.float64, device="cuda")))
        return rows[s["tokens"]] * s["scale"] * factor(case["n"], case["cols"])
    if case["op"] == "table gradient":
        out = s["dtable"].double() if case["add"] else torch.zeros_like(s["dtable"], dtype=torch.float64)
        dy = s["dy"].double() * factor(case["n"], case["cols"])
        used = s["tokens"] >= 0
        return out.index_put_((s["tokens"][used],), dy[used] * s["scale"], accumulate=True)
    x, w, rows = s["x"].double(), s["w"].double(), case["rows"]
    counted = s["labels"] >= 0
    c = s["weights"].double() if case["weighted"] else torch.full((rows,), 1 / max(1, int(counted.sum())),
                                                                  dtype=torch.float64, device="cuda")
    each = torch.zeros(rows, dtype=torch.float64, device="cuda")
    out = {"rows": each}
    if case["grads"]:
        dx = torch.zeros_like(x)
        dw = s["dw"].double() if case["add"] else torch.zeros_like(w)
    for part in torch.nonzero(counted)[:, 0].split(1024):
        z, y = x[part] @ w.T, s["labels"][part]
        log_p = z - torch.logsumexp(z, 1, keepdim=True)
        each[part] = -log_p.gather(1, y[:, None])[:, 0]
        if case["grads"]:
            d = log_p.exp_()
            d.scatter_add_(1, y[:, None], torch.full_like(y, -1, dtype=torch.float64)[:, None])
            d *= c[part, None]
            dx[part] = d @ w
            dw += d.T @ x[part]
    out["loss"] = (each * c).sum()
    if case["grads"]:
        out.update(dx=dx, dw=dw)
    return out
