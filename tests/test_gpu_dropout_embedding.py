"""Dropout, embedding and the embedding's gradient through the C ABI against the oracle in 64 bits.

Tolerances count roundings: half a step of the result's type, and half a step of fp32 for each product or sum before it."""
import numpy as np
import pytest

from oracle import language_oracle as L

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}           # relative
TINY = {"float32": 2.0 ** -150, "bfloat16": 2.0 ** -134, "float16": 2.0 ** -25}        # half of the smallest number
F32 = 2.0 ** -24


def torch_():
    import torch
    return torch


def B_():
    from paper_2101_10761_b200 import binding
    return binding


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def on_gpu(x, dtype, ld=None, shift=0):
    """(flat device buffer from the first element on, the whole buffer, values in 64 bits) of a matrix with rows ld apart;
    what lies between and around is NaN."""
    torch = torch_()
    rows, cols = x.shape
    ld = ld or cols
    t = torch.from_numpy(np.ascontiguousarray(x)).to(getattr(torch, dtype))
    store = torch.full((rows * ld + shift + 16,), float("nan"), dtype=t.dtype, device="cuda")
    view = store[shift:shift + rows * ld].view(rows, ld)
    view[:, :cols] = t.cuda()
    return store[shift:], store, t.double().numpy()


def rows_of(store, shift, rows, cols, ld):
    return store[shift:shift + rows * ld].view(rows, ld)[:, :cols].double().cpu().numpy()


def rest_is_nan(store, shift, rows, cols, ld):
    c = store.clone()
    c[shift:shift + rows * ld].view(rows, ld)[:, :cols] = float("nan")
    return bool(torch_().isnan(c).all())


def close(got, want, dtype, magnitude=None, roundings=0):
    """|got - want| within half a step of the type and `roundings` of fp32 on the sum of the terms' magnitudes."""
    magnitude = np.abs(want) if magnitude is None else magnitude
    bound = (HALF[dtype] * np.abs(want) + roundings * F32 * magnitude) * (1 + 2.0 ** -7) + TINY[dtype]
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (bad.sum(), np.abs(got - want)[bad].max(), np.argwhere(bad)[:5])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,shift", [(1, 0), (7, 0), (8, 0), (2049, 0), (2048, 1), (100003, 3), (1050000, 0)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(n, shift, dtype, residual):
    torch, B = torch_(), B_()
    r = rng(n + shift)
    x, _, hx = on_gpu(r.standard_normal((1, n)), dtype, shift=shift)
    res, _, hr = on_gpu(r.standard_normal((1, n)) * 3, dtype, shift=shift)
    out = torch.full((n + shift + 8,), float("nan"), dtype=x.dtype, device="cuda")
    p, seed, call = 0.3, (77 << 32) + n, 5 + (9 << 33)
    B.sidco_dropout(x, n, p, seed, call, out[shift:], residual=res if residual else None)
    torch.cuda.synchronize()
    dropped = L.dropout(hx[0], p, seed, call)
    want = dropped + (hr[0] if residual else 0)
    got = out[shift:shift + n].double().cpu().numpy()
    # factor and product: two roundings of the product; the sum: one of the result
    close(got, want, dtype, 2 * np.abs(dropped) + (np.abs(want) if residual else 0), 1)
    if not residual:
        assert np.array_equal(got == 0, dropped == 0)
    assert torch.isnan(out[:shift]).all() and torch.isnan(out[shift + n:]).all()


def test_dropout_in_place_and_backward_draw_the_same_mask():
    torch, B = torch_(), B_()
    n = 100001
    x = torch.ones(n, device="cuda")
    kept = x.clone()
    B.sidco_dropout(x, n, 0.5, 3, 4, x)
    B.sidco_dropout(kept, n, 0.5, 3, 4, kept, residual=kept)
    assert torch.equal(kept, x + 1) and set(x.unique().tolist()) == {0.0, 2.0}


def test_dropout_ends_of_p_and_what_is_dropped():
    torch, B = torch_(), B_()
    n = 4099
    x = torch.full((n,), float("nan"), device="cuda")
    x[::3] = float("inf")
    out = torch.empty_like(x)
    B.sidco_dropout(x, n, 1.0, 1, 1, out)
    assert bool((out == 0).all())
    B.sidco_dropout(x, n, 0.0, 1, 1, out)
    assert torch.equal(out.view(torch.int32), x.view(torch.int32))
    B.sidco_dropout(x, n, 0.4, 1, 1, out)
    kept = torch.from_numpy(L.factors(n, 0.4, 1, 1) > 0).cuda()
    assert torch.equal(out != 0, kept) and torch.equal(torch.isinf(out), kept & torch.isinf(x))
    B.sidco_dropout(x, 0, 0.4, 1, 1, out)


def test_dropout_step_is_read_when_the_kernel_runs():
    """A captured call draws a new mask for every value of the counter: the call number plus the counter, mod 2^64."""
    torch, B = torch_(), B_()
    n = 5000
    x, out = torch.ones(n, device="cuda"), torch.empty(n, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sidco_dropout(x, n, 0.5, 11, 2 ** 64 - 1, out, step=step)
        step += 1
    for k in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy() > 0, L.factors(n, 0.5, 11, 2 ** 64 - 1 + k) > 0)


def test_dropout_of_far_positions():
    """Elements on both sides of 2^32: their counters do not wrap."""
    torch, B = torch_(), B_()
    n = (1 << 32) + 1000
    x = torch.ones(n, dtype=torch.float16, device="cuda")
    B.sidco_dropout(x, n, 0.5, 21, 3, x)
    for at in (0, (1 << 31) - 400, (1 << 32) - 800, (1 << 32) + 200):
        block = np.arange(at // 4, at // 4 + 200, dtype=np.uint64)
        counters = np.stack([block & np.uint64(0xffffffff), block >> np.uint64(32), np.full_like(block, 3),
                             np.zeros_like(block)], 1)
        want = L.philox(counters, 21).reshape(-1) >= np.uint64(1 << 31)
        assert np.array_equal(x[at:at + 800].cpu().numpy() > 0, want), at


LOOKUPS = [  # n, vocab, cols, ld, ldo, shift, p
    (1, 1, 1, 1, 1, 0, 0.0), (5, 7, 3, 3, 3, 0, 0.3), (33, 10, 32, 32, 32, 0, 0.0), (64, 100, 8, 8, 8, 0, 0.6),
    (700, 1000, 1500, 1500, 1500, 0, 0.65), (17, 50, 1030, 1030, 1030, 0, 0.1), (40, 31, 129, 140, 133, 1, 0.4),
    (3, 9, 4100, 4104, 4100, 0, 0.5), (9, 4, 4096, 4096, 4096, 2, 0.2), (2000, 300, 12, 16, 20, 0, 0.5),
]


@pytest.mark.parametrize("table_type", TYPES)
@pytest.mark.parametrize("out_type", TYPES)
@pytest.mark.parametrize("case", LOOKUPS)
def test_embedding(case, table_type, out_type):
    torch, B = torch_(), B_()
    n, vocab, cols, ld, ldo, shift, p = case
    r = rng(n * 31 + cols)
    table, _, held = on_gpu(r.standard_normal((vocab, cols)), table_type, ld, shift)
    tokens = r.integers(-2, vocab, n)
    tokens[0] = 0
    wide = (n + cols) % 2 == 0
    t = torch.from_numpy(tokens).to(torch.int64 if wide else torch.int32).cuda()
    out = torch.full((n * ldo + shift + 16,), float("nan"), dtype=getattr(torch, out_type), device="cuda")
    B.sidco_embedding(table, vocab, cols, ld, t, n, 1.7, out[shift:], ldo, p=p, seed=n, call=cols)
    torch.cuda.synchronize()
    want = L.embedding(held, tokens, float(np.float32(1.7)), p, n, cols)
    got = rows_of(out, shift, n, cols, ldo)
    close(got, want, out_type, None, 3)                  # scale, factor, product
    assert np.array_equal(got == 0, want == 0)
    assert rest_is_nan(out, shift, n, cols, ldo)


def test_embedding_is_dropout_of_the_lookup():
    torch, B = torch_(), B_()
    n, vocab, cols = 300, 41, 101
    table = torch.randn(vocab, cols, device="cuda")
    t = torch.randint(0, vocab, (n,), device="cuda")
    y, z = torch.empty(n, cols, device="cuda"), torch.empty(n, cols, device="cuda")
    B.sidco_embedding(table, vocab, cols, cols, t, n, 1.0, y, cols)
    assert torch.equal(y, table[t])
    B.sidco_dropout(y, n * cols, 0.25, 8, 9, y)
    B.sidco_embedding(table, vocab, cols, cols, t, n, 1.0, z, cols, p=0.25, seed=8, call=9)
    assert torch.equal(y, z)


def test_embedding_reports_tokens_outside_the_table():
    torch, B = torch_(), B_()
    vocab, cols = 5, 6
    table = torch.randn(vocab, cols, device="cuda")
    status = torch.full((1,), 99, dtype=torch.int32, device="cuda")
    t = torch.tensor([4, 5, -1, 2 ** 40, 0], device="cuda")
    out = torch.empty(5, cols, device="cuda")
    B.sidco_embedding(table, vocab, cols, cols, t, 5, 1.0, out, cols, status=status)
    assert status.item() == B.EMBEDDING_ST_TOKEN
    assert torch.equal(out[[0, 4]], table[[4, 0]]) and bool((out[1:4] == 0).all())
    B.sidco_embedding(table, vocab, cols, cols, t[[0, 2, 4]], 3, 1.0, out, cols, status=status)
    assert status.item() == 0


GRADS = [  # n, vocab, cols, ld_dy, ldd, shift, p, kind of tokens
    (1, 1, 1, 1, 1, 0, 0.0, "any"), (5, 9, 3, 3, 3, 0, 0.3, "any"), (32, 300, 32, 32, 32, 0, 0.0, "any"),
    (33, 5, 130, 130, 130, 0, 0.5, "any"), (700, 1000, 1500, 1500, 1500, 0, 0.65, "any"), (700, 70000, 12, 16, 20, 0, 0.2, "any"),
    (5000, 40, 17, 20, 19, 1, 0.1, "skewed"), (4096, 256, 64, 64, 64, 0, 0.0, "one"), (4097, 3, 64, 64, 64, 2, 0.0, "one"),
    (40000, 5003, 65, 65, 65, 0, 0.1, "skewed"), (9000, 2, 8, 8, 8, 0, 0.0, "any"), (257, 17, 5, 5, 5, 0, 0.5, "none"),
    (100000, 66000, 4, 4, 4, 0, 0.0, "skewed"), (8192, 65536, 4, 4, 4, 0, 0.0, "falling"),
    (2048, 7, 300, 300, 300, 0, 0.3, "skewed"), (2049, 2048, 264, 264, 264, 0, 0.1, "any"), (1500, 1, 9, 9, 9, 0, 0.0, "any"),
    (2500, 30, 264, 272, 264, 8, 0.25, "skewed"),
]


def tokens_of(kind, n, vocab, r):
    if kind == "one":
        return np.full(n, vocab - 1)
    if kind == "none":
        return np.where(r.random(n) < 0.5, -1, vocab + 3)
    if kind == "falling":
        return (n - 1 - np.arange(n)) * 8 % vocab
    t = r.integers(0, vocab, n) if kind == "any" else np.minimum((r.pareto(0.6, n)).astype(np.int64), vocab - 1)
    t[r.random(n) < 0.05] = -7
    t[r.random(n) < 0.02] = vocab
    return t


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("case", GRADS)
@pytest.mark.parametrize("types", [(a, b) for a in TYPES for b in TYPES])
def test_embedding_grad(case, types, add):
    torch, B = torch_(), B_()
    n, vocab, cols, ld_dy, ldd, shift, p, kind = case
    r = rng(n * 7 + cols)
    tokens = tokens_of(kind, n, vocab, r)
    known = (tokens >= 0) & (tokens < vocab)
    values = r.standard_normal((n, cols))
    values[~known] = np.nan                              # behind padding: not read
    dy, _, held = on_gpu(values, types[0], ld_dy, shift)
    held[~known] = 0
    old, store, before = on_gpu(r.standard_normal((vocab, cols)), types[1], ldd, shift)
    t = torch.from_numpy(tokens).to(torch.int32 if add else torch.int64).cuda()
    need = B.sidco_embedding_grad_workspace_bytes(n, vocab, cols)
    ws = torch.full((need + 256,), 205, dtype=torch.uint8, device="cuda")
    kw = dict(p=p, seed=n, call=cols)
    B.sidco_embedding_grad(dy, ld_dy, t, n, vocab, cols, 0.8, old, ldd, ws, need, add=add, **kw)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 205).all())
    scale = float(np.float32(0.8))
    want = L.embedding_grad(held, tokens, vocab, scale, **kw) + (before if add else 0)
    magnitude = L.embedding_grad(np.abs(held), tokens, vocab, scale, **kw) + (np.abs(before) if add else 0)
    many = np.bincount(tokens[known], minlength=vocab)[:, None]
    got = rows_of(store, shift, vocab, cols, ldd)
    # factor and product per term, the sum of `many`, the scale, the addition
    close(got, want, types[1], magnitude, many + 4)
    untouched = many[:, 0] == 0
    assert np.array_equal(got[untouched], before[untouched] if add else np.zeros_like(before[untouched]))
    assert rest_is_nan(store, shift, vocab, cols, ldd)


def test_embedding_grad_repeats_bit_for_bit_and_across_streams():
    torch, B = torch_(), B_()
    n, vocab, cols = 30000, 900, 200
    t = torch.randint(0, vocab, (n,), device="cuda") // 7
    dy = torch.randn(n, cols, device="cuda")
    need = B.sidco_embedding_grad_workspace_bytes(n, vocab, cols)
    outs = []
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(6):
        with torch.cuda.stream(streams[i & 1]):
            out = torch.empty(vocab, cols, device="cuda")
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            B.sidco_embedding_grad(dy, cols, t, n, vocab, cols, 1.0, out, cols, ws, need)
            outs.append((out, ws))
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0][0], o) for o, _ in outs)


@pytest.mark.parametrize("n", [1000, 5000])
def test_embedding_grad_in_a_graph_follows_its_inputs(n):
    torch, B = torch_(), B_()
    vocab, cols = 300, 60
    t = torch.randint(0, vocab, (n,), device="cuda")
    dy, out = torch.randn(n, cols, device="cuda"), torch.empty(vocab, cols, device="cuda")
    need = B.sidco_embedding_grad_workspace_bytes(n, vocab, cols)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sidco_embedding_grad(dy, cols, t, n, vocab, cols, 1.0, out, cols, ws, need)
    for _ in range(3):
        t.copy_(torch.randint(-1, vocab, (n,), device="cuda"))
        dy.normal_()
        out.fill_(9)
        g.replay()
        want = L.embedding_grad(dy.double().cpu().numpy(), t.cpu().numpy(), vocab)
        assert np.allclose(out.cpu().numpy(), want, atol=1e-4)         # sums of some 20 terms below 5


def test_nothing_to_do():
    torch, B = torch_(), B_()
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    out = torch.full((4, 3), 5.0, device="cuda")
    B.sidco_embedding(None, 0, 3, 3, t, 4, 1.0, out, 3, table_type=0)           # a table without rows
    assert bool((out == 0).all())
    B.sidco_embedding(out, 4, 3, 3, None, 0, 1.0, None, 3, token_type=4, out_type=0)
    B.sidco_embedding_grad(None, 3, None, 0, 4, 3, 1.0, out.fill_(5), 3, None, 0, add=True, dy_type=0, token_type=3)
    assert bool((out == 5).all())
    B.sidco_embedding_grad(None, 3, None, 0, 4, 3, 1.0, out, 3, None, 0, dy_type=0, token_type=3)
    assert bool((out == 0).all())
