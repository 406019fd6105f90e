"""4-bit quantisation, reading back, product, compressor and mean through the C ABI against the oracle in 64 bits."""
import numpy as np
import pytest

from oracle import mx4_oracle as Q

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
GUARD = 77


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def torch_():
    import torch
    return torch


def B_():
    from paper_2101_10761_b200 import binding
    return binding


def guarded(n, shift=0):
    """n bytes with 64 marked ones on either side, 16-byte aligned plus `shift`."""
    torch = torch_()
    store = torch.full((n + 160,), GUARD, dtype=torch.uint8, device="cuda")
    return store, store[64 + shift:64 + shift + n]


def untouched(store, view, shift=0):
    n = view.numel()
    return bool((store[:64 + shift] == GUARD).all()) and bool((store[64 + shift + n:] == GUARD).all())


def values(seed, rows, cols):
    """Rows of very different scale, with zeros and exact ties among them."""
    r = rng(seed)
    x = r.standard_normal((rows, cols)) * np.exp(r.uniform(-8, 8, (rows, 1)))
    x[r.random((rows, cols)) < 0.1] = 0.0
    pick = r.random((rows, cols)) < 0.2
    x[pick] = np.sign(x[pick]) * 2.0 ** r.integers(-4, 5, pick.sum()) * r.choice([.75, 1.25, 1.75, 2.5, 3.5, 5], pick.sum())
    return x


def on_gpu(x, dtype, ld=None, shift=0):
    """x as a device matrix of leading dimension ld, its base `shift` elements off; and what it holds in 64 bits."""
    torch = torch_()
    rows, cols = x.shape
    ld = ld or cols
    t = torch.from_numpy(np.ascontiguousarray(x)).to(getattr(torch, dtype))
    store = torch.full((rows * ld + shift + 8,), float("nan"), dtype=t.dtype, device="cuda")
    view = store[shift:shift + rows * ld].view(rows, ld)
    view[:, :cols] = t.cuda()
    return store[shift:], t.double().numpy()


SHAPES = [(1, 1), (1, 32), (3, 45), (31, 33), (64, 8), (127, 129), (128, 128), (129, 257), (200, 300), (1, 5000),
          (5000, 1), (700, 1500)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_both_forms_exactly(rows, cols, dtype):
    torch, B = torch_(), B_()
    ld, shift = (cols, 0) if (rows + cols) % 2 else (cols + 5, 3)              # vector path and the other
    x, held = on_gpu(values(rows * 7 + cols, rows, cols), dtype, ld, shift)
    bufs = [guarded(n) for n in (B.sidco_mx4_code_bytes(rows, cols), B.sidco_mx4_scale_bytes(rows, cols),
                                 B.sidco_mx4_code_bytes(cols, rows), B.sidco_mx4_scale_bytes(cols, rows))]
    B.sidco_mx4_quantize(x, rows, cols, ld, *[v for _, v in bufs])
    torch.cuda.synchronize()
    assert all(untouched(s, v) for s, v in bufs)
    for h, (codes, scales) in ((held, bufs[:2]), (held.T, bufs[2:])):
        want_c, want_s, want_v = Q.quantize(h)
        assert np.array_equal(scales[1].cpu().numpy(), want_s)
        assert np.array_equal(codes[1].cpu().numpy(), want_c)
        r, c = h.shape
        for out_type in TYPES:
            out = torch.full((r * (c + 3) + 8,), 7.0, dtype=getattr(torch, out_type), device="cuda")
            B.sidco_mx4_dequantize(codes[1], scales[1], r, c, out, c + 3)
            got = out[:r * (c + 3)].view(r, c + 3).double().cpu().numpy()
            with np.errstate(over="ignore"):
                want = torch.from_numpy(want_v.astype(np.float32)).to(getattr(torch, out_type)).double().numpy()
            assert np.array_equal(got[:, :c], want)
            assert (got[:, c:] == 7.0).all()


def test_one_form_alone_is_the_same_as_both():
    torch, B = torch_(), B_()
    rows, cols = 150, 333
    x, held = on_gpu(values(1, rows, cols), "bfloat16")
    for r, c, h, alone in ((rows, cols, held, 0), (cols, rows, held.T, 1)):
        codes, scales = guarded(B.sidco_mx4_code_bytes(r, c)), guarded(B.sidco_mx4_scale_bytes(r, c))
        args = [codes[1], scales[1]]
        B.sidco_mx4_quantize(x, rows, cols, cols, *(args + [None, None] if alone == 0 else [None, None] + args))
        want_c, want_s, _ = Q.quantize(h)
        assert np.array_equal(codes[1].cpu().numpy(), want_c) and np.array_equal(scales[1].cpu().numpy(), want_s)
        assert untouched(*codes) and untouched(*scales)


def test_ends_of_the_range_and_non_finite_blocks():
    """Subnormals, the largest fp32 value, negative zeros, NaN and infinities, each in a block of its own."""
    torch, B = torch_(), B_()
    x = np.zeros((12, 64), np.float32)
    x[0, :4] = [2.0 ** -149, -2.0 ** -148, 2.0 ** -140, 0]
    x[1, :4] = [2.0 ** -127, 2.0 ** -126, 3 * 2.0 ** -128, -2.0 ** -129]
    x[2, :3] = [np.finfo(np.float32).max, -1e38, 1.0]
    x[3, :] = -0.0
    x[4, 3] = np.nan
    x[5, 40] = np.inf
    x[6, 2], x[6, 3] = -np.inf, np.nan
    x[7, :] = 6.0
    x[8, :] = -7.99
    x[9, :32] = 2.0 ** np.arange(-16, 16)
    x[10, 0] = 1.0
    x[11, :] = np.float32(1) + np.float32(2.0 ** -23)
    t = torch.from_numpy(x).cuda()
    codes = torch.empty(B.sidco_mx4_code_bytes(12, 64), dtype=torch.uint8, device="cuda")
    scales = torch.empty(B.sidco_mx4_scale_bytes(12, 64), dtype=torch.uint8, device="cuda")
    codes_t = torch.empty(B.sidco_mx4_code_bytes(64, 12), dtype=torch.uint8, device="cuda")
    scales_t = torch.empty(B.sidco_mx4_scale_bytes(64, 12), dtype=torch.uint8, device="cuda")
    B.sidco_mx4_quantize(t, 12, 64, 64, codes, scales, codes_t, scales_t)
    for h, c, s in ((x, codes, scales), (x.T, codes_t, scales_t)):
        want_c, want_s, want_v = Q.quantize(h)
        assert np.array_equal(c.cpu().numpy(), want_c) and np.array_equal(s.cpu().numpy(), want_s)
        out = torch.empty(h.shape, dtype=torch.float32, device="cuda")
        B.sidco_mx4_dequantize(c, s, *h.shape, out, h.shape[1])
        assert np.array_equal(out.cpu().numpy().astype(np.float64), want_v, equal_nan=True)


def operands(seed, rows, k, scale=1.0):
    """(codes, scales) on the device and the values in 64 bits."""
    torch = torch_()
    c, s, v = Q.quantize((rng(seed).standard_normal((rows, k)) * np.exp(rng(seed + 1).normal(0, 1, (rows, 1))) * scale))
    return torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), v


def ulp_half(dtype):
    """Half a unit in the last place, relative: 2^-p of a type with p significant bits."""
    return {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]


def check_product(got, a, b, c0, dtype):
    """|error| <= k 2^-23 sum |a||b| for fp32 sums in any order, and half a unit of the result's type."""
    exact = a @ b.T + (0 if c0 is None else c0)
    size = np.abs(a) @ np.abs(b).T + (0 if c0 is None else np.abs(c0))
    tol = (a.shape[1] + 2) * 2.0 ** -23 * size + ulp_half(dtype) * np.abs(exact) * (1 + 2.0 ** -8) + 2.0 ** -25
    assert (np.abs(got - exact) <= tol).all(), float((np.abs(got - exact) - tol).max())


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 300, 1500), (2, 129, 33), (5, 40, 64), (8, 260, 700), (9, 1000, 65), (16, 128, 2080),
            (17, 500, 256), (31, 33, 31), (33, 700, 288), (64, 64, 4100), (100, 90, 320), (128, 128, 128), (129, 127, 257),
            (130, 300, 1100), (256, 512, 96), (300, 130, 2048), (520, 600, 1500), (1000, 8, 500), (2000, 1, 129)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, dtype):
    torch, B = torch_(), B_()
    ac, as_, a = operands(m + 3 * k, m, k)
    bc, bs, b = operands(n + 5 * k, n, k, k ** -0.5)
    for ldc, shift, add in ((n, 0, False), (n + 3, 1, True), ((n + 7) // 8 * 8, 0, True)):
        c0 = rng(m + n).standard_normal((m, n))
        store, held = on_gpu(c0, dtype, ldc, shift)
        B.sidco_mx4_matmul(ac, as_, bc, bs, m, n, k, store, ldc, add)
        torch.cuda.synchronize()
        got = store[:m * ldc].view(m, ldc).double().cpu().numpy()
        assert np.isnan(got[:, n:]).all() and torch.isnan(store[m * ldc:]).all(), "wrote outside C"
        check_product(got[:, :n], a, b, held if add else None, dtype)
    assert B.sidco_wait_timeouts() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(5000, 1030, 300), (2560, 2304, 64), (300, 19000, 520), (19001, 100, 33), (2300, 2300, 1500)])
def test_large_product(m, n, k, dtype):
    """As test_product, at sizes that go by pairs of CTAs: aligned and unaligned C, ragged edges, more tiles than pairs."""
    torch, B = torch_(), B_()
    ac, as_, a = operands(m + 3 * k, m, k)
    bc, bs, b = operands(n + 5 * k, n, k, k ** -0.5)
    exact = torch.from_numpy(a).cuda() @ torch.from_numpy(b).cuda().T
    size = torch.from_numpy(np.abs(a)).cuda() @ torch.from_numpy(np.abs(b)).cuda().T
    held = torch.randn(m, n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(getattr(torch, dtype))
    for ldc, shift, add in (((n + 7) // 8 * 8, 0, False), ((n + 7) // 8 * 8 + 8, 8, True), (n + 3, 1, False), (n + 3, 0, True)):
        store = torch.full((m * ldc + shift + 8,), float("nan"), dtype=held.dtype, device="cuda")
        view = store[shift:shift + m * ldc].view(m, ldc)
        view[:, :n] = held
        B.sidco_mx4_matmul(ac, as_, bc, bs, m, n, k, store[shift:], ldc, add)
        assert torch.isnan(view[:, n:]).all() and torch.isnan(store[shift + m * ldc:]).all(), "wrote outside C"
        want, big = (exact + held.double(), size + held.double().abs()) if add else (exact, size)
        tol = (k + 2) * 2.0 ** -23 * big + ulp_half(dtype) * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -25
        assert ((view[:, :n].double() - want).abs() <= tol).all()
    assert B.sidco_wait_timeouts() == 0


@pytest.mark.parametrize("m,n,k", [(1, 200, 320), (20, 300, 700), (200, 300, 700), (5000, 1100, 700)])
def test_product_nan_block_stays_in_its_row_and_column(m, n, k):
    torch, B = torch_(), B_()
    r = rng(8)
    x, w = r.standard_normal((m, k)), r.standard_normal((n, k))
    x[m // 2, 40] = np.nan
    w[7, k - 1] = np.inf
    (ac, as_, a), (bc, bs, b) = Q.quantize(x), Q.quantize(w)
    t = [torch.from_numpy(v).cuda() for v in (ac, as_, bc, bs)]
    c = torch.zeros(m, n, device="cuda")
    B.sidco_mx4_matmul(*t, m, n, k, c, n)
    got = c.double().cpu().numpy()
    bad = np.zeros((m, n), bool)
    bad[m // 2], bad[:, 7] = True, True
    assert np.array_equal(np.isnan(got), bad)
    rows, cols = np.arange(m) != m // 2, np.arange(n) != 7
    check_product(got[rows][:, cols], a[rows], b[cols], None, "float32")


def test_product_of_nothing():
    torch, B = torch_(), B_()
    c = torch.full((4, 6), 3.0, device="cuda")
    B.sidco_mx4_matmul(None, None, None, None, 4, 5, 0, c, 6, True)
    assert (c == 3).all()
    B.sidco_mx4_matmul(None, None, None, None, 4, 5, 0, c, 6)
    assert (c[:, :5] == 0).all() and (c[:, 5] == 3).all()
    B.sidco_mx4_matmul(None, None, None, None, 0, 5, 32, None, 6, c_type=B.T_F32)


def test_product_repeats_bit_for_bit_and_on_another_stream():
    torch, B = torch_(), B_()
    for m, n, k in ((3, 1000, 2000), (300, 500, 1000)):
        ac, as_, _ = operands(1, m, k)
        bc, bs, _ = operands(2, n, k)
        outs = [torch.empty(m, n, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        for i, c in enumerate(outs):
            B.sidco_mx4_matmul(ac, as_, bc, bs, m, n, k, c, n, stream=side if i % 2 else None)
        torch.cuda.synchronize()
        assert all(torch.equal(outs[0], c) for c in outs)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,shift", [(1, 0), (31, 0), (32, 1), (33, 0), (1000, 3), (4096, 0), (269722, 0), (100001, 1)])
def test_compress_carries_the_residual_exactly(d, shift, dtype):
    torch, B = torch_(), B_()
    nb = -(-d // 32)
    res_store = torch.full((d + 16,), 5.0, device="cuda")
    res = res_store[shift:shift + d]
    res.zero_()
    want_res = np.zeros(d, np.float32)
    for call in range(3):
        g = torch.from_numpy(rng(d + call).laplace(0, 1e-3, d).astype(np.float32)).to(getattr(torch, dtype))
        grad = torch.zeros(d + 16, dtype=g.dtype, device="cuda")[shift:shift + d]
        grad.copy_(g)
        codes, scales = guarded(16 * nb), guarded(nb)
        B.sidco_mx4_compress(grad, res, d, codes[1], scales[1])
        torch.cuda.synchronize()
        want_c, want_s, _, want_res = Q.compress(g.float().numpy(), want_res)
        assert np.array_equal(codes[1].cpu().numpy(), want_c) and np.array_equal(scales[1].cpu().numpy(), want_s)
        assert np.array_equal(res.cpu().numpy(), want_res)
        assert untouched(*codes) and untouched(*scales)
        assert float(res_store[shift + d]) == 5.0


def test_compress_non_finite_blocks():
    torch, B = torch_(), B_()
    g = rng(9).standard_normal(200).astype(np.float32)
    g[40], g[100] = np.nan, -np.inf
    grad, res = torch.from_numpy(g).cuda(), torch.zeros(200, device="cuda")
    codes, scales = torch.empty(16 * 7, dtype=torch.uint8, device="cuda"), torch.empty(7, dtype=torch.uint8, device="cuda")
    B.sidco_mx4_compress(grad, res, 200, codes, scales)
    want_c, want_s, _, _ = Q.compress(g, np.zeros(200))
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    bad = np.zeros(200, bool)
    bad[32:64], bad[96:128] = True, True
    assert np.array_equal(np.isnan(res.cpu().numpy()), bad)


@pytest.mark.parametrize("d,workers,shift", [(1, 1, 0), (33, 2, 1), (1001, 3, 0), (4096, 8, 0), (5000, 9, 2), (12345, 64, 0)])
def test_mean_of_workers(d, workers, shift):
    """fp32 sums in worker order and one product by 1/N: N + 1 roundings of 2^-24 of the sum of magnitudes."""
    torch, B = torch_(), B_()
    parts = [Q.compress(rng(w).laplace(0, np.exp(w % 5), d), np.zeros(d)) for w in range(workers)]
    codes, scales = np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])
    store = torch.full((d + 16,), 5.0, device="cuda")
    out = store[shift:shift + d]
    B.sidco_mx4_mean(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), workers, d, out)
    exact = Q.mean(codes, scales, workers, d)
    size = np.mean([np.abs(p[2]) for p in parts], 0)
    assert (np.abs(out.double().cpu().numpy() - exact) <= (workers + 1) * 2.0 ** -24 * size).all()
    assert float(store[shift + d]) == 5.0 and (shift == 0 or float(store[shift - 1]) == 5.0)
    if workers == 1:
        assert np.array_equal(out.double().cpu().numpy(), exact)


def test_mean_of_a_nan_block():
    torch, B = torch_(), B_()
    g = np.ones(64, np.float32)
    g[3] = np.nan
    parts = [Q.compress(g, np.zeros(64)), Q.compress(np.ones(64), np.zeros(64))]
    out = torch.empty(64, device="cuda")
    B.sidco_mx4_mean(torch.from_numpy(np.concatenate([p[0] for p in parts])).cuda(),
                     torch.from_numpy(np.concatenate([p[1] for p in parts])).cuda(), 2, 64, out)
    assert torch.isnan(out[:32]).all() and (out[32:] == 1).all()


def test_calls_replay_in_a_graph():
    torch, B = torch_(), B_()
    m, n, k = 40, 200, 333
    x, w = torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda")
    bufs = [[torch.empty(f(r, k), dtype=torch.uint8, device="cuda") for f in (B.sidco_mx4_code_bytes, B.sidco_mx4_scale_bytes)]
            for r in (m, n)]
    c = torch.empty(m, n, device="cuda")

    def step():
        B.sidco_mx4_quantize(x, m, k, k, *bufs[0])
        B.sidco_mx4_quantize(w, n, k, k, *bufs[1])
        B.sidco_mx4_matmul(*bufs[0], *bufs[1], m, n, k, c, n)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in (1, 2):
        torch.manual_seed(seed)
        x.normal_()
        w.normal_()
        g.replay()
        torch.cuda.synchronize()
        again = c.clone()
        step()
        assert torch.equal(c, again)


def test_linear_layer_gradients_are_the_formulas():
    """Y, dX, dW of the layer against the products of the quantised operands in 64 bits, and against differences of the
    loss in the decoded operands (the product is linear in each, so differences are exact up to the products' sums)."""
    torch = torch_()
    from paper_2101_10761_b200.training import mx4_linear
    m, n, k = 70, 90, 150
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(m, k, generator=g, device="cuda").requires_grad_()
    w = (torch.randn(n, k, generator=g, device="cuda") / k ** 0.5).requires_grad_()
    dy = torch.randn(m, n, generator=g, device="cuda")
    y = mx4_linear(x.view(7, 10, k), w).view(m, n)
    y.backward(dy)
    X, W, D = (t.detach().double().cpu().numpy() for t in (x, w, dy))

    def rows(v):
        return Q.quantize(v)[2]

    def cols(v):
        return Q.quantize(v.T)[2]                              # the transpose, blocks along its rows
    check_product(y.detach().double().cpu().numpy(), rows(X), rows(W), None, "float32")
    check_product(x.grad.double().cpu().numpy(), rows(D), cols(W), None, "float32")
    check_product(w.grad.double().cpu().numpy(), cols(D), cols(X), None, "float32")
    # d/dw of sum(D_q * (X_q W^T)) by a difference of one entry
    dq, xq = cols(D).T, cols(X).T                              # [m, n], [m, k]
    for i, j in ((0, 0), (17, 149), (89, 75)):
        step = np.zeros((n, k))
        step[i, j] = 1.0
        diff = (dq * (xq @ (W + step).T)).sum() - (dq * (xq @ (W - step).T)).sum()
        assert abs(diff / 2 - float(w.grad[i, j])) <= 1e-4 * np.abs(dq).max() * np.abs(xq).max() * m


def test_linear_layer_of_no_rows_and_one_sided_gradients():
    torch = torch_()
    from paper_2101_10761_b200.training import mx4_linear
    w = torch.randn(20, 33, device="cuda").requires_grad_()
    y = mx4_linear(torch.zeros(0, 33, device="cuda"), w)
    y.sum().backward()
    assert y.shape == (0, 20) and w.grad.shape == w.shape and not w.grad.any()
    x = torch.randn(5, 33, device="cuda", dtype=torch.bfloat16).requires_grad_()
    y = mx4_linear(x, w.detach())
    assert y.dtype == torch.bfloat16
    y.sum().backward()                                         # (an expanded gradient: its rows are one value)
    assert x.grad.shape == x.shape and torch.isfinite(x.grad).all()


@pytest.mark.parametrize("exchange", ["mx4", "sparse"])
def test_example_learns(exchange):
    import importlib.util
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("four_bit_training", os.path.join(root, "examples", "four_bit_training.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses = ex.train(steps=60, exchange=exchange)
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0]
