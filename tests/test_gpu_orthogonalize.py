"""sidco_orthogonalize against the oracle in 64 bits, through the C ABI.

Tolerance: the result is rounded to bf16 (1.7e-3 of its norm) and comes from products of fp16 operands: about a dozen
roundings of 2^-12 (1.4e-4 in the mean), each scaled by at most the largest coefficient 3.45 before the next
normalisation, 1.7e-3 together; twice their sum is allowed, 7e-3 of the norm.  Momentum is one fp32 operation."""
import numpy as np
import pytest

from oracle import orthogonalize_oracle as N

pytestmark = pytest.mark.gpu

TOL = 7e-3


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def run(shapes, offsets, d, grads, moms, mu, nesterov, steps, dtype="float32", eps=1e-7, stream=None):
    import torch
    from paper_2101_10761_b200 import binding as B
    grad = torch.full((d,), float("nan")).to(getattr(torch, dtype))
    mom = torch.full((d,), float("nan"))
    for (r, c), o, g, m in zip(shapes, offsets, grads, moms):
        grad[o:o + r * c] = torch.from_numpy(g.reshape(-1)).to(grad.dtype)
        mom[o:o + r * c] = torch.from_numpy(m.reshape(-1)).float()
    grad, mom = grad.cuda(), mom.cuda() if mu is not None else None
    out = torch.full((d,), 7.0, dtype=torch.bfloat16, device="cuda")
    rows, cols = [r for r, _ in shapes], [c for _, c in shapes]
    need = B.sidco_orthogonalize_workspace_bytes(rows, cols)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")     # stale contents: NaN in every format
    torch.cuda.synchronize()
    B.sidco_orthogonalize(grad, mom, mu or 0.0, nesterov, offsets, rows, cols, steps, out, ws, need, eps, stream=stream)
    torch.cuda.synchronize()
    assert B.sidco_wait_timeouts() == 0
    assert bool((ws[need:] == 255).all()), "wrote behind the workspace"
    held = grad.double().cpu().numpy()
    return out.double().cpu().numpy(), None if mom is None else mom.double().cpu().numpy(), held


def check(shapes, mu=0.95, nesterov=True, steps=5, dtype="float32", gap=3, scale=1e-3, tol=TOL, kind="laplace"):
    offsets, at = [], 1
    for r, c in shapes:
        offsets.append(at)
        at += r * c + gap
    r_ = rng(sum(r * 31 + c for r, c in shapes) + steps)

    def draw(r, c):
        g = r_.laplace(0, 1.0, (r, c))
        if kind == "decaying":                                # singular values over two decades
            u, _, v = np.linalg.svd(g, full_matrices=False)
            g = u @ np.diag(np.logspace(0, -2, min(r, c))) @ v
        return g * scale
    grads = [draw(*s) for s in shapes]
    moms = [draw(*s).astype(np.float32) for s in shapes]
    out, mom, held = run(shapes, offsets, at, grads, moms, mu, nesterov, steps, dtype)
    seen = np.zeros(at, bool)
    for (r, c), o, m in zip(shapes, offsets, moms):
        if r * c == 0:
            continue
        g = held[o:o + r * c].reshape(r, c)
        want, want_m = N.orthogonalize(g, None if mu is None else m, float(np.float32(mu or 0)), nesterov, steps)
        err = np.linalg.norm(out[o:o + r * c].reshape(r, c) - want) / np.linalg.norm(want)
        assert err <= tol, ((r, c), err)
        if mu is not None:
            assert np.abs(mom[o:o + r * c].reshape(r, c) - want_m).max() <= 2.0 ** -23 * np.abs(want_m).max()
        seen[o:o + r * c] = True
    assert (out[~seen] == 7.0).all(), "wrote outside the matrices"
    if mu is not None:
        assert np.isnan(mom[~seen]).all()


@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (7, 1), (2, 2), (16, 27), (10, 64), (64, 10), (33, 65), (64, 64), (64, 576),
                                   (65, 64), (127, 130), (128, 128), (129, 128), (10, 512), (100, 1000), (1000, 100),
                                   (200, 200), (257, 300), (300, 257), (64, 3000), (512, 520), (640, 385), (128, 2048), (2048, 128), (100, 2049), (17, 1030)])
def test_single_matrices(shape):
    check([shape])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("nesterov", [False, True])
def test_types_and_momentum(dtype, nesterov):
    check([(60, 100), (150, 40), (200, 330)], nesterov=nesterov, dtype=dtype)


def test_without_momentum():
    check([(60, 100), (150, 140)], mu=None)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6, 7, 8])
def test_step_counts(steps):
    check([(40, 70), (150, 200), (260, 130)], steps=steps)


def test_a_model_of_many_shapes_in_one_call():
    check([(16, 27)] + [(16, 144)] * 6 + [(32, 144)] + [(32, 288)] * 5 + [(64, 288)] + [(64, 576)] * 5 + [(10, 64)]
          + [(300, 700), (2000, 150), (128, 1152), (1000, 513)])


def test_more_matrices_than_one_chain_takes():
    check([(3 + i % 20, 4 + i % 33) for i in range(300)])
    check([(129 + i % 3, 130 + i % 5) for i in range(131)])


def test_scales_far_from_one():
    for scale in (1e-18, 1e15):
        check([(50, 90), (200, 150)], scale=scale if scale > 1 else 1e-5)
    # below eps the update shrinks with the gradient, as the formula says
    out, _, held = run([(8, 9)], [0], 72, [rng(1).standard_normal((8, 9)) * 1e-9], [np.zeros((8, 9))], None, False, 5)
    want = N.iterate(held.reshape(8, 9), 5)
    assert np.linalg.norm(out.reshape(8, 9) - want) <= TOL * np.linalg.norm(want)


def test_decaying_spectra():
    check([(64, 200), (300, 300), (257, 1000)], kind="decaying", tol=TOL)


def test_zero_and_non_finite_matrices_leave_the_others_alone():
    shapes = [(20, 30), (150, 200), (20, 30), (64, 64)]
    r = rng(2)
    grads = [r.standard_normal(s) for s in shapes]
    grads[0][:] = 0.0
    grads[2][3, 4] = np.nan
    grads[3][0, 63] = np.inf
    offsets = [0, 600, 30600, 31200]
    out, _, held = run(shapes, offsets, 31200 + 4096, grads, [np.zeros(s) for s in shapes], None, False, 5)
    assert not out[:600].any()
    want = N.iterate(held[600:30600].reshape(150, 200), 5)
    assert np.linalg.norm(out[600:30600].reshape(150, 200) - want) <= TOL * np.linalg.norm(want)
    assert np.isnan(out[30600:31200]).all() and np.isnan(out[31200:]).all()


def test_no_matrices_and_empty_ones():
    import torch
    from paper_2101_10761_b200 import binding as B
    B.sidco_orthogonalize(None, None, 0.9, True, [], [], [], 5, None, None, 0, grad_type=B.T_F32)
    check([(0, 5), (30, 40), (7, 0)])
    torch.cuda.synchronize()


def test_repeats_bit_for_bit_on_streams_and_in_a_graph():
    import torch
    from paper_2101_10761_b200 import binding as B
    rows, cols, offsets = [64, 300, 130], [576, 200, 1000], [0, 36864, 96864]
    d = 96864 + 130000
    grad = torch.randn(d, generator=torch.Generator().manual_seed(1)).cuda()
    need = B.sidco_orthogonalize_workspace_bytes(rows, cols)
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.zeros(d, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for i in (0, 1):                                           # two workspaces, two streams at once
        B.sidco_orthogonalize(grad, None, 0, False, offsets, rows, cols, 5, outs[i], spaces[i], need,
                              stream=side if i else None)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sidco_orthogonalize(grad, None, 0, False, offsets, rows, cols, 5, outs[2], spaces[0], need)
    for _ in range(3):
        g.replay()
    B.sidco_orthogonalize(grad, None, 0, False, offsets, rows, cols, 5, outs[3], spaces[0], need)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0], o) for o in outs[1:])


def test_optimizer_object_takes_the_flat_gradient():
    import torch
    from paper_2101_10761_b200.training import OrthogonalizedUpdate
    shapes = [(40, 60), (100, 30)]
    opt = OrthogonalizedUpdate(shapes, mu=0.9, nesterov=True)
    grads = [rng(s).standard_normal(40 * 60 + 100 * 30).astype(np.float32) for s in (1, 2)]
    moms = [np.zeros((40, 60)), np.zeros((100, 30))]
    for g in grads:
        up = opt.step(torch.from_numpy(g).cuda()).double().cpu().numpy()
        for i, ((r, c), o) in enumerate(zip(shapes, opt.offsets)):
            want, moms[i] = N.orthogonalize(g[o:o + r * c].reshape(r, c), moms[i], float(np.float32(0.9)), True, 5)
            assert np.linalg.norm(up[o:o + r * c].reshape(r, c) - want) <= TOL * np.linalg.norm(want)
    with pytest.raises(ValueError):
        opt.step(torch.zeros(10, device="cuda"))


def test_both_kinds_follow_and_precede_the_stream():
    """Small matrices run beside the others on another stream; the call still starts after what the caller's stream holds
    and its results are there for what comes next."""
    import torch
    from paper_2101_10761_b200 import binding as B
    rows, cols, offsets = [64, 300, 16], [576, 200, 27], [0, 36864, 96864]
    d = 96864 + 432
    need = B.sidco_orthogonalize_workspace_bytes(rows, cols)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    source = torch.randn(d, device="cuda")
    want = torch.empty(d, dtype=torch.bfloat16, device="cuda")
    B.sidco_orthogonalize(source, None, 0, False, offsets, rows, cols, 5, want, ws, need)
    torch.cuda.synchronize()
    big = torch.randn(4096, 4096, device="cuda")
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(s):
            grad = torch.full((d,), float("nan"), device="cuda")
            out = torch.full((d,), 7.0, dtype=torch.bfloat16, device="cuda")
            for _ in range(8):
                big = big @ big * 1e-4                        # keeps the stream busy for a while
            grad.copy_(source)
            B.sidco_orthogonalize(grad, None, 0, False, offsets, rows, cols, 5, out, ws, need)
            got = out.clone()
            grad.fill_(float("nan"))
        s.synchronize()
        assert torch.equal(got, want)


def test_a_wait_that_runs_out_ends_the_kernel_and_is_counted():
    """One phase is withheld (its results are stored but not counted): the kernel gives up after the shortened limit, says
    so, and the next call is right again."""
    import torch
    from paper_2101_10761_b200 import binding as B
    rows, cols = [300], [200]
    need = B.sidco_orthogonalize_workspace_bytes(rows, cols)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    grad = torch.randn(60000, device="cuda")
    outs = [torch.zeros(60000, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.sidco_orthogonalize(grad, None, 0, False, [0], rows, cols, 5, outs[0], ws, need)
    assert B.sidco_wait_timeouts() == 0
    try:
        for drop in (0, 1, 5, 6):                             # a Gram product, a polynomial, a product, an application
            B.sidco_set_product_test_hooks(5000, drop)
            B.sidco_orthogonalize(grad, None, 0, False, [0], rows, cols, 5, outs[1], ws, need)
            torch.cuda.synchronize()
            assert B.sidco_wait_timeouts() > 0
    finally:
        B.sidco_set_product_test_hooks()
    B.sidco_orthogonalize(grad, None, 0, False, [0], rows, cols, 5, outs[1], ws, need)
    torch.cuda.synchronize()
    assert B.sidco_wait_timeouts() == 0 and torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("shape", [(16, 139), (16, 27), (139, 16), (33, 65), (64, 64), (64, 576), (10, 512), (5, 2048)])
def test_few_rows_keep_two_parts_of_their_products(shape):
    """With up to 64 rows (or columns) the squares are sums of two fp16 parts, 2^-22 each, so only X is rounded to fp16, once
    as it comes in and after each of three groups but the last: relative 2^-12 in the mean, each times at most 3.45, together
    1.5e-3 at worst.  Next to bf16's 1.7e-3 that makes sqrt(1.7^2 + 1.5^2) e-3 = 2.3e-3 of the norm."""
    check([shape, shape], tol=2.3e-3)
    check([shape, shape], tol=2.3e-3, dtype="bfloat16", nesterov=False)


@pytest.mark.parametrize("shape", [(150, 700), (700, 150), (300, 301), (130, 129)])
@pytest.mark.parametrize("low, high", [(0.0, 1e-3), (0.0, 1e7), (1e-6, 1e6), (0.0, 3e-30), (1e6, 1e6)])
@pytest.mark.parametrize("with_momentum", [False, True])
def test_norms_that_hide_in_one_entry(shape, low, high, with_momentum):
    """A matrix whose norm no sample of its entries tells: one entry holds it.  Beside it in the call a matrix like any."""
    r, c = shape
    r_ = rng(r + c)
    other = (140, 200)
    grads = [r_.laplace(0, 1, shape) * low, r_.laplace(0, 1, other)]
    grads[0][r // 3, c // 2 + 1] = high
    moms = [np.zeros(shape), r_.laplace(0, 1, other).astype(np.float32)]
    mu = 0.9 if with_momentum else None
    out, mom, held = run([shape, other], [0, r * c + 3], r * c + 3 + 28000, grads, moms, mu, with_momentum, 5, eps=0.0)
    for (rows, cols), o, m in zip([shape, other], [0, r * c + 3], moms):
        g = held[o:o + rows * cols].reshape(rows, cols)
        want, _ = N.orthogonalize(g, m if with_momentum else None, float(np.float32(mu or 0)), with_momentum, 5, eps=0.0)
        err = np.linalg.norm(out[o:o + rows * cols].reshape(rows, cols) - want) / np.linalg.norm(want)
        assert err <= TOL, ((rows, cols), err)
