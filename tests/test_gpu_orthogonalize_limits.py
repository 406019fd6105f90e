"""sidco_orthogonalize at the ends of its range, on both of its paths: (50, 90) and its like are small matrices, the others go
through the chain of products.  Tolerance as in test_gpu_orthogonalize."""
import numpy as np
import pytest

from oracle import orthogonalize_oracle as N
from test_gpu_orthogonalize import TOL, rng, run

pytestmark = pytest.mark.gpu

SMALL, LARGE, TALL = (50, 90), (150, 200), (300, 150)


def call(grads, moms=None, mu=None, nesterov=True, eps=1e-7, steps=5):
    """[(result, wanted)] of matrices side by side."""
    shapes = [g.shape for g in grads]
    offsets, at = [], 0
    for r, c in shapes:
        offsets.append(at)
        at += r * c + 3
    moms = moms or [np.zeros(s) for s in shapes]
    out, mom, held = run(shapes, offsets, at, grads, moms, mu, nesterov, steps, eps=eps)
    pairs = []
    for (r, c), o, m in zip(shapes, offsets, moms):
        with np.errstate(invalid="ignore", divide="ignore"):
            want, want_m = N.orthogonalize(held[o:o + r * c].reshape(r, c), None if mu is None else m.astype(np.float32),
                                           float(np.float32(mu or 0)), nesterov, steps, eps)
        if mu is not None:
            got_m = mom[o:o + r * c].reshape(r, c)
            fine = np.isfinite(want_m)
            assert np.array_equal(np.isnan(got_m), np.isnan(want_m))
            # (one rounding: 2^-24 of a normal number, half of 2^-149 below)
            assert (np.abs(got_m - want_m)[fine] <= 2.0 ** -23 * np.abs(want_m)[fine] + 2.0 ** -149).all()
        pairs.append((out[o:o + r * c].reshape(r, c), want))
    return pairs


def near(got, want, tol=TOL):
    assert np.isfinite(got).all()
    assert np.linalg.norm(got - want) <= tol * np.linalg.norm(want), np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("eps", [1e-7, 1e-20, 1e-37])
@pytest.mark.parametrize("mu", [None, 0.9])
def test_a_zero_matrix_stays_zero(eps, mu):
    r = rng(1)
    grads = [np.zeros(SMALL), np.zeros(LARGE), r.standard_normal(LARGE), np.zeros(TALL), r.standard_normal(SMALL)]
    got = call(grads, mu=mu, eps=eps)
    for i in (0, 1, 3):
        assert not got[i][0].any()
    near(*got[2])
    near(*got[4])


def test_a_zero_matrix_without_eps_is_not_a_number_as_the_formula_says():
    r = rng(2)
    got = call([np.zeros(SMALL), np.zeros(LARGE), r.standard_normal(LARGE), r.standard_normal(SMALL)], eps=0.0)
    assert np.isnan(got[0][0]).all() and np.isnan(got[1][0]).all()
    near(*got[2])
    near(*got[3])


@pytest.mark.parametrize("shape", [SMALL, LARGE, TALL])
@pytest.mark.parametrize("scale", [1e-40, 1e-37, 1e-30, 1e-18, 1e15, 1e30, 3e36])
@pytest.mark.parametrize("mu", [None, 0.9])
def test_any_scale_without_eps(shape, scale, mu):
    r = rng(3)
    grads = [r.laplace(0, 1, shape) * scale, r.laplace(0, 1, shape)]
    moms = [r.laplace(0, 1, shape) * scale, r.laplace(0, 1, shape)]
    for got, want in call(grads, moms, mu, eps=0.0):
        near(got, want)


@pytest.mark.parametrize("shape", [(600, 700), (700, 300)])
@pytest.mark.parametrize("scale", [1e-43, 1e-36, 1e-30, 1e30, 1e38])
def test_any_scale_that_the_samples_miss(shape, scale):
    g = np.zeros(shape)
    g[np.ix_([3, 77, 140], [2, 30, 31, 90, 149])] = np.arange(1, 16).reshape(3, 5) % 7 / 7 * scale
    for got, want in call([g, rng(4).standard_normal(shape)], eps=0.0):
        near(got, want)


@pytest.mark.parametrize("shape", [SMALL, LARGE, TALL])
@pytest.mark.parametrize("scale", [1e-9, 1e-11, 1e-18])
def test_below_eps_the_update_shrinks_with_the_gradient(shape, scale):
    """|U| 1e-2 to 1e-9 of eps.  X is held to 2^-39 at worst (fp16's 2^-25, 2^14 times), twice, times a^5 at most."""
    for got, want in call([rng(5).standard_normal(shape) * scale / np.sqrt(shape[0] * shape[1])], eps=1e-7):
        assert np.linalg.norm(got - want) <= TOL * np.linalg.norm(want) + 2 * 485 * 2.0 ** -39 * np.sqrt(got.size)


@pytest.mark.parametrize("mu", [None, 0.9])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_non_finite_matrices_leave_the_others_alone(bad, mu):
    r = rng(6)
    shapes = [LARGE, LARGE, TALL, SMALL, TALL, SMALL, LARGE]
    grads, moms = ([r.standard_normal(s) for s in shapes] for _ in range(2))
    grads[1][149, 199] = bad
    grads[2][0, 0] = bad
    grads[3][7, 8] = bad
    if mu is not None:
        moms[6][5, 5] = bad
    got = call(grads, moms, mu)
    for i in (1, 2, 3) + ((6,) if mu is not None else ()):
        assert np.isnan(got[i][0]).all()
    for i in (0, 4, 5) + ((6,) if mu is None else ()):
        near(*got[i])


def test_callers_on_two_streams_do_not_wait_for_each_other():
    """A call with matrices of both kinds behind a stream that is held up must not hold up a call on another stream.  (Of four
    pairs of streams: one pair, or what the library forks from it, may share a queue of the hardware.)"""
    import torch
    from paper_2101_10761_b200 import binding as B
    rows, cols, offsets = [64, 300, 16], [576, 200, 27], [0, 36864, 96864]
    d = 96864 + 432
    need = B.sidco_orthogonalize_workspace_bytes(rows, cols)
    grad = torch.randn(d, device="cuda")
    apart = 0
    for _ in range(4):
        spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
        outs = [torch.zeros(d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()

        def step(i):
            B.sidco_orthogonalize(grad, None, 0, False, offsets, rows, cols, 5, outs[i], spaces[i], need, stream=streams[i])
        for i in (0, 1):                                       # (what the first call of a stream sets up)
            step(i)
        torch.cuda.synchronize()
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[0]):
            torch.cuda._sleep(1_000_000_000)                   # cycles: about half a second
        step(0)
        step(1)
        done = [torch.cuda.Event() for _ in range(2)]
        for e, s in zip(done, streams):
            e.record(s)
        done[1].synchronize()
        apart += not done[0].query()
        torch.cuda.synchronize()
        assert outs[1].any() and torch.equal(outs[0], outs[1])
    assert apart, "the second stream always waited for the first"


def test_many_streams_one_after_the_other():
    """More streams than the library keeps streams of its own for."""
    import torch
    from paper_2101_10761_b200 import binding as B
    rows, cols, offsets = [64, 300], [576, 200], [0, 36864]
    need = B.sidco_orthogonalize_workspace_bytes(rows, cols)
    grad = torch.randn(96864, device="cuda")
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    want = torch.zeros(96864, dtype=torch.bfloat16, device="cuda")
    B.sidco_orthogonalize(grad, None, 0, False, offsets, rows, cols, 5, want, ws, need)
    torch.cuda.synchronize()
    for _ in range(40):
        s = torch.cuda.Stream()
        out = torch.zeros_like(want)
        s.wait_stream(torch.cuda.current_stream())
        B.sidco_orthogonalize(grad, None, 0, False, offsets, rows, cols, 5, out, ws, need, stream=s)
        s.synchronize()
        assert torch.equal(out, want)


FIRST = r'''
import sys
sys.path.insert(0, %r)
import torch
from paper_2101_10761_b200 import binding as B
x = torch.randn(300, 200, device="cuda")
rows, cols, offsets = [64, 300], [576, 200], [0, 36864]
need = B.sidco_orthogonalize_workspace_bytes(rows, cols)
grad = torch.randn(96864, device="cuda")
ws = torch.empty(need, dtype=torch.uint8, device="cuda")
outs = [torch.zeros(96864, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
codes = torch.empty(B.sidco_mx4_code_bytes(300, 200), dtype=torch.uint8, device="cuda")
scales = torch.empty(B.sidco_mx4_scale_bytes(300, 200), dtype=torch.uint8, device="cuda")
prods = [torch.zeros(300, 300, device="cuda") for _ in range(2)]
def step(i):
    B.sidco_mx4_quantize(x, 300, 200, 200, codes, scales)
    B.sidco_mx4_matmul(codes, scales, codes, scales, 300, 300, 200, prods[i], 300)
    B.sidco_orthogonalize(grad, None, 0, False, offsets, rows, cols, 5, outs[i], ws, need)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step(0)
g.replay()
torch.cuda.synchronize()
step(1)
torch.cuda.synchronize()
assert outs[0].any() and prods[0].any()
assert torch.equal(outs[0], outs[1]) and torch.equal(prods[0], prods[1])
print("same")
'''


def test_first_calls_of_a_process_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-c", FIRST % root], capture_output=True, text=True, timeout=300, cwd=root)
    assert p.returncode == 0 and p.stdout.strip().endswith("same"), p.stderr[-2000:]
