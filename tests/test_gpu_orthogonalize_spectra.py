"""sidco_orthogonalize on matrices whose rank is below their shorter side, as gradients of few rows are.

The formula keeps what is zero zero, but multiplies whatever the rounding of X adds there by up to a^steps (485 for five).
Tolerances: X enters every application as two fp16 parts (2^-22 of an entry at most, 2^-24 in the mean, times 485: 3e-5 of |X|),
in larger matrices as one part in the last two steps (2^-12, 1.4e-4 in the mean, times a^2 = 12: 1.7e-3); the products
of rounded s x s matrices add up to 1.7e-3 and bf16 1.7e-3 as for any spectrum.  Twice the sum of what applies, 7e-3 of
the norm, is allowed as for full rank; matrices with up to 64 rows or columns, whose s x s matrices have two parts
as well, keep 2.3e-3."""
import numpy as np
import pytest

from oracle import orthogonalize_oracle as N
from test_gpu_orthogonalize import TOL, rng, run

pytestmark = pytest.mark.gpu


def of_rank(shape, rank, seed, noise=0.0):
    r = rng(seed)
    u = r.standard_normal((shape[0], rank)) @ r.standard_normal((rank, shape[1]))
    if noise:
        e = r.standard_normal(shape)
        u += noise * np.linalg.norm(u) / np.linalg.norm(e) * e
    return u * 1e-3


def check(shapes, grads, moms=None, mu=None, nesterov=True, steps=5, dtype="float32", tol=TOL, eps=1e-7):
    offsets, at = [], 1
    for r, c in shapes:
        offsets.append(at)
        at += r * c + 3
    held_moms = moms or [np.zeros(s) for s in shapes]
    out, _, held = run(shapes, offsets, at, grads, held_moms, mu, nesterov, steps, dtype, eps=eps)
    for (r, c), o, m in zip(shapes, offsets, held_moms):
        g = held[o:o + r * c].reshape(r, c)
        want, _ = N.orthogonalize(g, None if mu is None else m.astype(np.float32), float(np.float32(mu or 0)), nesterov, steps,
                                  eps)
        err = np.linalg.norm(out[o:o + r * c].reshape(r, c) - want) / np.linalg.norm(want)
        assert err <= tol, ((r, c), err)


@pytest.mark.parametrize("rank", [1, 2, 8, 64])
@pytest.mark.parametrize("shape", [(100, 333), (1152, 128), (128, 2048), (130, 140), (257, 300), (300, 1000), (1000, 300),
                                   (512, 2304)])
def test_low_rank(shape, rank):
    check([shape], [of_rank(shape, rank, rank + sum(shape))])


@pytest.mark.parametrize("rank", [1, 2, 8, 32])
@pytest.mark.parametrize("shape", [(40, 70), (64, 576), (576, 64), (64, 64), (33, 2048)])
def test_low_rank_of_few_rows(shape, rank):
    check([shape], [of_rank(shape, rank, rank + sum(shape))], tol=2.3e-3)


@pytest.mark.parametrize("shape", [(64, 576), (128, 1152), (300, 1000)])
def test_low_rank_beside_a_little_noise(shape):
    check([shape], [of_rank(shape, 8, 5, noise=0.01)])


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("shape", [(40, 70), (150, 200), (700, 300)])
def test_low_rank_for_every_number_of_steps(shape, steps):
    check([shape], [of_rank(shape, 4, steps)], steps=steps)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("nesterov", [False, True])
def test_low_rank_with_momentum_beside_other_matrices(dtype, nesterov):
    shapes = [(60, 100), (300, 200), (150, 700), (200, 200)]
    r = rng(3)
    grads = [of_rank(s, 3, i) for i, s in enumerate(shapes[:3])] + [r.laplace(0, 1e-3, shapes[3])]
    moms = [of_rank(s, 5, 10 + i) for i, s in enumerate(shapes[:3])] + [r.laplace(0, 1e-3, shapes[3])]
    check(shapes, grads, moms, 0.95, nesterov, dtype=dtype)


def test_first_step_of_a_layer_with_a_batch_of_eight_rows():
    """dW = dY^T X of eight rows, momentum still zero."""
    for shape in ((300, 1000), (64, 576)):
        check([shape], [of_rank(shape, 8, 7)], mu=0.95)


def test_low_rank_that_the_samples_miss():
    """A block of 3 x 5 holds the norm, the rest is 1e-9 of it: the scale that 2048 of the entries suggest is far off, so X is
    written a second time."""
    for shape in ((300, 700), (700, 150)):
        g = of_rank(shape, 2, 1) * 1e-9
        g[np.ix_([3, 77, 140], [2, 30, 31, 90, 149])] = of_rank((3, 5), 1, 4)
        check([shape, shape], [g, of_rank(shape, 1, 2)], eps=0.0)
