"""Pins of the 4-bit and orthogonalisation oracles: brute force, hand-worked values and the singular-value form (CPU)."""
import numpy as np
import pytest

from oracle import mx4_oracle as Q
from oracle import orthogonalize_oracle as N


def test_grid_ties_and_saturation_by_hand():
    x = np.zeros(32)
    x[:16] = [4, 7.9, 5, 3.5, 2.5, 1.75, 1.25, .75, .25, .26, -.25, -.3, -6, -7, 4.99, 5.01]       # scale 1 (4 <= max < 8)
    code, byte = Q.encode_blocks(x[None])
    assert byte[0] == 127
    v = Q.decode_blocks(code, byte)[0]
    assert v[:16].tolist() == [4, 6, 4, 4, 2, 2, 1, 1, 0, .5, 0, -.5, -6, -6, 4, 6]
    assert np.signbit(v[10]) and code[0, 10] == 8


def test_codes_are_the_nearest_by_brute_force():
    r = np.random.Generator(np.random.PCG64(3))
    x = r.standard_normal((200, 32)) * np.exp(r.uniform(-60, 60, (200, 1)))
    code, byte = Q.encode_blocks(x)
    e = byte.astype(int) - 127
    top = np.abs(x).max(1)
    assert (top >= 4 * 2.0 ** e).all() and (top < 8 * 2.0 ** e).all()
    values = np.concatenate([Q.GRID, -Q.GRID])[:, None, None] * (2.0 ** e)[None, :, None]
    best = np.abs(values - x[None]).min(0)
    assert np.allclose(np.abs(Q.decode_blocks(code, byte) - x), best, rtol=1e-12, atol=0)


@pytest.mark.parametrize("top,byte", [(0.0, 0), (1.0, 125), (2.0 ** -126, 0), (2.0 ** -149, 0), (2.0 ** -124, 1),
                                      (np.float64(np.finfo(np.float32).max), 252), (np.inf, 255), (np.nan, 255)])
def test_scale_bytes_at_the_ends_of_the_range(top, byte):
    x = np.zeros((1, 32))
    x[0, 5] = top
    code, got = Q.encode_blocks(x)
    assert got[0] == byte
    if byte == 255:
        assert not code.any() and np.isnan(Q.decode_blocks(code, got)).all()


def test_tiled_scales_cover_every_byte_once():
    byte = (np.arange(300 * 9).reshape(300, 9) % 251 + 1).astype(np.uint8)
    t = Q.tile_scales(byte)
    assert t.size == 3 * 3 * 512 and np.count_nonzero(t) == byte.size and sorted(t[t > 0]) == sorted(byte.reshape(-1))
    assert t[0] == byte[0, 0] and t[16] == byte[1, 0] and t[4] == byte[32, 0] and t[1] == byte[0, 1]
    assert t[512] == byte[0, 4] and t[3 * 512] == byte[128, 0]


def test_compress_keeps_what_it_did_not_send():
    r = np.random.Generator(np.random.PCG64(4))
    g, res = r.laplace(0, 1e-3, 1001).astype(np.float32), r.laplace(0, 1e-4, 1001).astype(np.float32)
    codes, scales, value, after = Q.compress(g, res)
    assert codes.size == 16 * 32 and scales.size == 32
    assert np.abs(value + after.astype(np.float64) - (g + res)).max() <= 2.0 ** -24 * np.abs(g + res).max()
    assert np.array_equal(Q.mean(codes, scales, 1, 1001), value)


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (7, 7), (1, 4)])
def test_iteration_acts_on_the_singular_values(shape):
    r = np.random.Generator(np.random.PCG64(5))
    u = r.standard_normal(shape)
    left, s, right = np.linalg.svd(u, full_matrices=False)
    s = s / (np.sqrt((s * s).sum()) + 1e-7)
    for _ in range(5):
        s = N.A * s + N.B * s ** 3 + N.C * s ** 5
    assert np.allclose(N.iterate(u, 5), left @ np.diag(s) @ right, atol=1e-12)
    assert (np.abs(s - 1) < 0.35).all()


def test_one_step_of_a_scalar_and_momentum_by_hand():
    x = 3.0 / (3.0 + 1e-7)
    assert abs(N.iterate([[3.0]], 1)[0, 0] - (N.A * x + N.B * x ** 3 + N.C * x ** 5)) < 1e-15
    up, m = N.orthogonalize([[1.0]], [[2.0]], 0.5, True, 1)
    assert m[0, 0] == 2.0                                     # 0.5 * 2 + 1; the update is of 1 + 0.5 * 2
    assert np.allclose(up, N.iterate([[2.0]], 1))
    assert not N.iterate(np.zeros((3, 4)), 5).any()
