"""sidco_mx4_matmul with `add` at the lower end of fp32."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


# few rows, 128 x 128 tiles, pairs of CTAs with whole boxes and with odd rows
SIZES = [(20, 300, 64, 300), (300, 200, 64, 200), (5000, 1100, 64, 1104), (5000, 1100, 64, 1101)]


@pytest.mark.parametrize("m,n,k,ldc", SIZES)
def test_adding_nothing_leaves_c_as_it_is(m, n, k, ldc):
    """C + 0 is C, subnormal numbers included."""
    import torch
    from paper_2101_10761_b200 import binding as B
    r = np.random.Generator(np.random.PCG64(1))
    c0 = (r.integers(-(1 << 23), 1 << 23, (m, ldc)).astype(np.float64) * 2.0 ** -149).astype(np.float32)
    c0[::3] = r.standard_normal(c0[::3].shape)
    c = torch.from_numpy(c0).cuda()
    codes = [torch.zeros(B.sidco_mx4_code_bytes(rows, k), dtype=torch.uint8, device="cuda") for rows in (m, n)]
    scales = [torch.zeros(B.sidco_mx4_scale_bytes(rows, k), dtype=torch.uint8, device="cuda") for rows in (m, n)]
    B.sidco_mx4_matmul(codes[0], scales[0], codes[1], scales[1], m, n, k, c, ldc, True)
    assert np.array_equal(c.cpu().numpy(), c0)


@pytest.mark.parametrize("m,n,k,ldc", SIZES)
def test_subnormal_products_and_sums_are_kept(m, n, k, ldc):
    """C - 2^-126 of C between 2^-126 and 2^-125 is a subnormal number that fp32 holds exactly."""
    import torch
    from oracle import mx4_oracle as Q
    from paper_2101_10761_b200 import binding as B
    x, w = np.zeros((m, k)), np.zeros((n, k))
    w[:, 0] = 2.0 ** -63
    for exponent, add in ((-63, True), (-65, False)):
        x[:, 0] = -2.0 ** exponent
        operands = [torch.from_numpy(v).cuda() for q in (x, w) for v in Q.quantize(q)[:2]]
        c0 = ((1 + np.random.Generator(np.random.PCG64(2)).random((m, ldc))) * 2.0 ** -126).astype(np.float32)
        c = torch.from_numpy(c0).cuda()
        B.sidco_mx4_matmul(*operands, m, n, k, c, ldc, add)
        want = c0.astype(np.float64)
        want[:, :n] = want[:, :n] * add - 2.0 ** (exponent - 63)
        assert np.array_equal(c.cpu().numpy().astype(np.float64), want)


@pytest.mark.parametrize("shape", [(3, 0), (2, 3, 0), (0,), (0, 5), (5,)])
def test_linear_layer_of_empty_sums_and_of_a_single_row(shape):
    import torch
    from paper_2101_10761_b200.training import mx4_linear
    x = torch.ones(shape, device="cuda").requires_grad_()
    w = torch.ones(4, shape[-1], device="cuda").requires_grad_()
    y = mx4_linear(x, w)
    assert y.shape == shape[:-1] + (4,) and (y == shape[-1]).all()
    y.sum().backward()
    assert x.grad.shape == x.shape and (x.grad == 4).all()
    assert w.grad.shape == w.shape and (w.grad == x[..., :1].numel()).all()
