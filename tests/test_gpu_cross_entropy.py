"""Cross entropy of an output projection and its gradients through the C ABI against the oracle in 64 bits.

Tolerances.  u = half a step of the operands' type.  A logit is a sum of `hidden` exact products of 16-bit numbers, added 16
at a time to an fp32 accumulator that may cut instead of round: off by at most (hidden / 16 + 2) 2^-22 times the sum of the
products' magnitudes.  The loss is off by twice the largest of these, by the arguments of the exponentials (2^-22 of the
largest logit) and by sums and logarithm (2^-18 together).  The gradient of a logit is off by these and by two roundings,
so the gradients of the inputs by 2 u (+ u^2) of the sum of their terms' magnitudes, and by their own rounding.  As the
roundings are independent and each has at most u / sqrt(3) in the mean square, the whole gradient is within u (1 + 2^-3) of its norm."""
import numpy as np
import pytest

from oracle import language_oracle as L

pytestmark = pytest.mark.gpu

U = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}
TINY = {"bfloat16": 2.0 ** -134, "float16": 2.0 ** -25, "float32": 2.0 ** -150}


def torch_():
    import torch
    return torch


def B_():
    from paper_2101_10761_b200 import binding
    return binding


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def matrix(x, dtype, ld=None, shift=0, fill=float("nan")):
    """(flat buffer from the first element, whole buffer, values in 64 bits); NaN between the rows and around."""
    torch = torch_()
    rows, cols = x.shape
    ld = ld or cols
    t = torch.from_numpy(np.ascontiguousarray(x)).to(getattr(torch, dtype))
    store = torch.full((rows * ld + shift + 16,), fill, dtype=t.dtype, device="cuda")
    store[shift:shift + rows * ld].view(rows, ld)[:, :cols] = t.cuda()
    return store[shift:], store, t.double().numpy()


def inside(store, shift, rows, cols, ld):
    return store[shift:shift + rows * ld].view(rows, ld)[:, :cols]


def rest_is_nan(store, shift, rows, cols, ld):
    c = store.clone()
    inside(c, shift, rows, cols, ld).fill_(float("nan"))
    return bool(torch_().isnan(c).all())


def inputs(rows, vocab, hidden, seed, ignored=0.0, sharp=2.0):
    """Rows that know their label and rows that do not."""
    r = rng(seed)
    w = r.standard_normal((vocab, hidden)) * sharp / hidden ** 0.5
    labels = r.integers(0, vocab, rows)
    x = r.standard_normal((rows, hidden)) + r.random((rows, 1)) * 4 * w[labels]
    labels[r.random(rows) < ignored] = -100
    return x, w, labels


def call(x, w, labels, dtype, w_dtype=None, dw_dtype=None, weights=None, scale=1.0, grads=3, old=None, piece_rows=0,
         lds=(0, 0, 0, 0), shift=0, wide=True, status=None):
    """The call on fresh buffers; everything it wrote, and the values of its inputs in 64 bits."""
    torch, B = torch_(), B_()
    rows, hidden = x.shape
    vocab = w.shape[0]
    ldx, ldw, lddx, lddw = (hidden + a for a in lds)
    dw_dtype = dw_dtype or dtype
    gx, _, hx = matrix(x, dtype, ldx, shift)
    gw, _, hw = matrix(w, w_dtype or dtype, ldw, shift)
    if w_dtype == "float32":
        hw = torch.from_numpy(hw).to(getattr(torch, dtype)).double().numpy()
    y = torch.from_numpy(labels).to(torch.int64 if wide else torch.int32).cuda()
    c = None if weights is None else torch.from_numpy(weights).float().cuda()
    each, loss = torch.full((rows,), float("nan"), device="cuda"), torch.full((), float("nan"), device="cuda")
    dx, dx_store, _ = matrix(np.full((rows, hidden), np.nan), dtype, lddx, shift)
    dw, dw_store, held = matrix(np.full((vocab, hidden), np.nan) if old is None else old, dw_dtype, lddw, shift)
    need = B.sidco_linear_cross_entropy_workspace_bytes(gx, gw, ldw, rows, vocab, hidden, grads, piece_rows)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")       # NaN whatever is read unwritten
    B.sidco_linear_cross_entropy(gx, ldx, gw, ldw, y, rows, vocab, hidden, each, loss, dx if grads & 1 else None, lddx,
                                 dw if grads & 2 else None, lddw, ws, need, row_weights=c, scale=scale,
                                 add=old is not None, piece_rows=piece_rows, status=status)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 255).all()) and B.sidco_wait_timeouts() == 0
    assert rest_is_nan(dx_store, shift, rows, hidden, lddx) and rest_is_nan(dw_store, shift, vocab, hidden, lddw)
    return (each.double().cpu().numpy(), loss.double().item(), inside(dx_store, shift, rows, hidden, lddx).double().cpu().numpy(),
            inside(dw_store, shift, vocab, hidden, lddw).double().cpu().numpy(), hx, hw, held,
            None if c is None else c.double().cpu().numpy())


def check(got, labels, dtype, dw_dtype=None, scale=1.0, grads=3, add=False):
    each, loss, dx, dw, x, w, held, c = got
    dw_dtype = dw_dtype or dtype
    rows, hidden = x.shape
    scale = float(np.float32(scale))
    x = np.where((labels >= 0)[:, None], x, 0.0)
    want_each, want_loss, want_dx, want_dw = L.linear_cross_entropy(x, w, labels, c, scale)
    counted = (labels >= 0) & (labels < w.shape[0])
    size = np.where(counted, (np.abs(x) @ np.abs(w).T).max(1) * abs(scale), 0)
    logit = (hidden / 16 + 2) * 2.0 ** -22 * size + 2.0 ** -22 * size
    off = 2 * logit + 2.0 ** -18
    assert (np.abs(each - want_each) <= np.where(counted, off, 0)).all(), np.abs(each - want_each).max()
    weight = np.where(counted, c if c is not None else 1 / max(1, counted.sum()), 0.0)
    assert abs(loss - want_loss) <= (off * np.abs(weight)).sum() + 2.0 ** -23 * abs(want_loss)
    if not grads:
        return
    u = U[dtype]
    z = x @ w.T * scale
    d = np.exp(z - z.max(1, keepdims=True))
    d /= d.sum(1, keepdims=True)
    rows_at = np.flatnonzero(counted)
    d_label = d[rows_at, labels[rows_at]]
    d[rows_at, labels[rows_at]] = 1 - d_label
    d *= (weight * abs(scale))[:, None]
    # the error of a gradient of a logit: two roundings; the logits' own error (relative, and of 1 at the label)
    bad = d * ((2 * u + u * u) + 4 * off)[:, None] if np.ndim(off) else d * (2 * u + u * u + 4 * off)
    bad[rows_at, labels[rows_at]] += (weight * abs(scale) * 2 * off)[rows_at]
    if dtype == "float16":                               # below the smallest normal number, before and after the lift
        bad += np.where(counted, 1.0, 0.0)[:, None] * (np.abs(weight * scale).max() * 2.0 ** -36)
    if grads & 1:
        assert (dx[~counted] == 0).all()
        bound = bad @ np.abs(w) + u * np.abs(want_dx) * 1.01 + (hidden + 60) * 2.0 ** -22 * (d @ np.abs(w)) + TINY[dtype]
        assert (np.abs(dx - want_dx) <= bound).all(), (np.abs(dx - want_dx) / bound).max()
    if grads & 2:
        old = held if add else 0.0
        magnitude = d.T @ np.abs(x)
        bound = bad.T @ np.abs(x) + U[dw_dtype] * np.abs(want_dw + old) * 1.01 + (rows / 16 + 60) * 2.0 ** -22 * (magnitude + np.abs(old)) + TINY[dw_dtype]
        assert (np.abs(dw - (want_dw + old)) <= bound).all(), (np.abs(dw - want_dw - old) / bound).max()
    for on, a, b in ((1, dx, want_dx), (2, dw, want_dw)):
        if grads & on and not add and a.size > 500 and rows_at.size and not (dtype == "float16" and np.abs(b).max() < 1e-3):
            assert np.linalg.norm(a - b) <= u * 1.125 * np.linalg.norm(b), np.linalg.norm(a - b) / np.linalg.norm(b)


SHAPES = [(1, 1, 1), (1, 2, 3), (3, 10, 8), (5, 129, 64), (64, 256, 64), (65, 300, 65), (2, 127, 300), (257, 257, 130),
          (300, 1000, 257), (700, 1001, 150), (1500, 520, 96), (35, 5000, 512), (256, 512, 256), (130, 2600, 70)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_training_step(shape, dtype):
    x, w, labels = inputs(*shape, seed=sum(shape))
    check(call(x, w, labels, dtype), labels, dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", [(3, 10, 8), (300, 1000, 257), (700, 777, 64)])
def test_weights_scale_padding_strides_and_addition(shape, dtype):
    rows, vocab, hidden = shape
    x, w, labels = inputs(*shape, seed=1 + sum(shape), ignored=0.4)
    x[labels < 0] = np.nan                               # rows without a label may hold anything
    x[np.flatnonzero(labels < 0)[::2]] = np.inf
    r = rng(5)
    weights, old = r.random(rows) / rows, r.standard_normal((vocab, hidden)) * 1e-3
    weights[::5] = 0
    got = call(x, w, labels, dtype, weights=weights, scale=-0.7, old=old, lds=(3, 5, 1, 2), shift=1, wide=False)
    check(got, labels, dtype, scale=-0.7, add=True)
    got = call(x, w, labels, dtype, weights=weights * 1000, scale=1.3, lds=(8, 16, 4, 12))
    check(got, labels, dtype, scale=1.3)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dw_dtype", ["float32", None])
def test_master_weights_and_gradients_in_32_bits(dtype, dw_dtype):
    x, w, labels = inputs(333, 901, 190, seed=8, ignored=0.1)
    check(call(x, w, labels, dtype, w_dtype="float32", dw_dtype=dw_dtype), labels, dtype, dw_dtype)
    old = rng(6).standard_normal(w.shape) * 1e-3
    check(call(x, w, labels, dtype, w_dtype="float32", dw_dtype=dw_dtype, old=old, lds=(0, 1, 0, 3)), labels, dtype, dw_dtype,
          add=True)


@pytest.mark.parametrize("grads", [0, 1, 2])
def test_parts_of_the_result(grads):
    x, w, labels = inputs(300, 700, 100, seed=9, ignored=0.2)
    got = call(x, w, labels, "bfloat16", grads=grads)
    check(got, labels, "bfloat16", grads=grads)
    assert grads & 1 or np.isnan(got[2]).all()
    assert grads & 2 or np.isnan(got[3]).all()
    whole = call(x, w, labels, "bfloat16")
    assert np.array_equal(got[0], whole[0]) and got[1] == whole[1]
    assert not grads & 1 or np.array_equal(got[2], whole[2]) or np.allclose(got[2], whole[2], rtol=2.0 ** -7, atol=1e-7)


@pytest.mark.parametrize("dw_dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("ignored", [0.0, 0.3, 0.7])
@pytest.mark.parametrize("add", [False, True])
def test_pieces(add, ignored, dw_dtype):
    """Four pieces of 256 rows; with many rows ignored the last ones are empty."""
    x, w, labels = inputs(1000, 600, 140, seed=10, ignored=ignored)
    old = rng(7).standard_normal(w.shape) * 1e-3 if add else None
    got = call(x, w, labels, "bfloat16", dw_dtype=dw_dtype, piece_rows=200, old=old)
    check(got, labels, "bfloat16", dw_dtype, add=add)
    for grads in (0, 2):
        part = call(x, w, labels, "bfloat16", dw_dtype=dw_dtype, piece_rows=256, old=old, grads=grads)
        assert np.array_equal(part[0], got[0]) and part[1] == got[1]
        assert not grads or np.array_equal(part[3], got[3])


@pytest.mark.parametrize("dtype,dw_dtype,hidden,lddw", [("float16", "float16", 141, 0), ("bfloat16", "float32", 141, 2),
                                                        ("bfloat16", "bfloat16", 264, 0), ("float16", "float32", 40, 3)])
def test_pieces_added_to_rows_of_any_alignment(dtype, dw_dtype, hidden, lddw):
    x, w, labels = inputs(700, 500, hidden, seed=20, ignored=0.2)
    old = rng(9).standard_normal(w.shape) * 1e-3
    for shift in (0, 1):
        got = call(x, w, labels, dtype, dw_dtype=dw_dtype, piece_rows=256, old=old, lds=(0, 0, 0, lddw), shift=shift)
        check(got, labels, dtype, dw_dtype, add=True)


@pytest.mark.parametrize("rows,vocab,hidden", [(3, 70001, 24), (1, 300, 4097), (40, 33000, 72), (513, 257, 1028)])
def test_long_and_wide(rows, vocab, hidden):
    x, w, labels = inputs(rows, vocab, hidden, seed=rows + vocab + hidden)
    check(call(x, w, labels, "bfloat16"), labels, "bfloat16")


@pytest.mark.parametrize("hidden", [32, 33, 64, 96, 128, 129, 160, 256, 257, 288])
def test_last_tiles_of_every_width(hidden):
    x, w, labels = inputs(150, 256 + hidden, hidden, seed=hidden)
    check(call(x, w, labels, "float16"), labels, "float16")


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("piece_rows", [0, 256])
def test_no_label_at_all(dtype, piece_rows):
    x, w, labels = inputs(520, 300, 40, seed=11)
    labels[:] = -1
    x[:] = np.nan
    got = call(x, w, labels, dtype, piece_rows=piece_rows)
    assert (got[0] == 0).all() and got[1] == 0 and (got[2] == 0).all() and (got[3] == 0).all()
    old = rng(8).standard_normal(w.shape)
    got = call(x, w, labels, dtype, old=old, piece_rows=piece_rows)
    assert np.array_equal(got[3], got[6])


def test_labels_outside_the_vocabulary_are_reported():
    torch, B = torch_(), B_()
    x, w, labels = inputs(40, 50, 16, seed=12)
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    check(call(x, w, labels, "bfloat16", status=status), labels, "bfloat16")
    assert status.item() == 0
    labels[3], labels[9] = 50, 2 ** 33
    got = call(x, w, labels, "bfloat16", status=status)
    assert status.item() == B.CROSS_ENTROPY_ST_LABEL and got[0][3] == 0 and got[0][9] == 0
    labels[3] = labels[9] = -1
    check(got, labels, "bfloat16")


def test_sure_rows():
    """Rows that give their label nearly all: 1 - p is far below a step of the type, and the loss near zero."""
    x, w, labels = inputs(200, 300, 64, seed=13)
    x = x * 0.01 + w[labels] * 5
    got = call(x, w, labels, "bfloat16")
    check(got, labels, "bfloat16")
    assert np.median(got[0]) < 1e-3


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_equal_weights_cost_no_rounding(dtype):
    """Of 700 rows with 128 equal logits each, the gradients of the logits are -(1 - 2^-7) and 2^-7 times 1 / 700: stored times
    700 they are numbers of either type, so that dW is off by its own rounding and that of the fp32 sums alone."""
    x, _, labels = inputs(700, 128, 96, seed=15)
    each, loss, _, dw, hx, hw, _, _ = call(x, np.zeros((128, 96)), labels, dtype, grads=2)
    _, want_loss, _, want = L.linear_cross_entropy(hx, hw, labels, None, 1.0)
    d = np.full((700, 128), 2.0 ** -7 / 700)
    d[np.arange(700), labels] = (1 - 2.0 ** -7) / 700
    bound = U[dtype] * np.abs(want) * 1.01 + (700 / 16 + 4) * 2.0 ** -22 * (d.T @ np.abs(hx)) + TINY[dtype]
    assert (np.abs(dw - want) <= bound).all(), (np.abs(dw - want) / bound).max()
    assert abs(loss - want_loss) <= 2.0 ** -18


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_long_sums_are_not_short(dtype):
    """Losses near -s of rows whose label has the logit s, far below another of zero: sums of 8192 products that are cut to fp32
    512 times.  Cut by half a unit of 2^-23 each time, sums that grow evenly would be short by 0.36 x 512 x 2^-24 of s (what
    accumulators with more bits lose is less); in the mean over the rows, less than 0.1 times 512 x 2^-24 may be left."""
    r = rng(16)
    w = np.stack((r.standard_normal(8192) * 2 * 8192 ** -0.5, np.zeros(8192)))
    x = r.standard_normal((1000, 8192)) - 2 * (1 + r.random((1000, 1))) * w[0]
    each, _, _, _, hx, hw, _, _ = call(x, w, np.zeros(1000, dtype=np.int64), dtype, grads=0)
    s = hx @ hw[0]
    want = np.logaddexp(s, 0.0) - s
    assert abs((each - want).mean()) < 0.1 * 512 * 2.0 ** -24 * np.abs(s).mean(), (each - want).mean() / np.abs(s).mean()


def test_logits_of_any_size():
    """Logits of thousands, and equal ones; columns far below the others vanish."""
    x, w, labels = inputs(100, 400, 32, seed=14, sharp=600.0)
    check(call(x, w, labels, "bfloat16"), labels, "bfloat16")
    x[:] = 0
    got = call(x, w, labels, "bfloat16")
    assert np.abs(got[0] - np.log(400)).max() < 1e-5 and (got[3] == 0).all()
    check(got, labels, "bfloat16")


def test_infinite_logits():
    """A logit of -inf counts as probability 0 (its row of w gets no gradient from that row of x); NaN and +inf make the
    row's loss NaN and leave the other rows' losses."""
    torch = torch_()
    x, w, labels = inputs(20, 300, 16, seed=15)
    x = np.abs(x)
    w[7] = -np.inf                                       # in a half of a tile with others
    w[256:] = -np.inf                                    # a half of a tile by itself
    labels[:] = np.arange(20) + 8
    got = call(x, w, labels, "bfloat16", grads=2)
    kept = [i for i in range(256) if i != 7]
    want = L.linear_cross_entropy(got[4], got[5][kept], labels - 1)
    assert np.abs(got[0] - want[0]).max() < 1e-4
    assert (got[3][7] == 0).all() and (got[3][256:] == 0).all()
    x[4] = np.nan
    w[7] = 1.0
    w[256:] = 0.5
    x[5, 0] = np.inf
    got = call(x, w, labels, "bfloat16", grads=0)
    assert np.isnan(got[0][[4, 5]]).all() and np.isfinite(np.delete(got[0], [4, 5])).all() and np.isnan(got[1])


def test_repeats_bit_for_bit_and_across_streams():
    torch, B = torch_(), B_()
    rows, vocab, hidden = 600, 3000, 200
    x = torch.randn(rows, hidden, device="cuda").bfloat16()
    w = torch.randn(vocab, hidden, device="cuda").bfloat16() / 10
    y = torch.randint(0, vocab, (rows,), device="cuda")
    need = B.sidco_linear_cross_entropy_workspace_bytes(x, w, hidden, rows, vocab, hidden)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for i in range(6):
        with torch.cuda.stream(streams[i & 1]):
            out = [torch.empty(rows, device="cuda"), torch.empty((), device="cuda"), torch.empty_like(x),
                   torch.empty_like(w), torch.empty(need, dtype=torch.uint8, device="cuda")]
            B.sidco_linear_cross_entropy(x, hidden, w, hidden, y, rows, vocab, hidden, out[0], out[1], out[2], hidden,
                                         out[3], hidden, out[4], need)
            outs.append(out)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o[:4], outs[0]))


def test_in_a_graph_follows_its_inputs():
    torch, B = torch_(), B_()
    rows, vocab, hidden = 300, 500, 64
    x = torch.randn(rows, hidden, device="cuda").bfloat16()
    w = torch.randn(vocab, hidden, device="cuda").bfloat16() / 4
    y = torch.randint(0, vocab, (rows,), device="cuda")
    each, loss = torch.empty(rows, device="cuda"), torch.empty((), device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    need = B.sidco_linear_cross_entropy_workspace_bytes(x, w, hidden, rows, vocab, hidden)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sidco_linear_cross_entropy(x, hidden, w, hidden, y, rows, vocab, hidden, each, loss, dx, hidden, dw, hidden, ws, need)
    for k in range(3):
        x.normal_()
        y.copy_(torch.where(torch.rand(rows, device="cuda") < 0.3 * k, -1, torch.randint(0, vocab, (rows,), device="cuda")))
        g.replay()
        torch.cuda.synchronize()
        check((each.double().cpu().numpy(), loss.double().item(), dx.double().cpu().numpy(), dw.double().cpu().numpy(),
               x.double().cpu().numpy(), w.double().cpu().numpy(), None, None), y.cpu().numpy(), "bfloat16")


def test_no_rows():
    torch, B = torch_(), B_()
    loss, dw = torch.full((), 5.0, device="cuda"), torch.full((7, 4), 5.0, device="cuda")
    B.sidco_linear_cross_entropy(None, 4, None, 4, None, 0, 7, 4, None, loss, None, 4, dw, 4, None, 0, add=True, x_type=1,
                                 w_type=1, label_type=4)
    assert loss.item() == 0 and bool((dw == 5).all())
    B.sidco_linear_cross_entropy(None, 4, None, 4, None, 0, 7, 4, None, loss, None, 4, dw, 4, None, 0, x_type=1, w_type=1,
                                 label_type=4)
    assert bool((dw == 0).all())
