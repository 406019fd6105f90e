"""Argument errors of the matrix operators, found on the host before any CUDA call (no GPU), and the 4-bit exchange over
two gloo ranks."""
import ctypes
import json
import os
import socket
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x100000                                   # never dereferenced: every call below fails validation first
BIG = 1 << 31


@pytest.fixture(scope="module")
def B():
    from paper_2101_10761_b200 import binding, build
    build.build()
    return binding


def code(call, *args, **kw):
    from paper_2101_10761_b200 import binding
    with pytest.raises(binding.SidcoError) as e:
        call(*args, stream=0, **kw)
    return e.value.code


def test_sizes(B):
    assert B.sidco_mx4_code_bytes(3, 33) == 3 * 32 and B.sidco_mx4_code_bytes(0, 9) == 0
    assert B.sidco_mx4_scale_bytes(129, 129) == 2 * 2 * 512 and B.sidco_mx4_scale_bytes(1, 128) == 512
    for f in (B.sidco_mx4_code_bytes, B.sidco_mx4_scale_bytes):
        for bad in ((-1, 4), (4, -1), (BIG, 1), (1, BIG)):
            with pytest.raises(B.SidcoError) as e:
                f(*bad)
            assert e.value.code == -10


def test_quantize_refuses(B):
    q = B.sidco_mx4_quantize
    assert code(q, P, -1, 8, 8, P, P, x_type=0) == -10
    assert code(q, P, 8, BIG, BIG, P, P, x_type=0) == -10
    assert code(q, P, 8, 8, 8, P, P, x_type=3) == -13
    assert code(q, P, 8, 8, 8, P, P) == -13                       # a raw address without a type
    assert code(q, np.zeros(4, np.float64), 2, 2, 2, P, P) == -13
    assert code(q, P, 8, 8, 7, P, P, x_type=0) == -6
    assert code(q, P, 8, 8, 8, None, None, x_type=0) == -1
    assert code(q, P, 8, 8, 8, P, None, x_type=0) == -1
    assert code(q, P, 8, 8, 8, P, P, None, P, x_type=0) == -1
    assert code(q, None, 8, 8, 8, P, P, x_type=0) == -1
    assert code(q, P + 2, 8, 8, 8, P, P, x_type=0) == -14
    assert code(q, P, 8, 8, 8, P + 8, P, x_type=0) == -14
    assert code(q, P, 8, 8, 8, P, P + 4, x_type=1) == -14
    q(None, 0, 8, 8, P, P, x_type=0, stream=0)                    # nothing to do


def test_dequantize_refuses(B):
    q = B.sidco_mx4_dequantize
    assert code(q, P, P, -1, 8, P, 8, out_type=0) == -10
    assert code(q, P, P, 8, 8, P, 8, out_type=9) == -13
    assert code(q, P, P, 8, 8, P, 4, out_type=0) == -6
    assert code(q, P, None, 8, 8, P, 8, out_type=0) == -1
    assert code(q, P, P + 1, 8, 8, P, 8, out_type=0) == -14
    assert code(q, P, P, 8, 8, P + 1, 8, out_type=1) == -14


def test_matmul_refuses(B):
    f = B.sidco_mx4_matmul
    assert code(f, P, P, P, P, -1, 4, 4, P, 4, c_type=0) == -10
    assert code(f, P, P, P, P, 4, 4, BIG, P, 4, c_type=0) == -10
    assert code(f, P, P, P, P, 4, 4, 4, P, 4, c_type=-1) == -13
    assert code(f, P, P, P, P, 4, 4, 4, P, 3, c_type=0) == -6
    assert code(f, P, P, P, P, 4, 4, 4, None, 4, c_type=0) == -1
    assert code(f, P, P, P, None, 4, 4, 4, P, 4, c_type=0) == -1
    assert code(f, P, P + 8, P, P, 4, 4, 4, P, 4, c_type=0) == -14
    assert code(f, P, P, P, P, 4, 4, 4, P + 1, 4, c_type=2) == -14


def test_compress_and_mean_refuse(B):
    f = B.sidco_mx4_compress
    assert code(f, P, 2 * P, -1, P, P, grad_type=0) == -10
    assert code(f, P, 2 * P, BIG, P, P, grad_type=0) == -10
    assert code(f, P, 2 * P, 8, P, P, grad_type=4) == -13
    assert code(f, P, None, 8, P, P, grad_type=0) == -1
    assert code(f, P, 2 * P, 8, P + 4, P, grad_type=0) == -14
    assert code(f, P + 1, 2 * P, 8, P, P, grad_type=1) == -14
    assert code(f, P, P + 16, 8, P, P, grad_type=0) == -9
    assert code(f, P, P + 12, 8, P, P, grad_type=1) == -9
    g = B.sidco_mx4_mean
    assert code(g, P, P, 0, 8, P) == -6 and code(g, P, P, 65, 8, P) == -6
    assert code(g, P, P, 2, -8, P) == -10 and code(g, P, P, 2, BIG, P) == -10
    assert code(g, P, None, 2, 8, P) == -1
    assert code(g, P + 8, P, 2, 8, P) == -14 and code(g, P, P, 2, 8, P + 2) == -14


def test_orthogonalize_refuses(B):
    f = B.sidco_orthogonalize

    def call(grad=P, mom=2 * P, mu=0.9, off=(0,), rows=(8,), cols=(8,), steps=5, out=3 * P, ws=4 * P, n=1 << 30, eps=1e-7,
             t=0):
        return code(f, grad, mom, mu, True, off, rows, cols, steps, out, ws, n, eps, grad_type=t)
    assert call(rows=(-1,)) == -10 and call(cols=((1 << 22) + 1,)) == -10
    assert call(rows=(20000,), cols=(20000,)) == -10
    assert call(t=7) == -13
    assert call(mu=1.0) == -6 and call(mu=-0.1) == -6 and call(mu=float("nan")) == -6
    assert call(steps=0) == -6 and call(steps=33) == -6 and call(eps=-1.0) == -6
    big = dict(rows=(300,), cols=(200,))                          # (small matrices need no workspace)
    assert call(grad=None) == -1 and call(out=None) == -1 and call(ws=None, **big) == -1
    assert call(off=(-4,)) == -2
    assert call(off=(0, 63), rows=(8, 4), cols=(8, 4)) == -2 and call(off=(3, 0), rows=(8, 2), cols=(8, 2)) == -2    # overlap
    assert call(out=P + 16) == -9 and call(mom=P + 128) == -9 and call(mom=3 * P - 128) == -9
    assert call(grad=P + 2) == -14 and call(mom=P + 1) == -14 and call(out=P + 1) == -14
    need = B.sidco_orthogonalize_workspace_bytes([300], [200])
    assert call(n=need - 1, **big) == -8 and call(ws=4 * P + 8, **big) == -8
    assert B.sidco_orthogonalize_workspace_bytes([128, 2048], [2048, 5]) == 0
    with pytest.raises(ValueError):
        f(P, None, 0.9, True, [0], [8, 8], [8], 5, P, P, 1 << 30, grad_type=0, stream=0)
    with pytest.raises(B.SidcoError):
        B.sidco_orthogonalize_workspace_bytes([1 << 23], [4])
    assert B.sidco_orthogonalize_workspace_bytes([], []) == 0
    # a chain's workspace is reused by the next: many matrices cost no more than the largest chain
    assert B.sidco_orthogonalize_workspace_bytes([200] * 128, [150] * 128) == \
        B.sidco_orthogonalize_workspace_bytes([200] * 256, [150] * 256) > 0


def test_hooks_refuse(B):
    for bad in ((-1, -1), (3000000, -1), (0, -2)):
        with pytest.raises(B.SidcoError) as e:
            B.sidco_set_product_test_hooks(*bad)
        assert e.value.code == -6


def test_error_texts_name_the_reason(B):
    assert "type" in B.sidco_error_string(-13) and "aligned" in B.sidco_error_string(-14)


def test_matrix_helpers_refuse():
    import torch
    from paper_2101_10761_b200 import training as T
    with pytest.raises(ValueError):
        T.quantize(torch.zeros(4))
    with pytest.raises(ValueError):
        T.mx4_linear(torch.zeros(2, 4), torch.zeros(3, 5))


WORKER = r'''
import os, sys, json
sys.path.insert(0, %r)
import numpy as np, torch, torch.distributed as dist
from paper_2101_10761_b200.exchange import gather_mx4
from oracle import mx4_oracle as Q
dist.init_process_group("gloo", rank=int(os.environ["RANK"]), world_size=int(os.environ["WORLD_SIZE"]))
rank, d = dist.get_rank(), 1001
grads = [np.random.Generator(np.random.PCG64(w)).laplace(0, 1e-3, d).astype(np.float32) for w in range(2)]
codes, scales, value, _ = Q.compress(grads[rank], np.zeros(d))
c, s, n = gather_mx4(torch.from_numpy(codes), torch.from_numpy(scales))
assert n == 2
dense = Q.mean(c.numpy(), s.numpy(), n, d)
want = sum(Q.compress(g, np.zeros(d))[2] for g in grads) / 2
print(json.dumps({"ok": bool(np.array_equal(dense, want)), "sum": float(np.abs(dense).sum())}))
dist.destroy_process_group()
''' % ROOT


def test_two_ranks_exchange_quantised_gradients():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = str(s.getsockname()[1])
    procs = [subprocess.Popen([sys.executable, "-c", WORKER],
                              env=dict(os.environ, RANK=str(r), LOCAL_RANK=str(r), WORLD_SIZE="2", MASTER_ADDR="127.0.0.1",
                                       MASTER_PORT=port), cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
             for r in range(2)]
    recs = []
    for p in procs:
        out, err = p.communicate(timeout=600)
        assert p.returncode == 0, err[-3000:]
        recs.append(json.loads(out.strip().splitlines()[-1]))
    assert recs[0] == recs[1] and recs[0]["ok"] and recs[0]["sum"] > 0


def test_one_process_gathers_itself():
    import torch
    from paper_2101_10761_b200.exchange import gather_mx4
    c, s = torch.arange(32, dtype=torch.uint8), torch.arange(2, dtype=torch.uint8)
    got = gather_mx4(c, s)
    assert torch.equal(got[0], c) and torch.equal(got[1], s) and got[2] == 1
