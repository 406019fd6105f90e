"""Data-parallel training of a two-layer network with 4-bit products, 4-bit gradient exchange and orthogonalised updates.

    python examples/four_bit_training.py [--steps 60] [--exchange mx4|sparse]
    python -m torch.distributed.run --standalone --local-addr 127.0.0.1 --nproc-per-node N examples/four_bit_training.py

Every step: forward and backward through ``mx4_linear`` (quantise, product), the flat gradient through the
error-compensated compressor (``sidco_mx4_compress``, or ``sidco_compress`` with --exchange sparse), all-gather, dense
mean, momentum and orthogonalised update (``sidco_orthogonalize``), weights <- weights - lr * update.  The network learns
a fixed random network of the same shape; the loss of every tenth step is printed.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2101_10761_b200 import binding as B                                        # noqa: E402
from paper_2101_10761_b200.exchange import gather_mx4, gather_sparse                  # noqa: E402
from paper_2101_10761_b200.training import OrthogonalizedUpdate, mx4_linear           # noqa: E402


def train(steps=60, exchange="mx4", width=200, hidden=500, outputs=40, batch=700, lr=0.02, rank=0):
    """Returns the losses (before every step)."""
    dev = torch.device("cuda", torch.cuda.current_device())
    shapes = [(hidden, width), (outputs, hidden)]
    sizes = [r * c for r, c in shapes]
    d = sum(sizes)
    g = torch.Generator(device=dev).manual_seed(0)                                     # the same weights everywhere
    teacher = [torch.randn(s, generator=g, device=dev) / s[1] ** 0.5 for s in shapes]
    flat = torch.cat([(torch.randn(s, generator=g, device=dev) * 0.5 / s[1] ** 0.5).view(-1) for s in shapes])
    residual = torch.zeros(d, device=dev)
    mean = torch.empty(d, device=dev)
    blocks = -(-d // 32)
    codes = torch.empty(16 * blocks, dtype=torch.uint8, device=dev)
    scales = torch.empty(blocks, dtype=torch.uint8, device=dev)
    idx = torch.empty(d, dtype=torch.int32, device=dev)
    val = torch.empty(d, device=dev)
    count = torch.empty(len(shapes) + 1, dtype=torch.int32, device=dev)
    offsets = [0, sizes[0], d]
    update = OrthogonalizedUpdate(shapes, dev)
    data = torch.Generator(device=dev).manual_seed(1000 + rank)
    losses = []
    for step in range(steps):
        x = torch.randn(batch, width, generator=data, device=dev)
        target = torch.relu(x @ teacher[0].T) @ teacher[1].T
        leaf = flat.detach().requires_grad_()
        w = [p.view(s) for p, s in zip(leaf.split(sizes), shapes)]
        hid = torch.relu(mx4_linear(x.bfloat16(), w[0]))
        loss = (mx4_linear(hid, w[1]).float() - target).square().mean()
        loss.backward()
        if exchange == "mx4":
            B.sidco_mx4_compress(leaf.grad, residual, d, codes, scales)
            codes_all, scales_all, world = gather_mx4(codes, scales)
            B.sidco_mx4_mean(codes_all, scales_all, world, d, mean)
        else:
            B.sidco_compress(leaf.grad, residual, offsets, 0.05, B.SID_EXP, 2, idx, val, count)
            idx_all, val_all, counts, stride = gather_sparse(idx, val, int(count[-1]))
            B.sidco_aggregate(idx_all, val_all, counts, counts.numel(), stride, d, mean)
        flat -= lr * (1 - step / steps) * update.step(mean)
        losses.append(loss.detach())
    if exchange != "mx4":
        B.sidco_release(residual)
    return torch.stack(losses).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--exchange", choices=("mx4", "sparse"), default="mx4")
    a = ap.parse_args()
    rank = int(os.environ.get("RANK", 0))
    torch.cuda.set_device(int(os.environ.get("LOCAL_RANK", 0)))
    if int(os.environ.get("WORLD_SIZE", 1)) > 1:
        torch.distributed.init_process_group("nccl")
    losses = train(a.steps, a.exchange, rank=rank)
    if rank == 0:
        for i in list(range(0, a.steps, 10)) + [a.steps - 1]:
            print("step %3d  loss %.5f" % (i, losses[i]))
    if torch.distributed.is_initialized():
        torch.distributed.destroy_process_group()


if __name__ == "__main__":
    main()
