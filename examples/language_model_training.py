"""Data-parallel training of a small language model: lookup and dropout of the tokens, 4-bit linear layers with a residual,
cross entropy over the vocabulary, 4-bit gradient exchange and orthogonalised updates.

    python examples/language_model_training.py [--steps 60] [--untied] [--graph]
    python -m torch.distributed.run --standalone --local-addr 127.0.0.1 --nproc-per-node N examples/language_model_training.py

Every step: ``embedding`` (scaled, with dropout), ``mx4_linear`` twice with ``dropout`` onto the residual stream, and
``linear_cross_entropy`` against the next tokens, its weight the table itself unless --untied.  The flat gradient goes through
the error-compensated compressor and the all-gather to the orthogonalised update.  The text is a random walk over the words:
each is followed by one of four.  With --graph a step's forward and backward pass is captured once and replayed, the dropout
masks drawn anew by a counter on the device.  The loss of every tenth step is printed.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2101_10761_b200 import binding as B                                                       # noqa: E402
from paper_2101_10761_b200.exchange import gather_mx4                                                # noqa: E402
from paper_2101_10761_b200.training import (OrthogonalizedUpdate, dropout, embedding,                # noqa: E402
                                            linear_cross_entropy, mx4_linear)


class Model:
    """Parameters as views of one flat fp32 vector."""

    def __init__(self, vocab, width, hidden, tied, p, device):
        self.shapes = [(vocab, width), (hidden, width), (width, hidden)] + ([] if tied else [(vocab, width)])
        self.sizes = [r * c for r, c in self.shapes]
        g = torch.Generator(device=device).manual_seed(0)                              # the same weights everywhere
        self.flat = torch.cat([(torch.randn(s, generator=g, device=device) / s[1] ** 0.5).view(-1) for s in self.shapes])
        self.flat.requires_grad_()
        self.tied, self.p, self.width = tied, p, width
        self.step = torch.zeros(1, dtype=torch.int64, device=device)                   # number of the step, for the masks

    def loss(self, tokens, labels):
        w = [v.view(s) for v, s in zip(self.flat.split(self.sizes), self.shapes)]
        x = embedding(tokens, w[0], scale=self.width ** 0.5, p=self.p, seed=1, call=0, step=self.step, dtype=torch.bfloat16)
        y = mx4_linear(torch.relu(mx4_linear(x, w[1])), w[2])
        x = dropout(y, self.p, seed=2, call=0, step=self.step, residual=x)
        return linear_cross_entropy(x, w[0] if self.tied else w[3], labels, scale=self.width ** -0.5)


def text(next_words, sequences, length, g):
    """Tokens [sequences, length + 1], some of the sequences padded with -1 at their end."""
    device = next_words.device
    walk = [torch.randint(0, next_words.shape[0], (sequences,), generator=g, device=device)]
    for _ in range(length):
        pick = torch.randint(0, next_words.shape[1], (sequences,), generator=g, device=device)
        walk.append(next_words[walk[-1], pick])
    words = torch.stack(walk, 1)
    ends = torch.randint(length // 2, 2 * length, (sequences, 1), generator=g, device=device)
    return torch.where(torch.arange(length + 1, device=device) <= ends, words, -1)


def train(steps=60, tied=True, graph=False, vocab=1000, width=128, hidden=384, sequences=20, length=35, p=0.1, lr=0.02, rank=0):
    """Returns the losses (before every step)."""
    dev = torch.device("cuda", torch.cuda.current_device())
    model = Model(vocab, width, hidden, tied, p, dev)
    d = model.flat.numel()
    g = torch.Generator(device=dev).manual_seed(3)
    next_words = torch.randint(0, vocab, (vocab, 4), generator=g, device=dev)
    data = torch.Generator(device=dev).manual_seed(1000 + rank)
    blocks = -(-d // 32)
    residual, mean = torch.zeros(d, device=dev), torch.empty(d, device=dev)
    codes = torch.empty(16 * blocks, dtype=torch.uint8, device=dev)
    scales = torch.empty(blocks, dtype=torch.uint8, device=dev)
    update = OrthogonalizedUpdate(model.shapes, dev)
    tokens = torch.empty(sequences, length, dtype=torch.int64, device=dev)
    labels = torch.empty_like(tokens)

    def forward_backward():
        model.flat.grad = None
        loss = model.loss(tokens, labels)
        loss.backward()
        model.step.add_(1)                                                             # new masks in the next step
        return loss.detach()

    captured, loss = None, None
    losses = []
    for step in range(steps):
        words = text(next_words, sequences, length, data)
        tokens.copy_(words[:, :-1])
        labels.copy_(words[:, 1:])
        if graph and captured is None:
            side = torch.cuda.Stream()                                                 # (as captures ask for: a run beside)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                forward_backward()
                model.step.zero_()
            torch.cuda.current_stream().wait_stream(side)
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                loss = forward_backward()
        if graph:
            captured.replay()
        else:
            loss = forward_backward()
        B.sidco_mx4_compress(model.flat.grad, residual, d, codes, scales)
        codes_all, scales_all, world = gather_mx4(codes, scales)
        B.sidco_mx4_mean(codes_all, scales_all, world, d, mean)
        with torch.no_grad():
            model.flat -= lr * (1 - step / steps) * update.step(mean)
        losses.append(loss.clone())
    return torch.stack(losses).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--untied", action="store_true")
    ap.add_argument("--graph", action="store_true")
    a = ap.parse_args()
    rank = int(os.environ.get("RANK", 0))
    torch.cuda.set_device(int(os.environ.get("LOCAL_RANK", 0)))
    if int(os.environ.get("WORLD_SIZE", 1)) > 1:
        torch.distributed.init_process_group("nccl")
    losses = train(a.steps, not a.untied, a.graph, rank=rank)
    if rank == 0:
        for i in list(range(0, a.steps, 10)) + [a.steps - 1]:
            print("step %3d  loss %.5f" % (i, losses[i]))
    if torch.distributed.is_initialized():
        torch.distributed.destroy_process_group()


if __name__ == "__main__":
    main()
