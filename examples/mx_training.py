"""Two workers train a small network against the service, every product on 4-bit operands.

    python examples/mx_training.py [--steps 60]

Each worker, each step: pulls the fp32 master weights, quantises them along both directions, runs
forward and backward with ps_mx_matmul, clips its own gradient and writes it as bf16 to its push
buffer (Clip).  The service sums both workers' shards, clips the sum by the job's global norm and
applies Adam (ps_round_run_clipped).  The task: regress the outputs of a fixed random network.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2204_03211_b200 import binding as B  # noqa: E402

WORKERS, BATCH, D_IN, D_HIDDEN, D_OUT = 2, 512, 256, 640, 96
SHAPES = [(D_HIDDEN, D_IN), (D_OUT, D_HIDDEN)]


class Linear:
    """y = x w^T on 4-bit operands, with both gradients."""

    def __init__(self, shape, dtype=torch.bfloat16):
        n, k = shape
        both = lambda r, c: (B.MxTensor(r, c), B.MxTensor(c, r))  # noqa: E731
        self.w, self.x, self.dy = both(n, k), both(BATCH, k), both(BATCH, n)
        empty = lambda r, c: torch.empty(r, c, device="cuda", dtype=dtype)  # noqa: E731
        self.y, self.dx, self.dw = empty(BATCH, n), empty(BATCH, k), torch.empty(n, k, device="cuda")

    def load(self, w):
        B.ps_mx_quantize(w, *self.w)

    def forward(self, x):
        B.ps_mx_quantize(x, *self.x)
        return B.ps_mx_matmul(self.x[0], self.w[0], self.y)

    def backward(self, dy):
        """Returns dx = dy w; leaves dw = dy^T x."""
        B.ps_mx_quantize(dy, *self.dy)
        B.ps_mx_matmul(self.dy[1], self.x[1], self.dw)
        return B.ps_mx_matmul(self.dy[0], self.w[1], self.dx)


class Worker:
    def __init__(self, rank, teacher, local_norm):
        self.rank, self.teacher, self.local_norm = rank, teacher, local_norm
        self.layers = [Linear(s) for s in SHAPES]
        self.push = [torch.empty(s, device="cuda", dtype=torch.bfloat16) for s in SHAPES]
        self.clip = B.Clip([l.dw for l in self.layers], self.push)
        self.gen = torch.Generator(device="cuda").manual_seed(100 + rank)

    def step(self, weights):
        x = torch.randn(BATCH, D_IN, device="cuda", generator=self.gen).bfloat16()
        target = torch.relu(x.float() @ self.teacher[0].t()) @ self.teacher[1].t()
        for layer, w in zip(self.layers, weights):
            layer.load(w)
        h = self.layers[0].forward(x)
        y = self.layers[1].forward(torch.relu(h))
        diff = y.float() - target
        dh = self.layers[1].backward((diff * (2.0 / diff.numel())).bfloat16())
        self.layers[0].backward(torch.where(h > 0, dh, torch.zeros_like(dh)))
        self.clip.run(self.local_norm)
        return (diff * diff).mean()


def train(steps=60, max_norm=1.0, local_norm=2.0, lr=2e-3):
    """Returns the mean loss of every step and the gradient norms the service reported."""
    torch.cuda.set_device(0)
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda s, scale: torch.randn(s, device="cuda", generator=gen) * scale  # noqa: E731
    teacher = [rand(s, s[1] ** -0.5) for s in SHAPES]
    svc = B.Service(0, 1, 16 << 20)
    job = svc.register_job(opt=B.PS_ADAM, grad_dtype=B.PS_BF16, num_workers=WORKERS, lr=lr, grad_scale=1.0 / WORKERS)
    for b, s in enumerate(SHAPES):
        svc.register_block(job, b, s[0] * s[1], 0, rand(s, s[1] ** -0.5))
    weights = [svc.view(svc.pull(job, b), s[0] * s[1]).view(s) for b, s in enumerate(SHAPES)]
    workers = [Worker(w, teacher, local_norm) for w in range(WORKERS)]
    blocks = np.repeat(np.arange(len(SHAPES), dtype=np.int32), WORKERS)
    ranks = np.tile(np.arange(WORKERS, dtype=np.int32), len(SHAPES))
    ptrs = np.array([workers[w].push[b].data_ptr() for b, w in zip(blocks, ranks)], np.uint64)
    rnd = svc.round_prepare(np.full(len(blocks), job, np.int32), blocks, ranks, ptrs, [(job, b) for b in range(len(SHAPES))])
    norms = torch.zeros(steps, device="cuda")
    losses = []
    for t in range(steps):
        losses.append(sum(w.step(weights) for w in workers) / WORKERS)
        svc.round_run_clipped(rnd, max_norm, norms[t:])
    losses, norms = torch.stack(losses).tolist(), norms.tolist()
    assert B.ps_mx_status() == 0 and svc.device_status() == 0
    svc.close()
    return losses, norms


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    losses, norms = train(ap.parse_args().steps)
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %3d  loss %.4f  gradient norm %.4f" % (t, losses[t], norms[t]))
    print("last       loss %.4f" % losses[-1])
