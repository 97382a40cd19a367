"""Two workers train a next-word model against the service: Muon for its hidden matrix, Adam for its output weight.

    python examples/lm_training.py [--steps 60]

Each worker, each step: pulls the fp32 master weights, runs the hidden layer on 4-bit operands (ps_mx_matmul), takes
the loss over the vocabulary and both of its gradients without the scores ever being stored (CrossEntropy), and pushes
bf16 gradients.  The service sums both workers' shards; the hidden matrix belongs to a PS_MUON job (momentum and an
orthogonalised update), the output weight to a PS_ADAM job whose gradients it clips by their norm.  The task: words
follow one another by a fixed random rule, seen through fixed random features; a tenth of each batch is padding.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import mx_training as mx  # noqa: E402

from paper_2204_03211_b200 import binding as B  # noqa: E402

WORKERS, BATCH, VOCAB, D_IN, D_HIDDEN = 2, mx.BATCH, 1000, 256, 640


class Worker:
    def __init__(self, rank, features, rule):
        self.rank, self.features, self.rule = rank, features, rule
        self.hidden = mx.Linear((D_HIDDEN, D_IN))
        self.head = B.CrossEntropy(BATCH, VOCAB, D_HIDDEN)
        empty = lambda *s: torch.empty(s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        self.dh, self.push_hidden, self.push_out = empty(BATCH, D_HIDDEN), empty(D_HIDDEN, D_IN), empty(VOCAB, D_HIDDEN)
        self.clip = B.Clip([self.hidden.dw], [self.push_hidden])           # (with no limit: fp32 into the push buffer)
        self.gen = torch.Generator(device="cuda").manual_seed(100 + rank)

    def step(self, w_hidden, w_out):
        words = torch.randint(0, VOCAB, (BATCH,), device="cuda", generator=self.gen)
        targets = self.rule[words]
        targets[BATCH - BATCH // 10:] = -100
        scale = 1.0 / (BATCH - BATCH // 10)
        x = self.features[words]
        self.hidden.load(w_hidden)
        h = torch.relu(self.hidden.forward(x))
        w = w_out.bfloat16()
        loss, lse = self.head.forward(h, w, targets)
        self.head.backward(h, w, targets, lse, self.dh, self.push_out, scale=scale)
        self.hidden.backward(torch.where(h > 0, self.dh, torch.zeros_like(self.dh)))
        self.clip.run(float("inf"))
        self.last = (h, w, targets)
        return loss.sum() * scale


def train(steps=60, max_norm=1.0):
    """Returns the mean loss of every step, the norms of the output weight's gradients, and the workers."""
    torch.cuda.set_device(0)
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda s, scale: torch.randn(s, device="cuda", generator=gen) * scale  # noqa: E731
    features = rand((VOCAB, D_IN), 1.0).bfloat16()
    rule = torch.randperm(VOCAB, device="cuda", generator=gen)
    svc = B.Service(0, 1, 32 << 20)
    common = dict(grad_dtype=B.PS_BF16, num_workers=WORKERS, grad_scale=1.0 / WORKERS)
    muon = svc.register_job(opt=B.PS_MUON, lr=0.02, momentum=0.95, **common)
    adam = svc.register_job(opt=B.PS_ADAM, lr=5e-3, **common)
    svc.register_matrix(muon, 0, D_HIDDEN, D_IN, 0, rand((D_HIDDEN, D_IN), D_IN ** -0.5))
    svc.register_block(adam, 0, VOCAB * D_HIDDEN, 0, rand((VOCAB, D_HIDDEN), D_HIDDEN ** -0.5))
    w_hidden = svc.view(svc.pull(muon, 0), D_HIDDEN * D_IN).view(D_HIDDEN, D_IN)
    w_out = svc.view(svc.pull(adam, 0), VOCAB * D_HIDDEN).view(VOCAB, D_HIDDEN)
    workers = [Worker(r, features, rule) for r in range(WORKERS)]
    ranks, zeros = np.arange(WORKERS, dtype=np.int32), np.zeros(WORKERS, np.int32)

    def prepare(job, buffers):
        ptrs = np.array([t.data_ptr() for t in buffers], np.uint64)
        return svc.round_prepare(np.full(WORKERS, job, np.int32), zeros, ranks, ptrs, [(job, 0)])

    rounds = prepare(muon, [w.push_hidden for w in workers]), prepare(adam, [w.push_out for w in workers])
    norms = torch.zeros(steps, device="cuda")
    losses = []
    for t in range(steps):
        losses.append(sum(w.step(w_hidden, w_out) for w in workers) / WORKERS)
        svc.round_run(rounds[0])
        svc.round_run_clipped(rounds[1], max_norm, norms[t:])
    losses, norms = torch.stack(losses).tolist(), norms.tolist()
    assert B.ps_mx_status() == 0 and B.ps_xent_status() == 0 and svc.device_status() == 0
    svc.close()
    return losses, norms, workers


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    losses, norms, _ = train(ap.parse_args().steps)
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %3d  loss %.4f  gradient norm %.4f" % (t, losses[t], norms[t]))
    print("last       loss %.4f" % losses[-1])
