"""The language-model example: loss, gradients and both kinds of round run together."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_lm_training_runs_and_its_gradients_are_the_formulas():
    spec = importlib.util.spec_from_file_location("lm_training", os.path.join(ROOT, "examples", "lm_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms, workers = example.train(steps=4)
    assert all(math.isfinite(v) for v in losses) and all(n > 0 for n in norms)
    pushed = []
    for w in workers:
        h, wt, targets = (t.double() if t.is_floating_point() else t for t in w.last)
        keep = targets >= 0
        s = h @ wt.t()
        e = torch.softmax(s, 1)
        e[torch.arange(len(h)), targets.clamp(min=0)] -= 1
        e = e * keep[:, None] / keep.sum()
        for got, ref, size in ((w.dh, e @ wt, e.abs() @ wt.abs()), (w.push_out, e.t() @ h, e.abs().t() @ h.abs())):
            # one bf16 rounding of each entry of e and of the result, and 1e-5 for the scores' binary32 sums
            assert bool(((got.double() - ref).abs() <= (2.0 ** -8 + 1e-5) * size + 2.0 ** -8 * ref.abs() + 1e-12).all())
        pushed.append(w.push_out.double())
    # the service reports the norm of the mean of what was pushed (the last step's buffers are still there)
    assert abs(norms[-1] - float((sum(pushed) / len(pushed)).norm())) <= 1e-5 * norms[-1]
    again, _, _ = example.train(steps=2)
    assert again == losses[:2]              # nothing in a step depends on the order in which the GPU does things
