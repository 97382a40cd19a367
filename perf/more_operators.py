"""Cases for measuring the matrix operators around the service: Muon's step and the loss over a vocabulary.

Three operators, each in a plain form (elementary torch operations in 32 bits, norms in 64) and,
where `own` is true, through this package's entry points:

  ortho  matrices orthogonalised by five Newton-Schulz steps (a worker's, or a trainer's own, optimizer step)
  muon   one round of a PS_MUON job: sum of the workers' shards, momentum, orthogonalised update, decoupled
         weight decay, for all of the job's matrices
  xent   softmax cross entropy of tokens over a vocabulary, from activations and the output weight: the losses
         alone (evaluation), or with the gradients of both (a training step)

`listed()` and `draw()` give the cases, `prepare()` a case's inputs, `run()` one pass, `exact()`
what a pass returns computed in 64 bits, and `work()` the bytes and operations no pass can do without.
"""
import math

import numpy as np
import torch

own = False

F32, BF16 = "f32", "bf16"
DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
ESIZE = {F32: 4, BF16: 2}
STEPS, COEF, NORM_EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
LR, MOM, WD = 1e-3, 0.95, 0.1


# ---------------------------------------------------------------- cases

def listed():
    return [
        # the hidden matrices of a tiny model: the cost of the calls is what counts
        dict(name="ortho_8x64x256_f32", op="ortho", count=8, rows=64, cols=256, pad=0, src=F32, dst=F32),
        # a few odd-sized matrices, taller than wide, cut from a wider tensor
        dict(name="ortho_3x777x300", op="ortho", count=3, rows=777, cols=300, pad=5, src=F32, dst=F32),
        # the square projections of a six-layer, 512-wide transformer
        dict(name="ortho_24x512x512_bf16", op="ortho", count=24, rows=512, cols=512, pad=0, src=BF16, dst=BF16),
        # one feed-forward matrix of each of 24 layers, 1024 wide
        dict(name="ortho_24x1024x4096_bf16", op="ortho", count=24, rows=1024, cols=4096, pad=0, src=BF16, dst=BF16),
        # a two-layer, 128-wide model's round, two workers
        dict(name="muon_2layer_w2", op="muon", layers=2, width=128, W=2, dtype=F32),
        # the matrices of a six-layer, 512-wide transformer, eight workers
        dict(name="muon_6layer_w8", op="muon", layers=6, width=512, W=8, dtype=F32),
        # the matrices of 24 layers, 1024 wide (BERT-large-shaped), four workers, bf16 gradients: the largest round
        dict(name="muon_24layer_w4", op="muon", layers=24, width=1024, W=4, dtype=BF16),
        # evaluation: losses of a batch of odd length over a 30522-word vocabulary
        dict(name="xent_loss_1000x30522x1024", op="xent", T=1000, V=30522, D=1024, grads=False),
        # a few tokens of a tiny model, training
        dict(name="xent_37x500x64", op="xent", T=37, V=500, D=64, grads=True),
        # a training step's loss over a 33278-word vocabulary, 512 wide
        dict(name="xent_2048x33278x512", op="xent", T=2048, V=33278, D=512, grads=True),
        # the largest training step: 8192 tokens, 30522 words, 1024 wide
        dict(name="xent_8192x30522x1024", op="xent", T=8192, V=30522, D=1024, grads=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _len(rng, lo, hi):
    """A length spread over the logarithm of its range: as drawn (mostly odd), or the next multiple of 64."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.5 else (n + 63) // 64 * 64


def draw(rng):
    op = rng.choice(["ortho", "muon", "xent"])
    if op == "ortho":
        rows, cols = _len(rng, 1, 4096), _len(rng, 16, 4096)
        count = _log(rng, 1, 32)
        while count * rows * cols * min(rows, cols) > 24 * 1024 * 4096 * 1024:
            count, rows = max(1, count // 2), rows // 2 + 1
        return dict(op=op, count=count, rows=rows, cols=cols, pad=rng.choice([0, 0, 8, 5]), src=rng.choice([F32, BF16]),
                    dst=rng.choice([F32, BF16]))
    if op == "muon":
        return dict(op=op, layers=rng.randint(1, 8), width=_len(rng, 32, 1024), W=rng.choice([1, 2, 3, 4, 8]),
                    dtype=rng.choice([F32, BF16]))
    T, V, D = _len(rng, 1, 8192), _len(rng, 100, 50000), 8 * _len(rng, 8, 256)
    D -= rng.choice([0, 0, 0, 3])                                   # (mostly whole vectors: a model's width is)
    while T * V * D > 8192 * 30522 * 1024:
        T = T // 2 + 1
    return dict(op=op, T=T, V=V, D=D, grads=rng.random() < 0.6)


def _shapes(case):
    """Groups (count, rows, cols) of a muon case's matrices: the projections and the two feed-forward ones per layer."""
    L, d = case["layers"], case["width"]
    return [(4 * L, d, d), (L, 4 * d, d), (L, d, 4 * d)]


def _scale(rows, cols):
    """The usual factor that gives an orthogonalised update the size of Adam's."""
    return 0.2 * math.sqrt(max(rows, cols))


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _gradients(shape, g):
    """Like a layer's gradients: a few strong directions, a decaying rest, noise."""
    *lead, m, n = shape
    r = max(1, min(m, n) // 16)
    rand = lambda *s: torch.randn(*lead, *s, device="cuda", generator=g)  # noqa: E731
    decay = torch.logspace(0, -2, r, device="cuda")
    return (rand(m, r) * decay) @ rand(r, n) * 1e-2 + rand(m, n) * 1e-2


def _inputs(case, seed):
    g = _gen(seed)
    if case["op"] == "ortho":
        x = torch.empty(case["count"], case["rows"], case["cols"] + case["pad"], device="cuda", dtype=DTYPE[case["src"]])
        for k in range(case["count"]):
            x[k] = _gradients((case["rows"], case["cols"] + case["pad"]), g)
        return dict(x=x[:, :, :case["cols"]])
    if case["op"] == "muon":
        grads, params = [], []
        for count, m, n in _shapes(case):
            t = torch.empty(case["W"], count, m, n, device="cuda", dtype=DTYPE[case["dtype"]])
            for w in range(case["W"]):
                for k in range(count):
                    t[w, k] = _gradients((m, n), g)
            grads.append(t)
            params.append(torch.randn(count, m, n, device="cuda", generator=g) * 0.02)
        return dict(grads=grads, params=params)
    T, V, D = case["T"], case["V"], case["D"]
    x = torch.randn(T, D, device="cuda", generator=g).to(torch.bfloat16)
    w = (torch.randn(V, D, device="cuda", generator=g) * (2.0 / math.sqrt(D))).to(torch.bfloat16)
    # frequent words more often, and a padded end of the batch
    u = torch.rand(T, device="cuda", generator=g)
    targets = (u * u * u * V).long().clamp(max=V - 1)
    targets[T - T // 16:] = -100
    return dict(x=x, w=w, targets=targets, valid=T - T // 16)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    {"ortho": _prepare_ortho, "muon": _prepare_muon, "xent": _prepare_xent}[case["op"]](s, case)
    return s


def _prepare_ortho(s, case):
    if not own:
        return
    from paper_2204_03211_b200 import binding as B
    s["out"] = torch.empty(case["count"], case["rows"], case["cols"], device="cuda", dtype=DTYPE[case["dst"]])
    s["ortho"] = B.Ortho(list(s["x"].unbind(0)), list(s["out"].unbind(0)))
    s["stream"] = torch.cuda.current_stream()


def _prepare_muon(s, case):
    if not own:
        s["p"] = s["params"]
        s["v"] = [torch.zeros_like(p) for p in s["p"]]
        return
    from paper_2204_03211_b200 import binding as B
    groups = _shapes(case)
    pad = lambda n: (4 * n + 255) // 256 * 256  # noqa: E731
    svc = B.Service(torch.cuda.current_device(), 1, sum(2 * c * pad(m * n) for c, m, n in groups))
    job = svc.register_job(opt=B.PS_MUON, grad_dtype=B.PS_F32 if case["dtype"] == F32 else B.PS_BF16,
                           num_workers=case["W"], lr=LR, momentum=MOM, weight_decay=WD)
    torch.cuda.synchronize()
    blocks, workers, ptrs, where, es = [], [], [], [], ESIZE[case["dtype"]]
    for (count, m, n), params, grads in zip(groups, s.pop("params"), s["grads"]):
        for k in range(count):
            b = len(where)
            svc.register_matrix(job, b, m, n, 0, params[k], _scale(m, n))
            where.append((m, n))
            for w in range(case["W"]):
                blocks.append(b)
                workers.append(w)
                ptrs.append(grads.data_ptr() + es * (w * count + k) * m * n)
    s["round"] = svc.round_prepare(np.full(len(blocks), job, np.int32), np.array(blocks, np.int32),
                                   np.array(workers, np.int32), np.array(ptrs, np.uint64),
                                   [(job, b) for b in range(len(where))])
    # an empty arena hands its ranges out one after the other: a group's blocks are one tensor of (parameters, momentum)
    s["svc"], s["master"], b = svc, [], 0
    for count, m, n in groups:
        sec = pad(m * n) // 4
        flat = svc.view(svc.pull(job, b), 2 * count * sec).view(count, 2, sec)
        s["master"].append((flat[:, 0, :m * n].view(count, m, n), flat[:, 1, :m * n].view(count, m, n)))
        b += count
    s["stream"] = torch.cuda.current_stream()


def _prepare_xent(s, case):
    s["scale"] = 1.0 / max(1, s["valid"])                           # mean over the tokens that count
    if not own:
        return
    from paper_2204_03211_b200 import binding as B
    T, V, D = case["T"], case["V"], case["D"]
    s["xent"] = B.CrossEntropy(T, V, D)
    s["loss"], s["lse"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    if case["grads"]:
        s["dx"] = torch.empty(T, D, device="cuda", dtype=torch.bfloat16)
        s["dw"] = torch.empty(V, D, device="cuda", dtype=torch.bfloat16)
    s["stream"] = torch.cuda.current_stream()


# ---------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    return (OWN if own else PLAIN)[op](state)


def _newton_schulz(u):
    """Five steps for a stack of matrices, in 32 bits."""
    tall = u.shape[-2] > u.shape[-1]
    x = u.transpose(-2, -1) if tall else u
    norm = x.double().square().sum((-2, -1), keepdim=True).sqrt() + NORM_EPS
    x = (x.double() / norm).float()
    a, b, c = COEF
    for _ in range(STEPS):
        g = x @ x.transpose(-2, -1)
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.transpose(-2, -1) if tall else x


def _plain_ortho(s):
    return _newton_schulz(s["x"].float()).to(DTYPE[s["case"]["dst"]]).contiguous()


def _plain_muon(s):
    out = []
    for p, v, grads in zip(s["p"], s["v"], s["grads"]):
        g = grads.sum(0, dtype=torch.float32)
        v.mul_(MOM).add_(g)
        o = _newton_schulz(g + MOM * v)
        p.mul_(1 - LR * WD).sub_(o, alpha=LR * _scale(*p.shape[1:]))
        out.append((p, v))
    return out


def _plain_xent(s):
    x, w, t = s["x"].float(), s["w"].float(), s["targets"]
    logits = x @ w.t()
    keep = t >= 0
    at = t.clamp(min=0)[:, None]
    lse = torch.where(keep, torch.logsumexp(logits, 1), 0.0)
    loss = torch.where(keep, lse - logits.gather(1, at)[:, 0], 0.0)
    if not s["case"]["grads"]:
        return dict(loss=loss, lse=lse)
    d = torch.exp(logits - lse[:, None])
    d.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
    d *= (keep * s["scale"])[:, None]
    return dict(loss=loss, lse=lse, dx=(d @ w).to(torch.bfloat16), dw=(d.t() @ x).to(torch.bfloat16))


def _own_ortho(s):
    s["ortho"].run(s["stream"])
    return s["out"]


def _own_muon(s):
    s["svc"].round_run(s["round"], s["stream"])
    return s["master"]


def _own_xent(s):
    s["xent"].forward(s["x"], s["w"], s["targets"], s["loss"], s["lse"], stream=s["stream"])
    if not s["case"]["grads"]:
        return dict(loss=s["loss"], lse=s["lse"])
    s["xent"].backward(s["x"], s["w"], s["targets"], s["lse"], s["dx"], s["dw"], scale=s["scale"], stream=s["stream"])
    return dict(loss=s["loss"], lse=s["lse"], dx=s["dx"], dw=s["dw"])


PLAIN = dict(ortho=_plain_ortho, muon=_plain_muon, xent=_plain_xent)
OWN = dict(ortho=_own_ortho, muon=_own_muon, xent=_own_xent)


# ---------------------------------------------------------------- what a pass cannot do without

def _ns_flops(rows, cols):
    m, n = min(rows, cols), max(rows, cols)
    return STEPS * (m * m * n + m ** 3 + 2 * m * m * n)             # two of the three products are symmetric


def work(case):
    if case["op"] == "ortho":
        n = case["count"] * case["rows"] * case["cols"]
        return dict(bytes=n * (ESIZE[case["src"]] + ESIZE[case["dst"]]),
                    flops=case["count"] * _ns_flops(case["rows"], case["cols"]))
    if case["op"] == "muon":
        n = sum(c * m * k for c, m, k in _shapes(case))
        return dict(bytes=n * (case["W"] * ESIZE[case["dtype"]] + 16),
                    flops=sum(c * _ns_flops(m, k) for c, m, k in _shapes(case)))
    T, V, D = case["T"], case["V"], case["D"]
    if not case["grads"]:
        return dict(bytes=2 * D * (T + V) + 16 * T, flops=2 * T * V * D)
    return dict(bytes=4 * D * (T + V) + 16 * T, flops=6 * T * V * D)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_ortho(u):
    """All five steps are polynomials in the Gram matrix, which commute: they are multiplied up on the smaller side and
    meet the matrix once."""
    u = u.double()
    m, n = u.shape[-2:]
    u = u / (torch.linalg.matrix_norm(u)[..., None, None] + NORM_EPS)
    t = torch.einsum("...ik,...jk->...ij", u, u) if m <= n else torch.einsum("...ki,...kj->...ij", u, u)
    eye = torch.eye(t.shape[-1], dtype=torch.float64, device=t.device)
    total = eye.expand_as(t)
    for _ in range(STEPS):
        q = COEF[0] * eye + COEF[1] * t + COEF[2] * torch.matmul(t, t)
        total = torch.matmul(q, total)
        t = torch.matmul(torch.matmul(q, t), q)
    return torch.matmul(total, u) if m <= n else torch.matmul(u, total)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "ortho":
        return torch.stack([_exact_ortho(x) for x in s["x"]])
    if case["op"] == "muon":
        f = lambda v: float(np.float32(v))  # noqa: E731
        out = []
        for p, grads in zip(s["params"], s["grads"]):
            v = torch.zeros(p.shape, device="cuda", dtype=torch.float64)
            for w in range(case["W"]):
                v += grads[w].double()
            o = torch.stack([_exact_ortho((1 + f(MOM)) * x) for x in v])
            out.append((p.double() * (1 - f(LR) * f(WD)) - f(LR) * f(_scale(*p.shape[1:])) * o, v))
        return out
    T, V = case["T"], case["V"]
    x, w, t = s["x"].double(), s["w"].double(), s["targets"].cpu().numpy()
    logits = torch.einsum("td,vd->tv", x, w)
    top = logits.max(1, keepdim=True).values
    e = torch.exp(logits - top)
    z = e.sum(1, keepdim=True)
    rows = torch.tensor(np.flatnonzero((t >= 0) & (t < V)), device="cuda")
    words = s["targets"][rows]
    lse, loss = torch.zeros(T, device="cuda", dtype=torch.float64), torch.zeros(T, device="cuda", dtype=torch.float64)
    lse[rows] = (top + torch.log(z))[rows, 0]
    loss[rows] = lse[rows] - logits[rows, words]
    if not case["grads"]:
        return dict(loss=loss, lse=lse)
    del logits
    p = torch.zeros_like(e)
    p[rows] = e[rows] / z[rows]
    p[rows, words] -= 1
    p /= max(1, len(rows))
    return dict(loss=loss, lse=lse, dx=torch.einsum("tv,vd->td", p, w), dw=torch.einsum("tv,td->vd", p, x))
