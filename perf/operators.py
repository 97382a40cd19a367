"""Cases for measuring the operators that a training job runs around the aggregation service.

Four operators, each in a plain form (elementary torch operations in 32 bits) and, where `own`
is true, through this package's entry points:

  aggregate  one round of a job whose gradients are clipped by their global norm: sum of the
             workers' shards, norm over all of the job's tensors, clipping factor, optimizer update
  clip       the same norm and factor on one worker's gradients, written to its push buffer
  quantize   microscaled 4-bit floating point (blocks of 32, E2M1 values, power-of-two scales)
             along the rows, along the columns or both
  product    activations quantised in the call times a kept 4-bit weight
  linear     a training step of a linear layer on 4-bit operands: output and both gradients

`listed()` and `draw()` give the cases, `prepare()` a case's inputs, `run()` one pass, `exact()`
what a pass returns computed in 64 bits, and `work()` the bytes and operations no pass can do without.
"""
import math
import random

import numpy as np
import torch

own = False

F32, BF16 = "f32", "bf16"
DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
ESIZE = {F32: 4, BF16: 2}
LR, MOM, WD, B1, B2, EPS = 1e-3, 0.9, 1e-4, 0.9, 0.999, 1e-8


# ---------------------------------------------------------------- cases

def listed():
    return [
        # a small model's round: 16 equal blocks, four workers; the cost of the calls is part of it
        dict(name="aggregate_16x64k_w4", op="aggregate", tensors="equal", blocks=16, largest=65536, W=4,
             dtype=F32, opt="sgd", max_norm=1.0),
        # a six-layer, 512-wide transformer with a 33278-word vocabulary, eight workers, fp32 gradients
        dict(name="aggregate_6layer_w8", op="aggregate", tensors="transformer", layers=6, width=512, vocab=33278,
             W=8, dtype=F32, opt="sgd", max_norm=1.0),
        # BERT-large-shaped tensors, bf16 gradients of four workers, Adam: the largest round
        dict(name="aggregate_24layer_adam", op="aggregate", tensors="transformer", layers=24, width=1024, vocab=30522,
             W=4, dtype=BF16, opt="adam", max_norm=1.0),
        # one worker's gradients of a tiny model
        dict(name="clip_2layer", op="clip", tensors="transformer", layers=2, width=64, vocab=500, src=F32, dst=F32,
             max_norm=1.0),
        # one worker's fp32 gradients of BERT-large-shaped tensors into its bf16 push buffer
        dict(name="clip_24layer_to_bf16", op="clip", tensors="transformer", layers=24, width=1024, vocab=30522,
             src=F32, dst=BF16, max_norm=1.0),
        # activations of a short prompt, rows of no whole number of blocks
        dict(name="quantize_19x1000", op="quantize", rows=19, cols=1000, pad=0, dtype=BF16, ways="rows"),
        # activations or output gradients of a training batch: both directions are needed
        dict(name="quantize_8192x4096_both", op="quantize", rows=8192, cols=4096, pad=0, dtype=BF16, ways="both"),
        # one token through a feed-forward weight
        dict(name="product_1x4096x1024", op="product", M=1, N=4096, K=1024),
        # a few sequences' next-token scores over a 30522-word vocabulary
        dict(name="product_37x30522x1024", op="product", M=37, N=30522, K=1024),
        # a batch of prompts through a square weight
        dict(name="product_8192x4096x4096", op="product", M=8192, N=4096, K=4096),
        # a small layer's training step on a ragged batch
        dict(name="linear_300x256x1000", op="linear", T=300, K=256, N=1000),
        # a feed-forward layer's training step on 8192 tokens
        dict(name="linear_8192x1024x4096", op="linear", T=8192, K=1024, N=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _len(rng, lo, hi):
    """A length spread over the logarithm of its range: as drawn (mostly odd), or the next multiple of 64."""
    n = _log(rng, lo, hi)
    n = n if rng.random() < 0.5 else (n + 63) // 64 * 64
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["aggregate", "aggregate", "clip", "clip", "quantize", "quantize", "product", "product", "linear"])
    if op in ("aggregate", "clip"):
        c = dict(op=op, tensors="ragged", blocks=_log(rng, 1, 300), largest=_log(rng, 1000, 1 << 23),
                 shape_seed=rng.randrange(1 << 30), max_norm=rng.choice([0.1, 1.0, 1e6]))
        c.update(dict(W=rng.choice([1, 2, 3, 4, 8, 16]), dtype=rng.choice([F32, BF16]), opt=rng.choice(["sgd", "adam"]))
                 if op == "aggregate" else dict(src=rng.choice([F32, BF16]), dst=rng.choice([F32, BF16])))
        while sum(_sizes(c)) > (1 << 27):
            c["largest"] //= 2
        return c
    if op == "quantize":
        rows, cols = _len(rng, 1, 16384), _len(rng, 32, 8192)
        while rows * cols > (1 << 25):
            rows = rows // 2 + 1
        return dict(op=op, rows=rows, cols=cols, pad=rng.choice([0, 0, 8, 33]), dtype=rng.choice([F32, BF16]),
                    ways=rng.choice(["rows", "columns", "both"]))
    if op == "product":
        M, N, K = _len(rng, 1, 8192), _len(rng, 64, 32768), _len(rng, 64, 8192)
        while M * N * K > (1 << 37):
            N = N // 2 + 1
        return dict(op=op, M=M, N=N, K=K)
    T, K, N = _len(rng, 32, 8192), _len(rng, 64, 4096), _len(rng, 64, 4096)
    while T * K * N > (1 << 35):
        T = T // 2 + 1
    return dict(op=op, T=T, K=K, N=N)


def _sizes(case):
    """Element counts of the tensors of a case."""
    if case["tensors"] == "equal":
        return [case["largest"]] * case["blocks"]
    if case["tensors"] == "ragged":
        r = random.Random(case["shape_seed"])
        return [_log(r, 1, max(2, case["largest"])) for _ in range(case["blocks"])]
    d = case["width"]
    layer = [d * d, d] * 4 + [d, d] + [4 * d * d, 4 * d, 4 * d * d, d] + [d, d]
    return [case["vocab"] * d, 512 * d, d, d] + layer * case["layers"] + [d * d, d]


def _padded(sizes):
    """Sizes in a flat buffer whose tensors start at multiples of 64 elements."""
    return [(n + 63) // 64 * 64 for n in sizes]


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _zero_gaps(flat, sizes):
    off = 0
    for n, m in zip(sizes, _padded(sizes)):
        if m > n:
            flat[..., off + n:off + m] = 0
        off += m


def _activations(rows, cols, dtype, g, pad=0):
    """Unit normal values with a few channels twenty times as large and a run of padded (zero) rows at the end."""
    x = torch.randn(rows, cols + pad, device="cuda", generator=g)
    x[:, ::97] *= 20
    x[rows - rows // 16:] = 0
    return x.to(DTYPE[dtype])[:, :cols]


def _inputs(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op == "aggregate":
        sizes = _sizes(case)
        total = sum(_padded(sizes))
        grads = torch.empty(case["W"], total, device="cuda", dtype=DTYPE[case["dtype"]])
        for w in range(case["W"]):
            grads[w] = torch.randn(total, device="cuda", generator=g) * 1e-2
        _zero_gaps(grads, sizes)
        params = torch.randn(total, device="cuda", generator=g) * 0.05
        _zero_gaps(params, sizes)
        return dict(sizes=sizes, grads=grads, params=params)
    if op == "clip":
        sizes = _sizes(case)
        grads = (torch.randn(sum(_padded(sizes)), device="cuda", generator=g) * 1e-2).to(DTYPE[case["src"]])
        _zero_gaps(grads, sizes)
        return dict(sizes=sizes, grads=grads)
    if op == "quantize":
        return dict(x=_activations(case["rows"], case["cols"], case["dtype"], g, case["pad"]))
    if op == "product":
        return dict(x=_activations(case["M"], case["K"], BF16, g),
                    w=torch.randn(case["N"], case["K"], device="cuda", generator=g) * 0.02)
    return dict(x=_activations(case["T"], case["K"], BF16, g),
                w=torch.randn(case["N"], case["K"], device="cuda", generator=g) * 0.02,
                dy=(torch.randn(case["T"], case["N"], device="cuda", generator=g) * 1e-3).to(torch.bfloat16))


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    {"aggregate": _prepare_aggregate, "clip": _prepare_clip, "quantize": _prepare_quantize,
     "product": _prepare_product, "linear": _prepare_linear}[case["op"]](s, case)
    return s


def _prepare_aggregate(s, case):
    """The master copy lies as the service lays a job's blocks out: per block parameters, then state."""
    sections = 2 if case["opt"] == "sgd" else 3
    sizes, pads = s["sizes"], _padded(s["sizes"])
    starts = np.concatenate([[0], np.cumsum(pads)])
    s["pads"], s["step"] = pads, 0
    if not own:
        s["master"] = torch.zeros(sections * int(starts[-1]), device="cuda")
        views = [[s["master"][sections * int(a) + k * m:][:m] for a, m in zip(starts, pads)] for k in range(sections)]
        s["p"], s["state"] = views[0], views[1:]
        for p, a, m in zip(s["p"], starts, pads):
            p.copy_(s.get("params")[int(a):int(a) + m])
        return
    from paper_2204_03211_b200 import binding as B
    svc = B.Service(torch.cuda.current_device(), 1, 4 * sections * int(starts[-1]))
    job = svc.register_job(opt=B.PS_SGD if case["opt"] == "sgd" else B.PS_ADAM,
                           grad_dtype=B.PS_F32 if case["dtype"] == F32 else B.PS_BF16, num_workers=case["W"],
                           lr=LR, momentum=MOM, weight_decay=WD, beta1=B1, beta2=B2, eps=EPS)
    torch.cuda.synchronize()
    for b, n in enumerate(sizes):
        svc.register_block(job, b, n, 0, s["params"][int(starts[b]):])
    nb, W = len(sizes), case["W"]
    grads, es = s["grads"], ESIZE[case["dtype"]]
    blocks = np.repeat(np.arange(nb, dtype=np.int32), W)
    workers = np.tile(np.arange(W, dtype=np.int32), nb)
    ptrs = (grads.data_ptr() + es * (workers.astype(np.int64) * grads.shape[1] + starts[blocks])).astype(np.uint64)
    s["round"] = svc.round_prepare(np.full(nb * W, job, np.int32), blocks, workers, ptrs, [(job, b) for b in range(nb)])
    # an empty arena hands its ranges out one after the other: the job's blocks are one tensor
    _, first, _ = svc.block_location(job, 0)
    _, last, section = svc.block_location(job, nb - 1)
    if last + sections * section - first != 4 * sections * int(starts[-1]):
        raise RuntimeError("the job's blocks are not neighbours in the arena")
    s["master"] = svc.view(svc.pull(job, 0), sections * int(starts[-1]))
    s["svc"], s["norm"] = svc, torch.zeros(1, device="cuda")
    s["stream"] = torch.cuda.current_stream()


def _prepare_clip(s, case):
    if not own:
        return
    from paper_2204_03211_b200 import binding as B
    pads = _padded(s["sizes"])
    s["out"] = torch.zeros(sum(pads), device="cuda", dtype=DTYPE[case["dst"]])
    split = lambda flat: [v[:n] for v, n in zip(torch.split(flat, pads), s["sizes"])]  # noqa: E731
    s["clip"] = B.Clip(split(s["grads"]), split(s["out"]))
    s["norm"], s["stream"] = torch.zeros(1, device="cuda"), torch.cuda.current_stream()


def _prepare_quantize(s, case):
    if not own:
        return
    from paper_2204_03211_b200 import binding as B
    R, C, ways = case["rows"], case["cols"], case["ways"]
    empty = lambda r, c: torch.empty(r, c, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    s["q"], s["rows"] = (B.MxTensor(R, C), empty(R, C)) if ways != "columns" else (None, None)
    s["qt"], s["columns"] = (B.MxTensor(C, R), empty(C, R)) if ways != "rows" else (None, None)
    s["stream"] = torch.cuda.current_stream()


def _prepare_product(s, case):
    """The weight is kept in its 4-bit form; the fp32 one is not needed again."""
    w = s.pop("w")
    if not own:
        s["wv"] = _mx_values(w)
        return
    from paper_2204_03211_b200 import binding as B
    s["stream"] = torch.cuda.current_stream()
    s["wq"] = B.MxTensor(case["N"], case["K"])
    B.ps_mx_quantize(w, s["wq"], stream=s["stream"])
    s["xq"] = B.MxTensor(case["M"], case["K"])
    s["y"] = torch.empty(case["M"], case["N"], device="cuda", dtype=torch.bfloat16)


def _prepare_linear(s, case):
    if not own:
        return
    from paper_2204_03211_b200 import binding as B
    T, K, N = case["T"], case["K"], case["N"]
    for name, r, c in (("x", T, K), ("w", N, K), ("dy", T, N)):
        s[name + "_q"], s[name + "_qt"] = B.MxTensor(r, c), B.MxTensor(c, r)
    for name, r, c in (("y", T, N), ("dx", T, K), ("dw", N, K)):
        s[name] = torch.empty(r, c, device="cuda", dtype=torch.bfloat16)
    s["stream"] = torch.cuda.current_stream()


# ---------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    return (OWN if own else PLAIN)[op](state)


def _pow2(e):
    """2^e in 32 bits for whole e in [-127, 127], from its bits: torch.ldexp goes through pow, which rounds."""
    return torch.where(e == -127, 2.0 ** -127, ((e + 127) << 23).view(torch.float32))


def _mx_values(x):
    """The values that microscaled 4-bit floating point gives x, blocks of 32 along the last dimension, in 32 bits."""
    x = x.float()
    rows, cols = x.shape
    b = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    amax = b.abs().amax(-1, keepdim=True)
    # the scale puts the block's largest magnitude in [4, 8), above which E2M1 saturates at 6
    e = (torch.frexp(amax).exponent - 3).clamp(-127, 127)
    e = torch.where(amax > 0, e, torch.full_like(e, -127))
    a = b * _pow2(-e)
    mag = a.abs()
    step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
    q = ((mag / step).round() * step).clamp(max=6.0).copysign(a)
    v = torch.where(torch.isfinite(amax), q * _pow2(e), torch.nan)
    return v.view(rows, -1)[:, :cols]


def _factor(norm, max_norm):
    return torch.clamp(max_norm / (norm + 1e-6), max=1.0)


def _plain_aggregate(s):
    case = s["case"]
    s["step"] += 1
    G = s["grads"].sum(0, dtype=torch.float32)
    norm = (G * G).sum().sqrt()
    d = torch.split(G * _factor(norm, case["max_norm"]), s["pads"])
    d = torch._foreach_add(d, s["p"], alpha=WD)
    if case["opt"] == "sgd":
        torch._foreach_mul_(s["state"][0], MOM)
        torch._foreach_add_(s["state"][0], d)
        torch._foreach_add_(s["p"], s["state"][0], alpha=-LR)
    else:
        m, v = s["state"]
        torch._foreach_mul_(m, B1)
        torch._foreach_add_(m, d, alpha=1 - B1)
        torch._foreach_mul_(v, B2)
        torch._foreach_add_(v, torch._foreach_mul(torch._foreach_mul(d, d), 1 - B2))
        den = torch._foreach_sqrt(v)
        torch._foreach_div_(den, math.sqrt(1 - B2 ** s["step"]))
        torch._foreach_add_(den, EPS)
        torch._foreach_add_(s["p"], torch._foreach_div(m, den), alpha=-LR / (1 - B1 ** s["step"]))
    return dict(master=s["master"], norm=norm.view(1))


def _plain_clip(s):
    g = s["grads"].float()
    norm = (g * g).sum().sqrt()
    return dict(out=(g * _factor(norm, s["case"]["max_norm"])).to(DTYPE[s["case"]["dst"]]), norm=norm.view(1))


def _plain_quantize(s):
    ways, out = s["case"]["ways"], {}
    if ways != "columns":
        out["rows"] = _mx_values(s["x"]).to(torch.bfloat16)
    if ways != "rows":
        out["columns"] = _mx_values(s["x"].t()).to(torch.bfloat16)
    return out


def _plain_product(s):
    return (_mx_values(s["x"]) @ s["wv"].t()).to(torch.bfloat16)


def _plain_linear(s):
    x, w, dy = s["x"], s["w"], s["dy"]
    y = _mx_values(x) @ _mx_values(w).t()
    dx = _mx_values(dy) @ _mx_values(w.t()).t()
    dw = _mx_values(dy.t()) @ _mx_values(x.t()).t()
    return dict(y=y.to(torch.bfloat16), dx=dx.to(torch.bfloat16), dw=dw.to(torch.bfloat16))


def _own_aggregate(s):
    s["svc"].round_run_clipped(s["round"], s["case"]["max_norm"], s["norm"], s["stream"])
    return dict(master=s["master"], norm=s["norm"])


def _own_clip(s):
    s["clip"].run(s["case"]["max_norm"], s["norm"], s["stream"])
    return dict(out=s["out"], norm=s["norm"])


def _own_quantize(s):
    from paper_2204_03211_b200 import binding as B
    stream, out = s["stream"], {}
    B.ps_mx_quantize(s["x"], s["q"], s["qt"], stream)
    if s["q"] is not None:
        out["rows"] = B.ps_mx_dequantize(s["q"], s["rows"], stream)
    if s["qt"] is not None:
        out["columns"] = B.ps_mx_dequantize(s["qt"], s["columns"], stream)
    return out


def _own_product(s):
    from paper_2204_03211_b200 import binding as B
    B.ps_mx_quantize(s["x"], s["xq"], stream=s["stream"])
    return B.ps_mx_matmul(s["xq"], s["wq"], s["y"], s["stream"])


def _own_linear(s):
    from paper_2204_03211_b200 import binding as B
    st = s["stream"]
    B.ps_mx_quantize(s["x"], s["x_q"], s["x_qt"], st)
    B.ps_mx_quantize(s["w"], s["w_q"], s["w_qt"], st)
    B.ps_mx_matmul(s["x_q"], s["w_q"], s["y"], st)
    B.ps_mx_quantize(s["dy"], s["dy_q"], s["dy_qt"], st)
    B.ps_mx_matmul(s["dy_q"], s["w_qt"], s["dx"], st)
    B.ps_mx_matmul(s["dy_qt"], s["x_qt"], s["dw"], st)
    return dict(y=s["y"], dx=s["dx"], dw=s["dw"])


PLAIN = dict(aggregate=_plain_aggregate, clip=_plain_clip, quantize=_plain_quantize, product=_plain_product,
             linear=_plain_linear)
OWN = dict(aggregate=_own_aggregate, clip=_own_clip, quantize=_own_quantize, product=_own_product, linear=_own_linear)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "aggregate":
        n, states = sum(_sizes(case)), 1 if case["opt"] == "sgd" else 2
        return dict(bytes=n * (case["W"] * ESIZE[case["dtype"]] + 8 * (1 + states)),
                    flops=n * (case["W"] + 3 + (6 if states == 1 else 16)))
    if op == "clip":
        n = sum(_sizes(case))
        return dict(bytes=n * (ESIZE[case["src"]] + ESIZE[case["dst"]]), flops=3 * n)
    if op == "quantize":
        n, ways = case["rows"] * case["cols"], 2 if case["ways"] == "both" else 1
        return dict(bytes=n * (ESIZE[case["dtype"]] + 2 * ways), flops=4 * n * ways)
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return dict(bytes=2 * M * K + N * K * 17 / 32 + 2 * M * N, flops=2 * M * N * K)
    T, K, N = case["T"], case["K"], case["N"]
    return dict(bytes=2 * T * K + 4 * N * K + 2 * T * N + 2 * (T * N + T * K + N * K), flops=6 * T * K * N)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_round(case, s):
    sizes, pads = s["sizes"], _padded(s["sizes"])
    G = torch.zeros(s["grads"].shape[1], device="cuda", dtype=torch.float64)
    for w in range(case["W"]):
        G += s["grads"][w].double()
    norm = float(torch.sqrt(torch.sum(G ** 2)))
    f = np.float32
    lr, mom, wd, b1, b2 = (float(f(v)) for v in (LR, MOM, WD, B1, B2))
    p = s["params"].double()
    d = min(1.0, case["max_norm"] / (norm + 1e-6)) * G + wd * p
    if case["opt"] == "sgd":
        parts = [p - lr * d, d]
    else:
        m, v = (1 - b1) * d, (1 - b2) * d * d
        parts = [p - lr / (1 - b1) * m / (torch.sqrt(v) / math.sqrt(1 - b2) + float(f(EPS))), m, v]
    rows, off = [], 0
    for m in pads:
        rows += [q[off:off + m] for q in parts]
        off += m
    return dict(master=torch.cat(rows), norm=torch.tensor([norm], dtype=torch.float64))


def _exact_mx(x):
    """Nearest of the 4-bit values at the block's scale, in 64 bits: distances to all eight magnitudes, ties to the
    even code."""
    x = x.double()
    R, C = x.shape
    full = torch.zeros(R, (C + 31) // 32 * 32, device=x.device, dtype=torch.float64)
    full[:, :C] = x
    b = full.reshape(-1, 32)
    top = b.abs().max(1).values
    # the largest power of two that is at most the block's largest magnitude, from a table of exact ones
    powers = torch.tensor([2.0 ** k for k in range(-125, 129)], dtype=torch.float64, device=x.device)
    at = torch.searchsorted(powers, top.contiguous(), right=True) - 1
    scale = (powers[at.clamp(min=0)] / 4)[:, None]
    mags = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
    a = b.abs() / scale
    best, gap = torch.zeros_like(a), a.clone()
    for code in range(1, 8):
        g = (a - mags[code]).abs()
        take = (g < gap) | ((g == gap) & (code % 2 == 0))
        best = torch.where(take, mags[code], best)
        gap = torch.where(take, g, gap)
    return (torch.sign(b) * best * scale).reshape(R, -1)[:, :C]


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "aggregate":
        return _exact_round(case, s)
    if op == "clip":
        g = s["grads"].double()
        norm = float(torch.sqrt(torch.sum(g ** 2)))
        return dict(out=g * min(1.0, case["max_norm"] / (norm + 1e-6)), norm=torch.tensor([norm], dtype=torch.float64))
    if op == "quantize":
        out = {}
        if case["ways"] != "columns":
            out["rows"] = _exact_mx(s["x"])
        if case["ways"] != "rows":
            out["columns"] = _exact_mx(s["x"].t())
        return out
    if op == "product":
        return _exact_mx(s["x"]) @ _exact_mx(s["w"]).t()
    x, w, dy = s["x"], s["w"], s["dy"]
    return dict(y=_exact_mx(x) @ _exact_mx(w).t(), dx=_exact_mx(dy) @ _exact_mx(w.t()).t(),
                dw=_exact_mx(dy.t()) @ _exact_mx(x.t()).t())
