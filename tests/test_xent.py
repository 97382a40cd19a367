"""Cross entropy over a vocabulary (ps_xent_*): losses, log-sum-exps and both gradients against the formula in 64 bits,
the gradients also against differences of the 64-bit loss.

Tolerances, per element.  x and w are bf16 and their products exact; a score is a sum of D of them in binary32, off by at
most ds = 2 D 2^-24 (|x| |w|), each addition by a unit in the last place.  lse and loss carry the largest ds of their
row, the additions of V exponentials (each 2^-22 of its value) and roundings of lse: dl = max ds + (V / 64 + 16) 2^-23 +
2^-22 |lse|.  An entry p - [v = target] is off by p (ds + dl + 2^-21) before it is rounded to bf16 (2^-8 of it); sums over
n such entries add n 2^-23 of the sum of magnitudes, and the result is rounded once more."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2204_03211_b200 import binding as B

gpu = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def inputs(T, V, D, pad=0, seed=0, ignored=0.1, bits=64, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, D + pad, generator=g).to(BF).cuda()[:, :D]
    w = (torch.randn(V, D + pad, generator=g) * (spread / D ** 0.5)).to(BF).cuda()[:, :D]
    t = torch.randint(0, V, (T,), generator=g)
    t[torch.rand(T, generator=g) < ignored] = -100
    return x, w, t.to(torch.int64 if bits == 64 else torch.int32).cuda()


def formula(x, w, t, g):
    """loss, lse, dx, dw in 64 bits, and their tolerances (before the results' own rounding)."""
    x, w, t = x.double(), w.double(), t.long()
    T, V, D = x.shape[0], w.shape[0], x.shape[1]
    keep = (t >= 0) & (t < V)
    x = torch.where(keep[:, None], x, 0.0)                  # whatever an ignored row holds
    g = torch.where(keep, g.double(), 0.0)
    s = x @ w.t()
    ds = 2 * D * 2.0 ** -24 * (x.abs() @ w.abs().t())
    lse = torch.logsumexp(s, 1)
    dl = ds.max(1).values + (V / 64 + 16) * 2.0 ** -23 + 2.0 ** -22 * lse.abs()
    at = torch.where(keep, t, 0)[:, None]
    score = s.gather(1, at)[:, 0]
    p = torch.exp(s - lse[:, None])
    e = p.clone()
    e[torch.arange(T), at[:, 0]] -= 1
    de = p * (ds + dl[:, None] + 2.0 ** -21) * 1.01 + 2.0 ** -8 * e.abs()
    eg, deg = e * g[:, None], de * g.abs()[:, None]
    big = eg.abs() + deg
    zero = torch.zeros_like(lse)
    return dict(loss=torch.where(keep, lse - score, zero), lse=torch.where(keep, lse, zero),
                dx=eg @ w, dw=eg.t() @ x), \
        dict(loss=torch.where(keep, 2 * dl + 2.0 ** -23 * score.abs(), zero), lse=torch.where(keep, dl, zero),
             dx=deg @ w.abs() + V * 2.0 ** -23 * (big @ w.abs()), dw=deg.t() @ x.abs() + T * 2.0 ** -23 * (big.t() @ x.abs()))


def check(got, ref, tol, dtype=F32):
    u = torch.finfo(dtype).eps / 2
    off = (got.double() - ref).abs()
    allowed = tol + u * (ref.abs() + tol) + 1e-37
    assert torch.isfinite(got).all()
    assert bool((off <= allowed).all()), "off by up to %.3g of what is allowed" % float((off / allowed).max())


def run(T, V, D, pad=0, seed=0, bits=64, dw_dtype=BF, token_scale=False, scale=1.0, ignored=0.1, made_for=None):
    x, w, t = inputs(T, V, D, pad, seed, ignored, bits)
    ce = B.CrossEntropy(made_for or T, V, D, aligned=(D + pad) % 8 == 0)
    ts = None
    if token_scale:
        ts = torch.rand(T, generator=torch.Generator().manual_seed(7)).cuda() + 0.25
        ts[t < 0] = float("nan")                            # what ignored tokens hold does not matter
    loss, lse = ce.forward(x, w, t)
    dx = torch.full((T, D), 7.0, device="cuda", dtype=BF)
    dw = torch.full((V, D), 7.0, device="cuda", dtype=dw_dtype)
    ce.backward(x, w, t, lse, dx, dw, scale=scale, token_scale=ts)
    torch.cuda.synchronize()
    assert B.ps_xent_status() == 0
    f = np.float32(scale)
    ref, tol = formula(x, w, t, torch.full((T,), float(f), dtype=torch.float64, device="cuda") * (1 if ts is None else ts.double()))
    if ts is not None:                                      # for dw the factor is rounded into x: one more bf16 rounding
        tol["dw"] = tol["dw"] + 2.0 ** -8 * (formula(x, w, t, torch.where(t < 0, 0, f * ts).double().abs())[1]["dw"] * 2 ** 8)
    check(loss, ref["loss"], tol["loss"])
    check(lse, ref["lse"], tol["lse"])
    check(dx, ref["dx"], tol["dx"] * (1 + 2.0 ** -22) + 2.0 ** -22 * ref["dx"].abs(), BF)
    check(dw, ref["dw"], tol["dw"] * (1 + 2.0 ** -22) + 2.0 ** -22 * ref["dw"].abs(), dw_dtype)
    return loss, lse, dx, dw


SHAPES = [(1, 1, 1), (1, 2, 8), (3, 1, 5), (1, 1000, 64), (37, 500, 64), (128, 128, 64), (256, 256, 256), (257, 257, 257),
          (300, 1111, 96), (129, 4097, 72), (1000, 300, 40), (64, 8320, 512), (700, 2500, 264)]


@gpu
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_losses_and_gradients(T, V, D):
    run(T, V, D)


@gpu
@pytest.mark.parametrize("kw", [dict(bits=32), dict(dw_dtype=F32), dict(token_scale=True), dict(pad=8), dict(pad=3),
                                dict(pad=3, token_scale=True, dw_dtype=F32), dict(scale=1 / 7), dict(ignored=1.0),
                                dict(ignored=0.0), dict(made_for=4000), dict(scale=0.0)])
def test_variants(kw):
    run(301, 1500, 104, **kw)


@gpu
@pytest.mark.parametrize("T,V,D", [(5000, 7000, 64), (20000, 1500, 64)])
def test_several_pieces_of_the_vocabulary(T, V, D):
    """More entries than one piece of d holds: several launches, dx added up over them."""
    run(T, V, D, scale=1 / T)


@gpu
def test_few_tokens_many_words_share_out_the_vocabulary():
    run(40, 40000, 128)


@gpu
@pytest.mark.parametrize("T,V,D,kw", [(6000, 250, 72, {}), (3000, 100, 40, dict(dw_dtype=F32)), (2100, 300, 37, {}),
                                      (2500, 64, 24, dict(made_for=9000, pad=3, token_scale=True)), (1100, 1, 8, {})])
def test_many_tokens_few_words_share_out_the_tokens(T, V, D, kw):
    run(T, V, D, **kw)


@gpu
@pytest.mark.parametrize("dw_dtype", [BF, F32])
@pytest.mark.parametrize("D", [1, 8, 24, 33, 36, 40, 62, 264])
def test_rows_of_results_on_any_boundary(D, dw_dtype):
    """Results are stored 32 bytes, 16 bytes or an element at a time, the last along the rows."""
    run(270, 300, D, dw_dtype=dw_dtype)


@gpu
@pytest.mark.parametrize("T,V,D", [(70, 300, 767), (300, 700, 768), (33, 130, 1000), (600, 1, 1030)])
def test_widths_around_the_change_of_warps(T, V, D):
    """From 768 on eight warps read a tile's sums, below sixteen."""
    run(T, V, D)


@gpu
def test_gradient_against_differences():
    """Directional derivatives of the 64-bit loss, by central differences in 64 bits."""
    T, V, D = 50, 300, 48
    x, w, t = inputs(T, V, D, ignored=0.2)
    ce = B.CrossEntropy(T, V, D)
    _, lse = ce.forward(x, w, t)
    dx, dw = torch.empty(T, D, device="cuda", dtype=BF), torch.empty(V, D, device="cuda", dtype=F32)
    ce.backward(x, w, t, lse, dx, dw)

    def total(x, w):
        s = x @ w.t()
        keep = t >= 0
        return (torch.logsumexp(s, 1) - s.gather(1, t.clamp(min=0)[:, None])[:, 0])[keep].sum()

    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        a = torch.randn(T, D, device="cuda", generator=g, dtype=torch.float64)
        b = torch.randn(V, D, device="cuda", generator=g, dtype=torch.float64)
        h = 1e-5
        for da, db, got, ref in ((a, 0 * b, dx, a), (0 * a, b, dw, b)):
            slope = (total(x.double() + h * da, w.double() + h * db) - total(x.double() - h * da, w.double() - h * db)) / (2 * h)
            mine = (got.double() * ref).sum()
            # each entry of a gradient is off by at most two bf16 roundings of magnitudes no larger than these
            allowed = 2.0 ** -7 * ((got.double() * ref).abs().sum() + (ref.abs().sum(0) * got.double().abs().amax(0)).sum() / T) + 1e-4
            assert abs(float(slope - mine)) <= float(allowed)


@gpu
def test_what_ignored_rows_hold_does_not_matter():
    T, V, D = 200, 700, 64
    x, w, t = inputs(T, V, D, ignored=0.3)
    t[3], t[4] = V, 2 ** 40                                 # past the vocabulary: ignored too
    dirty = x.clone()
    dirty[~((t >= 0) & (t < V))] = float("nan")
    dirty[t == -100] = float("inf")
    ce = B.CrossEntropy(T, V, D)
    outs = []
    for z in (x, dirty):
        loss, lse = ce.forward(z, w, t)
        dx, dw = torch.empty(T, D, device="cuda", dtype=BF), torch.empty(V, D, device="cuda", dtype=BF)
        ce.backward(z, w, t, lse, dx, dw, scale=0.25)
        outs.append((loss, lse, dx, dw))
    for a, b in zip(*outs):
        assert torch.isfinite(a).all() and torch.equal(a, b)
    gone = ~((t >= 0) & (t < V))
    assert gone[3] and gone[4]
    for z in outs[0][:3]:
        assert not z[gone].any()


@gpu
@pytest.mark.parametrize("T,V,D", [(200, 700, 64), (300, 700, 37), (40, 40000, 128), (40, 40000, 77), (5000, 7000, 64)])
def test_what_w_holds_does_not_reach_ignored_rows(T, V, D):
    """One slice, many, several pieces; results along the rows and not.  An infinity or a NaN in w makes NaNs of every
    other token's gradient."""
    x, w, t = inputs(T, V, D, ignored=0.3)
    w[7, 0], w[V - 1, D - 1] = float("inf"), float("nan")
    gone = t < 0
    ce = B.CrossEntropy(T, V, D)
    loss, lse = ce.forward(x, w, t)
    ts = torch.where(gone, float("nan"), 0.5)
    dx = torch.full((T, D), 7.0, device="cuda", dtype=BF)
    ce.backward(x, w, t, lse, dx, None, scale=0.25, token_scale=ts)
    assert gone.any() and not gone.all()
    for z in (loss, lse, dx):
        assert bool((z[gone] == 0).all())
    assert dx[~gone].isnan().any(1).all()


@gpu
def test_nan_and_infinities_stay_in_their_rows():
    T, V, D = 70, 600, 64
    x, w, t = inputs(T, V, D, ignored=0.0)
    x[5, 3] = float("nan")
    x[6] = 0
    x[6, 0] = float("inf")                                  # scores of both infinities, and NaN where w is zero
    ce = B.CrossEntropy(T, V, D)
    loss, lse = ce.forward(x, w, t)
    dx, dw = torch.empty(T, D, device="cuda", dtype=BF), torch.empty(V, D, device="cuda", dtype=BF)
    ce.backward(x, w, t, lse, dx, dw)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[5] = bad[6] = True
    assert loss[bad].isnan().all() and torch.isfinite(loss[~bad]).all()
    assert dx[bad].isnan().any(1).all() and torch.isfinite(dx[~bad]).all()
    assert dw.isnan().any()                                 # (the sum over all tokens)


@gpu
def test_large_scores():
    """Scores in the thousands: exponentials by differences from the row's maximum, at either end of the vocabulary."""
    T, V, D = 33, 1000, 64
    x, w, t = inputs(T, V, D, ignored=0.0, spread=400.0)
    x[0], t[0] = 0, 5                                       # all scores equal
    t[1], t[2] = 0, V - 1
    ce = B.CrossEntropy(T, V, D)
    loss, lse = ce.forward(x, w, t)
    ref, tol = formula(x, w, t, torch.ones(T, device="cuda", dtype=torch.float64))
    check(loss, ref["loss"], tol["loss"])
    check(lse, ref["lse"], tol["lse"])


@gpu
@pytest.mark.parametrize("T,V,D", [(70_000, 300, 32_768), (300, 70_000, 32_768)])
def test_offsets_past_2_31(T, V, D):
    """Operands and results of 2.3 G elements: rows at both ends and around the 2^31st element against the formula."""
    x = torch.empty(T, D, device="cuda", dtype=BF)
    w = torch.empty(V, D, device="cuda", dtype=BF)
    g = torch.Generator(device="cuda").manual_seed(2)
    for m in (x, w):
        for r in range(0, m.shape[0], 4096):
            m[r:r + 4096] = torch.randn(m[r:r + 4096].shape, device="cuda", generator=g)
    w *= 0.01
    t = torch.randint(0, V, (T,), device="cuda", generator=g)
    ce = B.CrossEntropy(T, V, D)
    loss, lse = ce.forward(x, w, t)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ce.backward(x, w, t, lse, dx, dw)
    torch.cuda.synchronize()
    assert B.ps_xent_status() == 0
    edge = 2 ** 31 // D
    rows = [r for r in (0, 1, edge - 1, edge, edge + 1, T - 1) if r < T]
    words = [v for v in (0, edge - 1, edge, edge + 1, V - 1) if v < V]

    def scores(rs):                                         # in 64 bits, a part of the width at a time
        return sum(x[rs, c:c + 2048].double() @ w[:, c:c + 2048].double().t() for c in range(0, D, 2048))

    for r in rows:
        s = scores([r])[0]
        l = torch.logsumexp(s, 0)
        ds = 2 * D * 2.0 ** -24 * float((x[r].double().abs()[None] @ w[:1000].double().abs().t()).max()) * 4
        assert abs(float(lse[r]) - float(l)) <= ds + 1e-5
        assert abs(float(loss[r]) - float(l - s[t[r]])) <= 2 * ds + 1e-5
        e = torch.exp(s - l)
        e[t[r]] -= 1
        cols = [0, 5, D - 1]
        ref = e @ w[:, cols].double()
        tol = 2.0 ** -8 * (e.abs() @ w[:, cols].double().abs()) + 2.0 ** -8 * ref.abs() + ds
        assert bool(((dx[r, cols].double() - ref).abs() <= tol).all())
    if T <= 1000:                                           # (dw needs the scores of all tokens)
        s = scores(list(range(T)))
        e = torch.exp(s - torch.logsumexp(s, 1)[:, None])
        e[torch.arange(T), t] -= 1
    else:
        e = torch.cat([(lambda s: torch.exp(s - torch.logsumexp(s, 1)[:, None]))(scores(list(range(a, min(T, a + 5000)))))
                       for a in range(0, T, 5000)])
        e[torch.arange(T), t] -= 1
    cols = [0, 5, D - 1]
    ref = e[:, words].t() @ x[:, cols].double()
    tol = 2.0 ** -7 * (e[:, words].abs().t() @ x[:, cols].double().abs()) + 2.0 ** -8 * ref.abs()
    assert bool(((dw[words][:, cols].double() - ref).abs() <= tol).all())


@gpu
def test_no_tokens():
    ce = B.CrossEntropy(0, 90, 24)
    x, w = torch.empty(0, 24, device="cuda", dtype=BF), torch.randn(90, 24, device="cuda").to(BF)
    t = torch.empty(0, device="cuda", dtype=torch.int64)
    loss, lse = ce.forward(x, w, t)
    assert loss.numel() == lse.numel() == 0
    for dtype in (BF, F32):
        dw = torch.full((90, 30), 3.0, device="cuda", dtype=dtype)
        ce.backward(x, w, t, lse, torch.empty(0, 24, device="cuda", dtype=BF), dw[:, :24])
        assert not dw[:, :24].any() and bool((dw[:, 24:] == 3).all())


@gpu
def test_results_in_wider_rows_one_gradient_and_the_same_every_time():
    T, V, D = 150, 900, 72
    x, w, t = inputs(T, V, D)
    _, lse, dx0, dw0 = run(T, V, D)
    ce = B.CrossEntropy(T, V, D)
    for pad in (8, 5, 40):
        dx = torch.full((T, D + pad), 7.0, device="cuda", dtype=BF)
        dw = torch.full((V, D + pad), 7.0, device="cuda", dtype=BF)
        ce.backward(x, w, t, lse, dx[:, :D], dw[:, :D])
        assert torch.equal(dx[:, :D], dx0) and torch.equal(dw[:, :D], dw0)
        assert bool((dx[:, D:] == 7).all()) and bool((dw[:, D:] == 7).all())
    dx, dw = torch.empty_like(dx0), torch.empty_like(dw0)
    ce.backward(x, w, t, lse, dx=dx)
    ce.backward(x, w, t, lse, dw=dw)
    assert torch.equal(dx, dx0) and torch.equal(dw, dw0)


@gpu
def test_on_another_stream_and_captured():
    T, V, D = 300, 1000, 64
    ce = B.CrossEntropy(T, V, D)
    x, w, t = inputs(T, V, D)
    ref = run(T, V, D)
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dx, dw = torch.empty(T, D, device="cuda", dtype=BF), torch.empty(V, D, device="cuda", dtype=BF)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def step(s):
        ce.forward(x, w, t, loss, lse, stream=s)
        ce.backward(x, w, t, lse, dx, dw, stream=s)

    step(stream)
    stream.synchronize()
    for a, b in zip((loss, lse, dx, dw), ref):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    x2, w2, t2 = inputs(T, V, D, seed=9)
    x.copy_(x2), w.copy_(w2), t.copy_(t2)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((loss, lse, dx, dw), run(T, V, D, seed=9)):
        assert torch.equal(a, b)


def on_a_busy_stream(stream, call, fill, ms=200):
    """`call` behind work that keeps `stream` busy; then the current stream writes over `fill` bytes of freed memory, many
    times, in allocations of every size that could be served from what `call` released."""
    for busy in (0, ms):                                    # (first without: a kernel's first launch may wait for the device)
        with torch.cuda.stream(stream):
            torch.cuda._sleep(int(busy * 1.9e6) + 1)
        made = call()
        held = []
        for n in fill:
            held += [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        if busy == 0:
            del held, made[:]
            torch.cuda.synchronize()
    torch.cuda.current_stream().synchronize()
    assert not stream.query()                               # (it was busy all the while)
    stream.synchronize()


@gpu
@pytest.mark.parametrize("kind", ["torch", "number"])
@pytest.mark.parametrize("T,V,D", [(300, 5000, 64), (300, 5000, 61)])
def test_dropped_and_fresh_results_while_the_calls_wait(kind, T, V, D):
    """An object dropped right after its calls on another stream, results of its own making, and results dropped at once:
    none of their memory is the current stream's before the calls are done."""
    x, w, t = inputs(T, V, D)
    ref = run(T, V, D)
    stream = torch.cuda.Stream()
    given = stream if kind == "torch" else stream.cuda_stream
    dx, dw = torch.empty(T, D, device="cuda", dtype=BF), torch.empty(V, D, device="cuda", dtype=BF)
    torch.cuda.synchronize()
    out = []

    def call():
        junk = torch.full((B.ps_xent_sizes(T, V, D)[1],), 3, dtype=torch.uint8, device="cuda")
        torch.cuda._sleep(2_000_000)
        junk.fill_(9)                                       # (still to run when the workspace takes the memory over)
        del junk
        ce = B.CrossEntropy(T, V, D)
        loss, lse = ce.forward(x, w, t, stream=given)
        ce.backward(x, w, t, lse, dx, dw, stream=given)
        gone = ce.forward(x, w, t, stream=given)
        out.extend((loss, lse, dx, dw))
        if kind == "torch":
            del ce, gone
        else:
            out.append((ce, gone))                          # (dropping it waits, which is looked at below)
        return out

    on_a_busy_stream(stream, call, (T * 4, 1 << 20, *B.ps_xent_sizes(T, V, D)))
    for a, b in zip(out[:4], ref):
        assert torch.equal(a, b)
    if kind == "number":
        ce, _ = out.pop()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(20_000_000)
        ce.forward(x, w, t, stream=given)
        del ce, _
        assert stream.query()


@gpu
def test_made_inside_a_capture():
    """Workspace and results from the graph's memory; afterwards the object serves calls outside the graph as well."""
    T, V, D = 300, 1000, 64
    x, w, t = inputs(T, V, D)
    ref = run(T, V, D)
    dx, dw = torch.empty(T, D, device="cuda", dtype=BF), torch.empty(V, D, device="cuda", dtype=BF)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ce = B.CrossEntropy(T, V, D)
        stream = torch.cuda.current_stream()
        loss, lse = ce.forward(x, w, t, stream=stream)
        ce.backward(x, w, t, lse, dx, dw, stream=stream)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((loss, lse, dx, dw), ref):
        assert torch.equal(a, b)
    for other in (None, torch.cuda.Stream()):
        again = ce.forward(x, w, t, stream=other)
        torch.cuda.synchronize()
        assert torch.equal(again[0], ref[0]) and torch.equal(again[1], ref[1])


@gpu
def test_results_made_on_the_default_stream_beside_a_current_one():
    """No stream given is the default one, whatever is current."""
    T, V, D = 200, 700, 64
    x, w, t = inputs(T, V, D)
    ref = run(T, V, D)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        ce = B.CrossEntropy(T, V, D)
        loss, lse = ce.forward(x, w, t)
        torch.cuda.default_stream().synchronize()
        assert torch.equal(loss, ref[0]) and torch.equal(lse, ref[1])


def test_device_zero_is_a_device(monkeypatch):
    """Given as 0 it is GPU 0, whatever is current; not given it is the current one."""
    asked = []
    B.CrossEntropy, B.MxTensor                              # (loads the extension)

    class Asked(Exception):
        pass

    def empty(*a, device=None, **kw):
        asked.append(device)
        raise Asked

    monkeypatch.setattr(torch, "empty", empty)
    for make in (lambda d: B.CrossEntropy(10, 20, 8, d), lambda d: B.MxTensor(32, 64, d)):
        for device in (0, 1, "cuda:0", None):
            with pytest.raises(Asked):
                make(device)
    assert asked == [0, 1, "cuda:0", "cuda"] * 2


def test_memory_of_calls_on_other_streams_is_the_allocators_business(monkeypatch):
    """On made-up streams: the workspace is reported once for each torch stream, results come from the call's stream, and a
    stream given as a number makes the drop wait."""
    ops_ready = B.CrossEntropy                              # (loads the extension)
    log, now = [], []

    class Stream:
        def __init__(self, handle):
            self.cuda_stream = handle

        def record_event(self):
            return "made on %d" % self.cuda_stream

        def wait_event(self, e):
            log.append(("wait", self.cuda_stream, e))

    class Entered:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            now.append(self.s)

        def __exit__(self, *a):
            now.pop()

    class Memory:
        device = "cuda:0"

        def __init__(self, n):
            self.n, self.on = n, now[-1].cuda_stream

        def record_stream(self, s):
            log.append(("record", self.n, self.on, s.cuda_stream))

        data_ptr, numel, get_device = lambda self: 256, lambda self: self.n, lambda self: 0

    class Loss(ops_ready):
        def _forward(self, *a):
            log.append(("forward", a[3].on, a[4].on, a[5]))

        def _backward(self, *a):
            log.append(("backward",))

    now.append(Stream(0))
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch, "empty", lambda n, **kw: Memory(n))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream(0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream(handle))
    monkeypatch.setattr(torch.cuda, "stream", Entered)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: log.append("synchronize"))
    size = B.ps_xent_sizes(10, 20, 8)[0]
    class Tokens(list):
        device = "cuda:0"

    x = Tokens(range(10))
    ce, side = Loss(10, 20, 8), Stream(5)
    ce.forward(x, None, None)
    assert log == [("forward", 0, 0, None)]
    for k in range(2):
        del log[:]
        ce.forward(x, None, None, stream=side)
        results = [("record", 10, 5, 0)] * 2
        assert log == ([("wait", 5, "made on 0"), ("record", size, 0, 5)] if k == 0 else []) + results + [("forward", 5, 5, side)]
    del log[:]
    ce.backward(x, None, None, None, stream=side)
    assert log == [("backward",)]
    del ce
    assert log == [("backward",)]
    ce = Loss(10, 20, 8)
    ce.backward(x, None, None, None, stream=7)
    assert log[1:] == [("wait", 7, "made on 0"), ("backward",)]
    del ce
    assert log[-1] == "synchronize"


@gpu
def test_objects_from_several_host_threads():
    """One thread, stream and object each, results as on one thread, to the bit."""
    import threading
    sizes = [(300, 1000, 64), (37, 5000, 61), (1000, 300, 136), (5000, 7000, 64)]
    data = [inputs(*s, seed=k) for k, s in enumerate(sizes)]
    refs = [run(*s, seed=k) for k, s in enumerate(sizes)]
    torch.cuda.synchronize()
    errors = []

    def work(k):
        try:
            torch.cuda.set_device(0)
            stream, (T, V, D) = torch.cuda.Stream(), sizes[k]
            for it in range(20):
                with torch.cuda.stream(stream):
                    ce = B.CrossEntropy(T, V, D)
                    dx, dw = torch.empty(T, D, device="cuda", dtype=BF), torch.empty(V, D, device="cuda", dtype=BF)
                loss, lse = ce.forward(*data[k], stream=stream)
                ce.backward(*data[k], lse, dx, dw, stream=stream)
                stream.synchronize()
                assert all(torch.equal(a, b) for a, b in zip((loss, lse, dx, dw), refs[k]))
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(sizes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert B.ps_xent_status() == 0


@gpu
def test_the_binding_refuses():
    ce = B.CrossEntropy(10, 100, 16)
    x, w, t = inputs(10, 100, 16)
    _, lse = ce.forward(x, w, t)
    dx, dw = torch.empty(10, 16, device="cuda", dtype=BF), torch.empty(100, 16, device="cuda", dtype=BF)
    wrong = [lambda: ce.forward(x.float(), w, t), lambda: ce.forward(x, w.half(), t), lambda: ce.forward(x.cpu(), w, t),
             lambda: ce.forward(x, w, t.cpu()), lambda: ce.forward(x, w, t.to(torch.int16)), lambda: ce.forward(x, w, t[:5]),
             lambda: ce.forward(x, w[:50], t), lambda: ce.forward(x[:, :8], w[:, :8], t), lambda: ce.forward(x, w.t().contiguous().t(), t),
             lambda: ce.forward(x, w, t, loss=torch.empty(9, device="cuda")), lambda: ce.forward(x, w, t, lse=lse.double()),
             lambda: ce.forward(torch.cat([x, x]), w, torch.cat([t, t])), lambda: ce.backward(x, w, t, lse),
             lambda: ce.backward(x, w, t, lse[:3], dx, dw), lambda: ce.backward(x, w, t, None, dx, dw),
             lambda: ce.backward(x, w, t, lse, dx.float(), dw), lambda: ce.backward(x, w, t, lse, dx, dw.half()),
             lambda: ce.backward(x, w, t, lse, dx, dw, token_scale=lse[:4])]
    for call in wrong:
        with pytest.raises(B.PsError) as e:
            call()
        assert e.value.status == B.PS_ERR_BAD_ARG


def made_up(**kw):
    """A description whose addresses are never read: every call below is refused before anything runs."""
    d = dict(x=1 << 20, ldx=64, w=1 << 21, ldw=64, targets=1 << 22, target_bits=64, tokens=32, vocab=100, dim=64,
             workspace=1 << 24, workspace_bytes=B.ps_xent_sizes(32, 100, 64)[0])
    d.update(kw)
    return B.ps_xent(*[d[n] for n, _ in B.ps_xent._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(tokens=-1), B.PS_ERR_BAD_ARG), (dict(vocab=0), B.PS_ERR_BAD_ARG), (dict(dim=0), B.PS_ERR_BAD_ARG),
    (dict(tokens=(1 << 26) + 1), B.PS_ERR_BAD_ARG), (dict(vocab=(1 << 30) + 1), B.PS_ERR_BAD_ARG),
    (dict(dim=(1 << 24) + 1, ldx=1 << 25, ldw=1 << 25), B.PS_ERR_BAD_ARG), (dict(ldx=63), B.PS_ERR_BAD_ARG), (dict(ldw=10), B.PS_ERR_BAD_ARG),
    (dict(target_bits=16), B.PS_ERR_BAD_ARG), (dict(x=0), B.PS_ERR_BAD_ARG), (dict(w=0), B.PS_ERR_BAD_ARG),
    (dict(targets=0), B.PS_ERR_BAD_ARG), (dict(workspace=0), B.PS_ERR_BAD_ARG), (dict(x=(1 << 20) + 1), B.PS_ERR_ALIGN),
    (dict(w=(1 << 21) + 1), B.PS_ERR_ALIGN), (dict(targets=(1 << 22) + 4), B.PS_ERR_ALIGN),
    (dict(workspace=(1 << 24) + 128), B.PS_ERR_ALIGN), (dict(workspace_bytes=1000), B.PS_ERR_NOMEM),
    (dict(ldw=68, workspace_bytes=1000), B.PS_ERR_NOMEM),
    (dict(tokens=1 << 26, vocab=1 << 30, workspace_bytes=1 << 62), B.PS_ERR_TOO_LARGE)])
def test_refusals(kw, status):
    lib, q = B.load(), made_up(**kw)
    assert lib.ps_xent_forward(C.byref(q), 1 << 23, 1 << 23, None) == status
    assert lib.ps_xent_backward(C.byref(q), 1 << 23, 1.0, None, 1 << 25, 64, 1 << 26, B.PS_BF16, 64, None) == status


def test_refusals_of_results():
    lib, q = B.load(), made_up()
    fwd = lambda loss, lse: lib.ps_xent_forward(C.byref(q), loss, lse, None)  # noqa: E731
    assert fwd(None, None) == B.PS_ERR_BAD_ARG and fwd(2, None) == B.PS_ERR_ALIGN and fwd(None, 6) == B.PS_ERR_ALIGN

    def bwd(lse=1 << 23, ts=None, dx=1 << 25, lddx=64, dw=1 << 26, dtype=B.PS_BF16, lddw=64):
        return lib.ps_xent_backward(C.byref(q), lse, 1.0, ts, dx, lddx, dw, dtype, lddw, None)

    assert bwd(lse=None) == bwd(dx=None, dw=None) == bwd(dtype=2) == bwd(lddx=63) == bwd(lddw=63) == B.PS_ERR_BAD_ARG
    assert bwd(lse=2) == bwd(ts=2) == bwd(dx=(1 << 25) + 1) == bwd(dw=(1 << 26) + 2, dtype=B.PS_F32) == B.PS_ERR_ALIGN
    assert lib.ps_xent_forward(None, 1 << 23, None, None) == lib.ps_xent_status(None) == B.PS_ERR_BAD_ARG
    with pytest.raises(B.PsError):
        B.ps_xent_sizes(10, 0, 10)


def test_workspace_sizes_hold_for_every_smaller_batch():
    """A call of fewer tokens than the workspace was made for is cut differently and has to fit all the same: refused
    for NOMEM before it would be for the missing result."""
    lib = B.load()
    for V, D, most in ((30522, 1024, 8192), (500, 64, 3000), (100_000, 128, 70_000)):
        have = B.ps_xent_sizes(most, V, D)
        for T in sorted({1, 2, 31, 64, 200, 255, 256, 257, 549, 1000, 2048, 4095, 8192, 16384, 16385, 65536, most}):
            if T > most:
                continue
            for ld, size in ((D, have[0]), (D + 1, have[1])):
                q = made_up(tokens=T, vocab=V, dim=D, ldx=ld, ldw=ld, workspace_bytes=size)
                assert lib.ps_xent_forward(C.byref(q), None, None, None) == B.PS_ERR_BAD_ARG, (T, V, D, ld)
