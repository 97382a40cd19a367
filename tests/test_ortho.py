"""Orthogonalised matrices (ps_ortho_*) against the definition in 64 bits.

Tolerances, in the Frobenius norm relative to the result's.  fp32 results claim the precision of binary32 arithmetic:
four times what the same five steps are off when torch computes them in binary32 on the same matrix, plus what the last
step's operands of 22 bits may add where binary32 happens to be exact (a 1 x 1 matrix): X, E and F are rounded to 2^-23
of themselves and low x low is left out, 2^-22, together 2^-21 of the terms a X, b A X and c A A X, whose coefficients
add up to 10.3 for singular values near 1, over a result of at least 0.68 of X: 10.3 / 0.68 2^-21 < 2^-17.
bf16 results come from operands of 11 bits: three times what the steps are off when they are computed in 64 bits with
those operands rounded to fp16 (X to two halves, the diagonals of A and B kept), plus the bf16 rounding."""
import ctypes as C

import pytest
import torch

from paper_2204_03211_b200 import binding as B

gpu = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
STEPS, (KA, KB, KC), EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


def steps(g, dtype=torch.float64, rounded=False):
    """The five steps on the smaller side, in `dtype`; rounded: with the products' operands as fp16."""
    flip = g.shape[0] > g.shape[1]
    x = (g.t() if flip else g).double()
    x = (x / (x.square().sum().sqrt() + EPS)).to(dtype)

    def h(m):
        s = 2.0 ** 14 if m.shape[0] == m.shape[1] else 2.0 ** 12
        return (m * s).half().to(dtype) / s if rounded else m

    for _ in range(STEPS):
        xh = h(x)
        a = xh @ xh.t()
        if rounded:
            d = torch.diag(a)
            e = h(a - torch.diag(d))
            b = KB * e + KC * (e @ e + (d[:, None] + d[None, :]) * e)
            f = KB * d + KC * (torch.diag(e @ e) + d * d)
            b = b - torch.diag(torch.diag(b))
            x = (KA + f)[:, None] * x + h(b) @ xh
        else:
            x = KA * x + (KB * a + KC * (a @ a)) @ x
    return x.t() if flip else x


def off(a, b):
    return float((a.double() - b).norm() / b.norm().clamp(min=1e-30))


def matrix(rows, cols, kind, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, device="cuda", generator=g)
    if kind == "decaying":                                  # a few strong directions and little else
        r = max(1, min(rows, cols) // 8)
        x = (torch.randn(rows, r, device="cuda", generator=g) * torch.logspace(0, -3, r, device="cuda")) @ \
            torch.randn(r, cols, device="cuda", generator=g) + 1e-4 * x
    if kind == "spike":                                     # one entry holds nearly all of the norm
        x = 1e-3 * x
        x[rows // 2, cols // 3] = 50.0
    return x


def check(x, out):
    ref = steps(x)
    if out.dtype == F32:
        allowed = 4 * off(steps(x, torch.float32), ref) + 2.0 ** -17
    else:
        allowed = 3 * off(steps(x, rounded=True), ref) + 2.0 ** -8
    got = off(out, ref)
    assert got <= allowed, "off by %.3g, allowed %.3g" % (got, allowed)


SHAPES = [(1, 1), (1, 50), (50, 1), (2, 3), (16, 16), (31, 33), (64, 64), (65, 200), (128, 128), (129, 127), (300, 300),
          (128, 1000), (777, 300), (257, 513), (600, 130),
          (100, 2048), (2048, 77), (16, 300), (128, 257), (1, 1025), (100, 2049), (512, 128)]


@gpu
@pytest.mark.parametrize("kind", ["normal", "decaying", "spike"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_shapes(rows, cols, kind):
    x = matrix(rows, cols, kind)
    for src in (F32, BF):
        for dst in (F32, BF):
            s = x.to(src)
            out = torch.full((rows, cols), 9.0, device="cuda", dtype=dst)
            o = B.Ortho([s], [out])
            o.run()
            assert o.status() == 0
            check(s, out)


@gpu
@pytest.mark.parametrize("dst", [F32, BF])
def test_a_list_of_many_shapes(dst):
    """Pairs of CTAs (enough large tiles) and single ones, matrices of one tile next to matrices of many, empty ones; and a
    list of small ones only, which clusters of CTAs keep in shared memory."""
    tiny = [(3, 700), (64, 64), (0, 9), (128, 384), (1100, 90), (17, 1), (128, 128)] * 30
    small = [(5, 7), (0, 4), (200, 40), (128, 384), (3, 0), (130, 130), (64, 64)]
    for shapes in (tiny, small, small + [(512, 2100)] * 12, [(1100, 700)] * 15 + [(260, 30)]):
        xs = [matrix(r, c, "normal" if k % 2 else "decaying", k) for k, (r, c) in enumerate(shapes)]
        outs = [torch.full((r, c), 9.0, device="cuda", dtype=dst) for r, c in shapes]
        o = B.Ortho(xs, outs)
        o.run()
        assert o.status() == 0
        for x, out in list(zip(xs, outs))[:9] + list(zip(xs, outs))[-2:]:
            if x.numel():
                check(x, out)
        first = [t.clone() for t in outs]
        o.run()                                             # the same every time
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))


@gpu
@pytest.mark.parametrize("rows,cols,count", [(100, 4096, 3), (4095, 64, 2), (33, 2500, 14), (33, 2500, 15), (128, 4097, 1)])
def test_rows_of_thousands(rows, cols, count):
    """Up to 4096 columns one cluster of sixteen CTAs holds a matrix; longer lists, and wider ones, take the general form."""
    xs = [matrix(rows, cols, "normal", k) for k in range(count)]
    for dst in (F32, BF):
        outs = [torch.full((rows, cols), 9.0, device="cuda", dtype=dst) for _ in xs]
        o = B.Ortho(xs, outs)
        o.run()
        assert o.status() == 0
        for x, out in ((xs[0], outs[0]), (xs[-1], outs[-1])):
            check(x, out)


@gpu
def test_large_matrix_in_pairs():
    xs = [matrix(1024, 4096, "decaying", 3), matrix(4000, 1030, "normal", 4), matrix(2048, 2048, "normal", 5)] * 2
    for dst in (F32, BF):
        outs = [torch.empty(x.shape, device="cuda", dtype=dst) for x in xs]
        o = B.Ortho(xs, outs)
        o.run()
        assert o.status() == 0
        for x, out in zip(xs[:3], outs):
            check(x, out)
        assert all(torch.equal(outs[k], outs[k + 3]) for k in range(3))


@gpu
def test_offsets_past_2_31():
    """Rows 2^23 elements apart: the last one starts past the 2^31st element of either tensor."""
    m, n, ld = 300, 520, 1 << 23
    base, to = torch.empty(m, ld, device="cuda"), torch.empty(m, ld, device="cuda", dtype=BF)
    for rows, cols in ((m, n), (m, 100)):                   # the general form, and the small one
        x, out = base[:rows, :cols], to[:rows, :cols]
        x.copy_(matrix(rows, cols, "normal"))
        o = B.Ortho([x], [out])
        o.run()
        assert o.status() == 0
        check(x, out)


@gpu
def test_long_rows():
    """Sums over 200 000 elements, and as many columns of a result."""
    for rows, cols in ((3, 200_000), (140, 100_000), (100_000, 140)):
        x = matrix(rows, cols, "normal")
        for dst in (F32, BF):
            out = torch.empty(rows, cols, device="cuda", dtype=dst)
            o = B.Ortho([x], [out])
            o.run()
            assert o.status() == 0
            check(x, out)


@gpu
def test_rows_of_wider_tensors_and_in_place():
    base = torch.randn(90, 300, device="cuda")
    wide = torch.full((90, 200), 5.0, device="cuda")
    src = base[10:70, 7:107]
    B.Ortho([src], [wide[:60, 1:101]]).run()
    torch.cuda.synchronize()
    check(src, wide[:60, 1:101])
    wide[:60, 1:101] = 5.0
    assert bool((wide == 5.0).all())                        # nothing else was written
    a, b = torch.randn(40, 40, device="cuda"), torch.randn(40, 40, device="cuda")
    ra, rb = a.clone(), b.clone()
    B.Ortho([a, b], [b, a]).run()                           # all sources are read before a result is written
    torch.cuda.synchronize()
    check(ra, b)
    check(rb, a)
    c = matrix(150, 90, "normal").to(BF)
    rc = c.clone()
    B.Ortho([c]).run()
    torch.cuda.synchronize()
    check(rc, c)


@gpu
@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
def test_scales(scale):
    x = matrix(96, 160, "normal") * scale
    out = torch.empty(96, 160, device="cuda")
    B.Ortho([x], [out]).run()
    torch.cuda.synchronize()
    if scale == 1e-30:                                      # next to the 1e-7 beside the norm
        assert float(out.abs().max()) < 1e-18
    else:
        check(x, out)


@gpu
def test_zeros_nan_and_infinities():
    ok = matrix(70, 90, "normal")
    xs = [torch.zeros(70, 90, device="cuda"), ok.clone(), ok.clone(), ok]
    xs[1][69, 89], xs[2][0, 0] = float("nan"), float("-inf")
    for dst in (F32, BF):
        outs = [torch.empty(70, 90, device="cuda", dtype=dst) for _ in xs]
        o = B.Ortho(xs, outs)
        o.run()
        assert o.status() == 0
        assert not outs[0].any() and outs[1].isnan().all() and outs[2].isnan().all()
        check(ok, outs[3])


@gpu
def test_on_another_stream_and_captured():
    x, out = matrix(200, 260, "normal"), torch.empty(200, 260, device="cuda")
    o = B.Ortho([x], [out])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    o.run(stream)
    stream.synchronize()
    check(x, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.run(torch.cuda.current_stream())
    x.copy_(matrix(200, 260, "decaying", 8))
    graph.replay()
    torch.cuda.synchronize()
    check(x, out)


@gpu
def test_the_binding_refuses():
    a, b = torch.randn(8, 9, device="cuda"), torch.randn(8, 9, device="cuda")
    for srcs, dsts in (([a], [b.t()]), ([a.cpu()], [b]), ([a], [b.cpu()]), ([a.half()], [b]), ([a, b.to(BF)], [a, b]),
                       ([a.t()], [b.t()]), ([a[0]], [b[0]]), ([a], [a, b]), ([a], [b[:, :8]])):
        with pytest.raises(B.PsError) as e:
            B.Ortho(srcs, dsts)
        assert e.value.status == B.PS_ERR_BAD_ARG


def test_refusals():
    lib, h = B.load(), C.c_void_p()

    def create(src=(4096, 4, 8, 8), dst=(8192, 4, 8, 8), st=B.PS_F32, dt=B.PS_F32, n=1, device=0):
        s, d = (B.ps_matrix * 1)(src), (B.ps_matrix * 1)(dst)
        return lib.ps_ortho_create(C.byref(h), device, n, s, st, d, dt)

    bad = B.PS_ERR_BAD_ARG
    assert create(src=(0, 4, 8, 8)) == create(dst=(0, 4, 8, 8)) == create(src=(4096, 4, 8, 7)) == create(dst=(8192, 4, 8, 7)) == bad
    assert create(dst=(8192, 8, 4, 8)) == create(src=(4096, -1, 8, 8)) == create(st=2) == create(dt=-1) == create(device=-1) == bad
    assert create(n=-1) == create(src=(4096, (1 << 24) + 1, 8, 8), dst=(8192, (1 << 24) + 1, 8, 8)) == bad
    s, d = (B.ps_matrix * 2)((4096, 4, 8, 8), (4096, 4, 8, 8)), (B.ps_matrix * 2)((8192, 4, 8, 8), (8192, 4, 8, 8))
    assert lib.ps_ortho_create(C.byref(h), 0, 2, s, B.PS_F32, d, B.PS_F32) == bad          # two results in one place
    assert create(src=(4098, 4, 8, 8)) == create(dst=(8193, 4, 8, 8), dt=B.PS_BF16) == B.PS_ERR_ALIGN
    big = (1 << 21, 1 << 21, 1 << 21)
    assert create(src=(4096, *big), dst=(8192, *big)) == B.PS_ERR_TOO_LARGE
    assert lib.ps_ortho_create(None, 0, 0, None, 0, None, 0) == lib.ps_ortho_create(C.byref(h), 0, 1, None, 0, None, 0) == bad
    for call in (lambda: lib.ps_ortho_run(None, None), lambda: lib.ps_ortho_status(None, None), lambda: lib.ps_ortho_destroy(None)):
        assert call() == B.PS_ERR_BAD_HANDLE
    assert not h.value


@gpu
def test_handles_from_several_host_threads():
    """One thread, stream and list each, made and run at the same time: results as on one thread, to the bit."""
    import threading
    gen = torch.Generator(device="cuda").manual_seed(4)
    lists = [[torch.randn(s, device="cuda", generator=gen) for s in shapes] for shapes in
             ([(64, 256)] * 5, [(777, 300), (130, 130)], [(128, 1000)] * 3, [(700, 900)] * 4, [(40, 2000), (2000, 40)])]
    alone = []
    for l in lists:
        outs = [torch.empty_like(t) for t in l]
        o = B.Ortho(l, outs)
        o.run()
        torch.cuda.synchronize()
        o.close()
        alone.append(outs)
    errors = []

    def work(k):
        try:
            torch.cuda.set_device(0)
            stream = torch.cuda.Stream()
            for it in range(20):
                with torch.cuda.stream(stream):
                    outs = [torch.zeros_like(t) for t in lists[k]]
                o = B.Ortho(lists[k], outs)
                for _ in range(3):
                    o.run(stream)
                stream.synchronize()
                assert o.status() == 0 and all(torch.equal(a, b) for a, b in zip(outs, alone[k]))
                o.close()
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(lists))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
