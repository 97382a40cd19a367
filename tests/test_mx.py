"""Microscaled 4-bit operands: quantisation both ways, the values read back, and the product with
its gradients, against plain numpy in 64 bits.  Quantisation is defined to the bit, so it is compared
for equality; the product's tolerance is derived from the number of additions."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2204_03211_b200 import binding as B

MAGS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx_ref(x):
    """The values a matrix takes on in the format, blocks of 32 along its rows, in 64 bits (NaN blocks as NaN)."""
    x = np.asarray(x, dtype=np.float64)
    R, Cc = x.shape
    full = np.zeros((R, -(-Cc // 32) * 32))
    full[:, :Cc] = x
    out = np.empty_like(full)
    for r in range(R):
        for b in range(0, full.shape[1], 32):
            v = full[r, b:b + 32]
            if not np.isfinite(v).all():
                out[r, b:b + 32] = np.nan
                continue
            top = np.abs(v).max()
            e = max(int(np.frexp(top)[1]) - 3, -127) if top else -127
            a = np.abs(v) / 2.0 ** e
            d = np.abs(a[:, None] - MAGS[None])
            code = np.empty(32, dtype=int)
            for i in range(32):
                best = np.flatnonzero(d[i] == d[i].min())              # two at a tie: the even code
                code[i] = next((k for k in best if k % 2 == 0), best[0])
            out[r, b:b + 32] = np.copysign(MAGS[code], v) * 2.0 ** e
    return out[:, :Cc]


def as64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def same(got, ref):
    return np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[~np.isnan(ref)], ref[~np.isnan(ref)])


def quantized(x, transposed=False):
    r, c = x.shape
    q = B.MxTensor(c, r) if transposed else B.MxTensor(r, c)
    B.ps_mx_quantize(x, None if transposed else q, q if transposed else None)
    return q


def values(q, dtype=torch.float32):
    return B.ps_mx_dequantize(q, torch.empty(q.rows, q.cols, device="cuda", dtype=dtype))


def tricky(rows, cols, dtype, seed):
    """Values over many binades: whole blocks of zeros, subnormal and huge blocks, every tie of the format, signed
    zeros, and blocks with an infinity or a NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=g).float())
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.75, -0.25, -0.75, -2.5, -5.0, 0.0, -0.0])
    for r in range(rows):
        k = r % 9
        if k == 1:
            x[r] = 0
        elif k == 2:
            x[r] = ties[torch.randint(0, 16, (cols,), generator=g)]
            x[r, ::32] = 4.5
        elif k == 3:
            x[r] *= 2.0 ** -130
        elif k == 4:
            x[r] = torch.sign(x[r]) * 3e38
        elif k == 5:
            x[r, cols // 2] = float("inf")
        elif k == 6:
            x[r, -1] = float("nan")
        elif k == 7:
            x[r] = torch.exp2(torch.randint(-8, 3, (cols,), generator=g).float())
    return x.to(dtype).cuda()


SHAPES = [(1, 1), (1, 31), (1, 32), (3, 33), (9, 64), (18, 127), (33, 129), (129, 40), (130, 257), (64, 1000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_both_ways(rows, cols, dtype):
    x = tricky(rows, cols, dtype, rows * 1000 + cols)
    ref, ref_t = mx_ref(as64(x)), mx_ref(as64(x).T)
    q, qt = B.MxTensor(rows, cols), B.MxTensor(cols, rows)
    for t in (q.codes, q.scales, qt.codes, qt.scales):
        t.fill_(0xFF)                       # padding has to be written, not found
    B.ps_mx_quantize(x, q, qt)
    for out in (torch.float32, torch.bfloat16):
        assert same(as64(values(q, out)), ref)
        assert same(as64(values(qt, out)), ref_t)
    assert same(as64(values(quantized(x))), ref)
    assert same(as64(values(quantized(x, True))), ref_t)
    one, one_t = quantized(x), quantized(x, True)
    assert torch.equal(one.codes, q.codes) and torch.equal(one_t.codes, qt.codes)


@pytest.mark.gpu
def test_quantize_strides_alignment_and_streams():
    base = torch.randn(70, 301, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for dtype in (torch.float32, torch.bfloat16):
        b = base.to(dtype)
        side.wait_stream(torch.cuda.current_stream())
        for off, width in ((0, 300), (1, 300), (3, 40), (8, 128)):
            x = b[:, off:off + width]                   # row stride 301: no vector loads
            q, qt = B.MxTensor(70, width), B.MxTensor(width, 70)
            wide = torch.full((70, width + 5), 7.0, device="cuda", dtype=dtype)
            side.wait_stream(torch.cuda.current_stream())
            B.ps_mx_quantize(x, q, qt, side)
            B.ps_mx_dequantize(q, wide[:, :width], side)
            side.synchronize()
            assert same(as64(wide[:, :width]), mx_ref(as64(x)))
            assert (wide[:, width:] == 7.0).all()
            assert same(as64(values(qt)), mx_ref(as64(x).T))


def check_product(M, N, K, dtype, seed=0, scale=True):
    g = torch.Generator().manual_seed(seed)
    a = torch.randn(M, K, generator=g)
    b = torch.randn(N, K, generator=g)
    if scale:                               # blocks of very different size: additions do round
        a *= torch.exp2(torch.randint(-12, 12, (M, 1), generator=g).float())
        a[:, : K // 2] *= 2.0 ** 11
        b[:, K // 3:] *= 2.0 ** -7
    a, b = a.cuda(), b.cuda()
    qa, qb = quantized(a), quantized(b)
    va, vb = as64(values(qa)), as64(values(qb))
    wide = torch.full((M, N + 3), 5.0, device="cuda", dtype=dtype)
    out = wide[:, :N] if M % 2 else torch.full((M, N), 5.0, device="cuda", dtype=dtype)
    B.ps_mx_matmul(qa, qb, out)
    got, ref = as64(out), va @ vb.T
    # K products, exact; each addition may lose one unit in the last of 24 bits of a partial sum, which is at
    # most the sum of the magnitudes; a bf16 result is rounded once more, to 8 bits
    bound = K * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T)
    if dtype is torch.bfloat16:
        bound = bound * (1 + 2.0 ** -8) + np.abs(ref) * 2.0 ** -8
    assert (np.abs(got - ref) <= bound).all(), np.max(np.abs(got - ref) - bound)
    assert (wide[:, N:] == 5.0).all()
    assert B.ps_mx_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 1), (1, 128, 32), (1, 1000, 2050), (2, 129, 256), (7, 5, 100), (16, 640, 512), (17, 300, 4096),
    (64, 1024, 257), (65, 65, 65), (300, 1, 512), (257, 20, 4000), (128, 128, 128), (127, 129, 385), (500, 700, 1500),
    (129, 2500, 64), (2500, 257, 511),
])
def test_product(M, N, K, dtype):
    check_product(M, N, K, dtype, M * 7 + N * 3 + K)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(4000, 2817, 300), (2305, 4100, 1024), (20000, 250, 96), (1201, 1100, 600), (1024, 2048, 31),
                                   (2049, 2304, 2600)])
def test_product_of_many_tiles(M, N, K, dtype):
    """Tiles of 128 x 128 and of CTA pairs, several per CTA, with edges in both directions."""
    check_product(M, N, K, dtype)


@pytest.mark.gpu
def test_pairs_poison_only_what_they_should():
    """A NaN in the last block of rows, and results that end inside a tile, in the pairs' tiles."""
    a, b = torch.randn(2600, 320, device="cuda"), torch.randn(2500, 320, device="cuda")
    a[2599, 319] = float("nan")
    b[2499, 0] = float("-inf")
    out = torch.full((2601, 2503), 3.0, device="cuda", dtype=torch.bfloat16)
    B.ps_mx_matmul(quantized(a), quantized(b), out[:2600, :2500])
    bad = torch.zeros(2600, 2500, dtype=torch.bool, device="cuda")
    bad[2599] = True
    bad[:, 2499] = True
    assert torch.equal(out[:2600, :2500].isnan(), bad)
    assert (out[2600] == 3.0).all() and (out[:, 2500:] == 3.0).all()


@pytest.mark.gpu
def test_product_is_repeatable_and_poisons_only_its_rows():
    a, b = torch.randn(70, 900, device="cuda"), torch.randn(200, 900, device="cuda")
    a[3, 40] = float("nan")
    b[11, 899] = float("inf")
    qa, qb = quantized(a), quantized(b)
    first = B.ps_mx_matmul(qa, qb, torch.empty(70, 200, device="cuda"))
    for _ in range(3):
        again = B.ps_mx_matmul(qa, qb, torch.empty(70, 200, device="cuda"))
        assert torch.equal(first.view(torch.int32), again.view(torch.int32))
    bad = torch.zeros(70, 200, dtype=torch.bool, device="cuda")
    bad[3] = True
    bad[:, 11] = True
    assert torch.equal(first.isnan(), bad)


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", [(1, 32, 64), (40, 64, 96), (130, 300, 70)])
def test_gradients_of_a_layer(T, K, N):
    """dx = dy w and dw = dy^T x: against the formula on the operands' values, and against differences of
    sum(dy * y), which are exact because every value involved is one the format holds."""
    g = torch.Generator().manual_seed(T)
    grid = torch.tensor([-4.0, -3.0, -1.5, -0.5, 0.0, 1.0, 2.0, 3.0, 4.0])
    draw = lambda r, c: grid[torch.randint(0, 9, (r, c), generator=g)]  # noqa: E731
    x, w, dy = draw(T, K), draw(N, K), draw(T, N)
    for t in (x, w, dy):
        t[::32, :] = 4.0                    # every block along either direction has the scale 1
        t[:, ::32] = 4.0
    x, w, dy = x.cuda(), w.cuda(), dy.cuda()
    out = lambda r, c: torch.empty(r, c, device="cuda")  # noqa: E731
    dx = as64(B.ps_mx_matmul(quantized(dy), quantized(w, True), out(T, K)))
    dw = as64(B.ps_mx_matmul(quantized(dy, True), quantized(x, True), out(N, K)))
    assert np.array_equal(dx, as64(dy) @ as64(w))           # integers times a quarter: exact in binary32
    assert np.array_equal(dw, as64(dy).T @ as64(x))
    loss = lambda xx, ww: (as64(dy) * as64(B.ps_mx_matmul(quantized(xx), quantized(ww), out(T, N)))).sum()  # noqa: E731
    at = loss(x, w)
    for i, j in ((T - 1, K - 1), (T // 2, K // 3)):
        if i % 32 and j % 32:
            xx = x.clone()
            xx[i, j] = 2.0 if float(x[i, j]) != 2.0 else 3.0
            assert (loss(xx, w) - at) / float(xx[i, j] - x[i, j]) == dx[i, j]
    for i, j in ((N - 1, K - 1), (N // 2, K // 3)):
        if i % 32 and j % 32:
            ww = w.clone()
            ww[i, j] = 2.0 if float(w[i, j]) != 2.0 else 3.0
            assert (loss(x, ww) - at) / float(ww[i, j] - w[i, j]) == dw[i, j]


@pytest.mark.gpu
def test_empty_products_and_stream_order():
    assert B.ps_mx_matmul(B.MxTensor(0, 64), quantized(torch.ones(5, 64, device="cuda")),
                          torch.empty(0, 5, device="cuda")).shape == (0, 5)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        x = torch.randn(512, 2048, device="cuda")
        w = torch.randn(512, 2048, device="cuda")
        q, qw, y = B.MxTensor(512, 2048), B.MxTensor(512, 2048), torch.empty(512, 512, device="cuda")
        outs = []
        for k in range(8):                  # operands are overwritten while earlier products are still queued
            B.ps_mx_quantize(x + k, q, stream=s)
            B.ps_mx_quantize(w, qw, stream=s)
            outs.append(B.ps_mx_matmul(q, qw, y, s).clone())
        s.synchronize()
        for k in range(8):
            ref = B.ps_mx_matmul(quantized_on(x + k, s), qw, torch.empty_like(y), s)
            s.synchronize()
            assert torch.equal(outs[k], ref)


def quantized_on(x, s):
    q = B.MxTensor(*x.shape)
    B.ps_mx_quantize(x, q, stream=s)
    return q


# ---- refusals: before any device call, so they need no GPU ------------------------------------------------

def raw(rows, cols, codes=1 << 20, scales=1 << 21):
    return B.ps_mx(codes, scales, rows, cols)


def test_sizes():
    n, m = C.c_size_t(), C.c_size_t()
    lib = B.load()
    for rows, cols, codes, scales in ((1, 1, 16, 1024), (128, 256, 128 * 128, 1024), (129, 257, 129 * 144, 4096),
                                      (0, 64, 0, 0)):
        assert lib.ps_mx_sizes(rows, cols, C.byref(n), C.byref(m)) == B.PS_OK
        assert (n.value, m.value) == (codes, scales)
    for rows, cols in ((-1, 4), (4, 0), (1 << 31, 4), (4, 1 << 31)):
        assert lib.ps_mx_sizes(rows, cols, C.byref(n), C.byref(m)) == B.PS_ERR_BAD_ARG


def test_refusals():
    lib = B.load()
    ref = C.byref
    q = lambda *a, **k: ref(raw(*a, **k))  # noqa: E731
    x = 1 << 22
    bad, align = B.PS_ERR_BAD_ARG, B.PS_ERR_ALIGN
    quant = lambda *a: lib.ps_mx_quantize(*a, None)  # noqa: E731
    assert quant(x, 7, 4, 64, 64, q(4, 64), None) == bad              # type
    assert quant(x, B.PS_F32, 4, 64, 64, None, None) == bad           # nothing wanted
    assert quant(x, B.PS_F32, -1, 64, 64, q(4, 64), None) == bad
    assert quant(x, B.PS_F32, 4, 0, 64, q(4, 64), None) == bad
    assert quant(x, B.PS_F32, 4, 64, 63, q(4, 64), None) == bad       # stride shorter than a row
    assert quant(None, B.PS_F32, 4, 64, 64, q(4, 64), None) == bad
    assert quant(x, B.PS_F32, 4, 64, 64, q(4, 65), None) == bad       # shapes
    assert quant(x, B.PS_F32, 4, 64, 64, None, q(4, 64)) == bad       # the transpose has x's columns as rows
    assert quant(x, B.PS_F32, 4, 64, 64, q(4, 64, codes=0), None) == bad
    assert quant(x + 2, B.PS_F32, 4, 64, 64, q(4, 64), None) == align
    assert quant(x + 1, B.PS_BF16, 4, 64, 64, q(4, 64), None) == align
    assert quant(x, B.PS_F32, 4, 64, 64, q(4, 64, codes=(1 << 20) + 8), None) == align
    assert quant(x, B.PS_F32, 4, 64, 64, q(4, 64, scales=(1 << 20) + 4), None) == align
    assert quant(None, B.PS_F32, 0, 64, 64, q(0, 64), None) == B.PS_OK
    deq = lambda *a: lib.ps_mx_dequantize(*a, None)  # noqa: E731
    assert deq(None, B.PS_F32, x, 64) == bad
    assert deq(q(4, 64), 9, x, 64) == bad
    assert deq(q(4, 64), B.PS_F32, x, 63) == bad
    assert deq(q(4, 64), B.PS_F32, None, 64) == bad
    assert deq(q(4, 64), B.PS_F32, x + 2, 64) == align
    assert deq(q(0, 64), B.PS_F32, None, 64) == B.PS_OK
    mul = lambda *a: lib.ps_mx_matmul(*a, None)  # noqa: E731
    assert mul(q(4, 64), q(5, 96), B.PS_F32, x, 5) == bad             # contraction lengths
    assert mul(q(4, 64), q(5, 64), B.PS_F32, x, 4) == bad             # stride shorter than a row
    assert mul(q(4, 64), q(5, 64), 3, x, 5) == bad
    assert mul(q(4, 64), None, B.PS_F32, x, 5) == bad
    assert mul(q(4, 64), q(5, 64), B.PS_F32, None, 5) == bad
    assert mul(q(4, 64), q(5, 64), B.PS_F32, x + 2, 5) == align
    assert mul(q(0, 64), q(5, 64), B.PS_F32, None, 5) == B.PS_OK
    assert lib.ps_mx_status(None) == bad


def test_binding_refuses_wrong_arguments():
    q = B.MxTensor(4, 64, device="cpu")
    assert (q.rows, q.cols, q.shape) == (4, 64, (4, 64))
    x = torch.zeros(4, 64)
    with pytest.raises(B.PsError) as e:                          # not on a GPU
        B.ps_mx_quantize(x, q)
    assert e.value.status == B.PS_ERR_BAD_ARG
    with pytest.raises(B.PsError):
        B.ps_mx_dequantize(q, x)
    with pytest.raises(B.PsError):
        B.MxTensor(4, 0)
    for call in (lambda: B.ps_mx_quantize(), lambda: B.ps_mx_quantize(x, x), lambda: B.ps_mx_quantize(x, q, None, None, 1),
                 lambda: B.ps_mx_quantize(x, q, q=q), lambda: B.ps_mx_quantize(x, bias=q), lambda: B.ps_mx_matmul(q, q),
                 lambda: B.ps_mx_matmul(q, "b", x), lambda: B.MxTensor()):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(AttributeError):
        B.ps_mx_quantise


@pytest.mark.gpu
def test_binding_checks_shapes_and_types_and_takes_keywords():
    x, q = torch.randn(8, 64, device="cuda"), B.MxTensor(8, 64)
    qt = B.MxTensor(64, 8)
    assert B.ps_mx_quantize(x, qt=qt, stream=torch.cuda.current_stream()) is None
    B.ps_mx_quantize(x=x, q=q, stream=torch.cuda.current_stream().cuda_stream)
    out = torch.empty(8, 8, device="cuda")
    assert B.ps_mx_matmul(q, b=q, out=out) is out and out.equal(values(q) @ values(q).t())
    for bad in (lambda: B.ps_mx_matmul(q, q, torch.empty(8, 9, device="cuda")), lambda: B.ps_mx_matmul(q, qt, out),
                lambda: B.ps_mx_quantize(x, qt), lambda: B.ps_mx_quantize(x), lambda: B.ps_mx_quantize(x.double(), q),
                lambda: B.ps_mx_quantize(x[0], q), lambda: B.ps_mx_quantize(x.t(), qt), lambda: B.ps_mx_dequantize(q, out),
                lambda: B.ps_mx_quantize(x[:1].expand(8, 64), q)):
        with pytest.raises(B.PsError) as e:
            bad()
        assert e.value.status == B.PS_ERR_BAD_ARG
    with pytest.raises(AttributeError):
        B.ps_mx_quantize(x, q, stream="main")


PLACES = r"""
import ctypes, sys
sys.path.insert(0, sys.argv[1])
from paper_2204_03211_b200 import binding as B
B.load()
from paper_2204_03211_b200 import _ops


class Tensor:
    is_cuda, dtype = True, "f32"

    def __init__(self, rows, cols, device):
        self.shape, self.device = (rows, cols), device
        self.is_cuda = device >= 0

    def stride(self):
        return self.shape[1], 1

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 1 << 20


def refused(call, *args):
    try:
        call(*args)
    except B.PsError as e:
        assert e.status == B.PS_ERR_BAD_ARG, e
        return
    raise AssertionError("launched")


pretend = ctypes.CDLL(sys.argv[2])              # the current device is 0; launches are counted
_ops.setup("f32", "bf16", B._raise_op)
made = lambda r, c, d: _ops.Operand(1 << 21, 1 << 22, r, c, d)
x, far = Tensor(8, 64, 0), Tensor(8, 64, 1)
q, q_far, host = made(8, 64, 0), made(8, 64, 1), made(8, 64, -1)
qt, qt_far, out, out_far = made(64, 8, 0), made(64, 8, 1), Tensor(8, 8, 0), Tensor(8, 8, 1)
refused(_ops.ps_mx_quantize, x, host)
refused(_ops.ps_mx_quantize, x, q_far)
refused(_ops.ps_mx_quantize, x, q, qt_far)
refused(_ops.ps_mx_quantize, x, None, qt_far)
refused(_ops.ps_mx_quantize, far, q)
refused(_ops.ps_mx_quantize, far, q_far)        # all on one GPU, but not on the current one
refused(_ops.ps_mx_quantize, Tensor(8, 64, -1), host)
refused(_ops.ps_mx_dequantize, host, x)
refused(_ops.ps_mx_dequantize, q_far, x)
refused(_ops.ps_mx_dequantize, q, far)
refused(_ops.ps_mx_dequantize, q_far, far)
refused(_ops.ps_mx_matmul, q, host, out)
refused(_ops.ps_mx_matmul, host, q, out)
refused(_ops.ps_mx_matmul, q, q_far, out)
refused(_ops.ps_mx_matmul, q, q, out_far)
refused(_ops.ps_mx_matmul, q_far, q_far, out_far)
assert pretend.pretend_launches() == 0
_ops.ps_mx_quantize(x, q, qt)
_ops.ps_mx_dequantize(q, x)
assert pretend.pretend_launches() == 2          # these are where they should be
pretend.cudaSetDevice(1)
_ops.ps_mx_quantize(far, q_far)
refused(_ops.ps_mx_quantize, x, q)
assert pretend.pretend_launches() == 3
"""


def test_buffers_off_the_current_device_are_refused(tmp_path):
    """No kernel is launched on memory that the current device cannot reach: host buffers, another GPU's.  With made-up
    addresses, on a runtime that only keeps count."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    B.MxTensor(1, 1, device="cpu")              # (builds and loads what the child uses)
    pretend = str(tmp_path / "pretend.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", pretend,
                    os.path.join(root, "tests", "c", "pretend_cuda.c")], check=True)
    run = subprocess.run([sys.executable, "-c", PLACES, root, pretend], env=dict(os.environ, LD_PRELOAD=pretend),
                         capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_row_strides_whose_offsets_pass_31_bits(dtype):
    """The last rows of every matrix lie beyond 2^31 elements: the same bits as from packed ones."""
    R, C, ld = 70_000, 96, 32_000
    wide = torch.empty(R, ld, device="cuda", dtype=dtype)
    x = wide[:, :C]
    x.copy_(torch.randn(R, C, device="cuda"))
    packed = x.contiguous()
    q, qt, pq, pqt = B.MxTensor(R, C), B.MxTensor(C, R), B.MxTensor(R, C), B.MxTensor(C, R)
    B.ps_mx_quantize(x, q, qt)
    B.ps_mx_quantize(packed, pq, pqt)
    for a, b in ((q, pq), (qt, pqt)):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    B.ps_mx_dequantize(q, x)
    assert torch.equal(x, B.ps_mx_dequantize(q, torch.empty_like(packed)))
    for n in (5, 90):                       # few rows: one CTA per tile; more: CTA pairs
        w = quantized(torch.randn(n, C, device="cuda"))
        B.ps_mx_matmul(q, w, wide[:, :n])
        assert torch.equal(wide[:, :n], B.ps_mx_matmul(q, w, torch.empty(R, n, device="cuda", dtype=dtype)))
    del wide, x
    long = torch.empty(16, 140_000_000, device="cuda", dtype=dtype)[:, :R]      # few rows far apart: the swapped product
    w = quantized(torch.randn(16, C, device="cuda"))
    B.ps_mx_matmul(w, q, long)
    assert torch.equal(long, B.ps_mx_matmul(w, q, torch.empty(16, R, device="cuda", dtype=dtype)))
    assert B.ps_mx_status() == 0


@pytest.mark.gpu
def test_operands_of_more_than_two_gigabytes():
    """Codes of 2.1 GB in either direction, from rows that repeat every 1024: so do codes, values and products."""
    period, times, C = 1024, 1024, 4128
    rows = period * times + 5
    base = torch.randn(period, C, device="cuda").bfloat16()
    x = torch.empty(rows, C, device="cuda", dtype=torch.bfloat16)
    x[:period * times].view(times, period, C)[:] = base
    x[period * times:] = base[:5]
    q, qt, bq, bqt = B.MxTensor(rows, C), B.MxTensor(C, rows), B.MxTensor(period, C), B.MxTensor(C, period)
    B.ps_mx_quantize(x, q, qt)
    B.ps_mx_quantize(base, bq, bqt)
    assert q.codes.numel() > 1 << 31 and qt.codes.numel() > 1 << 31
    codes, want = q.codes.view(rows, -1), bq.codes.view(period, -1)
    assert (codes[:period * times].view(times, period, -1) == want).all() and torch.equal(codes[period * times:], want[:5])
    t, want_t = qt.codes.view(C, -1), bqt.codes.view(C, -1)
    for k in range(0, times, 128):
        part = t[:, k * period // 2:(k + 128) * period // 2].reshape(C, 128, period // 2)
        assert (part == want_t[:, None]).all()
    w = quantized(torch.randn(16, C, device="cuda"))
    y, small = torch.empty(rows, 16, device="cuda"), B.ps_mx_matmul(bq, w, torch.empty(period, 16, device="cuda"))
    B.ps_mx_matmul(q, w, y)
    # (the same sums in the same order, whatever the number of tiles, where K is not split: up to rounding otherwise)
    assert (y[:period * times].view(times, period, 16) == y[:period]).all() and torch.equal(y[period * times:], y[:5])
    # at most one unit in the last of 24 bits of a partial sum per addition
    bound = C * 2.0 ** -23 * (values(bq).abs() @ values(w).abs().t())
    assert ((y[:period] - small).abs() <= 2 * bound).all()
    x.fill_(7.0)
    B.ps_mx_dequantize(q, x)
    assert (x[:period * times].view(times, period, C) == values(bq, torch.bfloat16)).all()
    assert B.ps_mx_status() == 0


@pytest.mark.gpu
def test_calls_from_several_host_threads():
    """One thread, stream and set of operands each; every result has the bits of the one-thread call."""
    import threading
    sizes = [(1, 1000, 512), (300, 256, 1000), (700, 900, 2048), (2100, 2500, 320)]
    inputs = [(torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda")) for m, n, k in sizes]
    want = [B.ps_mx_matmul(quantized(a), quantized(b), torch.empty(a.shape[0], b.shape[0], device="cuda")) for a, b in inputs]
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            torch.cuda.set_device(0)
            a, b = inputs[i]
            stream = torch.cuda.Stream()
            qa, qb = B.MxTensor(*a.shape), B.MxTensor(*b.shape)
            out = torch.zeros_like(want[i])
            torch.cuda.synchronize()
            for _ in range(50):
                B.ps_mx_quantize(a, qa, stream=stream)
                B.ps_mx_quantize(b, qb, stream=stream)
                B.ps_mx_matmul(qa, qb, out, stream)
                stream.synchronize()
                assert torch.equal(out, want[i])
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(sizes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and B.ps_mx_status() == 0, errors
