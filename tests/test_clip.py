"""Gradients clipped by their global norm: in the service's aggregate and on a worker's own tensors.

The norm is checked against 64 bits.  Given the norm the kernel reports, every later operation is one
binary32 rounding, so parameters, state and clipped tensors are compared for equality."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2204_03211_b200 import binding as B

f32 = np.float32


def factor(norm, max_norm):
    if np.isinf(max_norm):
        return f32(1)
    with np.errstate(all="ignore"):
        f = f32(max_norm) / (f32(norm) + f32(1e-6))
    return f32(1) if f >= 1 else f


def to_bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)


class Ref:
    """One block: numpy in binary32, one rounding per operation."""

    def __init__(self, hp, p):
        self.hp, self.p = hp, p.copy()
        self.s0, self.s1, self.t = np.zeros_like(p), np.zeros_like(p), 0

    def scaled_sum(self, grads):
        G = grads[0].astype(f32)
        for g in grads[1:]:
            G = G + g.astype(f32)
        return G * f32(self.hp["grad_scale"])

    def apply(self, G, c):
        hp = self.hp
        self.t += 1
        d = G * c + f32(hp["weight_decay"]) * self.p
        if hp["opt"] == B.PS_SGD:
            self.s0 = f32(hp["momentum"]) * self.s0 + d
            self.p = self.p - f32(hp["lr"]) * self.s0
        else:
            b1, b2 = f32(hp["beta1"]), f32(hp["beta2"])
            self.s0 = b1 * self.s0 + (f32(1) - b1) * d
            self.s1 = b2 * self.s1 + (f32(1) - b2) * (d * d)
            ss = f32(float(f32(hp["lr"])) / (1.0 - float(b1) ** self.t))
            sbc2 = f32(np.sqrt(1.0 - float(b2) ** self.t))
            self.p = self.p - ss * (self.s0 / (np.sqrt(self.s1) / sbc2 + f32(hp["eps"])))


def hparams(opt, dtype, W, grad_scale=1.0):
    return dict(opt=opt, grad_dtype=dtype, num_workers=W, lr=0.05, momentum=0.9, weight_decay=1e-3, beta1=0.9, beta2=0.99,
                eps=1e-8, grad_scale=grad_scale)


class World:
    """A service and the references of its blocks, fed the same gradients."""

    def __init__(self, jobs, sizes, contexts=1, seed=0):
        self.rng = np.random.default_rng(seed)
        self.svc = B.Service(0, contexts, 3 * sum(4 * n + 4096 for s in sizes for n in s) + (1 << 20))
        self.jobs, self.sizes, self.ref = jobs, sizes, {}
        for j, (hp, ns) in enumerate(zip(jobs, sizes)):
            assert self.svc.register_job(**hp) == j
            for b, n in enumerate(ns):
                p = self.rng.normal(0, 0.05, n).astype(f32)
                self.svc.register_block(j, b, n, 0, p)
                self.ref[j, b] = Ref(hp, p)
        self.ready = list(self.ref)

    def gradients(self, shift=0, spread=1e-2):
        """Device shards and the same values on the host; shift > 0 leaves the shards unaligned."""
        self.dev, self.host = {}, {}
        for (j, b), r in self.ref.items():
            for w in range(self.jobs[j]["num_workers"]):
                g = torch.from_numpy(self.rng.normal(0, spread, len(r.p) + shift).astype(f32))
                if self.jobs[j]["grad_dtype"] == B.PS_BF16:
                    g = g.to(torch.bfloat16)
                self.host[j, b, w] = g[shift:].float().numpy()
                self.dev[j, b, w] = g.cuda()[shift:]

    def push(self):
        for (j, b, w), g in self.dev.items():
            self.svc.push(j, b, w, g)

    def sums(self):
        return {k: r.scaled_sum([self.host[k[0], k[1], w] for w in range(r.hp["num_workers"])]) for k, r in self.ref.items()}

    def check(self, max_norm, norms):
        """norms: what the kernel reported, one per job.  Compares everything and advances the references."""
        sums = self.sums()
        for j in range(len(self.jobs)):
            true = np.sqrt(sum((sums[k].astype(np.float64) ** 2).sum() for k in sums if k[0] == j))
            # binary64 sums and square root, rounded once to 24 bits
            assert abs(float(norms[j]) - true) <= 1.01 * 2.0 ** -24 * true
            c = factor(norms[j], max_norm)
            for (jj, b), r in self.ref.items():
                if jj != j:
                    continue
                r.apply(sums[jj, b], c)
                got = self.svc.view(self.svc.pull(jj, b), len(r.p)).cpu().numpy()
                assert np.array_equal(got, r.p), (jj, b, np.flatnonzero(got != r.p)[:5])
                a0, a1, _ = self.svc.block_state(jj, b)
                assert np.array_equal(self.svc.view(a0, len(r.p)).cpu().numpy(), r.s0)
                if a1:
                    assert np.array_equal(self.svc.view(a1, len(r.p)).cpu().numpy(), r.s1)
                sq, step = self.svc.block_stats(jj, b)
                want = (sums[jj, b].astype(np.float64) ** 2).sum()
                assert step == r.t and abs(sq - want) <= 1e-12 * want
        assert self.svc.device_status() == 0


TINY, MIXED = [1, 5, 33, 1024], [300_001, 7, 65536, 256, 255, 257, 1, 90_000]


@pytest.mark.gpu
@pytest.mark.parametrize("opt", [B.PS_SGD, B.PS_ADAM])
@pytest.mark.parametrize("dtype", [B.PS_F32, B.PS_BF16])
@pytest.mark.parametrize("W", [1, 2, 5])
@pytest.mark.parametrize("sizes,inline", [(TINY, 1), (TINY, 0), (MIXED, 1)])
def test_aggregate_clipped(opt, dtype, W, sizes, inline):
    world = World([hparams(opt, dtype, W, 0.5)], [sizes], seed=W)
    world.svc.set_option(B.PS_OPT_INLINE_TABLE, inline)
    norms = torch.full((1,), -1.0, device="cuda")
    for it, max_norm in enumerate((0.05, 1e4, 0.7)):
        world.gradients(shift=it % 2)
        world.push()
        world.svc.aggregate_clipped(world.ready, max_norm, norms)
        world.check(max_norm, norms.cpu().numpy())
    world.svc.close()


@pytest.mark.gpu
def test_more_sums_than_shared_memory_holds():
    """14 million elements: most sums go through the buffer; a second, smaller call uses it again."""
    sizes = [9_000_001, 3, 4_999_999, 64]
    world = World([hparams(B.PS_SGD, B.PS_F32, 2)], [sizes])
    norms = torch.zeros(1, device="cuda")
    for max_norm in (1.0, 2.0):
        world.gradients()
        world.push()
        world.svc.aggregate_clipped(world.ready, max_norm, norms)
        world.check(max_norm, norms.cpu().numpy())
    world.svc.close()


@pytest.mark.gpu
def test_several_jobs_have_their_own_norms():
    jobs = [hparams(B.PS_SGD, B.PS_F32, 16), hparams(B.PS_ADAM, B.PS_BF16, 2), hparams(B.PS_SGD, B.PS_BF16, 3, 2.0)]
    world = World(jobs, [[5000, 120_001], [70_000, 9], [333] * 90])
    world.gradients()
    for j in (1, 2):
        for k in world.dev:
            if k[0] == j:
                world.dev[k] *= 4 ** j
                world.host[k] = world.host[k] * f32(4 ** j)
    world.push()
    norms = torch.zeros(3, device="cuda")
    order = sorted(world.ready, key=lambda t: (-t[0], t[1]))       # job 2 is named first
    world.svc.aggregate_clipped(order, 0.9, norms)
    world.check(0.9, norms.cpu().numpy()[::-1])
    world.svc.close()


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", [1, 2])
def test_a_factor_of_one_changes_nothing(kernel):
    """Norm below the limit, and an infinite limit: the same bits as ps_aggregate."""
    jobs = [hparams(B.PS_SGD, B.PS_F32, 3), hparams(B.PS_ADAM, B.PS_BF16, 4)]
    a, b = World(jobs, [MIXED, TINY], seed=5), World(jobs, [MIXED, TINY], seed=5)
    b.svc.set_option(B.PS_OPT_KERNEL, kernel)
    norms = torch.zeros(2, device="cuda")
    for limit in (1e9, float("inf")):
        a.gradients()
        b.gradients()
        a.push()
        b.push()
        a.svc.aggregate_clipped(a.ready, limit, norms)
        b.svc.aggregate(b.ready)
        a.check(limit, norms.cpu().numpy())
        for k, r in a.ref.items():
            n = len(r.p)
            assert torch.equal(a.svc.view(a.svc.pull(*k), n), b.svc.view(b.svc.pull(*k), n))
    a.svc.close()
    b.svc.close()


@pytest.mark.gpu
def test_nonfinite_gradients():
    for bad, want in ((float("nan"), "nan"), (float("inf"), "zero")):
        world = World([hparams(B.PS_SGD, B.PS_F32, 2)], [[1000, 50]])
        world.gradients()
        world.dev[0, 0, 1][77] = bad
        world.push()
        norms = torch.zeros(1, device="cuda")
        before = world.svc.view(world.svc.pull(0, 1), 50).cpu().numpy()
        world.svc.aggregate_clipped(world.ready, 1.0, norms)
        after0 = world.svc.view(world.svc.pull(0, 0), 1000).cpu().numpy()
        after1 = world.svc.view(world.svc.pull(0, 1), 50).cpu().numpy()
        if want == "nan":
            assert np.isnan(norms.item()) and np.isnan(after0).all() and np.isnan(after1).all()
        else:                                # the factor is 0: only weight decay moves the other elements
            assert np.isinf(norms.item()) and np.isnan(after0[77]) and np.isfinite(np.delete(after0, 77)).all()
            hp = world.jobs[0]
            assert np.array_equal(after1, before - f32(hp["lr"]) * (f32(hp["weight_decay"]) * before))
        world.svc.close()


@pytest.mark.gpu
def test_zero_gradients_are_not_scaled():
    world = World([hparams(B.PS_SGD, B.PS_F32, 2)], [[3000]])
    world.gradients()
    for k in world.dev:
        world.dev[k].zero_()
        world.host[k][:] = 0
    world.push()
    norms = torch.full((1,), 9.0, device="cuda")
    world.svc.aggregate_clipped(world.ready, 1.0, norms)
    world.check(1.0, norms.cpu().numpy())
    assert norms.item() == 0.0
    world.svc.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.PS_F32, B.PS_BF16])
@pytest.mark.parametrize("row_len", [8, 400])
def test_row_sparse_shards(dtype, row_len):
    rows, W = 700, 3
    world = World([hparams(B.PS_SGD, dtype, W)], [[rows * row_len, 1000]])
    world.gradients()
    keep = []
    for w in range(W):
        ids = np.sort(world.rng.choice(rows, 40 + w, replace=False)).astype(np.int32)
        full = world.dev[0, 0, w].view(rows, row_len)
        world.host[0, 0, w] = np.where(np.isin(np.arange(rows), ids)[:, None],
                                       world.host[0, 0, w].reshape(rows, row_len), f32(0)).reshape(-1)
        if w == 1:                           # one dense worker among them
            d = torch.from_numpy(world.host[0, 0, w]).to(full.dtype).cuda()
            keep.append(d)
            world.svc.push(0, 0, w, d)
        else:
            di = torch.from_numpy(ids).cuda()
            v = full[di.long()].contiguous()
            keep += [di, v]
            world.svc.push_rows(0, 0, w, di, len(ids), row_len, v)
        world.svc.push(0, 1, w, world.dev[0, 1, w])
    norms = torch.zeros(1, device="cuda")
    world.svc.aggregate_clipped(world.ready, 0.3, norms)
    world.check(0.3, norms.cpu().numpy())
    world.svc.close()


@pytest.mark.gpu
@pytest.mark.parametrize("overlap", [0, 1])
def test_prepared_rounds_alternate_with_other_calls(overlap):
    """Clipped and plain runs of one prepared round, a migration between them, and a second stream."""
    world = World([hparams(B.PS_ADAM, B.PS_F32, 2)], [[40_000, 129]], contexts=2)
    svc = world.svc
    svc.set_option(B.PS_OPT_OVERLAP, overlap)
    world.gradients()
    dev = world.dev
    keys = list(dev)
    i32 = lambda k: np.array([x[k] for x in keys], np.int32)  # noqa: E731
    rid = svc.round_prepare(i32(0), i32(1), i32(2), np.array([dev[k].data_ptr() for k in keys], np.uint64), world.ready)
    norms = torch.zeros(1, device="cuda")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for it in range(6):
        s = streams[it % 2]
        if it == 3:
            svc.migrate_blocks(world.ready, 1, s)
        if it % 3 == 1:
            svc.round_run(rid, s)
            svc.join(s)
            torch.cuda.synchronize()
            sums = world.sums()
            for k, r in world.ref.items():
                r.apply(sums[k], f32(1))
        else:
            svc.round_run_clipped(rid, 0.25, norms, s)
            torch.cuda.synchronize()
            world.check(0.25, norms.cpu().numpy())
    for _ in range(4):                       # nothing waits in between: steps of one block follow one another
        svc.round_run_clipped(rid, 0.25, norms, streams[0])
        svc.round_run_clipped(rid, 0.25, norms, streams[1])
    torch.cuda.synchronize()
    sums, c = world.sums(), factor(norms.item(), 0.25)
    for k, r in world.ref.items():
        for _ in range(8):
            r.apply(sums[k], c)
        assert np.array_equal(svc.view(svc.pull(*k), len(r.p)).cpu().numpy(), r.p)
    assert svc.launch_stats(4)[3]["launches"] == 12
    svc.close()


@pytest.mark.gpu
def test_the_factor_is_the_gradients_scale_by_differences():
    """Without momentum and weight decay the update is -lr * c(G) * G; its derivative along a direction D of the
    gradients is compared with a difference quotient of the formula in 64 bits."""
    n, lr, limit, h = 4096, 1.0, 0.5, 1e-3
    rng = np.random.default_rng(3)
    G, D = rng.normal(0, 1e-2, n).astype(f32), rng.normal(0, 1e-2, n).astype(f32)

    def update(g):
        svc = B.Service(0, 1, 1 << 20)
        j = svc.register_job(opt=B.PS_SGD, num_workers=1, lr=lr)
        svc.register_block(j, 0, n, 0)
        d = torch.from_numpy(g.astype(f32)).cuda()
        svc.push(j, 0, 0, d)
        svc.aggregate_clipped([(j, 0)], limit)
        torch.cuda.synchronize()
        out = svc.view(svc.pull(j, 0), n).cpu().numpy().astype(np.float64)
        svc.close()
        return out

    G64, D64 = G.astype(np.float64), D.astype(np.float64)
    norm = np.sqrt((G64 ** 2).sum())
    assert norm > limit
    exact = -lr * limit / norm * (D64 - G64 * (G64 @ D64) / norm ** 2)     # d/dG of limit * G / |G|
    quotient = (update(G + h * D) - update(G - h * D)) / (2 * h)
    # inputs and outputs carry 2^-24 relative, divided by 2h; the quotient's own error is of order h^2
    tol = (4 * 2.0 ** -24 / (2 * h) + 10 * h * h) * (np.abs(G64).max() + np.abs(D64).max())
    assert np.abs(quotient - exact).max() <= tol


# ---- a worker's own tensors ---------------------------------------------------------------------------

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.gpu
@pytest.mark.parametrize("src,dst", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("sizes,shift", [([1], 0), ([7, 8, 2048, 2049, 1], 0), ([100_003, 64, 5], 1), ([3_000_000, 17], 0),
                                         ([300] * 200, 0)])
def test_clip_tensors(src, dst, sizes, shift):
    g = torch.Generator().manual_seed(sum(sizes))
    hosts = [(torch.randn(n, generator=g) * 0.1).to(DT[src]) for n in sizes]
    srcs = [torch.cat([torch.zeros(shift, dtype=DT[src]), h]).cuda()[shift:] for h in hosts]
    dsts = [torch.full((n + shift,), 3.0, device="cuda", dtype=DT[dst])[shift:] for n in sizes]
    clip = B.Clip(srcs, dsts)
    norm = torch.zeros(1, device="cuda")
    true = np.sqrt(sum(float((h.double() ** 2).sum()) for h in hosts))
    for limit in (0.2, 1e6, float("inf"), 0.05):
        clip.run(limit, norm)
        # eight squares are added with at most sixteen roundings of 2^-24, the rest in binary64; half of it reaches the root
        assert abs(norm.item() - true) <= 9 * 2.0 ** -24 * true
        c = torch.tensor(factor(norm.item(), limit))
        for h, d in zip(hosts, dsts):
            assert torch.equal((h.float() * c).to(DT[dst]), d.cpu())
    assert clip.status() == 0
    clip.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_clip_in_place(dt):
    hosts = [(torch.randn(n) * 0.1).to(DT[dt]) for n in (5000, 1, 0, 70_001)]
    dev = [h.clone().cuda() for h in hosts]
    clip, norm = B.Clip(dev), torch.zeros(1, device="cuda")
    clip.run(1e6, norm)
    assert all(torch.equal(h, d.cpu()) for h, d in zip(hosts, dev))
    clip.run(0.5, norm)
    c = torch.tensor(factor(norm.item(), 0.5))
    assert all(torch.equal((h.float() * c).to(DT[dt]), d.cpu()) for h, d in zip(hosts, dev))
    clip.close()


@pytest.mark.gpu
def test_clip_extreme_values():
    """Squares that leave binary32's range, both ways, and non-finite elements."""
    norm = torch.zeros(1, device="cuda")
    for v in (1e30, 1e-30):
        x = torch.full((1000,), v, device="cuda")
        clip = B.Clip([x], [torch.empty_like(x)])
        clip.run(1.0, norm)
        true = float(f32(v)) * np.sqrt(1000.0)
        assert abs(norm.item() - true) <= 2.0 ** -23 * true
        clip.close()
    for bad in (float("nan"), float("inf")):
        x = torch.ones(100, device="cuda")
        x[50] = bad
        out = torch.empty_like(x)
        clip = B.Clip([x], [out])
        clip.run(1.0, norm)
        if np.isnan(bad):
            assert np.isnan(norm.item()) and out.isnan().all()
        else:
            assert np.isinf(norm.item()) and out.isnan().sum() == 1 and (out[:50] == 0).all()
        clip.close()
    empty = B.Clip([torch.empty(0, device="cuda")])
    norm.fill_(5)
    empty.run(1.0, norm)
    assert norm.item() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("src,dst,shift", [("f32", "f32", 0), ("bf16", "f32", 1), ("f32", "bf16", 0)])
@pytest.mark.parametrize("units", [63, 64, 65, 127, 128, 129, 255, 256, 257, 296, 297])
def test_clip_lists_around_the_limits_of_a_launch(units, src, dst, shift):
    """Units of 2048 elements: a tensor of many with a ragged end, tensors of one unit, empty tensors between them."""
    sizes = [5, 0, 2048 * (units - 4) - 3, 2048, 0, 2047, 1]
    g = torch.Generator().manual_seed(units)
    hosts = [torch.randn(n, generator=g).to(DT[src]) for n in sizes]
    srcs = [torch.cat([torch.zeros(shift, dtype=DT[src]), h]).cuda()[shift:] for h in hosts]
    dsts = [torch.full((n + shift,), 3.0, device="cuda", dtype=DT[dst])[shift:] for n in sizes]
    true = np.sqrt(sum(float((h.double() ** 2).sum()) for h in hosts))
    norm = torch.zeros(1, device="cuda")
    clip = B.Clip(srcs, dsts)
    clip.run(0.5, norm)
    assert abs(norm.item() - true) <= 9 * 2.0 ** -24 * true
    c = torch.tensor(factor(norm.item(), 0.5))
    for h, d in zip(hosts, dsts):
        assert torch.equal((h.float() * c).to(DT[dst]), d.cpu())
    assert clip.status() == 0
    clip.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [700, 40_000, 262_144])
def test_clips_that_follow_one_another_read_what_the_one_before_wrote(n):
    x = torch.randn(n) * 3
    bufs = [x.clone().cuda()] + [torch.full((n,), 7.0, device="cuda") for _ in range(8)]
    norms = torch.zeros(8, device="cuda")
    clips = [B.Clip([bufs[k]], [bufs[k + 1]]) for k in range(8)]
    for _ in range(20):
        for k in range(8):
            clips[k].run(64.0 / 2 ** k, norms[k:])
        h = x
        got = norms.cpu()
        for k in range(8):
            assert abs(got[k].item() - float(h.double().norm())) <= 9 * 2.0 ** -24 * float(h.double().norm())
            h = h * torch.tensor(factor(got[k].item(), 64.0 / 2 ** k))
            assert torch.equal(h, bufs[k + 1].cpu())
        for b in bufs[1:]:
            b.fill_(7.0)
    for c in clips:
        c.close()


@pytest.mark.gpu
def test_clip_on_streams():
    a, b = torch.randn(1_000_000, device="cuda"), torch.randn(1_000_000, device="cuda")
    out = [torch.empty_like(a) for _ in range(2)]
    clips, norms = [B.Clip([a], [out[0]]), B.Clip([b], [out[1]])], torch.zeros(2, device="cuda")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for k in range(2):
            clips[k].run(1.0, norms[k:], streams[k])
    torch.cuda.synchronize()
    for k, t in enumerate((a, b)):
        assert torch.equal(out[k].cpu(), t.cpu() * torch.tensor(factor(norms[k].item(), 1.0)))


# ---- refusals: no GPU needed ----------------------------------------------------------------------------

def test_aggregate_refusals():
    svc = B.Service(B.PS_DEVICE_NONE, 1, 1 << 20)
    lib = B.load()
    j = svc.register_job(num_workers=2)
    svc.register_block(j, 0, 100)
    ready = B.make_tasks([(j, 0)])
    call = lambda t, n, m, out=None: lib.ps_aggregate_clipped(svc.handle, t, n, m, out, None)  # noqa: E731
    assert call(ready, 1, 1.0) == B.PS_ERR_NOT_READY
    for w in range(2):
        svc.push(j, 0, w, 4096)
    for m in (0.0, -1.0, float("nan")):
        assert call(ready, 1, m) == B.PS_ERR_BAD_ARG
    assert call(ready, 1, 1.0, 2) == B.PS_ERR_BAD_ARG
    assert call(B.make_tasks([(j, 3)]), 1, 1.0) == B.PS_ERR_BAD_ARG
    assert call(B.make_tasks([(j, 0), (j, 0)]), 2, 1.0) == B.PS_ERR_DUPLICATE
    assert call(None, 1, 1.0) == B.PS_ERR_BAD_ARG
    assert call(ready, 1, 1.0) == B.PS_ERR_NO_DEVICE
    assert lib.ps_aggregate_clipped(None, ready, 1, 1.0, None, None) == B.PS_ERR_BAD_HANDLE
    assert lib.ps_round_run_clipped(svc.handle, 0, 1.0, None, None, None) == B.PS_ERR_BAD_ARG
    rid = svc.round_prepare(None, None, None, None, [(j, 0)])
    assert lib.ps_round_run_clipped(svc.handle, rid, 0.0, None, None, None) == B.PS_ERR_BAD_ARG
    assert lib.ps_round_run_clipped(svc.handle, rid, 1.0, None, None, None) == B.PS_ERR_NO_DEVICE


def test_clip_refusals():
    lib = B.load()
    h = C.c_void_p()
    ptrs = lambda *a: (C.c_void_p * len(a))(*a)  # noqa: E731
    ns = (C.c_size_t * 1)(10)
    make = lambda *a: lib.ps_clip_create(C.byref(h), *a)  # noqa: E731
    ok = ptrs(4096)
    bad, align = B.PS_ERR_BAD_ARG, B.PS_ERR_ALIGN
    assert lib.ps_clip_create(None, 0, 1, ok, 0, ok, 0, ns) == bad
    assert make(-1, 1, ok, 0, ok, 0, ns) == bad
    assert make(0, -1, ok, 0, ok, 0, ns) == bad
    assert make(0, 1, None, 0, ok, 0, ns) == bad
    assert make(0, 1, ok, 5, ok, 0, ns) == bad
    assert make(0, 1, ok, 0, ok, 5, ns) == bad
    assert make(0, 1, ptrs(None), 0, ok, 0, ns) == bad
    assert make(0, 1, ok, 0, ok, 1, ns) == bad                   # in place, but of another type
    assert make(0, 1, ptrs(4098), 0, ok, 0, ns) == align
    assert make(0, 1, ok, 0, ptrs(4097), 1, ns) == align
    assert lib.ps_clip_run(None, 1.0, None, None) == B.PS_ERR_BAD_HANDLE
    assert lib.ps_clip_status(None, None) == B.PS_ERR_BAD_HANDLE
    assert lib.ps_clip_destroy(None) == B.PS_ERR_BAD_HANDLE


@pytest.mark.gpu
def test_more_than_64_jobs_are_refused():
    svc = B.Service(0, 1, 1 << 20)
    grads = torch.ones(64, device="cuda")
    for j in range(65):
        svc.register_job(num_workers=1)
        svc.register_block(j, 0, 64)
        svc.push(j, 0, 0, grads)
    with pytest.raises(B.PsError) as e:
        svc.aggregate_clipped([(j, 0) for j in range(65)], 1.0)
    assert e.value.status == B.PS_ERR_TOO_LARGE
    norms = torch.zeros(64, device="cuda")
    svc.aggregate_clipped([(j, 0) for j in range(64)], 1.0, norms)       # the pushes are still there
    assert (norms == 8.0).all()
    svc.close()


@pytest.mark.gpu
def test_a_view_keeps_its_service():
    """A view of service-owned memory outlives the last other reference to the service."""
    import gc
    import weakref
    svc = B.Service(0, 1, 1 << 20)
    j = svc.register_job(num_workers=1)
    svc.register_block(j, 0, 64)
    view, seen = svc.view(svc.pull(j, 0), 64), weakref.ref(svc)
    del svc
    gc.collect()
    assert seen() is not None                # checked on the host before the memory is read
    assert (view == 0).all()
    del view
    gc.collect()
    assert seen() is None


@pytest.mark.gpu
@pytest.mark.parametrize("opt,dtype,W,shift", [
    (B.PS_SGD, B.PS_F32, 3, 0), (B.PS_ADAM, B.PS_BF16, 4, 0), (B.PS_SGD, B.PS_BF16, 5, 0), (B.PS_ADAM, B.PS_F32, 1, 0),
    (B.PS_SGD, B.PS_BF16, 2, 1), (B.PS_SGD, B.PS_F32, 1, 0), (B.PS_SGD, B.PS_BF16, 2, 0), (B.PS_ADAM, B.PS_BF16, 1, 0),
])
def test_large_launches_keep_or_read_again(opt, dtype, W, shift):
    """More elements than shared memory holds, chunks that end in fewer than a vector: shards of few bytes per element
    are read again, others' sums are kept; unaligned ones take the scalar path throughout."""
    world = World([hparams(opt, dtype, W)], [[8_000_003, 130_005, 7, 1]], seed=W)
    norms = torch.zeros(1, device="cuda")
    for limit in (0.5, 1e9):
        world.gradients(shift=shift)
        world.push()
        world.svc.aggregate_clipped(world.ready, limit, norms)
        world.check(limit, norms.cpu().numpy())
    assert world.svc.launch_info()["kernel"] == "clip_inline"
    world.svc.close()


class PretendFloats:
    """What the binding asks a tensor of norms for; its address is never used, because every call has to be refused."""

    def __init__(self, n, device=0, dtype=torch.float32, contiguous=True):
        self.n, self.device, self.dtype, self.contiguous = n, device, dtype, contiguous

    def get_device(self):
        return self.device

    def numel(self):
        return self.n

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 1 << 20


def wrong_norms(n):
    return [torch.zeros(n), np.zeros(n, f32), [0.0] * n, PretendFloats(n, device=-1), PretendFloats(n - 1),
            PretendFloats(n, dtype=torch.float64), PretendFloats(n, dtype=torch.bfloat16)] + [
                PretendFloats(n, contiguous=False)] * (n > 1)


def test_norms_go_to_floats_on_the_gpu_only():
    """A kernel writes one float per job: host memory, another type and too few entries would be writes out of place."""
    svc = B.Service(B.PS_DEVICE_NONE, 1, 1 << 20)
    every = []
    for j in range(3):
        assert svc.register_job(num_workers=1) == j
        for b in range(2):
            svc.register_block(j, b, 64)
            svc.push(j, b, 0, 4096)
            every.append((j, b))
    B._SVC_DEVICE[svc.handle] = 0                # the tensors' device: nothing here gets as far as a launch
    rid = svc.round_prepare(None, None, None, None, every)
    one = svc.round_prepare(None, None, None, None, every[:2])
    calls = [(3, lambda x: svc.aggregate_clipped(every, 1.0, x)), (3, lambda x: svc.aggregate_clipped(B.make_tasks(every), 1.0, x)),
             (3, lambda x: svc.round_run_clipped(rid, 1.0, x)), (1, lambda x: svc.aggregate_clipped(every[:2], 1.0, x)),
             (1, lambda x: svc.round_run_clipped(one, 1.0, x))]
    for n, call in calls:
        for x in wrong_norms(n) + [PretendFloats(n, device=1)]:
            with pytest.raises(B.PsError) as e:
                call(x)
            assert e.value.status == B.PS_ERR_BAD_ARG
        for x in (None, 4096, np.uint64(4096), PretendFloats(n), PretendFloats(n + 5)):
            with pytest.raises(B.PsError) as e:
                call(x)
            assert e.value.status == B.PS_ERR_NO_DEVICE
    svc.round_release(rid)
    handle = svc.handle
    assert [k for k in B._ROUND_JOBS if k[0] == handle] == [(handle, one)]
    svc.close()
    assert handle not in B._SVC_DEVICE and not [k for k in B._ROUND_JOBS if k[0] == handle]


def test_a_clips_norm_goes_to_a_float_on_its_gpu_only():
    B.load()
    clip = B.Clip.__new__(B.Clip)                # no handle: the library refuses what the binding lets through
    clip.handle, clip.device = None, 0
    for x in wrong_norms(1) + [PretendFloats(1, device=1)]:
        with pytest.raises(B.PsError) as e:
            clip.run(1.0, x)
        assert e.value.status == B.PS_ERR_BAD_ARG
    for x in (None, 4096, PretendFloats(3)):
        with pytest.raises(B.PsError) as e:
            clip.run(1.0, x)
        assert e.value.status == B.PS_ERR_BAD_HANDLE


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where there is no GPU")
def test_a_clips_tensors_lie_on_one_gpu():
    """One launch reads and writes them all; on a GPU that cannot reach one of them it would fault."""
    here, far, host = PretendFloats(8), PretendFloats(8, device=1), PretendFloats(8, device=-1)
    for t in (here, far, host):
        t.is_cuda = True
    for srcs, dsts, device in (([here, far], None, None), ([here], [far], None), ([far], [here], None), ([here], None, 1),
                               ([here], [here], 1), ([here, here], [here, far], 0), ([host], None, None),
                               ([torch.zeros(8)], None, None), ([here], [host], None)):
        with pytest.raises(B.PsError) as e:
            B.Clip(srcs, dsts, device)
        assert e.value.status == B.PS_ERR_BAD_ARG


DEVICES = r"""
import ctypes as C, sys
sys.path.insert(0, sys.argv[1])
from paper_2204_03211_b200 import binding as B
lib, pretend = B.load(), C.CDLL(sys.argv[2])


def current():
    d = C.c_int(-1)
    assert pretend.cudaGetDevice(C.byref(d)) == 0
    return d.value


for n in (1000, 10_000_000):                    # a short list, a long one
    for mine in (0, 1):
        assert pretend.cudaSetDevice(mine) == 0
        h, st = C.c_void_p(), C.c_int(-1)
        ptr, size, before = (C.c_void_p * 1)(1 << 20), (C.c_size_t * 1)(n), pretend.pretend_launches()
        assert lib.ps_clip_create(C.byref(h), 1, 1, ptr, 0, ptr, 0, size) == 0 and current() == mine
        assert lib.ps_clip_run(h, 1.0, None, None) == 0 and current() == mine
        assert pretend.pretend_launches() == before + 1 and pretend.pretend_launch_device() == 1
        assert lib.ps_clip_status(h, C.byref(st)) == 0 and st.value == 0 and current() == mine
        assert lib.ps_clip_destroy(h) == 0 and current() == mine
        assert lib.ps_clip_create(C.byref(h), 2, 1, ptr, 0, ptr, 0, size) == B.PS_ERR_CUDA and current() == mine
        assert lib.ps_clip_create(C.byref(h), 1, 0, None, 0, None, 0, None) == 0
        assert lib.ps_clip_run(h, 1.0, 1 << 20, None) == 0 and current() == mine
        assert lib.ps_clip_destroy(h) == 0
"""


def test_clips_leave_the_current_device_alone(tmp_path):
    """Other calls launch on the thread's current device: a clip on another one, or its collection, must not change it.
    On a runtime of two made-up devices that only keeps count."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    B.load()
    pretend = str(tmp_path / "pretend.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", pretend,
                    os.path.join(root, "tests", "c", "pretend_cuda.c")], check=True)
    run = subprocess.run([sys.executable, "-c", DEVICES, root, pretend], env=dict(os.environ, LD_PRELOAD=pretend),
                         capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


@pytest.mark.gpu
def test_a_round_after_one_that_gave_up_waiting():
    """With a limit of one cycle every CTA but the last gives up at the barrier and returns; the service reports it, and
    the next round, on blocks that the failed ones did not touch, is like any other: nothing is left over in the counters
    from which chunks are claimed (14 million elements: more chunks than CTAs)."""
    import time
    hp = hparams(B.PS_SGD, B.PS_F32, 2)
    world = World([hp, hp], [[9_000_001, 4_999_999], [5_000_003, 8_999_997, 5]], seed=11)
    svc, norms = world.svc, torch.zeros(1, device="cuda")
    failed, sound = [k for k in world.ready if k[0] == 0], [k for k in world.ready if k[0] == 1]
    keep = []                                # gradients that are in use until the launch has ended
    for _ in range(3):
        world.gradients()
        for (j, b, w), g in world.dev.items():
            if j == 0:
                svc.push(j, b, w, g)
        keep.append(world.dev)
        torch.cuda.synchronize()
        svc.set_option(B.PS_OPT_WAIT_CYCLES, 1)
        t0 = time.perf_counter()
        svc.aggregate_clipped(failed, 1.0, norms)
        assert svc.device_status() != 0 and time.perf_counter() - t0 < 5.0
    svc.set_option(B.PS_OPT_WAIT_CYCLES, 4_000_000_000)
    world.ref = {k: world.ref[k] for k in sound}
    world.jobs = [dict(hp, num_workers=2)] * 2
    for limit in (0.5, 1e9):
        world.gradients()
        world.push()
        svc.aggregate_clipped(sound, limit, norms)
        torch.cuda.synchronize()
        sums = world.sums()
        true = np.sqrt(sum((v.astype(np.float64) ** 2).sum() for v in sums.values()))
        assert abs(norms.item() - true) <= 1.01 * 2.0 ** -24 * true
        for k, r in world.ref.items():
            r.apply(sums[k], factor(norms.item(), limit))
            assert np.array_equal(svc.view(svc.pull(*k), len(r.p)).cpu().numpy(), r.p)
    svc.close()


def test_dynamic_shared_memory_says_how_it_is_aligned():
    """Every such array is accessed with 128-bit loads or copied to in bulk; an array of floats promises 4 bytes only, and
    where it starts then depends on the static arrays in front of it."""
    import glob
    import os
    import re
    src = os.path.join(os.path.dirname(os.path.abspath(B.__file__)), "csrc")
    found = [(os.path.basename(p), re.sub(r"\s+", " ", m)) for p in glob.glob(os.path.join(src, "*.cu*"))
             for m in re.findall(r"extern __shared__[^;]*;", open(p).read())]
    assert len(found) >= 5
    for name, text in found:
        if "unsigned char smem_raw[]" in text:       # bytes, whose kernel rounds their address up itself
            continue
        align = re.search(r"__align__\((\d+)\)", text)
        assert align and int(align.group(1)) >= 16, (name, text)


def true_norm(hosts):
    """The norm in 64 bits: squares of binary32 numbers are exact, math.fsum rounds their sum once."""
    import math
    return math.sqrt(math.fsum((np.concatenate([h.float().numpy() for h in hosts]).astype(np.float64) ** 2).tolist()))


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 1000, 524_288, 524_289, 1_000_003])
@pytest.mark.parametrize("values", ["0.000873832", "-3.3e37", "1.7e-42", "normal", "binades"])
def test_the_norm_is_the_nearest_float(src, n, values):
    """On both sides of the limit of short lists, aligned and not, with equal elements too, whose roundings would all
    point the same way.

    A thread adds at most a few thousand exact squares in binary64, the rest is a tree: a relative error of the sum below
    2^-53 * 4096 = 2^-41, half of that in the root, which at 2^24 units per binade is less than 2^-17 of a unit in the
    last place; the root's and the reference's own roundings (2^-52) are smaller still."""
    g = torch.Generator().manual_seed(n)
    if values == "normal":
        h = torch.randn(n, generator=g) * 0.01
    elif values == "binades":
        h = torch.randn(n, generator=g) * torch.exp2(torch.randint(-60, 60, (n,), generator=g).float())
    else:
        h = torch.full((n,), float(values))
    h = h.to(DT[src])
    true, norms = true_norm([h]), []
    for shift in (0, 1, 3):
        x = torch.cat([torch.zeros(shift, dtype=DT[src]), h]).cuda()[shift:]
        out, norm = torch.empty_like(x), torch.zeros(1, device="cuda")
        clip = B.Clip([x], [out])
        clip.run(0.05, norm)
        got = norm.cpu().numpy()[0]
        norms.append(got)
        if true < float(np.finfo(f32).max):
            assert abs(float(got) - true) <= (0.5 + 2.0 ** -10) * float(np.spacing(got)), (got, true)
        else:
            assert np.isinf(got)
        assert torch.equal(out.cpu(), (h.float() * torch.tensor(factor(got, 0.05))).to(DT[src]))
        clip.close()
    assert np.isinf(norms).all() or max(norms) - min(norms) <= np.spacing(norms[0])


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[1 << 20, 1 << 18, 4096, 3 << 20], [9_000_000, 1 << 18, 4096, 20_000_000]])
def test_clipped_rounds_are_profiled(sizes):
    """The device time that blocks are assigned by is recorded for clipped rounds too (with and without the buffer of kept
    sums), and only when it is asked for; it changes no result."""
    world = World([hparams(B.PS_SGD, B.PS_F32, 3)], [sizes], seed=4)
    svc, norms = world.svc, torch.zeros(1, device="cuda")
    for it, on in enumerate((0, 1, 1, 0)):
        svc.set_option(B.PS_OPT_PROFILE, on)
        world.gradients()
        world.push()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        e0.record()
        svc.aggregate_clipped(world.ready, 0.5, norms)
        e1.record()
        torch.cuda.synchronize()
        wall = e0.elapsed_time(e1) * 1e3
        prof = [svc.block_profile(*k) for k in world.ready]
        if not on:
            assert prof == [(0.0, 0.0)] * 4 and svc.job_profile(0) == (0.0, 0.0, 0)
        else:
            busy, span = [p[0] for p in prof], [p[1] for p in prof]
            assert min(busy) > 0 and min(span) > 0
            assert busy[3] > busy[0] > busy[1] > busy[2]            # ordered like the sizes
            assert max(span) <= wall * 1.05 + 5.0                  # (the timer's resolution)
            total, whole, n = svc.job_profile(0)
            assert n == 4 and abs(total - sum(busy)) < 1e-6
            assert total <= svc.launch_info()["grid"] * (wall * 1.05 + 5.0)
            assert max(span) - 1e-6 <= whole <= wall * 1.05 + 5.0
        world.check(0.5, norms.cpu().numpy())
    svc.close()


NOMEM = r"""
import ctypes as C, sys
import numpy as np
sys.path.insert(0, sys.argv[1])
from paper_2204_03211_b200 import binding as B
lib, new = B.load(), C.CDLL(sys.argv[2])
i32 = lambda *a: np.array(a, np.int32)
failures = 0
for k in range(1, 20):
    svc = B.Service(0, 1, 1 << 20)
    svc.set_option(B.PS_OPT_OVERLAP, 1)
    rounds = []
    for j in range(4):                          # two launches that run on, a round held back behind them, the one in question
        svc.register_job(num_workers=1)
        svc.register_block(j, 0, 64)
        rounds.append(svc.round_prepare(i32(j), i32(0), i32(0), np.array([1 << 20], np.uint64), [(j, 0)], B.PS_ROUND_INPUTS_COMPLETE))
    for r in rounds[:3]:
        svc.round_run(r)
    new.fail_new(k)
    rc = lib.ps_round_run_clipped(svc.handle, rounds[3], 1.0, None, None, None)
    new.fail_new(0)
    assert rc in (B.PS_OK, B.PS_ERR_NOMEM), rc
    failures += rc != B.PS_OK
    svc.push(3, 0, 0, 1 << 20)                  # DUPLICATE if a failed call had left its push behind
    svc.aggregate_clipped([(3, 0)], 1.0)
    svc.close()
assert failures >= 4 and rc == B.PS_OK, (failures, rc)      # (a sort does without its buffer; the last ones came after the call)
"""


def test_a_clipped_round_that_runs_out_of_memory_takes_its_pushes_back(tmp_path):
    """Every allocation of a clipped round fails once, those of the held-back round that goes out before it included."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    B.load()
    pretend, failing = str(tmp_path / "pretend.so"), str(tmp_path / "failing.so")
    subprocess.run(["gcc", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", pretend,
                    os.path.join(root, "tests", "c", "pretend_cuda.c")], check=True)
    subprocess.run(["g++", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", failing,
                    os.path.join(root, "tests", "c", "failing_new.cpp")], check=True)
    run = subprocess.run([sys.executable, "-c", NOMEM, root, failing],
                         env=dict(os.environ, LD_PRELOAD=pretend + ":" + failing), capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [0, 1])
def test_a_tensor_of_more_than_two_to_the_31_elements(shift):
    """Offsets past 32 bits on both sides: markers on either side of 2^31 and at the end, equal elements elsewhere, whose
    sum of squares is known."""
    n, v = (1 << 31) + 4099, 2.0 ** -10
    x = torch.full((n + shift,), v, device="cuda", dtype=torch.bfloat16)[shift:]
    at = [0, (1 << 31) - 1, 1 << 31, (1 << 31) + 2049, n - 1]
    for k, i in enumerate(at):
        x[i] = 8.0 * (k + 1)
    out, norm = torch.zeros(n + shift, device="cuda", dtype=torch.bfloat16)[shift:], torch.zeros(1, device="cuda")
    clip = B.Clip([x], [out])
    clip.run(1.0, norm)
    got = norm.cpu().numpy()[0]
    true = np.sqrt((n - len(at)) * v * v + sum((8.0 * (k + 1)) ** 2 for k in range(len(at))))
    # binary64 throughout (all squares here are multiples of 2^-20 and their sum is below 2^33: it is even exact)
    assert abs(float(got) - true) <= (0.5 + 2.0 ** -10) * float(np.spacing(got))
    c = torch.tensor(factor(got, 1.0))
    for k, i in enumerate(at):
        assert out[i].cpu() == (torch.tensor(8.0 * (k + 1)) * c).to(torch.bfloat16)
        out[i] = (torch.tensor(v) * c).to(torch.bfloat16)
    assert (out == (torch.tensor(v) * c).to(torch.bfloat16).item()).all()
    clip.close()


@pytest.mark.gpu
def test_clips_from_several_host_threads():
    """Handles are independent: one thread, stream and list each, results as on one thread."""
    import threading
    lists = [[torch.randn(n, device="cuda") for n in ns] for ns in ([100_000, 5], [700_000], [64] * 40, [3_000_001, 17])]
    torch.cuda.synchronize()
    errors = []

    def work(k):
        try:
            torch.cuda.set_device(0)
            stream, norm = torch.cuda.Stream(), torch.zeros(1, device="cuda")
            outs = [torch.empty_like(t) for t in lists[k]]
            torch.cuda.synchronize()
            for it in range(30):
                clip = B.Clip(lists[k], outs)
                limit = 0.5 + it
                clip.run(limit, norm, stream)
                stream.synchronize()
                c = torch.tensor(factor(norm.item(), limit))
                true = true_norm([t.cpu() for t in lists[k]]) if it == 0 else true
                assert abs(norm.item() - true) <= float(np.spacing(f32(norm.item())))
                assert all(torch.equal(o.cpu(), t.cpu() * c) for o, t in zip(outs, lists[k]))
                clip.close()
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(lists))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("n", [100, 65_537, 524_288, 600_001])
@pytest.mark.parametrize("shift", [0, 1])
def test_infinities_and_nans_in_short_and_long_lists(src, n, shift):
    """One of them at the start, at each place of a vector, in the tail: an infinity gives the factor 0, a NaN, also beside
    an infinity, NaN throughout."""
    h = torch.ones(n + shift, dtype=DT[src])
    x, out, norm = h.cuda()[shift:], torch.empty(n + shift, device="cuda", dtype=DT[src])[shift:], torch.zeros(1, device="cuda")
    clip = B.Clip([x, x[:0]], [out, out[:0]])
    inf, nan = float("inf"), float("nan")
    for at in [0, 1, 2, 3, 4, 7, n // 2, n - 1]:
        for bad in (inf, -inf, nan):
            x[at] = bad
            clip.run(1.0, norm)
            if np.isnan(bad):
                assert norm.isnan().all() and out.isnan().all()
            else:
                assert norm.isposinf().all() and out[at].isnan() and out.isnan().sum() == 1 and (out == 0).sum() == n - 1
                x[n - 1 - at] = nan
                clip.run(1.0, norm)
                assert norm.isnan().all() and out.isnan().all()
                x[n - 1 - at] = 1.0
            x[at] = 1.0
    clip.run(1e9, norm)                      # and nothing of it is left
    assert abs(norm.item() - n ** 0.5) <= 0.51 * float(np.spacing(f32(n ** 0.5))) and torch.equal(out, x)
    clip.close()
