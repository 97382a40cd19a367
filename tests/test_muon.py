"""PS_MUON jobs of the service: sums, momentum and the orthogonalised update.

The sum, the momentum and the statistics are defined to the bit (binary32, worker order) and compared for equality.  The
update comes from the orthogonalisation: the parameters may be off by lr * update_scale times what test_ortho.py allows
an fp32 result (a bound on the Frobenius norm), plus three roundings of a parameter."""
import numpy as np
import pytest
import torch

from paper_2204_03211_b200 import binding as B
from test_ortho import off, steps

gpu = pytest.mark.gpu
LR, MOM, WD = 0.02, 0.95, 0.1


class World:
    """One PS_MUON job and what its blocks should hold, in 64 bits from binary32 momentum."""

    def __init__(self, shapes, W=3, dtype=B.PS_F32, grad_scale=1.0, contexts=1, seed=0, svc=None, scales=None):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.shapes, self.W, self.dtype, self.gs = shapes, W, dtype, grad_scale
        self.svc = svc or B.Service(0, contexts, (1 << 22) + sum(8 * r * c for r, c in shapes))
        self.job = self.svc.register_job(opt=B.PS_MUON, grad_dtype=dtype, num_workers=W, lr=LR, momentum=MOM, weight_decay=WD,
                                         grad_scale=grad_scale)
        self.scales = scales or [0.2 * max(s) ** 0.5 for s in shapes]
        self.p, self.v = [], []
        for b, s in enumerate(shapes):
            p = self.rand(s) * 0.05
            self.svc.register_matrix(self.job, b, *s, 0, p, None if scales is None else scales[b])
            self.p.append(p.double())
            self.v.append(torch.zeros(s, device="cuda"))
        self.tol = [0.0] * len(shapes)
        self.keep = []

    def rand(self, s):
        return torch.randn(s, device="cuda", generator=self.gen)

    def shards(self, b, off_by=0):
        n = self.shapes[b][0] * self.shapes[b][1]
        t = torch.float32 if self.dtype == B.PS_F32 else torch.bfloat16
        out = []
        for _ in range(self.W):
            flat = torch.empty(n + off_by, device="cuda", dtype=t)[off_by:]
            flat.copy_((self.rand((n,)) * 1e-2).to(t))
            out.append(flat)
        return out

    def expect(self, b, shards):
        """One aggregate of block b: what its state has to be, and the norm of the sum."""
        g = shards[0].float()
        for s in shards[1:]:
            g = g + s.float()                               # binary32, worker order
        g = (g * np.float32(self.gs)).view(self.shapes[b])
        m = np.float32(MOM)
        v = self.v[b] * m + g
        u = g + v * m
        self.v[b] = v
        o = steps(u)
        rate = float(np.float32(float(np.float32(LR)) * float(np.float32(self.scales[b]))))
        decay = float(np.float32(1.0 - float(np.float32(LR)) * float(np.float32(WD))))
        self.p[b] = self.p[b] * decay - rate * o
        self.tol[b] = self.tol[b] * decay + rate * (4 * off(steps(u, torch.float32), o) + 2.0 ** -17) * float(o.norm()) + \
            3 * 2.0 ** -24 * float(self.p[b].norm())
        return float(g.double().square().sum())

    def push(self, b, shards):
        self.keep.append(shards)
        for w in reversed(range(self.W)):
            self.svc.push(self.job, b, w, shards[w])

    def step(self, blocks=None, off_by=0, stream=None, extra=()):
        blocks = list(range(len(self.shapes))) if blocks is None else blocks
        sq = {}
        for b in blocks:
            s = self.shards(b, off_by)
            self.push(b, s)
            sq[b] = self.expect(b, s)
        torch.cuda.synchronize()
        self.svc.aggregate([(self.job, b) for b in blocks] + list(extra), stream)
        return sq

    def check(self, steps_done=None, sq=None):
        torch.cuda.synchronize()
        assert self.svc.device_status() == 0
        for b, s in enumerate(self.shapes):
            n = s[0] * s[1]
            p = self.svc.view(self.svc.pull(self.job, b), n).view(s)
            v = self.svc.view(self.svc.block_state(self.job, b)[0], n).view(s)
            assert torch.equal(v, self.v[b]), "momentum of block %d" % b
            far = float((p.double() - self.p[b]).norm())
            assert far <= self.tol[b] + 1e-12, "block %d: off by %.3g, allowed %.3g" % (b, far, self.tol[b])
            if steps_done is not None:
                got, step = self.svc.block_stats(self.job, b)
                assert step == (steps_done[b] if isinstance(steps_done, list) else steps_done)
                if sq and b in sq:
                    assert abs(got - sq[b]) <= 1e-9 * sq[b]


@gpu
@pytest.mark.parametrize("W,dtype,gs,off_by", [(1, B.PS_F32, 1.0, 0), (4, B.PS_F32, 0.25, 0), (3, B.PS_BF16, 1.0, 0),
                                               (2, B.PS_F32, 1.0, 1), (5, B.PS_BF16, 0.5, 3), (40, B.PS_BF16, 1.0, 0)])
def test_rounds(W, dtype, gs, off_by):
    """Every kind of matrix, several iterations, aligned and unaligned shards."""
    w = World([(64, 64), (1, 200), (200, 1), (130, 257), (300, 70), (128, 512), (1, 1)], W, dtype, gs)
    for t in range(3):
        sq = w.step(off_by=off_by)
    w.check(3, sq)


@gpu
def test_large_blocks():
    w = World([(1024, 1024), (1024, 2048), (2048, 520)] * 3, 2)
    for t in range(2):
        w.step()
    w.check(2)


@gpu
def test_subsets_and_update_scales():
    """Blocks that become ready in changing groups: tables of several sets, the same workspace."""
    w = World([(96, 200), (64, 64), (300, 100), (40, 40)], 2, scales=[1.0, 0.0, -0.5, 2.0])
    done = [0] * 4
    for group in ([0, 1], [2], [3, 0], [0, 1], [1, 2, 3], [2], [0, 1, 2, 3], [3]):
        w.step(group)
        for b in group:
            done[b] += 1
    w.check(done)


@gpu
def test_more_sets_than_are_kept():
    w = World([(8, 8)] * 12, 1)
    done = [0] * 12
    for k in range(80):                                     # 66 different pairs
        group = sorted({k % 12, (k * 5 + 1 + k // 12) % 12})
        w.step(group)
        for b in group:
            done[b] += 1
    w.check(done)


@gpu
@pytest.mark.parametrize("overlap", [0, 1])
def test_beside_other_jobs(overlap):
    """One list with blocks of PS_MUON, SGD and Adam jobs: the others get what they get alone, to the bit."""
    svc, alone = B.Service(0, 1, 1 << 26), B.Service(0, 1, 1 << 26)
    svc.set_option(B.PS_OPT_OVERLAP, overlap)
    w = World([(100, 60), (64, 256)], 2, svc=svc)
    kinds = [dict(opt=B.PS_SGD, lr=0.1, momentum=0.9, weight_decay=1e-4), dict(opt=B.PS_ADAM, lr=1e-3)]
    jobs = [(svc.register_job(num_workers=2, **k), alone.register_job(num_workers=2, **k)) for k in kinds]
    init = torch.randn(5000, device="cuda")
    for a, b in jobs:
        svc.register_block(a, 0, 5000, 0, init)
        alone.register_block(b, 0, 5000, 0, init)
    for t in range(3):
        grads = [[torch.randn(5000, device="cuda") for _ in range(2)] for _ in jobs]
        for (a, b), gs in zip(jobs, grads):
            for k, g in enumerate(gs):
                svc.push(a, 0, k, g)
                alone.push(b, 0, k, g)
        w.step(extra=[(a, 0) for a, _ in jobs])
        alone.aggregate([(b, 0) for _, b in jobs])
        svc.join()
        torch.cuda.synchronize()
    w.check(3)
    for a, b in jobs:
        assert torch.equal(svc.view(svc.pull(a, 0), 5000), alone.view(alone.pull(b, 0), 5000))
    kinds = {v["kernel"]: v["launches"] for v in svc.launch_stats(5)}
    assert kinds["ps_aggregate_muon_kernel"] == 3


@gpu
@pytest.mark.parametrize("flags", [0, B.PS_ROUND_INPUTS_COMPLETE])
def test_prepared_rounds_and_streams(flags):
    """Rounds replayed on changing streams without waiting in between: they follow one another by themselves."""
    w = World([(150, 90), (64, 300)], 3)
    w.svc.set_option(B.PS_OPT_OVERLAP, 1)
    bufs = [w.shards(b) for b in range(2)]
    blocks = np.repeat(np.arange(2, dtype=np.int32), 3)
    ranks = np.tile(np.arange(3, dtype=np.int32), 2)
    ptrs = np.array([bufs[b][r].data_ptr() for b, r in zip(blocks, ranks)], np.uint64)
    rnd = w.svc.round_prepare(np.full(6, w.job, np.int32), blocks, ranks, ptrs, [(w.job, 0), (w.job, 1)], flags)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for t in range(7):
        for b in range(2):
            w.expect(b, bufs[b])
        w.svc.round_run(rnd, streams[t % 3])
    w.check(7)
    out = np.zeros(2, np.uint64)
    w.svc.round_run(rnd, None, out)
    for b in range(2):
        w.expect(b, bufs[b])
    assert list(out) == [w.svc.pull(w.job, b) for b in range(2)]
    w.check(8)


@gpu
def test_migration_and_unregistration():
    w = World([(64, 100), (120, 50), (33, 77)], 2, contexts=2)
    w.step()
    w.svc.migrate_blocks([(w.job, 0), (w.job, 2)], 1)
    w.step()
    w.svc.migrate_block(w.job, 0, 0)
    w.step()
    w.check(3)
    # to another service and back, with momentum and step
    other = World([(120, 50)], 2)
    n, step = w.svc.block_export(w.job, 1)
    lane = torch.empty(n, device="cuda", dtype=torch.uint8)
    w.svc.block_export(w.job, 1, lane, n)
    torch.cuda.synchronize()
    other.svc.block_import(other.job, 0, lane, n, step)
    other.p[0], other.v[0], other.tol[0] = w.p[1], w.v[1], w.tol[1]
    other.step()
    other.check(4)
    w.svc.unregister_block(w.job, 1)
    w.svc.register_matrix(w.job, 1, 50, 20)
    w.shapes[1], w.scales[1] = (50, 20), 0.2 * 50 ** 0.5
    w.p[1], w.v[1], w.tol[1] = torch.zeros(50, 20, device="cuda", dtype=torch.float64), torch.zeros(50, 20, device="cuda"), 0.0
    w.step()
    w.check([4, 1, 4])


@gpu
def test_push_from_host_memory_and_profile():
    w = World([(48, 80)], 2)
    w.svc.set_option(B.PS_OPT_PROFILE, 1)
    s = w.shards(0)
    host = [x.cpu() for x in s]
    for k, h in enumerate(host):
        w.svc.push_host(w.job, 0, k, h)
    w.svc.aggregate([(w.job, 0)])
    w.expect(0, s)
    w.check(1)
    busy, span = w.svc.block_profile(w.job, 0)
    assert busy > 0 and span > 0


@gpu
def test_not_finite_gradients_stay_in_their_block():
    w = World([(40, 40), (64, 30)], 1)
    bad = torch.zeros(1600, device="cuda")
    bad[7] = float("inf")
    good = w.shards(1)
    w.svc.push(w.job, 0, 0, bad)
    w.push(1, good)
    w.expect(1, good)
    w.svc.aggregate([(w.job, 0), (w.job, 1)])
    torch.cuda.synchronize()
    assert w.svc.device_status() == 0
    assert w.svc.view(w.svc.pull(w.job, 0), 1600).isnan().all()
    p = w.svc.view(w.svc.pull(w.job, 1), 64 * 30).view(64, 30)
    assert float((p.double() - w.p[1]).norm()) <= w.tol[1]


@gpu
def test_a_failed_call_changes_nothing():
    w = World([(40, 40), (64, 30)], 2)
    s = w.shards(0)
    w.push(0, s)
    for ready, status in (([(w.job, 0), (w.job, 1)], B.PS_ERR_NOT_READY), ([(w.job, 0), (w.job, 0)], B.PS_ERR_DUPLICATE)):
        with pytest.raises(B.PsError) as e:
            w.svc.aggregate(ready)
        assert e.value.status == status
    with pytest.raises(B.PsError) as e:
        w.svc.aggregate_clipped([(w.job, 0)], 1.0)
    assert e.value.status == B.PS_ERR_BAD_ARG
    w.expect(0, s)
    w.svc.aggregate([(w.job, 0)])
    w.check([1, 0])


def planning():
    s = B.Service(B.PS_DEVICE_NONE, 1, 1 << 24)
    return s, s.register_job(opt=B.PS_MUON, num_workers=2)


def refused(status, call, *a):
    with pytest.raises(B.PsError) as e:
        call(*a)
    assert e.value.status == status


def test_registration_refuses():
    s, j = planning()
    sgd = s.register_job(opt=B.PS_SGD, num_workers=2)
    bad = B.PS_ERR_BAD_ARG
    refused(bad, s.register_block, j, 0, 100)
    refused(bad, s.register_matrix, sgd, 0, 10, 10)
    refused(bad, s.register_matrix, 9, 0, 10, 10)
    for rows, cols in ((0, 5), (5, 0), (-1, 5), ((1 << 20) + 1, 1)):
        refused(bad, s.register_matrix, j, 0, rows, cols)
    for scale in (float("nan"), float("inf")):
        refused(bad, s.register_matrix, j, 0, 4, 4, 0, None, scale)
    refused(bad, s.register_matrix, j, 0, 4, 4, 1)
    refused(B.PS_ERR_NOMEM, s.register_matrix, j, 0, 4096, 4096)
    s.register_matrix(j, 0, 30, 40)
    refused(B.PS_ERR_DUPLICATE, s.register_matrix, j, 0, 30, 40)
    refused(bad, s.register_job, 3)


def test_planning_knows_matrices():
    """Arena ranges, pushes, readiness and the chunk table work without a device; computing does not."""
    s, j = planning()
    s.register_matrix(j, 0, 300, 100)
    s.register_matrix(j, 1, 7, 9)
    assert s.arena_info(0)[0] == 2 * (120_064 + 256)         # parameters and momentum
    for b in range(2):
        for w in range(2):
            s.push(j, b, w, 4096 * (1 + b * 2 + w))
    refused(B.PS_ERR_BAD_ARG, s.push_rows, j, 0, 0, 4096, 1, 100, 4096)
    plan = s.plan([(j, 0), (j, 1)])
    assert sum(c.elem_count for c in plan) == 30_063
    refused(B.PS_ERR_NO_DEVICE, s.aggregate, [(j, 0), (j, 1)])
    refused(B.PS_ERR_NO_DEVICE, s.aggregate_clipped, [(j, 0)], 1.0)
    n, step = s.block_export(j, 0)
    assert n == 2 * 120_064 and step == 0


def test_noalloc_refuses():
    d = B.ps_job_desc(B.PS_MUON, B.PS_F32, 1, 0.1, 0.9, 0, 0, 0, 0, 1)
    refused(B.PS_ERR_BAD_ARG, B.ps_aggregate_block_noalloc, d, 1, 16, 4096, 8192, None, [4096])


def test_sharded_service_registers_what_it_owns():
    from paper_2204_03211_b200 import sharded
    sh = sharded.ShardedService(1, 2, B.PS_DEVICE_NONE, 1, 1 << 20)
    j = sh.register_job(opt=B.PS_MUON, grad_dtype=B.PS_F32, num_workers=1, lr=0.1, momentum=0.9, weight_decay=0.0)
    sh.set_owners({(j, 0): 0, (j, 1): 1})
    assert not sh.register_matrix(j, 0, 8, 4) and sh.register_matrix(j, 1, 4, 8)
    assert sh.svc.arena_info(0)[0] == 2 * 256
    refused(B.PS_ERR_BAD_ARG, sh.register_block, j, 1, 32)
    sh.close()

FAILURES = r"""
import ctypes as C, sys
import numpy as np
sys.path.insert(0, sys.argv[1])
from paper_2204_03211_b200 import binding as B
B.load()
fake = C.CDLL(sys.argv[2])
fake.last_copy_from.restype = C.c_void_p
SIDES = [int(n) for n in sys.argv[3].split(",")]
i32 = lambda *a: np.array(a, np.int32)
at = 1 << 20


def world():
    svc = B.Service(0, 1, 1 << 22)
    svc.register_job(opt=B.PS_MUON, num_workers=2)
    svc.register_job(opt=B.PS_SGD, num_workers=2)
    for b, n in enumerate(SIDES):
        svc.register_matrix(0, b, n, n)
    svc.register_block(1, 0, 5000)
    ready = [(0, b) for b in range(len(SIDES))] + [(1, 0)]
    pushes = [(j, b, w) for j, b in ready for w in range(2)]
    return svc, ready, [i32(*c) for c in zip(*pushes)], np.full(len(pushes), at, np.uint64)


def steps(svc, ready):
    return [svc.block_export(j, b)[1] for j, b in ready]


def call(how, svc, ready, lists, ptrs):
    if how == "aggregate":
        svc.aggregate(ready)
    elif how == "round":
        svc.round(*lists, ptrs, ready)
    else:
        svc.round_run(svc.round_prepare(*lists, ptrs, ready))


for how in ("aggregate", "round", "prepared"):
    k, kinds = 0, set()
    while True:
        k += 1
        svc, ready, lists, ptrs = world()
        if how == "aggregate":
            svc.push_batch(*lists, ptrs)
        before = fake.launches_seen()
        fake.fail_cuda(k)
        status = B.PS_OK
        try:
            call(how, svc, ready, lists, ptrs)
        except B.PsError as e:
            status = e.status
        failed = fake.calls_seen() >= k
        fake.fail_cuda(0)
        launched, table, done = fake.launches_seen() - before, fake.last_copy_from(), steps(svc, ready)
        if not failed:
            assert status == B.PS_OK and done == [1] * len(ready), (how, k, status, done)
            break
        assert status in (B.PS_ERR_NOMEM, B.PS_ERR_CUDA), (how, k, status)
        kinds.add((status, launched))
        # what went out has taken its pushes: the other job's launch is first, then the sums
        assert done == [int(launched >= 2)] * len(SIDES) + [int(launched >= 1)], (how, k, launched, done)
        if status == B.PS_ERR_NOMEM:
            assert launched == 0, (how, k, launched)
        # what did not is as it was, and everybody can go on
        if how == "aggregate":
            missing = [i for i, (j, b) in enumerate(zip(lists[0], lists[1])) if done[ready.index((j, b))]]
            svc.push_batch(*[c[missing] for c in lists], ptrs[missing])
        call(how, svc, ready, lists, ptrs)
        assert steps(svc, ready) == [d + 1 for d in done], (how, k)
        if launched >= 2:                       # the sums may still read their table
            assert fake.last_copy_from() != table, (how, k)
        svc.close()
    assert {n for _, n in kinds} >= {0, 1, 2} and (B.PS_ERR_NOMEM, 0) in kinds and k > 10, (how, k, kinds)
"""


@pytest.mark.parametrize("sides", ["40,64", "40,200"])
def test_what_fails_half_way_leaves_every_block_usable(tmp_path, sides):
    """One list with blocks of two jobs, small matrices and larger ones; every call of the CUDA runtime that can fail does,
    once.  Pushes are consumed by what was launched and by nothing else, and no launch's table is written again too early."""
    made_up_runtime(tmp_path, FAILURES, sides)


def made_up_runtime(tmp_path, script, *args, front="failing_cuda.c"):
    """Runs `script` on the runtime of tests/c/pretend_cuda.c, with another of those files in front of it."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    B.load()
    libs = []
    for name in (front, "pretend_cuda.c"):
        libs.append(str(tmp_path / (name + ".so")))
        subprocess.run(["g++" if name.endswith("pp") else "gcc", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-o", libs[-1],
                        os.path.join(root, "tests", "c", name), "-ldl"], check=True)
    run = subprocess.run([sys.executable, "-c", script, root, libs[0], *args],
                         env=dict(os.environ, LD_PRELOAD=":".join(libs)), capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


CHANGING_SETS = r"""
import ctypes as C, random, sys
sys.path.insert(0, sys.argv[1])
from paper_2204_03211_b200 import binding as B
B.load()
fake = C.CDLL(sys.argv[2])
LAYERS, PER = 24, 6
N = LAYERS * PER
svc = B.Service(0, 2, 1 << 25)
svc.register_job(opt=B.PS_MUON, num_workers=1)
for b in range(N):
    svc.register_matrix(0, b, 40 + b % 7, 64 if b % PER else 200)
rng = random.Random(3)


def go(blocks):
    for b in blocks:
        svc.push(0, b, 0, 1 << 20)
    svc.aggregate([(0, b) for b in blocks])


def costs(call):
    before = fake.mallocs_seen(), fake.stops_seen(), fake.copies_seen()
    call()
    return tuple(a - b for a, b in zip((fake.mallocs_seen(), fake.stops_seen(), fake.copies_seen()), before))


def iteration(shuffled):
    everything = list(range(N))
    layers = [everything[i:i + PER] for i in range(0, N, PER)]
    lists = [everything] + layers + [[b] for b in everything]
    for l in lists:
        if shuffled:
            rng.shuffle(l)
        go(l)
    return len(lists)


for sort in (1, 0):
    svc.set_option(B.PS_OPT_SORT_TASKS, sort)
    count = iteration(False)
    for k in range(20):                     # task tables in flight may still grow, each slot once
        go(list(range(N)))
    # a step that walks all of it again, in the same order or as things become ready, costs one table per aggregate
    for shuffled in (False, True, True):
        assert costs(lambda: iteration(shuffled)) == (0, 0, count), (sort, shuffled)
# options that do not touch the chunks keep the tables, too
svc.set_option(B.PS_OPT_PROFILE, 1)
svc.set_option(B.PS_OPT_OVERLAP, 1)
assert costs(lambda: iteration(True)) == (0, 0, count)
# a block that moves drops the sets that it belongs to
svc.migrate_block(0, 7, 1)
assert costs(lambda: go([8])) == (0, 0, 1)
mallocs, stops, copies = costs(lambda: go([7]))
assert stops == 0 and copies > 1
assert costs(lambda: go([7])) == (0, 0, 1)
# sets that are new every time: tables are made, but what was there before is not freed, and nothing is waited for
for k in range(3 * N):
    go(rng.sample(range(N), 5))
mallocs, stops, copies = costs(lambda: [go(rng.sample(range(N), 5)) for _ in range(500)])
assert stops == 0 and mallocs == 0, (mallocs, stops)
svc.close()
"""


def test_sets_of_blocks_that_change_from_call_to_call(tmp_path):
    """144 matrices, all at once, layer by layer and one by one, listed in changing orders; then sets that never recur.  Tables
    are made once for a set, and making them neither frees memory nor waits for the device."""
    made_up_runtime(tmp_path, CHANGING_SETS)


@gpu
def test_listed_in_any_order_with_options_that_change():
    w = World([(64, 64), (300, 70), (64, 64), (128, 512), (200, 130), (64, 64)], 2)
    gen = np.random.default_rng(0)
    for t, (option, value) in enumerate(((B.PS_OPT_SORT_TASKS, 0), (B.PS_OPT_CHUNK_ELEMS, 1024), (B.PS_OPT_PROFILE, 1),
                                         (B.PS_OPT_CHUNK_ELEMS, 0), (B.PS_OPT_SORT_TASKS, 1), (B.PS_OPT_OVERLAP, 1))):
        w.svc.set_option(option, value)
        w.step([int(b) for b in gen.permutation(6)])
    w.check(6)


@gpu
def test_sets_that_never_recur():
    """More sets than are kept, in a row without waiting: tables are made in the memory of older ones."""
    w = World([(8, 8), (16, 8), (8, 150), (24, 24), (9, 9), (130, 8), (8, 40), (12, 12), (8, 9), (20, 20)], 1)
    bufs = [w.shards(b) for b in range(10)]
    done, k = [0] * 10, 0
    for mask in list(range(1, 150)) * 2:
        group = [b for b in range(10) if (mask * 37 % 1023 + 1) >> b & 1]
        for b in group:
            w.push(b, bufs[b])
            w.expect(b, bufs[b])
            done[b] += 1
        w.svc.aggregate([(w.job, b) for b in reversed(group)])
    w.check(done)


def work(shape):
    m, n = min(shape), max(shape)
    return 5.0 * (3 * m * m * n + m ** 3)


@gpu
@pytest.mark.parametrize("shapes", [[(1024, 1024), (512, 512), (512, 2048), (1536, 700)],       # the general form
                                    [(64, 256), (128, 128), (128, 900), (100, 256)]])           # the small one
def test_device_times_cover_the_orthogonalisation(shapes):
    """What the planner weighs tasks by: a span as long as the call takes on the GPU, not as the sums alone do, and CTA-time
    that fits into it, four units per SM; results are untouched."""
    w = World(shapes, 2)
    w.step()                                                # (tables)
    w.svc.set_option(B.PS_OPT_PROFILE, 1)
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for b in range(len(shapes)):
        s = w.shards(b)
        w.push(b, s)
        w.expect(b, s)
    torch.cuda.synchronize()
    e0.record()
    w.svc.aggregate([(w.job, b) for b in range(len(shapes))])
    e1.record()
    torch.cuda.synchronize()
    wall = e0.elapsed_time(e1) * 1e3
    busy, span, blocks = w.svc.job_profile(w.job)
    assert blocks == len(shapes)
    # (the clock that kernels read ticks once a microsecond or so; the events enclose the launches of three kernels)
    assert 0.5 * wall - 20.0 <= span <= wall * 1.05 + 5.0
    each = [w.svc.block_profile(w.job, b) for b in range(len(shapes))]
    assert abs(sum(b for b, _ in each) - busy) <= 1e-6 * busy and max(s for _, s in each) <= span + 1e-6
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert busy <= 4 * sms * (wall * 1.05 + 5.0) * 2        # (the CTAs before the products are more than four on an SM)
    w.check(2)
    w.svc.set_option(B.PS_OPT_PROFILE, 0)
    w.step()
    torch.cuda.synchronize()
    assert w.svc.job_profile(w.job) == (0.0, 0.0, 0)
    w.check(3)
    # alone, the sums take a part of it that can be told: the larger product has the longer time
    if shapes[0] == (1024, 1024):
        w.svc.set_option(B.PS_OPT_PROFILE, 1)
        alone = []
        for b in range(len(shapes)):
            for _ in range(2):
                w.step([b])
            torch.cuda.synchronize()
            alone.append(w.svc.block_profile(w.job, b)[0])
        order = sorted(range(len(shapes)), key=lambda b: work(shapes[b]))
        assert alone[order[0]] < alone[order[-1]]


@gpu
def test_rounds_from_several_host_threads():
    """One service, a job, a stream and a thread each, lists that share nothing but the workspace."""
    import threading
    svc = B.Service(0, 1, 1 << 26)
    worlds = [World(shapes, 2, seed=k, svc=svc) for k, shapes in
              enumerate(([(64, 64), (300, 70)], [(128, 512)], [(200, 130), (33, 50), (8, 8)], [(513, 260)]))]
    bufs = [[w.shards(b) for b in range(len(w.shapes))] for w in worlds]
    torch.cuda.synchronize()
    errors, ROUNDS = [], 12

    def work(k):
        try:
            torch.cuda.set_device(0)
            w, stream = worlds[k], torch.cuda.Stream()
            for t in range(ROUNDS):
                ready = list(range(len(w.shapes)))
                for b in ready:
                    for r in range(w.W):
                        svc.push(w.job, b, r, bufs[k][b][r])
                svc.aggregate([(w.job, b) for b in (ready if t % 2 else ready[::-1])], stream)
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(worlds))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for k, w in enumerate(worlds):
        for _ in range(ROUNDS):
            for b in range(len(w.shapes)):
                w.expect(b, bufs[k][b])
        w.check(ROUNDS)


NOMEM = r"""
import ctypes as C, sys
sys.path.insert(0, sys.argv[1])
from paper_2204_03211_b200 import binding as B
lib, new = B.load(), C.CDLL(sys.argv[2])
svc = B.Service(0, 1, 1 << 22)
muon, sgd = svc.register_job(opt=B.PS_MUON, num_workers=2), svc.register_job(num_workers=2)
used = 0
for block in range(40):                         # (growth of the tables is among them)
    for call in (lambda: lib.ps_register_matrix(svc.handle, muon, block, 8, 8, 0, None, 1.0),
                 lambda: lib.ps_register_block(svc.handle, sgd, block, 64, 0, None)):
        k = rc = 0
        while k == 0 or rc != B.PS_OK:
            k += 1
            new.fail_new(k)
            rc = call()
            new.fail_new(0)
            assert rc in (B.PS_OK, B.PS_ERR_NOMEM), rc
            assert svc.arena_info(0)[0] == used + (512 if rc == B.PS_OK else 0), (block, k)
        assert k > 3 and call() == B.PS_ERR_DUPLICATE
        used += 512
svc.close()
"""


def test_registration_that_runs_out_of_memory(tmp_path):
    """Every allocation of a registration fails once: NOMEM, nothing is taken, and the next attempt succeeds."""
    made_up_runtime(tmp_path, NOMEM, front="failing_new.cpp")
