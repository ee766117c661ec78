"""Tensor sets and handles of the training-step operators on the GPU where their life is not the simplest one: several host threads,
side streams, an Ops that goes before its sets, parameters of mixed kinds, long chunks.

Tolerances (u = 2^-24) are those of test_gpu_training.py: norm 12 u, m 4 u and v 5 u of the magnitudes of their terms, p 3 u |p| + u |p1| +
24 u of the update with those magnitudes in m's place.
"""
import os
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import torch
    from paper_2609_23898_b200 import training
    assert torch.cuda.is_available()
    o = training.Ops()
    yield o
    o.status()


def test_a_set_used_at_once_on_a_side_stream(ops):
    """A non-blocking stream does not wait for the copies that made the set (2.6 MB of records here)."""
    import torch
    from paper_2609_23898_b200 import training as R
    flat = torch.full((20000 * 100,), 2.0, device="cuda")
    grads = list(flat.split(100))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(5):
            o = R.Ops()
            s = R.TensorSet(o, grads=grads)
            out = s.grad_norm(1.0)
            o.status()
            n64 = 2 * np.sqrt(flat.numel())
            assert abs(out[0].item() - n64) <= 12 * U * n64


def f64(t):
    return t.detach().double().cpu().numpy()


FIRST_PRODUCTS = """
import ctypes as C, threading, torch
from paper_2609_23898_b200 import cerar, training as R
torch.cuda.init()
n = 16
jobs = []
for i in range(n):
    o = R.Ops()
    q, = o.quantize(torch.ones(16, 128, device="cuda"), R.BY_ROW)
    jobs.append((o, q, torch.zeros(16, 16, device="cuda"), torch.cuda.Stream()))
torch.cuda.synchronize()
start, status = threading.Barrier(n), [None] * n
def work(i):
    o, q, out, s = jobs[i]
    start.wait()
    status[i] = cerar.lib.cerar_fp8_matmul(o._h, q.at, 0, q.at, 1, out.data_ptr(), 0, 16, 0, s.cuda_stream)
threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert status == [0] * n, status
assert all(bool((j[2] == 128).all()) for j in jobs)
"""


FIRST_AGGREGATION = """
import threading, torch
from paper_2609_23898_b200 import cerar
N, c, d = 4, 32, 32 * 4096
plan = cerar.Plan.create(N, c, cerar.EPSILON, 1e-2)
plan.set_kernel_mode(3)
g = torch.randn(N, d, device="cuda")
out, want, ws = torch.empty_like(g), torch.empty_like(g), torch.empty(plan.workspace_bytes(d) // 4, device="cuda")
s = torch.cuda.current_stream().cuda_stream
errors = []
def work():
    try:
        plan.allreduce_sim(g, d, out, d, ws, d, 1.0 / N, s)
    except Exception as e:
        errors.append(e)
t = threading.Thread(target=work)
t.start()
t.join()
assert not errors, errors
plan.allreduce_sim(g, d, want, d, ws, d, 1.0 / N, s)
torch.cuda.synchronize()
plan.device_status(s)
assert torch.equal(out, want)
"""


def test_first_products_of_several_threads():
    """Each thread with a handle of its own, as the header allows: the first call of a process sets up what all of them share."""
    for _ in range(3):
        r = subprocess.run([sys.executable, "-c", FIRST_PRODUCTS], cwd=ROOT, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stdout + r.stderr


def test_first_aggregation_of_a_thread():
    """The tensor-core contraction from a host thread that has not touched the device before."""
    r = subprocess.run([sys.executable, "-c", FIRST_AGGREGATION], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


def test_a_plan_used_at_once_on_a_side_stream():
    """The aggregation's own tables, as those of a set above."""
    import torch
    from paper_2609_23898_b200 import cerar
    N, c, d = 4, 8, 8 * 4096
    g = torch.randn(N, d, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    with torch.cuda.stream(side):
        for _ in range(5):
            plan = cerar.Plan.create(N, c, cerar.EPSILON, 1e-2)
            out, ws = torch.empty_like(g), torch.empty(plan.workspace_bytes(d) // 4, device="cuda")
            plan.allreduce_sim(g, d, out, d, ws, d, 1.0 / N, side.cuda_stream)
            plan.device_status(side.cuda_stream)
            outs.append(out)
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_an_ops_that_goes_before_its_sets():
    import torch
    from paper_2609_23898_b200 import cerar, training as R
    o = R.Ops()
    s = R.TensorSet(o, grads=[torch.ones(10, device="cuda")], params=[torch.ones(10, device="cuda")])
    o.destroy()
    for call in (lambda: s.grad_norm(1.0), lambda: s.adamw(lr=0.1, step=1), lambda: s.set_grads([torch.zeros(10, device="cuda")]), o.status):
        with pytest.raises(cerar.CerarError) as e:
            call()
        assert e.value.status == 1


def test_parameters_of_mixed_kinds_in_one_set(ops):
    """bfloat16 with and without a master copy and float32 in one set: the bits of a set of each kind (the stochastic one comes
    first: its random bits go by its place)."""
    import torch
    from paper_2609_23898_b200 import training as R
    torch.manual_seed(3)
    sizes = [700, 1300, 5, 2049]
    grads = [torch.randn(n, device="cuda") * 1e-3 for n in sizes]
    start = [torch.randn(n, device="cuda") * 0.02 for n in sizes]
    types = [torch.bfloat16, torch.bfloat16, torch.float32, torch.bfloat16]
    with_master = [False, True, False, True]

    def run(which, masters_of):
        p = [start[i].to(types[i]) for i in which]
        c = masters_of([start[i].clone() if with_master[i] else None for i in which])
        s = R.TensorSet(ops, grads=[grads[i] for i in which], params=p, masters=c, weight_decay=[0.1 * i for i in which])
        for step in (1, 2):
            s.adamw(lr=1e-2, step=step, seed=step)
        m = [s.m[a:a + grads[i].numel()] for a, i in zip(s.state_offsets, which)]
        return p, c or [None] * len(which), m

    p, c, m = run(range(4), lambda x: x)
    for which, masters_of in (([0], lambda x: None), ([1, 3], lambda x: x), ([2], lambda x: [None])):
        ps, cs, ms = run(which, masters_of)
        for j, i in enumerate(which):
            assert torch.equal(p[i], ps[j]) and torch.equal(m[i], ms[j])
            assert (c[i] is None) == (cs[j] is None) == (not with_master[i])
            if with_master[i]:
                assert torch.equal(c[i], cs[j]) and torch.equal(p[i], c[i].bfloat16())
    with pytest.raises(ValueError):
        R.TensorSet(ops, grads=grads, params=[s.bfloat16() for s in start], masters=[None, start[1][:5], None, None])
    with pytest.raises(ValueError):
        R.TensorSet(ops, grads=grads, params=[s.bfloat16() for s in start], masters=[None] * 3)
    with pytest.raises(TypeError):
        R.TensorSet(ops, grads=grads, params=[s.bfloat16() for s in start], masters=[None, start[1].bfloat16(), None, None])


LONG = [8192 * 1200 + 5, 7, 2049, 8193, 8191, 0, 3, 10_000_001, 16384]        # 19.9 million: chunks of four times 2048 elements


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_norm_of_long_chunks(ops, dtype, offset):
    import torch
    from paper_2609_23898_b200 import training as R
    torch.manual_seed(offset)
    flat = torch.randn(sum(LONG) + 8, device="cuda").to(getattr(torch, dtype))
    flat[:offset] = float("nan")
    flat[offset + sum(LONG):] = float("nan")
    g = list(flat[offset:offset + sum(LONG)].split(LONG))
    s = R.TensorSet(ops, grads=g)
    n64 = float(flat[offset:offset + sum(LONG)].double().square().sum().sqrt())
    a = s.grad_norm(1.0)
    assert abs(a[0].item() - n64) <= 12 * U * n64 and a[2].item() == 1 and torch.equal(a, s.grad_norm(1.0))
    for at in (0, 8192 * 1200 + 4, sum(LONG[:7]) + 9_999_999, sum(LONG) - 1):   # every element counts
        keep = flat[offset + at].clone()
        flat[offset + at] = float("inf")
        assert s.grad_norm(1.0)[2].item() == 0
        flat[offset + at] = keep


@pytest.mark.parametrize("grad", ["float32", "bfloat16"])
@pytest.mark.parametrize("param,offset", [("float32", 0), ("float32", 1), ("master", 0), ("master", 2)])
def test_adamw_of_long_chunks(ops, param, offset, grad):
    import torch
    from paper_2609_23898_b200 import training as R
    torch.manual_seed(7 + offset)
    total = sum(LONG)
    cut = lambda t: list(t[offset:offset + total].split(LONG))  # noqa: E731
    gflat = (torch.randn(total + 8, device="cuda") * 1e-3).to(getattr(torch, grad))
    pflat = torch.randn(total + 8, device="cuda") * 0.02
    cflat = pflat.bfloat16() if param == "master" else None
    edges = [torch.cat((t[:offset], t[offset + total:])) for t in (pflat, cflat) if t is not None]
    s = R.TensorSet(ops, grads=cut(gflat), params=cut(cflat if param == "master" else pflat), masters=cut(pflat) if param == "master" else None,
                    weight_decay=[0.1 * (i % 2) for i in range(len(LONG))])
    s.m.normal_(std=3e-4)
    s.v.exponential_(1.0).mul_(2.5e-7)
    m0, v0, p0 = s.m.double(), s.v.double(), pflat.double()
    clip = torch.tensor([2.0, 0.5, 1.0], device="cuda")
    s.adamw(lr=3e-3, step=3, clip=clip)
    at = offset
    for i, n in enumerate(LONG):
        a = s.state_offsets[i]
        g, m, v, p = 0.5 * gflat[at:at + n].double(), m0[a:a + n], v0[a:a + n], p0[at:at + n]
        terms = (0.9 * m).abs() + (0.1 * g).abs()
        m1, v1 = 0.9 * m + (1 - 0.9) * g, 0.95 * v + (1 - 0.95) * g * g
        root = (v1 / (1 - 0.95 ** 3)).sqrt() + 1e-8
        p1 = p - 3e-3 * float(np.float32(0.1 * (i % 2))) * p - 3e-3 / (1 - 0.9 ** 3) * m1 / root
        bound = 3 * U * p.abs() + 24 * U * 3e-3 / (1 - 0.9 ** 3) * terms / root + U * p1.abs()
        assert bool(((s.m[a:a + n].double() - m1).abs() <= 4 * U * terms).all())
        assert bool(((s.v[a:a + n].double() - v1).abs() <= 5 * U * v1).all())
        assert bool(((pflat[at:at + n].double() - p1).abs() <= bound).all())
        at += n
    now = [torch.cat((t[:offset], t[offset + total:])) for t in (pflat, cflat) if t is not None]
    assert all(torch.equal(x, y) for x, y in zip(edges, now))
    if param == "master":
        assert torch.equal(cflat[offset:offset + total], pflat[offset:offset + total].bfloat16())


@pytest.mark.parametrize("grad", ["float32", "bfloat16"])
@pytest.mark.parametrize("param,bits", [("float32", 32), ("master", 32), ("float32", 8), ("master", 8)])
def test_adamw_rounds_as_the_header_says(ops, param, bits, grad):
    """32-bit states have the bits of the formula in binary32, operation by operation (numpy's are rounded to nearest).  Parameters of zero
    show the update by itself: within 2^-21 of its formula in 64 bits from those states (root 2^-23, its product with the correction 2^-24,
    quotient 2^-22, last product 2^-24)."""
    import torch
    from paper_2609_23898_b200 import training as R
    f = np.float32
    n, lr, b1, b2, step = 100_000, 3e-3, 0.9, 0.95, 7
    rng = np.random.default_rng(bits)
    g = torch.from_numpy((rng.standard_normal(n) * 1e-3).astype(f)).cuda().to(getattr(torch, grad))
    p = torch.zeros(n, device="cuda", dtype=torch.float32 if param == "float32" else torch.bfloat16)
    c = torch.zeros(n, device="cuda") if param == "master" else None
    s = R.TensorSet(ops, grads=[g], params=[p], masters=None if c is None else [c], state_bits=bits)
    if bits == 32:
        s.m.normal_(std=3e-4)
        s.v.exponential_(1.0).mul_(2.5e-7)
        m, v = s.m.cpu().numpy()[:n], s.v.cpu().numpy()[:n]
    else:
        s.adamw(lr=lr, betas=(b1, b2), eps=1e-8, step=1, seed=1)           # states that have something in them
        p.zero_()
        if c is not None:
            c.zero_()
        wide = lambda t, w: (t.float() * w.repeat_interleave(256)).cpu().numpy()[:n]  # noqa: E731
        m, r = wide(s.m, s.m_scale), wide(s.v, s.v_scale)
        v = r * r
    s.adamw(lr=lr, betas=(b1, b2), eps=0.0, step=step, seed=2)
    g = g.float().cpu().numpy()
    m = f(b1) * m + f(1 - b1) * g
    v = f(b2) * v + f(1 - b2) * (g * g)
    if bits == 32:
        assert np.array_equal(s.m.cpu().numpy()[:n], m) and np.array_equal(s.v.cpu().numpy()[:n], v)
    m, v = m.astype(np.float64), v.astype(np.float64)
    want = -float(f(lr / (1 - b1 ** step))) * m / (np.sqrt(v) * float(f(1 / np.sqrt(1 - b2 ** step))))
    got = f64(p if c is None else c)
    assert (np.abs(got - want) <= 2.0 ** -21 * np.abs(want)).all()
    if c is not None:
        assert torch.equal(p, c.bfloat16())
