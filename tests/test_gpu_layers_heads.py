"""Norms of queries and keys for each head with the rotation by position (layers.head_norm, head_norm_backward, HeadNorm) against the
formulas in 64 bits, on the GPU.

Tolerances, in units u = 2^-24 and for a head of d values.  The sum of squares is within (d + 1) u of itself (d products and additions in any
order), the mean and + eps 2 u more, the root of a relative error e has e / 2, the reciprocal root's own error is 2 u at most: r is
within (d + 3) / 2 + 2 <= d / 2 + 4 of itself.  z = w r x: 2 more.  y = a c - b s: 2 more of |a| + |b|, the table's rounding 1: every y is within
(d / 2 + 9) u (|a| + |b|), and half a step of the result.  Gradient: dz has 3 u (|dy_a| + |dy_b|), n = r x (d / 2 + 5) u; dn = w dz one more; the mean of
dn n over d values: (d + d / 2 + 11) u mean |dn n|; dx = r (dn - n mean): with all that, (2 d + 24) u r (|dn| + |n| mean |dn n|) where dn's bound
is taken from |dy_a| + |dy_b|.  dw: a sum of N rows' terms dz n in any order: (N + d / 2 + 10) u sum (|dy_a| + |dy_b|) |n|.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ops():
    import torch
    from paper_2609_23898_b200 import training
    assert torch.cuda.is_available()
    o = training.Ops()
    yield o
    o.status()


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def partner(x, rot, pairs):
    """The value that each one is turned with (itself beyond the turned ones)."""
    import torch
    if rot == 0:
        return x
    t = x[..., :rot]
    p = t.roll(rot // 2, -1) if pairs == "halves" else t.unflatten(-1, (rot // 2, 2)).flip(-1).flatten(-2)
    return torch.cat((p, x[..., rot:]), -1)


def turn(z, table, pos, pairs, sign):
    """z with its first values turned: y_a = a c - b s, y_b = b c + a s (sign = -1: back)."""
    import torch
    rot = 0 if table is None else 2 * table.size(1)
    if rot == 0:
        return z
    c, s = table[pos.clamp(0, table.size(0) - 1).long()].double().unbind(-1)
    if pairs == "halves":
        c, s = torch.cat((c, c), -1), torch.cat((-s, s), -1)
    else:
        c, s = torch.stack((c, c), -1).flatten(-2), torch.stack((-s, s), -1).flatten(-2)
    y = z[..., :rot] * c[:, None] + sign * partner(z, rot, pairs)[..., :rot] * s[:, None]
    return torch.cat((y, z[..., rot:]), -1)


def exact(x, w, table, pos, pairs, eps):
    import torch
    x = x.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + float(np.float32(eps)))
    w = torch.ones(x.size(-1), dtype=torch.float64, device=x.device) if w is None else w.double()
    z = x * r * w
    live = (pos >= 0)[:, None, None]
    y = torch.where(live, turn(z, table, pos, pairs, 1), 0.0)
    rot = 0 if table is None else 2 * table.size(1)
    return y, z.abs() + partner(z, rot, pairs).abs()


def exact_grad(dy, x, w, table, pos, pairs, eps):
    import torch
    x, d = x.double(), x.size(-1)
    live = (pos >= 0)[:, None, None]
    x, dy = torch.where(live, x, 0.0), torch.where(live, dy.double(), 0.0)
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + float(np.float32(eps)))
    w = torch.ones(d, dtype=torch.float64, device=x.device) if w is None else w.double()
    n, dz = x * r, turn(dy, table, pos, pairs, -1)
    rot = 0 if table is None else 2 * table.size(1)
    size = (dy.abs() + partner(dy, rot, pairs).abs())
    dn = dz * w
    dx = torch.where(live, r * (dn - n * (dn * n).mean(-1, keepdim=True)), 0.0)
    sn = size * w.abs()
    return dx, r * (sn + n.abs() * (sn * n.abs()).mean(-1, keepdim=True)), (dz * n).sum((0, 1)), (size * n.abs()).sum((0, 1))


def near(got, want, size, units):
    import torch
    bound = size * (units * U) + want.abs() * (torch.finfo(got.dtype).eps / 2) * 1.01 + 1e-300
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (float((off / bound).max()), off.shape)


CASES = [  # tokens, query heads, key heads, dim, rotated, pairs, type, weights' type
    (1, 1, 1, 2, 2, "halves", "f32", "f32"), (1, 16, 4, 128, 128, "halves", "bf16", "bf16"), (5, 3, 2, 64, 64, "neighbours", "bf16", "f32"),
    (77, 4, 1, 80, 80, "halves", "bf16", "bf16"), (33, 7, 7, 72, 72, "neighbours", "bf16", "bf16"), (129, 5, 3, 96, 32, "halves", "f32", "f32"),
    (40, 2, 2, 96, 32, "neighbours", "bf16", "f32"), (19, 3, 1, 256, 256, "halves", "bf16", None), (9, 2, 1, 512, 512, "neighbours", "f32", "bf16"),
    (21, 2, 3, 512, 128, "halves", "bf16", "bf16"), (50, 3, 2, 34, 34, "halves", "bf16", "bf16"), (31, 1, 2, 6, 2, "neighbours", "f32", "f32"),
    (64, 2, 1, 26, 26, "halves", "bf16", "f32"), (11, 9, 4, 128, 0, "halves", "bf16", "bf16"), (700, 8, 2, 16, 16, "halves", "bf16", "bf16"),
    (6000, 9, 1, 64, 64, "halves", "bf16", "bf16"), (3000, 1, 3, 128, 96, "neighbours", "bf16", "f32"), (1200, 10, 2, 512, 512, "halves", "bf16", None),
    (3, 2, 2, 510, 254, "halves", "f32", "f32"), (2500, 12, 4, 128, 128, "halves", "f32", "f32"), (2500, 32, 8, 128, 64, "halves", "bf16", "bf16"),
]


def inputs(tokens, hq, hk, dim, rotated, ty, wty, layout, seed=0):
    import torch
    from paper_2609_23898_b200 import layers
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + tokens)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    if layout == "joint":                     # slices of one projection
        qkv = normal(tokens, hq + 2 * hk, dim).to(types()[ty])
        q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
    elif layout == "by head":                 # heads outermost in memory
        q, k = (normal(h, tokens, dim).to(types()[ty]).transpose(0, 1) for h in (hq, hk))
    elif layout == "odd":                     # rows on no boundary but their elements'
        q, k = (normal(tokens, h, dim + 1).to(types()[ty])[:, :, 1:] for h in (hq, hk))
    else:                                     # a head's values not next to one another
        q, k = (normal(tokens, dim, h).to(types()[ty]).transpose(1, 2) for h in (hq, hk))
    w = [None, None] if wty is None else [(1 + 0.3 * normal(dim)).to(types()[wty]) for _ in range(2)]
    dy = [normal(tokens, h, dim).to(types()[ty]) for h in (hq, hk)]
    return q, k, w, dy, g


@pytest.mark.parametrize("layout", ["joint", "by head", "odd", "transposed"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_and_gradient(ops, case, layout):
    import torch
    from paper_2609_23898_b200 import layers
    tokens, hq, hk, dim, rotated, pairs, ty, wty = case
    q, k, w, (dq, dk), g = inputs(tokens, hq, hk, dim, rotated, ty, wty, layout)
    eps = 1e-5
    table = layers.rotation_table(ops, 3000, rotated) if rotated else None
    pos = torch.randint(-300, 3000, (tokens,), device="cuda", generator=g)
    if layout == "odd":
        pos = pos.int()
    y = layers.head_norm(ops, q, k, w[0], w[1], table, pos, eps=eps, pairs=pairs)
    for got, x, wi in zip(y, (q, k), w):
        want, size = exact(x, wi, table, pos, pairs, eps)
        assert got.shape == x.shape and got.dtype == x.dtype
        near(got, want, size, dim / 2 + 9)
    dw = [torch.full((dim,), 3.0, device="cuda") for _ in range(2)]
    dx = layers.head_norm_backward(ops, dq, dk, q, k, w[0], w[1], table, pos, dwq=dw[0], dwk=dw[1], eps=eps, pairs=pairs)
    for got, gw, x, wi, dy in zip(dx, dw, (q, k), w, (dq, dk)):
        want, size, dww, dws = exact_grad(dy, x, wi, table, pos, pairs, eps)
        near(got, want, size, 2 * dim + 24)
        near(gw, dww + 3, dws + 3, tokens * x.size(1) + dim / 2 + 12)
    if layout == "joint":                     # without accumulate, into bfloat16, one of them not wanted; one part alone
        b = torch.full((dim,), 9.0, device="cuda").bfloat16()
        layers.head_norm_backward(ops, dq, dk, q, k, w[0], w[1], table, pos, dwk=b, accumulate=False, eps=eps, pairs=pairs)
        near(b, dww, dws, tokens * hk + dim / 2 + 12)
        alone, none = layers.head_norm(ops, q, None, w[0], None, table, pos, eps=eps, pairs=pairs)
        assert none is None and torch.equal(alone, y[0])
        dalone, none = layers.head_norm_backward(ops, dq, None, q, None, w[0], None, table, pos, eps=eps, pairs=pairs)
        assert none is None and torch.equal(dalone, dx[0])


def test_gradient_against_differences(ops):
    """The derivative along a direction of sum(y c), from the exact forward in 64 bits at two nearby points, against dx and dw."""
    import torch
    from paper_2609_23898_b200 import layers
    for pairs in ("halves", "neighbours"):
        q, k, w, (dq, dk), g = inputs(13, 3, 2, 24, 24, "f32", "f32", "joint")
        table, pos = layers.rotation_table(ops, 50, 16), torch.arange(13, device="cuda")
        dw = [torch.zeros(24, device="cuda") for _ in range(2)]
        dx = layers.head_norm_backward(ops, dq, dk, q, k, w[0], w[1], table, pos, dwq=dw[0], dwk=dw[1], pairs=pairs)
        h = 1e-5
        for x, wi, dy, dxi, dwi in zip((q, k), w, (dq, dk), dx, dw):
            vx, vw = torch.randn(x.shape, device="cuda", dtype=torch.float64), torch.randn(24, device="cuda", dtype=torch.float64)
            f = [(exact(x.double() + s * h * vx, wi.double() + s * h * vw, table, pos, pairs, 1e-6)[0] * dy.double()).sum() for s in (1, -1)]
            along = float(f[0] - f[1]) / (2 * h)
            got = float((dxi.double() * vx).sum() + (dwi.double() * vw).sum())
            assert abs(along - got) < 1e-4 * (float((dxi.double() * vx).abs().sum()) + 1)


def test_rotation_table(ops):
    """Against 64 bits: cosines and sines are off by half a step of binary32 at most, also of far positions."""
    import torch
    from paper_2609_23898_b200 import layers
    for first, rows, dim, base in ((0, 5, 2, 10000.0), (0, 300, 128, 10000.0), (1_000_000, 50, 64, 500000.0), (-3, 7, 6, 100.0)):
        t = layers.rotation_table(ops, rows, dim, base=base, first=first)
        freq = torch.tensor([base ** (-2.0 * j / dim) for j in range(dim // 2)], dtype=torch.float64)
        a = torch.arange(first, first + rows, dtype=torch.float64)[:, None] * freq
        want = torch.stack((a.cos(), a.sin()), -1).cuda()
        assert t.shape == (rows, dim // 2, 2)
        assert float((t.double() - want).abs().max()) <= U + 1e-9 * (abs(first) + rows) * 1e-6
    t = layers.rotation_table(ops, 4, 4, freqs=[0.5, 0.0])
    assert torch.equal(t[:, 1], torch.tensor([1.0, 0.0], device="cuda").expand(4, 2))
    assert layers.rotation_table(ops, 0, 8).shape == (0, 4, 2) and layers.rotation_table(ops, 3, 0).shape == (3, 0, 2)
    for bad in (dict(dim=5), dict(dim=4, freqs=[1.0]), dict(dim=-2)):
        with pytest.raises(ValueError):
            layers.rotation_table(ops, 3, **bad)
    from paper_2609_23898_b200 import cerar
    with pytest.raises(cerar.CerarError):
        layers.rotation_table(ops, 3, 4, freqs=[float("nan"), 1.0])
    with pytest.raises(cerar.CerarError):
        layers.rotation_table(ops, 3, 514)


def test_positions(ops):
    """Of every token; of one sequence for all; counted; with leading dimensions; a single new token; strided."""
    import torch
    from paper_2609_23898_b200 import layers
    table = layers.rotation_table(ops, 64, 32)
    q = torch.randn(3, 20, 4, 32, device="cuda").bfloat16()
    k = torch.randn(3, 20, 2, 32, device="cuda").bfloat16()
    one = torch.arange(20, device="cuda")
    a = layers.head_norm(ops, q, k, None, None, table, one)
    for pos in (None, one.expand(3, 20), one.int(), torch.stack((one, one), 1)[:, 0]):
        b = layers.head_norm(ops, q, k, None, None, table, pos)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    t = layers.head_norm(ops, q[:, 7:8], k[:, 7:8], None, None, table, one[7:8])
    assert torch.equal(t[0], a[0][:, 7:8]) and torch.equal(t[1], a[1][:, 7:8])
    e = layers.head_norm(ops, q[:0], k[:0], None, None, table)
    assert e[0].shape == (0, 20, 4, 32)
    e = layers.head_norm(ops, q[:, :, :0], k, None, None, table)
    assert e[0].shape == (3, 20, 0, 32) and torch.equal(e[1], a[1])
    dw = torch.full((32,), 4.0, device="cuda")
    layers.head_norm_backward(ops, q[:0], k[:0], q[:0], k[:0], None, None, table, dwq=dw, accumulate=False)
    assert not bool(dw.any())


def test_positions_beyond_the_table_and_padding(ops):
    import torch
    from paper_2609_23898_b200 import cerar, layers
    table = layers.rotation_table(ops, 10, 16)
    q = torch.randn(4, 2, 16, device="cuda")
    ops.status()
    y, _ = layers.head_norm(ops, q, None, None, None, table, torch.tensor([9, 10, -1, 2 ** 40], device="cuda"))
    with pytest.raises(cerar.CerarError) as e:
        ops.status()
    assert e.value.status == 10 and bool(y[0].any()) and not bool(y[1:].any())
    q[1:] = float("nan")                                           # rows of padding may hold anything
    w = torch.ones(16, device="cuda")
    for how in (0, 1):
        dw = torch.zeros(16, device="cuda")
        dx, _ = layers.head_norm_backward(ops, q if how else torch.ones_like(q), None, q if how else q.nan_to_num(), None, w, None, table,
                                          torch.tensor([9, -1, -5, -2 ** 40], device="cuda"), dwq=dw)
        assert not bool(dx[1:].any()) and bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dw).all())
    ops.status()


def test_rows_that_are_zero_or_not_finite(ops):
    import torch
    from paper_2609_23898_b200 import layers
    q = torch.zeros(3, 1, 8, device="cuda")
    q[1, 0, 2] = float("inf")
    q[2, 0, 1] = float("nan")
    y, _ = layers.head_norm(ops, q, None, None, None, None)
    assert not bool(y[0].any()) and bool(torch.isnan(y[1, 0, 2])) and bool(torch.isnan(y[2]).all())
    dy = torch.ones_like(q)
    dx, _ = layers.head_norm_backward(ops, dy, None, q, None, None, None, None, eps=1e-4)
    assert torch.allclose(dx[0], torch.full_like(dx[0], 100.0), rtol=1e-6)


def test_results_in_place_of_slices(ops):
    """out: slices of a joint gradient; what lies beside them stays."""
    import torch
    from paper_2609_23898_b200 import layers
    qkv = torch.randn(30, 8, 64, device="cuda").bfloat16()
    q, k = qkv[:, :4], qkv[:, 4:6]
    table = layers.rotation_table(ops, 30, 64)
    dy = torch.randn(30, 6, 64, device="cuda").bfloat16()
    a = layers.head_norm_backward(ops, dy[:, :4], dy[:, 4:], q, k, None, None, table)
    joint = torch.full_like(qkv, 2.0)
    b = layers.head_norm_backward(ops, dy[:, :4], dy[:, 4:], q, k, None, None, table, out=(joint[:, :4], joint[:, 4:6]))
    assert torch.equal(joint[:, :4], a[0]) and torch.equal(joint[:, 4:6], a[1]) and bool((joint[:, 6:] == 2).all()) and b[0].data_ptr() == joint.data_ptr()
    c = layers.head_norm(ops, q, k, None, None, table, out=(joint[:, :4], joint[:, 4:6]))
    d = layers.head_norm(ops, q, k, None, None, table)
    assert torch.equal(c[0], d[0]) and torch.equal(joint[:, 4:6], d[1])


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_table_on_any_boundary(ops, pairs):
    """A table that begins 8 bytes behind a boundary gives what one on it gives."""
    import torch
    from paper_2609_23898_b200 import layers
    q, k, w, dy, _ = inputs(300, 6, 2, 128, 128, "bf16", "bf16", "joint")
    table = layers.rotation_table(ops, 300, 128)
    off = torch.empty(table.numel() + 2, device="cuda")[2:].view_as(table).copy_(table)
    assert off.data_ptr() % 16 == 8
    for t in (table, off):
        dw = [torch.zeros(128, device="cuda") for _ in range(2)]
        got = [*layers.head_norm(ops, q, k, *w, t, pairs=pairs), *layers.head_norm_backward(ops, *dy, q, k, *w, t, dwq=dw[0], dwk=dw[1], pairs=pairs), *dw]
        if t is table:
            want = got
    pos = torch.arange(300, device="cuda")
    for x, wi, d, a, dwb in zip((q, k), w, dy, got[2:4], got[4:]):
        exact_dx, size, exact_dw, dws = exact_grad(d, x, wi, table, pos, pairs, 1e-6)
        near(a, exact_dx, size, 2 * 128 + 24)
        near(dwb, exact_dw, dws, 300 * x.size(1) + 64 + 12)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("ty,dim,heads,pairs,layout", [("bf16", 128, 21, "halves", "joint"), ("bf16", 64, 3, "neighbours", "by head"), ("f32", 128, 9, "halves", "by head"),
                                                       ("bf16", 70, 5, "halves", "odd"), ("f32", 30, 2, "neighbours", "odd"), ("bf16", 512, 7, "halves", "joint")])
@pytest.mark.parametrize("tokens", [1, 333])
def test_in_place(ops, ty, dim, heads, pairs, layout, tokens):
    """Results where q and k, gradients where either q and k or their results' gradients were: the same bits as next to them."""
    import torch
    from paper_2609_23898_b200 import layers
    q, k, w, dy, _ = inputs(tokens, heads, 2, dim, dim, ty, "f32", layout)
    table, pos = layers.rotation_table(ops, 400, dim), torch.arange(tokens, device="cuda").flip(0)
    pos[::5] = -1
    want = layers.head_norm(ops, q, k, *w, table, pos, pairs=pairs)
    grads = layers.head_norm_backward(ops, *dy, q, k, *w, table, pos, pairs=pairs)
    over = [d.clone() for d in dy]
    layers.head_norm_backward(ops, *over, q, k, *w, table, pos, pairs=pairs, out=over)
    assert torch.equal(over[0], grads[0]) and torch.equal(over[1], grads[1])
    # (a second pair with the same strides as q and k)
    q2, k2, _, _, _ = inputs(tokens, heads, 2, dim, dim, ty, "f32", layout)
    layers.head_norm(ops, q2, k2, *w, table, pos, pairs=pairs, out=(q2, k2))
    assert torch.equal(q2, want[0]) and torch.equal(k2, want[1])
    layers.head_norm_backward(ops, *dy, q, k, *w, table, pos, pairs=pairs, out=(q, k))
    assert torch.equal(q, grads[0]) and torch.equal(k, grads[1])


@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("dty", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,hq,hk", [(1, 1, 1), (77, 6, 2), (2000, 16, 16), (50, 3, 0)])
def test_weights_that_queries_and_keys_share(ops, tokens, hq, hk, dty, accumulate):
    """One weight vector and one dw for both: it gets the two sums.  Terms are 0, 1 and -1 but for r, two steps of binary32 off one at most; fewer than
    256 of them, so sums are within 256 (2^-22 + 2^-24 256) < 2^-7 of whole numbers below 256, which bfloat16 holds."""
    import torch
    from paper_2609_23898_b200 import cerar, layers
    dim = 64
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    q, k = (torch.where(torch.rand(tokens, h, dim, device="cuda", generator=g) < 0.5, -1.0, 1.0) for h in (hq, hk))
    dq, dk = (torch.where(torch.rand(tokens, h, dim, device="cuda", generator=g) < 1 / (8 * tokens), 1.0, 0.0) for h in (hq, hk))
    w = torch.ones(dim, device="cuda")
    apart = [torch.full((dim,), 3.0, device="cuda") for _ in range(2)]
    # eps so small beside 1 that r is 1
    layers.head_norm_backward(ops, dq, dk, q, k, w, w, None, dwq=apart[0], dwk=apart[1], eps=1e-12, accumulate=accumulate)
    start = 3.0 if accumulate else 0.0
    dw = torch.full((dim,), 3.0, device="cuda", dtype=types()[dty])
    layers.head_norm_backward(ops, dq, dk, q, k, w, w, None, dwq=dw, dwk=dw, eps=1e-12, accumulate=accumulate)
    sums = [(d * x).double().sum((0, 1)) for d, x in ((dq, q), (dk, k))]
    assert float((apart[0] - start - sums[0]).abs().max()) <= 2 ** -7 and float((dw.double() - start - sums[0] - sums[1]).abs().max()) <= 2 ** -7
    both = torch.zeros(dim + 8, device="cuda", dtype=types()[dty])
    with pytest.raises(cerar.CerarError):
        layers.head_norm_backward(ops, dq, dk, q, k, w, w, None, dwq=both[:dim], dwk=both[8:], eps=1e-12)


def test_autograd(ops):
    import torch
    from paper_2609_23898_b200 import layers
    q, k, w, (dq, dk), _ = inputs(12, 3, 2, 32, 32, "f32", "f32", "joint")
    q, k = q.contiguous().requires_grad_(), k.contiguous().requires_grad_()
    table, pos = layers.rotation_table(ops, 50, 32), torch.arange(12, device="cuda")
    dw = [torch.zeros(32, device="cuda") for _ in range(2)]
    y = layers.HeadNorm.apply(q, k, w[0], w[1], ops, table, pos, dw[0], dw[1])
    torch.autograd.backward(y, (dq, dk))
    ref = [torch.zeros(32, device="cuda") for _ in range(2)]
    want = layers.head_norm_backward(ops, dq, dk, q.detach(), k.detach(), w[0], w[1], table, pos, dwq=ref[0], dwk=ref[1])
    assert torch.equal(q.grad, want[0]) and torch.equal(k.grad, want[1]) and torch.equal(dw[0], ref[0]) and torch.equal(dw[1], ref[1])
    # only one of the results is used; inputs without gradients; queries alone
    for d in dw:
        d.zero_()
    y = layers.HeadNorm.apply(q.detach(), k.detach(), w[0], w[1], ops, table, pos, dw[0], dw[1])
    y[0].backward(dq)
    assert torch.equal(dw[0], ref[0]) and not bool(dw[1].any())
    dw[0].zero_()
    y, none = layers.HeadNorm.apply(q, None, w[0], None, ops, table, pos, dw[0])
    assert none is None
    y.backward(dq)
    assert torch.equal(dw[0], ref[0])
    with pytest.raises(ValueError):
        layers.HeadNorm.apply(q, k, w[0].clone().requires_grad_(), w[1], ops, table, pos)
    with pytest.raises(RuntimeError):
        y = layers.HeadNorm.apply(q, k, w[0], w[1], ops, table, pos)
        g, = torch.autograd.grad(y[0].sum(), [q], create_graph=True)
        torch.autograd.grad(g.sum(), [q])


def test_refusals(ops):
    import torch
    from paper_2609_23898_b200 import cerar, layers
    q, k = torch.randn(5, 2, 16, device="cuda"), torch.randn(5, 1, 16, device="cuda")
    w = torch.ones(16, device="cuda")
    table = layers.rotation_table(ops, 10, 16)

    def bad(error, *a, **b):
        with pytest.raises(error):
            layers.head_norm(ops, *a, **b)

    bad(TypeError, q.half(), k.half(), w, w, table)
    bad(ValueError, q, k.bfloat16(), w, w, table)
    bad(ValueError, q, k[:4], w, w, table)
    bad(ValueError, q[0], None, w, None, table)
    bad(ValueError, q.cpu(), k, w, w, table)
    bad(ValueError, q, k, w[:8], w, table)
    bad(TypeError, q, k, w, w.bfloat16(), table)
    bad(ValueError, q, k, w, w, table.double())
    bad(ValueError, q, k, w, w, table, torch.zeros(4, dtype=torch.int64, device="cuda"))
    bad(TypeError, q, k, w, w, table, torch.zeros(5, device="cuda"))
    bad(ValueError, q, k, w, w, table, pairs="thirds")
    bad(ValueError, q, k, w, w, table, out=(q[:4], k))
    bad(cerar.CerarError, q, k, w, w, layers.rotation_table(ops, 10, 18))
    bad(cerar.CerarError, q, k, w, w, table, eps=0.0)
    bad(cerar.CerarError, q, k, w, w, table, eps=float("nan"))
    bad(cerar.CerarError, torch.randn(2, 2, 514, device="cuda"), None, None, None, None)
    bad(cerar.CerarError, torch.randn(2, 2, 15, device="cuda"), None, None, None, None)
    bad(cerar.CerarError, q, None, None, None, None, out=(torch.zeros(2, 16, device="cuda").expand(5, 2, 16), None))
    with pytest.raises(ValueError):
        layers.head_norm_backward(ops, q, None, q, k, w, w, table)
    with pytest.raises(ValueError):
        layers.head_norm_backward(ops, q[:4], k, q, k, w, w, table)
    with pytest.raises(TypeError):
        layers.head_norm_backward(ops, q, k, q, k, w, w, table, dwq=torch.zeros(16, device="cuda"), dwk=torch.zeros(16, device="cuda").bfloat16())


def test_captured_and_replayed(ops):
    import torch
    from paper_2609_23898_b200 import layers
    q, k, w, (dq, dk), _ = inputs(500, 4, 2, 64, 64, "bf16", "bf16", "joint")
    table, pos = layers.rotation_table(ops, 1000, 64), torch.arange(500, device="cuda")
    dw = [torch.zeros(64, device="cuda") for _ in range(2)]

    def both(dw):
        y = layers.head_norm(ops, q, k, w[0], w[1], table, pos)
        return y + layers.head_norm_backward(ops, dq, dk, q, k, w[0], w[1], table, pos, dwq=dw[0], dwk=dw[1], accumulate=False)

    both(dw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a = both(dw)
    pos += 77
    dq.normal_()
    q.normal_()
    g.replay()
    e = [torch.zeros(64, device="cuda") for _ in range(2)]
    b = both(e)
    assert all(torch.equal(x, y) for x, y in zip(a + tuple(dw), b + tuple(e)))
