"""bfloat16 products and the gated feed-forward block (layers.matmul, gated, gated_backward, Gated) on the GPU.

Products: operands are small integers, which bfloat16 holds exactly, and all sums stay below 2^24: results are equal to those in 64 bits, rounded once
where the result is bfloat16.  No tolerance.

Block: against the formulas in 64 bits, by intervals.  A sum of K products from the tensor cores is within e S of itself, S the sum of the magnitudes,
e = 2^-23 (264 + K / 4096), in the gate's own products 2^-23 (8 + K / 16).  A value rounded to bfloat16 is off by 2^-8 of itself more, one kept in 24 bits by 2^-16.  The activation and its derivative move by at most 1.13 and 1 (their
own largest slopes) times what their argument moves, and the hardware's exponential and quotient are 2^-20 (1 + |g|) off.  An interval around every
factor gives one around every product, and sums of those give the ones behind the next product.
"""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import torch
    from paper_2609_23898_b200 import training
    assert torch.cuda.is_available()
    o = training.Ops()
    yield o
    o.status()


def whole(rng, *shape):
    import torch
    return torch.from_numpy(rng.integers(-4, 5, shape).astype(np.float32)).cuda().bfloat16()


def tile(m, n, k):
    from paper_2609_23898_b200 import cerar
    split = C.c_int()
    return cerar.lib.cerar_matmul_bf16_tile(m, n, k, 148, C.byref(split)), split.value


def stored(t, how):
    """The same values, lying in memory in another way."""
    import torch
    if how == "plain":
        return t
    if how == "strided":
        return torch.cat((t, t), 1)[:, :t.size(1)]
    if how == "offset":
        return torch.cat((t[:1, :1].flatten(), t.flatten()))[1:].view(t.shape)
    return t.t().contiguous().t()


SIZES = [(1, 1, 1), (1, 8, 64), (3, 5, 7), (16, 128, 64), (128, 128, 128), (130, 131, 133), (127, 257, 65), (1, 2048, 4096), (5, 72, 8192), (300, 1000, 520),
         (520, 300, 1500), (256, 256, 64), (257, 511, 200), (2500, 2600, 72), (1031, 4100, 333), (64, 64, 20000), (2304, 2304, 4160), (3952, 9, 1071), (105, 3965, 886), (58, 8, 684),
         (277, 2069, 2511), (9, 3142, 566), (1000, 2040, 16400)]


@pytest.mark.parametrize("trans_a", [False, True])
@pytest.mark.parametrize("trans_b", [False, True])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_products(ops, m, n, k, trans_a, trans_b):
    import torch
    from paper_2609_23898_b200 import layers
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    a, b = whole(rng, *((k, m) if trans_a else (m, k))), whole(rng, *((n, k) if trans_b else (k, n)))
    want = (a.double().t() if trans_a else a.double()) @ (b.double().t() if trans_b else b.double())
    for dtype in (torch.float32, torch.bfloat16):
        got = layers.matmul(ops, a, b, trans_a=trans_a, trans_b=trans_b, dtype=dtype)
        assert got.dtype == dtype and torch.equal(got, want.to(dtype))
        # added to, into a slice that lies on no boundary, with guards around it
        flat = torch.full((3 + m * n + 5,), 2.0, device="cuda", dtype=dtype)
        out = flat[3:3 + m * n].view(m, n)
        layers.matmul(ops, a, b, trans_a=trans_a, trans_b=trans_b, out=out, accumulate=True)
        assert torch.equal(out, (want + 2).to(dtype)) and bool((flat[:3] == 2).all()) and bool((flat[3 + m * n:] == 2).all())
        wide = torch.full((m, n + 8), 3.0, device="cuda", dtype=dtype)
        layers.matmul(ops, a, b, trans_a=trans_a, trans_b=trans_b, out=wide[:, :n], accumulate=True)
        assert torch.equal(wide[:, :n], (want + 3).to(dtype)) and bool((wide[:, n:] == 3).all())


def test_all_tiles_and_splits_are_tested():
    shapes = [tile(*s) for s in SIZES]
    assert {t for t, _ in shapes} == {0, 1, 2} and {form for form, s in shapes if s > 1} == {0, 1, 2}, shapes


@pytest.mark.parametrize("how_a", ["plain", "strided", "offset", "transposed"])
@pytest.mark.parametrize("how_b", ["strided", "offset", "transposed"])
def test_products_of_any_strides(ops, how_a, how_b):
    import torch
    from paper_2609_23898_b200 import layers
    rng = np.random.default_rng(1)
    for m, n, k in ((40, 72, 48), (41, 73, 51)):
        a, b = whole(rng, m, k), whole(rng, k, n)
        assert torch.equal(layers.matmul(ops, stored(a, how_a), stored(b, how_b), dtype=torch.float32), (a.double() @ b.double()).float())


def test_what_lies_between_rows_is_not_used(ops):
    import torch
    from paper_2609_23898_b200 import layers
    rng = np.random.default_rng(2)
    for m, n, k in ((100, 60, 50), (700, 2000, 100)):
        a, b = torch.full((m, 104), float("nan"), device="cuda").bfloat16(), torch.full((k, n + 12), float("nan"), device="cuda").bfloat16()
        a[:, :k], b[:, :n] = whole(rng, m, k), whole(rng, k, n)
        assert torch.equal(layers.matmul(ops, a[:, :k], b[:, :n], dtype=torch.float32), (a[:, :k].double() @ b[:, :n].double()).float())


def test_empty_products(ops):
    import torch
    from paper_2609_23898_b200 import layers
    e = torch.empty
    kw = dict(device="cuda", dtype=torch.bfloat16)
    assert layers.matmul(ops, e(0, 8, **kw), e(8, 4, **kw)).shape == (0, 4)
    assert layers.matmul(ops, e(3, 8, **kw), e(8, 0, **kw)).shape == (3, 0)
    assert not bool(layers.matmul(ops, e(3, 0, **kw), e(0, 4, **kw)).any())
    out = torch.ones(3, 4, device="cuda")
    layers.matmul(ops, e(3, 0, **kw), e(0, 4, **kw), out=out, accumulate=True)
    assert bool((out == 1).all())


def test_infinities_and_nan_stay_in_their_rows_and_columns(ops):
    import torch
    from paper_2609_23898_b200 import layers
    rng = np.random.default_rng(3)
    a, b = whole(rng, 300, 200), whole(rng, 200, 400)
    want = a.double() @ b.double()
    a[7, 3], a[290, 199] = float("nan"), float("inf")
    got = layers.matmul(ops, a, b, dtype=torch.float32)
    rows = torch.ones(300, dtype=torch.bool, device="cuda")
    rows[[7, 290]] = False
    assert torch.equal(got[rows], want[rows].float()) and bool(torch.isnan(got[7]).all()) and not bool(torch.isfinite(got[290][b[199] != 0]).any())


def test_long_sums(ops):
    """|C - exact| <= 2^-23 (264 + K / 4096) sum |A| |B| in binary32."""
    import torch
    from paper_2609_23898_b200 import layers
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    for m, n, k in ((130, 140, 30000), (2304, 2304, 9000)):
        a, b = torch.randn(m, k, device="cuda", generator=g).abs().bfloat16(), torch.randn(n, k, device="cuda", generator=g).abs().bfloat16()
        got, want = layers.matmul(ops, a, b, trans_b=True, dtype=torch.float32).double(), a.double() @ b.double().t()
        assert bool(((got - want).abs() <= 2.0 ** -23 * (264 + k / 4096) * want).all())


# ---------------------------------------------------------------------------------------------------- the block

def act_of(g, act):
    """act(g), act'(g), in 64 bits."""
    import torch
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if act == "gelu":
        c = torch.special.ndtr(g)
        return g * c, c + g * torch.exp(-g * g / 2) / np.sqrt(2 * np.pi)
    if act == "gelu_tanh":
        k = np.sqrt(2 / np.pi)
        t = torch.tanh(k * (g + 0.044715 * g ** 3))
        return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t * t) / 2 * k * (1 + 3 * 0.044715 * g * g)
    return g.clamp(min=0), (g > 0).double()


class Near:
    """A matrix in 64 bits and how far off it may be."""

    def __init__(self, v, off):
        self.v, self.off = v, off

    def __mul__(self, o):
        return Near(self.v * o.v, (self.v.abs() + self.off) * (o.v.abs() + o.off) - self.v.abs() * o.v.abs())

    def kept(self, u=2.0 ** -8):
        return Near(self.v, self.off * (1 + u) + self.v.abs() * u)

    def product(self, w, k):
        e = 2.0 ** -23 * max(264 + k / 4096, 8 + k / 16)
        return Near(self.v @ w, self.off @ w.abs() * (1 + e) + e * (self.v.abs() @ w.abs()))

    def plus_one(self):
        """Added to one in binary32: half a step of the sum, 2^-24 (1 + |v| + off), more."""
        return Near(self.v + 1, self.off + 2.0 ** -24 * (1 + self.v.abs() + self.off))

    def holds(self, got):
        d = (got.double() - self.v).abs()
        assert bool((d <= self.off * 1.001 + 1e-30).all()), float((d / (self.off + 1e-30)).max())


def exactly(t):
    return Near(t.double(), t.double() * 0)


def block(x, w_in, w_out, dy, act):
    """Intervals of y, dx, dw_in, dw_out before the rounding of the result."""
    f, (t, d) = w_out.size(1), x.shape
    x, w_in, w_out, dy = x.double(), w_in.double(), w_out.double(), dy.double()
    g, u = exactly(x).product(w_in[:f].t(), d), exactly(x).product(w_in[f:].t(), d)

    def around(g, slope, which):
        v = act_of(g.v, act)[which]
        off = g.off * slope + 2.0 ** -20 * (1 + g.v.abs())
        if act == "relu" and which == 1:
            off = (g.v.abs() <= g.off).double()
        return Near(v, off)

    h = (around(g, 1.13, 0) * u).kept()
    y = h.product(w_out.t(), f)
    gk, uk = g.kept(2.0 ** -16), u.kept(2.0 ** -16)
    dh = exactly(dy).product(w_out, w_out.size(0))
    dg, du = (dh * uk * around(gk, 1.0, 1)).kept(), (dh * around(gk, 1.13, 0)).kept()
    import torch
    dgu = Near(torch.cat((dg.v, du.v), 1), torch.cat((dg.off, du.off), 1))
    dx = dgu.product(w_in, 2 * f)
    dw_in = Near(dgu.v.t().contiguous(), dgu.off.t().contiguous()).product(x, t)
    h = (around(gk, 1.13, 0) * uk).kept()
    dw_out = Near(h.v.t().contiguous(), h.off.t().contiguous()).product(dy, t)
    return y, dx, dw_in, Near(dw_out.v.t(), dw_out.off.t())


def weights(t, d, f, o, seed=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + t + d + f)

    def normal(*s, std=1.0):
        return (torch.randn(*s, device="cuda", generator=g) * std).bfloat16()

    return normal(t, d), normal(2 * f, d, std=1.5 * d ** -0.5), normal(o, f, std=f ** -0.5), normal(t, o)


BLOCKS = [(1, 8, 8, 8), (1, 2048, 300, 64), (5, 33, 40, 17), (130, 72, 129, 72), (64, 64, 64, 64), (300, 136, 200, 264), (77, 1000, 24, 8), (1, 64, 8192, 128), (2, 72, 140, 9000),
          (1500, 136, 2104, 136), (2304, 200, 2310, 72), (2049, 200, 1027, 72), (700, 4200, 260, 40), (3, 1, 1, 1), (105, 886, 1983, 886), (3900, 1071, 5, 1071), (1000, 16400, 1020, 72), (1000, 40, 2040, 16400), (4096, 8, 2048, 512)]


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("t,d,f,o", BLOCKS)
def test_block(ops, t, d, f, o, act):
    import torch
    from paper_2609_23898_b200 import layers
    x, w_in, w_out, dy = weights(t, d, f, o)
    y, kept = layers.gated(ops, x, w_in, w_out, activation=act, keep=True)
    assert torch.equal(y, layers.gated(ops, x, w_in, w_out, activation=act)) and y.shape == (t, o) and y.dtype == torch.bfloat16
    dw_in, dw_out = torch.ones(2 * f, d, device="cuda"), torch.ones(o, f, device="cuda")
    dx = layers.gated_backward(ops, dy, kept, w_in, w_out, dw_in, dw_out)
    ey, edx, ewi, ewo = block(x, w_in, w_out, dy, act)
    ey.kept().holds(y)
    edx.kept().holds(dx)
    ewi.plus_one().holds(dw_in)
    ewo.plus_one().holds(dw_out)
    b_in, b_out = torch.full((2 * f, d), 5.0, device="cuda").bfloat16(), torch.full((o, f), 5.0, device="cuda").bfloat16()
    layers.gated_backward(ops, dy, kept, w_in, w_out, b_in, b_out, accumulate=False, need_dx=False)
    ewi.kept().holds(b_in)
    ewo.kept().holds(b_out)
    only = layers.gated_backward(ops, dy, kept, w_in, w_out, None, None)
    assert torch.equal(only, dx)


def test_block_tiles():
    for shapes in ([tile(t, 2 * f, d) for t, d, f, o in BLOCKS], [tile(t, f, o) for t, d, f, o in BLOCKS]):
        assert {t for t, _ in shapes} == {0, 1, 2} and {form for form, s in shapes if s > 1} == {0, 1, 2}, shapes


def test_gradient_against_differences(ops):
    """The block's derivative along a direction, from the formula in 64 bits at two nearby points."""
    import torch
    from paper_2609_23898_b200 import layers
    for act in ("silu", "gelu", "gelu_tanh"):
        x, w_in, w_out, dy = weights(40, 24, 32, 16)
        y, kept = layers.gated(ops, x, w_in, w_out, activation=act, keep=True)
        d = [torch.zeros(64, 24, device="cuda"), torch.zeros(16, 32, device="cuda")]
        dx = layers.gated_backward(ops, dy, kept, w_in, w_out, *d)
        along = [torch.randn(t.shape, dtype=torch.float64, device="cuda") for t in (x, w_in, w_out)]

        def f(s):
            a, b, c = (t.double() + s * v for t, v in zip((x, w_in, w_out), along))
            g, u = a @ b[:32].t(), a @ b[32:].t()
            return float((((act_of(g, act)[0] * u) @ c.t()) * dy.double()).sum())

        slope = (f(1e-6) - f(-1e-6)) / 2e-6
        terms = [(g.double() * v) for g, v in zip((dx, *d), along)]
        got, size = sum(float(t.sum()) for t in terms), sum(float(t.square().sum()) for t in terms) ** 0.5
        # every term carries some five roundings to bfloat16 of random signs: 5 sigma of 2^-8 sqrt(5 / 3) times their norm
        assert abs(got - slope) < 5 * 2.0 ** -8 * (5 / 3) ** 0.5 * size, (got, slope, size)


def test_block_of_any_strides_and_shapes(ops):
    import torch
    from paper_2609_23898_b200 import layers
    x, w_in, w_out, dy = weights(60, 40, 48, 24)
    want, kept = layers.gated(ops, x, w_in, w_out, keep=True)
    dwi, dwo = torch.zeros(96, 40, device="cuda"), torch.zeros(24, 48, device="cuda")
    dx = layers.gated_backward(ops, dy, kept, w_in, w_out, dwi, dwo)
    for how in ("strided", "offset", "transposed"):
        y, kept = layers.gated(ops, stored(x, how), stored(w_in, how), stored(w_out, how), keep=True)
        a, b = torch.zeros_like(dwi), torch.zeros_like(dwo)
        got = layers.gated_backward(ops, stored(dy, how), kept, stored(w_in, how), stored(w_out, how), a, b)
        assert torch.equal(y, want) and torch.equal(got, dx) and torch.equal(a, dwi) and torch.equal(b, dwo)
    y, kept = layers.gated(ops, x.view(3, 20, 40), w_in, w_out, keep=True)
    assert torch.equal(y, want.view(3, 20, 24))
    assert torch.equal(layers.gated_backward(ops, dy.view(3, 20, 24), kept, w_in, w_out, None, None), dx.view(3, 20, 40))
    assert torch.equal(layers.gated(ops, x[0], w_in, w_out), layers.gated(ops, x[:1], w_in, w_out)[0])
    e, kept = layers.gated(ops, x[:0], w_in, w_out, keep=True)
    a, b = torch.ones_like(dwi), torch.ones_like(dwo)
    assert e.shape == (0, 24) and layers.gated_backward(ops, dy[:0], kept, w_in, w_out, a, b, accumulate=False).shape == (0, 40)
    assert not bool(a.any()) and not bool(b.any())
    one = torch.ones((), device="cuda").bfloat16().expand(60, 24)
    assert torch.equal(layers.gated_backward(ops, one, layers.gated(ops, x, w_in, w_out, keep=True)[1], w_in, w_out, None, None),
                       layers.gated_backward(ops, one.contiguous(), layers.gated(ops, x, w_in, w_out, keep=True)[1], w_in, w_out, None, None))


def test_rows_do_not_touch_one_another(ops):
    """A token that is NaN leaves the others' results as they are."""
    import torch
    from paper_2609_23898_b200 import layers
    for t, d, f in ((50, 64, 80), (2000, 128, 2048)):
        x, w_in, w_out, dy = weights(t, d, f, d)
        want = layers.gated(ops, x, w_in, w_out)
        x[t // 2] = float("nan")
        y = layers.gated(ops, x, w_in, w_out)
        rest = torch.arange(t, device="cuda") != t // 2
        assert torch.equal(y[rest], want[rest]) and bool(torch.isnan(y[t // 2]).all())


def test_autograd(ops):
    import torch
    from paper_2609_23898_b200 import layers
    x, w_in, w_out, dy = weights(50, 40, 48, 40)
    xa = x.view(5, 10, 40).requires_grad_()
    a, b = torch.zeros(96, 40, device="cuda"), torch.zeros(40, 48, device="cuda")
    y = layers.Gated.apply(xa, w_in, w_out, ops, a, b)
    y.backward(dy.view(5, 10, 40))
    _, kept = layers.gated(ops, x.detach(), w_in, w_out, keep=True)
    c, d = torch.zeros_like(a), torch.zeros_like(b)
    dx = layers.gated_backward(ops, dy, kept, w_in, w_out, c, d)
    assert torch.equal(xa.grad.view(50, 40), dx) and torch.equal(a, c) and torch.equal(b, d)
    # weights' gradients where x is data; frozen weights; nothing wanted; weights changed in between; a second derivative
    y = layers.Gated.apply(x.detach(), w_in, w_out, ops, a, None, "relu")
    assert y.requires_grad
    y.backward(dy)
    y = layers.Gated.apply(xa, w_in, w_out, ops, None, None)
    g, = torch.autograd.grad(y, [xa], dy.view(5, 10, 40), retain_graph=True)
    assert torch.equal(g.view(50, 40), dx)
    w_in.mul_(1)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y, [xa], dy.view(5, 10, 40))
    assert not layers.Gated.apply(x.detach(), w_in, w_out, ops, None, None).requires_grad
    with torch.no_grad():
        assert not layers.Gated.apply(xa, w_in, w_out, ops, a, b).requires_grad
    with pytest.raises(ValueError):
        layers.Gated.apply(x, w_in.clone().requires_grad_(), w_out, ops, a, b)
    with pytest.raises(RuntimeError):
        y = layers.Gated.apply(xa, w_in, w_out, ops, None, None)
        g, = torch.autograd.grad(y.float().sum(), [xa], create_graph=True)
        torch.autograd.grad(g.float().sum(), [xa])


def test_refusals(ops):
    import torch
    from paper_2609_23898_b200 import layers
    x, w_in, w_out, dy = weights(10, 16, 24, 16)
    _, kept = layers.gated(ops, x, w_in, w_out, keep=True)
    dw = torch.zeros(48, 16, device="cuda")
    for error, a in ((TypeError, (x.float(), w_in, w_out)), (TypeError, (x, w_in.float(), w_out)), (TypeError, (x, w_in, w_out.half())),
                     (ValueError, (x, w_in[:47], w_out)), (ValueError, (x[:, :8], w_in, w_out)), (ValueError, (x.cpu(), w_in, w_out)),
                     (ValueError, (x, w_in.cpu(), w_out)), (ValueError, (x, w_in[0], w_out))):
        with pytest.raises(error):
            layers.gated(ops, *a)
    with pytest.raises(ValueError):
        layers.gated(ops, x, w_in, w_out, activation="tanh")
    for error, a in ((ValueError, (dy[:9], kept, w_in, w_out, None, None)), (ValueError, (dy, kept, w_in, w_out, dw[:40], None)),
                     (ValueError, (dy, kept, w_in, w_out, dw.t(), None)), (TypeError, (dy, kept, w_in, w_out, dw.double(), None)),
                     (TypeError, (dy.float(), kept, w_in, w_out, dw, None)),
                     (ValueError, (dy, (kept[0], kept[1][:6143], kept[2]), w_in, w_out, None, None)),          # shorter than these sizes' is
                     (ValueError, (dy, (kept[0], kept[1].cpu(), kept[2]), w_in, w_out, None, None)),
                     (ValueError, (dy, kept, torch.zeros(128, 16, device="cuda").bfloat16(), torch.zeros(16, 64, device="cuda").bfloat16(), None, None))):
        with pytest.raises(error):
            layers.gated_backward(ops, *a)
    for error, a, kw in ((TypeError, (x.float(), w_in.t()), {}), (ValueError, (x, w_in), {}), (ValueError, (x, w_in.t()), dict(accumulate=True)),
                         (ValueError, (x, w_in.t()), dict(out=dw)), (ValueError, (x[0], w_in.t()), {}), (TypeError, (x, w_in.t()), dict(dtype=torch.float16))):
        with pytest.raises(error):
            layers.matmul(ops, *a, **kw)
    square = torch.zeros(16, 16, device="cuda").bfloat16()
    for a in ((square, w_in[:16].clone()), (w_in[:16].clone(), square), (square, square)):
        with pytest.raises(ValueError):
            layers.matmul(ops, *a, out=square)


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("t,d,f", [(64, 256, 512), (333, 520, 1377), (2, 64, 96), (512, 1024, 1024), (700, 96, 2000), (40, 2048, 64)])
def test_passes_one_behind_the_other(ops, t, d, f, captured):
    """Many passes without a pause, whose workspaces lie where those before them had theirs, give what each gives alone: kernels that begin early
    neither read what is not there yet nor write what is still read."""
    import torch
    from paper_2609_23898_b200 import layers
    cases = [weights(t, d, f, d, seed=s) for s in range(12)]

    def run(case):
        x, w_in, w_out, dy = case
        y, kept = layers.gated(ops, x, w_in, w_out, keep=True)
        dw = torch.ones_like(w_in, dtype=torch.float32), torch.ones_like(w_out, dtype=torch.float32)
        return y, layers.gated_backward(ops, dy, kept, w_in, w_out, *dw), *dw

    want = []
    for case in cases:
        want.append(run(case))
        torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = [run(case) for case in cases]
        for _ in range(3):
            graph.replay()
    else:
        got = [run(case) for case in cases]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    ops.status()


def test_captured_and_replayed(ops):
    import torch
    from paper_2609_23898_b200 import layers
    x, w_in, w_out, dy = weights(300, 64, 136, 64)
    dw = [torch.zeros(272, 64, device="cuda"), torch.zeros(64, 136, device="cuda")]

    def both(a, b):
        y, kept = layers.gated(ops, x, w_in, w_out, keep=True)
        return y, layers.gated_backward(ops, dy, kept, w_in, w_out, a, b, accumulate=False)

    both(*dw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a = both(*dw)
    x.normal_()
    w_in.normal_(0, 0.1)
    g.replay()
    e = [torch.zeros_like(t) for t in dw]
    b = both(*e)
    assert all(torch.equal(p, q) for p, q in zip((*a, *dw), (*b, *e)))
