"""Infinities, NaN and values at the ends of the range in the layers' inputs and weights, on the GPU: they show where the formulas say, and nowhere else.

Head norms: a row that holds an infinity has r = 0 by the formula, so that its other values become zero, or NaN where they are turned with it; which results are infinite, NaN or
finite is compared with the formula in 64 bits.  Finite ones: zero exactly (forward), or within the bounds of the other tests of these layers: a sum of N rows' terms
dz n within (N + d / 2 + 12) 2^-24 of the sum of their magnitudes.  Exact results otherwise.
"""
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


def same_kind(got, want):
    """Infinite with the same sign, NaN, or finite, in the same places."""
    import torch
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf])


def turned(z, table, pairs, sign):
    """The first values of z (tokens, heads, d) turned by angles of `table` (tokens, pairs, 2)."""
    import torch
    rot = 2 * table.size(1)
    if rot == 0:
        return z
    c, s = (sign ** i * t[:, None] for i, t in enumerate(table.double().unbind(-1)))
    t = z[..., :rot]
    a, b = t.chunk(2, -1) if pairs == "halves" else (t[..., 0::2], t[..., 1::2])
    y = (a * c - b * s, b * c + a * s)
    return torch.cat((torch.cat(y, -1) if pairs == "halves" else torch.stack(y, -1).flatten(-2), z[..., rot:]), -1)


# d, rotated: chunks of 16, 8, 4 and 2 bytes, of values that are not turned, and of ones that are
FORMS = [("bf16", 128, 64), ("bf16", 128, 0), ("bf16", 128, 128), ("bf16", 72, 24), ("bf16", 36, 4), ("bf16", 34, 2), ("bf16", 10, 0), ("f32", 128, 64), ("f32", 64, 0),
         ("f32", 12, 4), ("f32", 10, 4), ("f32", 16, 16)]


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("ty,d,rot", FORMS)
def test_an_infinity_stays_where_the_formula_has_it(ops, ty, d, rot, pairs):
    """One infinite value in every row in turn: of x forward, of dy backward."""
    import torch
    from paper_2609_23898_b200 import layers
    dtype = torch.float32 if ty == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(d + rot)
    n = 2 * d
    x = (1 + torch.rand(n, 3, d, device="cuda", generator=g)).to(dtype)
    dy = (1 + torch.rand(n, 3, d, device="cuda", generator=g)).to(dtype)
    w = 1 + torch.rand(d, device="cuda", generator=g)
    table = layers.rotation_table(ops, n + 1, rot, first=1)[:n].contiguous()
    at, sign = torch.arange(n, device="cuda") % d, torch.where(torch.arange(n, device="cuda") < d, 1.0, -1.0)
    bad = x.clone()
    bad[torch.arange(n, device="cuda"), 1, at] = (sign * float("inf")).to(dtype)
    y, _ = layers.head_norm(ops, bad, None, w, None, table if rot else None, pairs=pairs)
    # r = 1 / sqrt(inf) = 0
    b = bad.double()
    r = 1 / torch.sqrt((b * b).mean(-1, keepdim=True) + 1e-6)
    want = turned(b * r * w.double(), table, pairs, 1)
    same_kind(y, want)
    assert not bool(y[:, 1][torch.isfinite(y[:, 1])].any())
    # backward: a row's dx is all infinite or NaN; the other rows' and the other columns of dw are what they would be
    bad = dy.clone()
    bad[torch.arange(n, device="cuda"), 1, at] = (sign * float("inf")).to(dtype)
    for row in (0, d - 1, min(d, rot + 1), d + d // 2):
        one = dy.clone()
        one[row] = bad[row]
        dw = torch.zeros(d, device="cuda")
        dx, _ = layers.head_norm_backward(ops, one, None, x, None, w, None, table if rot else None, dwq=dw, pairs=pairs)
        v = x.double()
        r = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6)
        dz = turned(one.double(), table, pairs, -1)
        terms = dz * v * r
        exact = terms.sum((0, 1))
        same_kind(dw, exact)
        finite = torch.isfinite(exact)
        mag = one.double().abs().nan_to_num(posinf=0)
        size = (mag + roll(mag, rot, pairs)) * v * r
        assert bool(((dw.double() - exact).abs()[finite] <= size.sum((0, 1))[finite] * (3 * n + d / 2 + 12) * U).all())
        dn = dz * w.double()
        same_kind(dx, r * (dn - v * r * (dn * v * r).mean(-1, keepdim=True)))


def roll(t, rot, pairs):
    """The value that each one is turned with (itself beyond the turned ones)."""
    import torch
    if rot == 0:
        return t
    a = t[..., :rot]
    p = a.roll(rot // 2, -1) if pairs == "halves" else a.unflatten(-1, (rot // 2, 2)).flip(-1).flatten(-2)
    return torch.cat((p, t[..., rot:]), -1)


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("ty,d,rot", FORMS)
def test_padding_is_zero_whatever_the_weights_are(ops, ty, d, rot, pairs):
    import torch
    from paper_2609_23898_b200 import layers
    dtype = torch.float32 if ty == "f32" else torch.bfloat16
    x, dy = (torch.randn(60, 3, d, device="cuda").to(dtype) for _ in range(2))
    table = layers.rotation_table(ops, 60, rot) if rot else None
    pos = torch.arange(60, device="cuda")
    pos[::3] = -1
    for value in (float("inf"), float("-inf"), float("nan")):
        for where in (slice(None), slice(1, 2), slice(d - 1, d)):
            w = torch.ones(d, device="cuda")
            w[where] = value
            y, _ = layers.head_norm(ops, x, None, w, None, table, pos, pairs=pairs)
            dw = torch.zeros(d, device="cuda")
            dx, _ = layers.head_norm_backward(ops, dy, None, x, None, w, None, table, pos, dwq=dw, pairs=pairs)
            assert not bool(y[::3].any()) and not bool(dx[::3].any()) and bool(torch.isfinite(dw).all())
            assert not bool(torch.isfinite(y[1::3]).all()) and not bool(torch.isfinite(dx[1::3]).any())


@pytest.mark.parametrize("outputs", [1, 8192])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_activations_far_out(ops, act, outputs):
    """Beyond 10^4 every activation is g or 0 and its derivative 1 or 0, up to the ends of the range: one token, one input, one hidden value with u = 1, dh = 1."""
    import torch
    from paper_2609_23898_b200 import layers
    one = torch.ones(1, 1, device="cuda").bfloat16()
    w_out = torch.ones(outputs, 1, device="cuda").bfloat16()
    dy = torch.zeros(1, outputs, device="cuda").bfloat16()
    dy[0, outputs // 2] = 1
    for size in (1e4, 1e10, 1e19, 3e19, 1e20, 3e38):
        for sign in (1, -1):
            w_in = torch.tensor([[sign * size], [1.0]], device="cuda").bfloat16()
            y, kept = layers.gated(ops, one, w_in, w_out, activation=act, keep=True)
            dw_in, dw_out = torch.zeros(2, 1, device="cuda"), torch.zeros(outputs, 1, device="cuda")
            layers.gated_backward(ops, dy, kept, w_in, w_out, dw_in, dw_out)
            g = float(w_in[0, 0]) if sign > 0 else 0.0
            assert bool((y == g).all()) and float(dw_in[0, 0]) == (1.0 if sign > 0 else 0.0) and float(dw_in[1, 0]) == g, (size, sign, dw_in)
            assert float(dw_out[outputs // 2, 0]) == g
