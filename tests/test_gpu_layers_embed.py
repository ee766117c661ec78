"""Embedding lookup and its gradient (layers.embed, embed_backward, Embed) against the formulas in 64 bits, on the GPU.

Tolerances.  Lookup: one product in binary32 and one rounding: |y - s t| <= |s t| (eps_out / 2 + 2^-24 (1 + 2^-8)) (the scale reaches the kernel in
binary32: 2^-24 more).  Gradient: a sum of n values in any order of binary32 additions is within n 2^-24 sum |values| of itself; then the
product with the scale, the addition to what is there, and a rounding to the result's type.
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


def half_step(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def table_of(v, d, dtype, how, seed=0):
    """A v x d table: alone, as the left part of wider rows (odd strides), or off any boundary but its elements'."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if how == "plain":
        return torch.randn(v, d, device="cuda", generator=g).to(dtype)
    if how == "strided":
        return torch.randn(v, d + 3, device="cuda", generator=g).to(dtype)[:, :d]
    return torch.randn(v * d + 1, device="cuda", generator=g).to(dtype)[1:].view(v, d)


@pytest.mark.parametrize("how", ["plain", "strided", "offset"])
@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,width,ids", [(1, 1, 1, "i64"), (1, 7, 8, "i32"), (3, 50, 2048, "i64"), (130, 33, 130, "i32"), (257, 1000, 519, "i64"),
                                                    (1000, 5, 64, "i64"), (65, 9, 5001, "i32")])
def test_lookup(ops, how, src, dst, tokens, vocab, width, ids):
    import torch
    from paper_2609_23898_b200 import layers
    t = table_of(vocab, width, types()[src], how)
    rng = np.random.default_rng(tokens)
    i = torch.from_numpy(rng.integers(-2, vocab, tokens)).cuda().to(torch.int32 if ids == "i32" else torch.int64)
    s = 1.7
    y = layers.embed(ops, t, i, scale=s, dtype=types()[dst])
    want = torch.where((i >= 0)[:, None], t.double()[i.clamp(min=0).long()] * s, 0.0)
    assert y.dtype == types()[dst] and y.shape == (tokens, width)
    bound = want.abs() * (half_step(y.dtype) + 3 * U)
    assert bool(((y.double() - want).abs() <= bound).all())


def test_lookup_shapes_and_emptiness(ops):
    import torch
    from paper_2609_23898_b200 import layers
    t = table_of(10, 12, torch.bfloat16, "plain")
    i = torch.arange(24, device="cuda").view(2, 3, 4) % 10
    assert torch.equal(layers.embed(ops, t, i), t[i])
    assert torch.equal(layers.embed(ops, t, i.transpose(0, 2)), t[i.transpose(0, 2)])
    assert layers.embed(ops, t, i[:0]).shape == (0, 3, 4, 12)
    assert layers.embed(ops, t, torch.tensor(3, device="cuda")).shape == (12,)
    assert layers.embed(ops, t[:, :0], i).shape == (2, 3, 4, 0)
    assert torch.equal(layers.embed(ops, t[:0], torch.full((2,), -1, device="cuda")), torch.zeros(2, 12, dtype=t.dtype, device="cuda"))


def test_special_values_are_looked_up_as_they_are(ops):
    import torch
    from paper_2609_23898_b200 import layers
    t = torch.tensor([[float("inf"), float("nan"), -0.0, 1e-40]], device="cuda")
    y = layers.embed(ops, t, torch.tensor([0, -1], device="cuda"))
    assert y[0, 0] == float("inf") and torch.isnan(y[0, 1]) and torch.equal(y[1], torch.zeros(4, device="cuda"))
    assert torch.equal(y[0, 2:].view(torch.int32), t[0, 2:].view(torch.int32))


def test_ids_beyond_the_table_are_reported(ops):
    import torch
    from paper_2609_23898_b200 import layers, cerar
    t = table_of(10, 16, torch.float32, "plain")
    d = torch.zeros(10, 16, device="cuda")
    i = torch.tensor([3, 10, 2 ** 40, -2 ** 40], device="cuda")
    ops.status()
    y = layers.embed(ops, t, i)
    with pytest.raises(cerar.CerarError) as e:
        ops.status()
    assert e.value.status == 10
    ops.status()                                                   # reported once
    assert torch.equal(y[0], t[3]) and not bool(y[1:].any())
    layers.embed_backward(ops, torch.ones(4, 16, device="cuda"), i, d)
    with pytest.raises(cerar.CerarError):
        ops.status()
    assert bool((d[3] == 1).all()) and float(d.sum()) == 16


def ids_of(kind, tokens, vocab, seed):
    import torch
    rng = np.random.default_rng(seed)
    if kind == "one":
        i = np.full(tokens, vocab // 2)
    elif kind == "few":
        i = rng.integers(0, min(vocab, 3), tokens)
    elif kind == "zipf":
        i = np.minimum(np.exp(rng.random(tokens) * np.log(vocab + 1)).astype(np.int64) - 1, vocab - 1)
    elif kind == "padded":
        i = rng.integers(-vocab, vocab, tokens)
    elif kind == "padding":
        i = np.full(tokens, -1)
    else:
        i = rng.integers(0, vocab, tokens)
    return torch.from_numpy(i.astype(np.int64)).cuda()


def check_grad(ops, i, dy, dtable, s, accumulate):
    import torch
    from paper_2609_23898_b200 import layers
    before = dtable.clone()
    layers.embed_backward(ops, dy, i, dtable, scale=s, accumulate=accumulate)
    v, w = dtable.shape
    live = i >= 0
    flat = i[live]
    want, size = torch.zeros(v, w, dtype=torch.float64, device="cuda"), torch.zeros(v, w, dtype=torch.float64, device="cuda")
    want.index_add_(0, flat, dy[live].double())
    size.index_add_(0, flat, dy[live].double().abs())
    n = torch.bincount(flat, minlength=v)[:, None].double()
    want, size = want * s, size * abs(s)
    if accumulate:
        want, size = want + before.double(), size + before.double().abs()
    # n additions, the scale's rounding and product, the addition to what is there; then the result's rounding
    bound = size * (n + 4) * U * 1.01 + want.abs() * half_step(dtable.dtype) * 1.01
    off = (dtable.double() - want).abs()
    assert bool((off <= bound).all()), float((off - bound).max())
    none = (n == 0).expand(v, w)
    assert torch.equal(dtable[none], before[none] if accumulate else torch.zeros_like(before[none]))
    return dtable


@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("kind", ["uniform", "one", "few", "zipf", "padded", "padding"])
@pytest.mark.parametrize("tokens,vocab,width,src,dst", [(1, 3, 5, "f32", "f32"), (4, 40, 64, "bf16", "f32"), (5, 1, 8, "bf16", "bf16"), (300, 70, 1030, "bf16", "f32"),
                                                        (1333, 503, 519, "f32", "f32"), (4096, 999, 128, "f32", "bf16"), (4097, 5000, 136, "bf16", "f32"),
                                                        (9001, 77, 24, "bf16", "f32"), (40000, 2000, 66, "bf16", "bf16")])
def test_gradient(ops, tokens, vocab, width, src, dst, kind, accumulate):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    i = ids_of(kind, tokens, vocab, tokens)
    dy = torch.randn(tokens, width, device="cuda", generator=g).to(types()[src])
    d = torch.randn(vocab, width, device="cuda", generator=g).to(types()[dst])
    check_grad(ops, i, dy, d, 0.37, accumulate)


@pytest.mark.parametrize("vocab", [1 << 9, (1 << 9) - 1, 1 << 18, (1 << 18) + 1, (1 << 27) + 5])
def test_gradient_of_large_vocabularies(ops, vocab):
    """One, two, three and four digits of the keys, and keys at the digits' borders."""
    import torch
    tokens = 6000
    i = ids_of("uniform", tokens, vocab, 3)
    i[:3] = torch.tensor([vocab - 1, 0, vocab - 1])
    i[100:104] = -1
    dy = torch.randn(tokens, 2, device="cuda")
    check_grad(ops, i, dy, torch.zeros(vocab, 2, device="cuda"), 1.0, True)


def test_gradient_strides_and_guards(ops):
    """Slices of a larger vector: nothing beside them is touched; dy transposed, expanded, a slice."""
    import torch
    from paper_2609_23898_b200 import layers
    i = ids_of("uniform", 700, 50, 1)
    for width, off in ((64, 0), (64, 1), (33, 3)):
        flat = torch.full((off + 50 * width + 7,), 5.0, device="cuda")
        d = flat[off:off + 50 * width].view(50, width)
        d.zero_()
        dy = torch.randn(700, width, device="cuda")
        check_grad(ops, i, dy, d, 1.0, False)
        assert bool((flat[:off] == 5).all()) and bool((flat[off + 50 * width:] == 5).all())
        first = d.clone()
        layers.embed_backward(ops, dy.t().contiguous().t(), i, d, accumulate=False)
        assert torch.equal(first, d)
        wide = torch.full((50, width + 5), 7.0, device="cuda")
        layers.embed_backward(ops, torch.cat((dy, dy), 1)[:, :width], i, wide[:, 2:2 + width], accumulate=False)
        assert torch.equal(first, wide[:, 2:2 + width]) and bool((wide[:, :2] == 7).all()) and bool((wide[:, 2 + width:] == 7).all())
        layers.embed_backward(ops, torch.ones((), device="cuda").expand(700, width), i, d, accumulate=False)
        assert torch.equal(d, torch.bincount(i, minlength=50)[:, None].float().expand(50, width))


def test_gradient_is_deterministic_and_padding_is_not_read(ops):
    import torch
    from paper_2609_23898_b200 import layers
    for tokens in (2000, 20000):
        i = ids_of("zipf", tokens, 100, 5)
        i[::7] = -1
        dy = torch.randn(tokens, 96, device="cuda").bfloat16()
        a, b = torch.zeros(100, 96, device="cuda"), torch.zeros(100, 96, device="cuda")
        layers.embed_backward(ops, dy, i, a)
        dy[::7] = float("nan")
        layers.embed_backward(ops, dy, i, b)
        assert torch.equal(a, b)


def test_long_offsets(ops):
    """Rows beyond 2^31 elements from the table's start."""
    import torch
    from paper_2609_23898_b200 import layers
    v, w = 1_100_000, 2048
    t = torch.empty(v, w, dtype=torch.bfloat16, device="cuda")
    i = torch.tensor([v - 1, 0, v - 2, v - 1], device="cuda")
    t[i] = torch.randn(4, w, device="cuda").bfloat16()
    assert torch.equal(layers.embed(ops, t, i), t[i])
    t[i] = 0
    dy = torch.randn(4, w, device="cuda").bfloat16()
    layers.embed_backward(ops, dy, i, t)
    assert torch.equal(t[v - 2], dy[2]) and torch.equal(t[0], dy[1]) and torch.equal(t[v - 1], (dy[0].float() + dy[3].float()).bfloat16())


def test_autograd(ops):
    import torch
    from paper_2609_23898_b200 import layers
    t = torch.randn(20, 24, device="cuda")
    d = torch.zeros(20, 24, device="cuda")
    i = torch.randint(0, 20, (3, 5), device="cuda")
    y = layers.Embed.apply(t, i, ops, d, 2.0)
    dy = torch.randn_like(y)
    y.backward(dy)
    ref = t.clone().requires_grad_()
    (2.0 * torch.nn.functional.embedding(i, ref)).backward(dy)
    assert torch.allclose(d, ref.grad, rtol=0, atol=float(dy.abs().max()) * 15 * 16 * U)
    y = layers.Embed.apply(t, i, ops, d, 2.0)
    i.add_(0)                                                      # changed in place since: refused, as autograd does
    with pytest.raises(RuntimeError):
        y.backward(dy)
    assert not layers.Embed.apply(t, i, ops, None, 2.0).requires_grad
    with pytest.raises(ValueError):
        layers.Embed.apply(ref, i, ops, d, 1.0)
    with pytest.raises(RuntimeError):
        y = layers.Embed.apply(t, i, ops, d, 2.0)
        g, = torch.autograd.grad(y, [y], dy, create_graph=True)
        x = torch.ones(1, device="cuda", requires_grad=True)
        z = layers.Embed.apply(t, i, ops, d, 2.0) * x
        a, = torch.autograd.grad(z.sum(), [x], create_graph=True)
        torch.autograd.grad(a, [x])


def test_refusals(ops):
    import torch
    from paper_2609_23898_b200 import layers
    t, i = torch.randn(4, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    dy = torch.randn(3, 8, device="cuda")
    with pytest.raises(TypeError):
        layers.embed(ops, t.half(), i)
    with pytest.raises(TypeError):
        layers.embed(ops, t, i.float())
    with pytest.raises(TypeError):
        layers.embed(ops, t, i, dtype=torch.float16)
    with pytest.raises(ValueError):
        layers.embed(ops, t.cpu(), i)
    with pytest.raises(ValueError):
        layers.embed(ops, t, i.cpu())
    with pytest.raises(ValueError):
        layers.embed(ops, t.t(), i)
    with pytest.raises(ValueError):
        layers.embed_backward(ops, dy[:2], i, t)
    with pytest.raises(ValueError):
        layers.embed_backward(ops, dy[:, :7], i, t)
    with pytest.raises(ValueError):
        layers.embed_backward(ops, dy, i, t.t())
    with pytest.raises(TypeError):
        layers.embed_backward(ops, dy, i, t.double())


def test_captured_and_replayed(ops):
    import torch
    from paper_2609_23898_b200 import layers
    t, d = torch.randn(500, 64, device="cuda"), torch.zeros(500, 64, device="cuda")
    i, dy = ids_of("uniform", 5000, 500, 1), torch.randn(5000, 64, device="cuda")
    layers.embed(ops, t, i)
    layers.embed_backward(ops, dy, i, d, accumulate=False)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = layers.embed(ops, t, i)
        layers.embed_backward(ops, dy, i, d, accumulate=False)
    i.copy_(ids_of("zipf", 5000, 500, 2))
    dy.normal_()
    g.replay()
    assert torch.equal(y, t[i])
    e = torch.zeros_like(d)
    layers.embed_backward(ops, dy, i, e, accumulate=False)
    assert torch.equal(d, e)
