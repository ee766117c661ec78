"""Training-step operators (8-bit products and conversions, gradient norm, AdamW) on the GPU against the 64-bit
restatement in oracle/training.py.

Tolerances, fixed before the first run (u = 2^-24):
  conversion   none: x 2^-e is exact and the code is the nearest one, so codes and scales are equal
  product      |C - C64| <= 2 u (128 + blocks + 4) sum |A||B| (+ half the distance of two bfloat16 numbers at C64); the sums
               have 128 terms per block and one per block, the 2 is for adders that truncate
  norm         4 u relative (binary64 sums; one rounding for the norm, two more for the coefficient), plus 8 u for the
               binary32 sums of eight squares
  AdamW        m: 4 u of the magnitudes of its two terms (they may cancel); v: 5 u; p: 3 u |p| + u |p1| + 24 u of the update
               with those magnitudes in m's place
  8-bit states, bfloat16 parameters  the kept value is the one the random bits ask for, unless the 64-bit number is within
               the bounds above of the point where the choice turns: then its neighbour is right too
"""
import ctypes as C

import numpy as np
import pytest

from oracle import training as T

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


def dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def f64(t):
    return t.detach().double().cpu().numpy()


SHAPE = {0: (1, 128), 1: (128, 1), 2: (128, 128)}             # BY_ROW, BY_COLUMN, BY_BLOCK


def oracle_scales(q):
    """Scales of a Quantized in the oracle's [row blocks, column blocks] order."""
    s = f64(q.scales)
    return s.T if q.scaling == 0 else s


# ---------------------------------------------------------------------------------------------------- conversion

@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols,ldx,offset", [(1, 1, 1, 0), (1, 128, 128, 0), (1, 2048, 2048, 0), (128, 128, 128, 0), (127, 129, 129, 0),
                                                  (130, 5, 9, 0), (300, 1000, 1000, 0), (257, 384, 400, 4), (100, 200, 203, 3), (16, 131, 132, 1)])
def test_quantize(ops, rows, cols, ldx, offset, dtype):
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(rows * 1000 + cols)
    x = rng.standard_normal((rows, cols)) * 10.0 ** rng.uniform(-5, 5, (1, cols)) * 10.0 ** rng.uniform(-3, 3, (rows, 1))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    buf = torch.full((rows * ldx + offset + 8,), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    view = buf[offset:].as_strided((rows, cols), (ldx, 1), storage_offset=offset)
    view.copy_(dev(x))
    want = f64(view)
    for forms in ([0], [1], [2], [0, 1], [2, 0], [1, 2], [0, 1, 2]):
        for q in ops.quantize(view, *forms):
            qc, qs = T.quantize(want, *SHAPE[q.scaling])
            assert np.array_equal(oracle_scales(q), qs), (forms, q.scaling)
            assert np.array_equal(f64(q.codes), qc), (forms, q.scaling)
            assert np.array_equal(f64(q.dequantize()), T.dequantize(qc, qs, *SHAPE[q.scaling]))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_special_values(ops, dtype):
    import torch
    from paper_2609_23898_b200 import training as R
    x = np.random.default_rng(0).standard_normal((260, 300))
    x[3, 5], x[3, 200], x[130, 7], x[259, 299] = np.nan, np.inf, -np.inf, np.nan
    x[10, :] = 0.0
    x[:, 20] = 0.0
    x[40, :128], x[41, :128], x[42, :128] = 3e38, 1e-38, 1e-42               # scale at its bounds
    x[128:256, 128:256] = 0.0
    x[200, 140:150] = np.inf                                                # a block whose finite part is zero
    t = dev(x).to(getattr(torch, dtype))
    want = f64(t)
    for q in ops.quantize(t, 0, 1, 2):
        qc, qs = T.quantize(want, *SHAPE[q.scaling])
        assert np.array_equal(oracle_scales(q), qs)
        assert np.array_equal(f64(q.codes), qc, equal_nan=True)


def test_quantize_of_nothing(ops):
    import torch
    for shape in ((0, 5), (5, 0), (0, 0)):
        for q in [*ops.quantize(torch.empty(*shape, device="cuda"), 0, 1, 2), *ops.quantize(torch.empty(*shape, device="cuda"), 1)]:
            assert tuple(q.codes.shape) == shape and q.dequantize().shape == shape


def test_quantize_writes_nothing_else(ops):
    """Codes between cols and ld, scales beyond the matrix and the bytes behind it keep what they hold."""
    import torch
    from paper_2609_23898_b200 import cerar
    rows, cols, ld = 131, 70, 96
    x = torch.randn(rows, cols, device="cuda")
    for scaling, (nr, nc) in {0: (1, rows), 1: (2, cols), 2: (2, 1)}.items():
        codes = torch.full((rows * ld + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        scales = torch.full((nr, nc + 3), -7.0, device="cuda")
        d = cerar.Fp8Matrix(codes.data_ptr(), scales.data_ptr(), rows, cols, ld, nc + 3, scaling)
        cerar._check(cerar.lib.cerar_fp8_quantize(ops._h, x.data_ptr(), 0, cols, C.addressof(d), 1, torch.cuda.current_stream().cuda_stream))
        body = codes[:rows * ld].view(rows, ld)
        assert bool((body[:, cols:] == 0xA5).all()) and bool((codes[rows * ld:] == 0xA5).all())
        assert bool((scales[:, nc:] == -7.0).all()) and bool((scales[:, :nc] > 0).all())


# ---------------------------------------------------------------------------------------------------- products

def random_matrix(rng, rows, cols, scaling, nan=(), pow2=False):
    """A Quantized with codes over the whole format and positive scales (any, or powers of two), and its 64-bit values."""
    from paper_2609_23898_b200 import training as R
    import torch
    codes = np.delete(np.arange(256), [0x7F, 0xFF])[rng.integers(0, 254, (rows, cols))].astype(np.uint8)
    codes[rng.random((rows, cols)) < 0.5] &= 0xBF                            # more of the smaller values
    for r, c in nan:
        codes[r, c] = 0x7F
    nr, nc = -(-rows // 128), -(-cols // 128)
    shape = {0: (nc, rows), 1: (nr, cols), 2: (nr, nc)}[scaling]
    e = rng.uniform(-6, 3, shape)
    scales = (2.0 ** (np.floor(e) if pow2 else e)).astype(np.float32)
    ld = -(-cols // 16) * 16 + 16 * int(rng.integers(0, 3))
    buf = torch.full((rows, ld), 0x7F, dtype=torch.uint8, device="cuda")      # NaN between the rows: must not be read as data
    buf[:, :cols] = dev(codes)
    wide = torch.full((shape[0], shape[1] + 3), float("nan"), device="cuda")
    wide[:, :shape[1]] = dev(scales)
    q = R.Quantized(buf[:, :cols], wide[:, :shape[1]], scaling)
    s = scales.T if scaling == 0 else scales
    return q, T.dequantize(T.e4m3_values()[codes], s.astype(np.float64), *SHAPE[scaling])


def product_bound(a, b, blocks, c64, bf16):
    half = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(c64), 1e-37))) - 8) if bf16 else 0      # 8 significant bits
    return 2 * U * (128 + blocks + 4) * (np.abs(a) @ np.abs(b)) * (1 + bf16 * 2.0 ** -7) + half + 1e-30


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 1, 128), (1, 300, 2048), (5, 64, 100), (128, 256, 128), (127, 255, 129), (129, 257, 127), (64, 1031, 300),
                                   (333, 200, 1000), (256, 512, 384), (700, 900, 640), (2, 2500, 16), (1500, 3, 272), (130, 130, 4100), (16, 16, 20000)])
@pytest.mark.parametrize("trans_a,trans_b", [(False, True), (False, False), (True, False), (True, True)])
@pytest.mark.parametrize("pow2", [False, True])
def test_product(ops, m, n, k, trans_a, trans_b, pow2):
    import torch
    rng = np.random.default_rng(m * 7 + n * 3 + k + 2 * trans_a + trans_b)
    for a_block, b_block, bf16 in ((False, False, False), (False, True, True), (True, False, True), (True, True, False)):
        A, a = random_matrix(rng, *((k, m) if trans_a else (m, k)), 2 if a_block else int(trans_a), pow2=pow2)
        B, b = random_matrix(rng, *((n, k) if trans_b else (k, n)), 2 if b_block else int(not trans_b), pow2=pow2)
        assert A.desc.pow2 == B.desc.pow2 == int(pow2)
        a, b = (a.T if trans_a else a), (b.T if trans_b else b)
        c64 = a @ b
        c = ops.matmul(A, B, trans_a=trans_a, trans_b=trans_b, dtype=torch.bfloat16 if bf16 else torch.float32)
        assert (np.abs(f64(c) - c64) <= product_bound(a, b, -(-k // 128), c64, bf16)).all(), (a_block, b_block)


@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("m,n,k,ldc,offset", [(128, 256, 256, 256, 0), (200, 130, 300, 137, 3), (1, 77, 128, 77, 1), (300, 260, 2000, 264, 8), (257, 128, 136, 130, 2)])
def test_product_accumulates_into_a_strided_buffer(ops, m, n, k, ldc, offset, bf16, pow2):
    """C + A B; what lies between the rows of C and around it stays; twice the same bits."""
    import torch
    rng = np.random.default_rng(m + n)
    A, a = random_matrix(rng, k, m, 1, pow2=pow2)
    B, b = random_matrix(rng, k, n, 1, pow2=pow2)
    dt = torch.bfloat16 if bf16 else torch.float32
    start = torch.randn(m * ldc + offset + 64, device="cuda").to(dt) * 100
    runs = []
    for _ in range(2):
        buf = start.clone()
        view = buf.as_strided((m, n), (ldc, 1), offset)
        c0 = f64(view)
        ops.matmul(A, B, trans_a=True, out=view, accumulate=True)
        runs.append(buf)
    c64 = c0 + a.T @ b
    bound = product_bound(a.T, b, -(-k // 128), c64, bf16) + 2 * U * (np.abs(c0) + np.abs(c64))
    assert (np.abs(f64(runs[0].as_strided((m, n), (ldc, 1), offset)) - c64) <= bound).all()
    assert torch.equal(runs[0], runs[1])
    mask = torch.ones_like(start, dtype=torch.bool)
    mask.as_strided((m, n), (ldc, 1), offset).fill_(False)
    assert torch.equal(runs[0][mask], start[mask])


@pytest.mark.parametrize("pow2", [False, True])
def test_product_nan_stays_in_its_row_and_column(ops, pow2):
    import torch
    rng = np.random.default_rng(5)
    A, a = random_matrix(rng, 300, 500, 0, nan=[(7, 3), (299, 499)], pow2=pow2)
    B, b = random_matrix(rng, 400, 500, 2, nan=[(11, 250)], pow2=pow2)
    c = f64(ops.matmul(A, B, trans_b=True, dtype=torch.float32))
    want = np.zeros((300, 400), bool)
    want[[7, 299], :] = True
    want[:, 11] = True
    assert np.array_equal(np.isnan(c), want)


def test_product_scale_that_is_no_power_of_two_after_all(ops):
    """Declared powers of two, one scale changed afterwards: its row, and nothing else, is NaN."""
    import torch
    rng = np.random.default_rng(6)
    A, a = random_matrix(rng, 200, 700, 0, pow2=True)
    B, b = random_matrix(rng, 300, 700, 2, pow2=True)
    A.scales[3, 77] = 0.75
    c = f64(ops.matmul(A, B, trans_b=True, dtype=torch.float32))
    want = np.zeros((200, 300), bool)
    want[77] = True
    assert np.array_equal(np.isnan(c), want)


def test_product_extreme_scales(ops):
    """Scales at the ends of what the conversion writes (2^-100, 2^100), whose products leave the range of one side only."""
    import torch
    rng = np.random.default_rng(8)
    A, a = random_matrix(rng, 130, 300, 0, pow2=True)
    B, b = random_matrix(rng, 140, 300, 0, pow2=True)
    A.scales[:, :65], A.scales[:, 65:] = 2.0 ** 100, 2.0 ** -100
    B.scales.fill_(2.0 ** -20)
    a, b = f64(A.dequantize()), f64(B.dequantize())
    c64 = a @ b.T
    c = f64(ops.matmul(A, B, trans_b=True, dtype=torch.float32))
    assert (np.abs(c - c64) <= product_bound(a, b.T, 3, c64, False)).all()


def test_product_of_nothing(ops):
    import torch
    from paper_2609_23898_b200 import training as R
    A, _ = random_matrix(np.random.default_rng(0), 5, 40, 0)
    empty = R.Quantized.empty(0, 40, 0, "cuda")
    assert ops.matmul(A, empty, trans_b=True).shape == (5, 0)
    assert ops.matmul(empty, A, trans_b=True).shape == (0, 5)
    k0 = R.Quantized.empty(5, 0, 0, "cuda")
    out = torch.full((5, 5), 3.0, device="cuda")
    ops.matmul(k0, k0, trans_b=True, out=out, accumulate=True)
    assert bool((out == 3).all())
    ops.matmul(k0, k0, trans_b=True, out=out)
    assert bool((out == 0).all())


def test_product_offsets_beyond_32_bits(ops):
    """An output of more than 2^31 elements: rows near the end land where they belong."""
    import torch
    rng = np.random.default_rng(9)
    m, n, k = 70001, 32768, 16
    A, a = random_matrix(rng, m, k, 0)
    B, b = random_matrix(rng, n, k, 2)
    out = torch.full((m * n,), float("nan"), dtype=torch.bfloat16, device="cuda").view(m, n)
    ops.matmul(A, B, trans_b=True, out=out)
    assert not bool(torch.isnan(out).any())
    for r in (0, 1, 65535, 65536, 69999, 70000):
        c64 = a[r:r + 1] @ b.T
        assert (np.abs(f64(out[r:r + 1]) - c64) <= product_bound(a[r:r + 1], b.T, 1, c64, True)).all(), r


def test_product_on_another_stream_and_in_a_graph(ops):
    import torch
    rng = np.random.default_rng(3)
    A, a = random_matrix(rng, 200, 700, 0)
    B, b = random_matrix(rng, 300, 700, 0)
    want = ops.matmul(A, B, trans_b=True, dtype=torch.float32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.zeros(200, 300, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ops.matmul(A, B, trans_b=True, out=out)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    out.zero_()
    with torch.cuda.graph(graph):
        ops.matmul(A, B, trans_b=True, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


# ---------------------------------------------------------------------------------------------------- a linear layer

def test_linear_gradients_against_differences(ops):
    """Inputs the format holds exactly (small integers), so y, dx and dw are those of the layer itself: equal to the formulas, and
    to central differences of sum(dy y), which is linear in x and in w, in 64 bits."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(1)
    t, n, k = 150, 70, 200
    x, w, dy = (rng.integers(-8, 9, s).astype(np.float64) for s in ((t, k), (n, k), (t, n)))
    xt = dev(x, torch.float32).requires_grad_()
    wq, = ops.quantize(dev(w, torch.float32), R.BY_BLOCK)
    dw = torch.ones(n, k, device="cuda")
    y = R.Linear8.apply(xt.view(10, 15, k), wq, ops, dw)
    assert y.shape == (10, 15, n)
    y.backward(dev(dy, torch.float32).view(10, 15, n))
    assert np.array_equal(f64(y).reshape(t, n), x @ w.T)
    assert np.array_equal(f64(xt.grad), dy @ w)
    assert np.array_equal(f64(dw), 1 + dy.T @ x)
    loss = lambda x, w: float((dy * (x @ w.T)).sum())  # noqa: E731
    for _ in range(20):
        i, j, o = rng.integers(t), rng.integers(k), rng.integers(n)
        e = np.zeros_like(x); e[i, j] = 0.5
        assert abs(loss(x + e, w) - loss(x - e, w) - f64(xt.grad)[i, j]) <= 1e-9 * np.abs(dy @ w).max()
        e = np.zeros_like(w); e[o, j] = 0.5
        assert abs(loss(x, w + e) - loss(x, w - e) - (f64(dw)[o, j] - 1)) <= 1e-9 * np.abs(dy.T @ x).max()


def test_linear_backward_parts(ops):
    """dx alone and dw alone are the same bits as both together; bfloat16 layer; dw into a slice of a flat vector."""
    import torch
    from paper_2609_23898_b200 import training as R
    torch.manual_seed(0)
    x, w, dy = (torch.randn(s, device="cuda", dtype=torch.bfloat16) for s in ((200, 100), (60, 100), (200, 60)))
    wq, = ops.quantize(w, R.BY_BLOCK)
    y, xc = R.linear(ops, x, wq)
    flat = torch.zeros(1 + 60 * 100 + 5, device="cuda")
    dw = flat[1:1 + 6000].view(60, 100)                                   # starts off every vector boundary
    dx = R.linear_backward(ops, dy, xc, wq, dw)
    assert dx.dtype == torch.bfloat16 and flat[0] == 0 and bool((flat[6001:] == 0).all())
    assert torch.equal(dx, R.linear_backward(ops, dy, xc, wq, None))
    dw2 = torch.zeros(60, 100, device="cuda")
    assert R.linear_backward(ops, dy, xc, wq, dw2, need_dx=False) is None
    assert torch.equal(dw, dw2)
    # against the layer without any rounding: each factor is within 2^-4 of its value or of 2^-9 / 448 of its block's top
    for got, a, b in ((y, x, w.t()), (dx, dy, w), (dw, dy.t(), x)):
        a, b = f64(a), f64(b)
        da, db = np.abs(a) / 16 + np.abs(a).max() * 2.0 ** -17, np.abs(b) / 16 + np.abs(b).max() * 2.0 ** -17
        assert (np.abs(f64(got) - a @ b) <= (da @ np.abs(b) + np.abs(a) @ db + da @ db) * 1.01 + 2.0 ** -8 * np.abs(a @ b)).all()


# ---------------------------------------------------------------------------------------------------- norm

def tensors_of(rng, sizes, dtype, offset, std=1.0):
    """Tensors of the given sizes end to end in one buffer that starts `offset` elements after an aligned address."""
    import torch
    flat = torch.empty(sum(sizes) + offset + 4, dtype=dtype, device="cuda")
    flat.copy_(dev(rng.standard_normal(flat.numel()) * std))
    out, at = [], offset
    for n in sizes:
        out.append(flat[at:at + n])
        at += n
    return flat, out


SIZES = [[1], [256, 2048, 4096], [255, 257, 1, 0, 2047, 2049, 3], [100000, 7, 4096 * 3], [1 << 20]]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("sizes", SIZES + [[0], []])
def test_norm(ops, sizes, offset, dtype):
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(len(sizes))
    for std in (1.0, 1e-3, 1e15, 1e-18):
        _, g = tensors_of(rng, sizes, getattr(torch, dtype), offset, std)
        s = R.TensorSet(ops, grads=g)
        for max_norm in (1.0, 0.0, 1e20):
            norm, coef, finite = f64(s.grad_norm(max_norm))
            n64, c64, f = T.grad_norm([f64(t) for t in g], max_norm)
            assert abs(norm - n64) <= 12 * U * n64 and abs(coef - c64) <= 16 * U * c64 + 1e-44 and finite == f == 1.0
        a, b = s.grad_norm(1.0), s.grad_norm(1.0)
        assert torch.equal(a, b)


def test_norm_special_values(ops):
    import torch
    from paper_2609_23898_b200 import training as R
    g = torch.randn(5000, device="cuda")
    s = R.TensorSet(ops, grads=[g[:3000], g[3000:]])
    for bad in (float("inf"), float("-inf"), float("nan")):
        g[4999] = bad
        norm, coef, finite = f64(s.grad_norm(1.0))
        assert not np.isfinite(norm) and coef == 0 and finite == 0
    g.zero_()
    assert np.array_equal(f64(s.grad_norm(1.0)), [0, 1, 1])
    g[7] = 1e-30                                                            # its square is no binary32 number
    assert abs(f64(s.grad_norm(1.0))[0] - float(g[7])) <= 12 * U * 1e-30
    g[7], g[4000] = 1e30, 1e30
    n64 = np.sqrt(2) * float(g[7])
    assert abs(f64(s.grad_norm(1.0))[0] - n64) <= 12 * U * n64
    g.fill_(3e38)                                                           # finite gradients, norm above the largest number
    assert np.array_equal(f64(s.grad_norm(1.0)), [np.inf, 0, 0])


def test_set_grads(ops):
    import torch
    from paper_2609_23898_b200 import training as R
    a = [torch.full((n,), 2.0, device="cuda") for n in [3] * 700]
    b = [torch.full((n,), 1.0, device="cuda") for n in [3] * 700]
    s = R.TensorSet(ops, grads=a)
    first = s.grad_norm()
    s.set_grads(b)
    second = s.grad_norm()
    assert abs(float(first[0]) - 2 * np.sqrt(2100)) < 1e-4 and abs(float(second[0]) - np.sqrt(2100)) < 1e-4
    with pytest.raises(ValueError):
        s.set_grads(b[:-1])
    with pytest.raises(TypeError):
        s.set_grads([t.bfloat16() for t in b])


# ---------------------------------------------------------------------------------------------------- AdamW

HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8)


def between(kept, x, error, spacing, offset, least=0.0):
    """Whether kept is what the random offset makes of a magnitude within `error` of x (the kept value grows with the
    magnitude, across the places where the spacing changes too)."""
    ends = []
    for y in (np.maximum(x - error, 0.0), x + error):
        d = spacing(y)
        ends.append(np.maximum(np.floor(y / d + offset) * d, least))
    return (kept >= ends[0]) & (kept <= ends[1])


def check_state8(codes, scales, want, error, bits16, floor_one):
    """Codes and scales of one tensor against the 64-bit moments (which binary32 has within `error`) and the random bits."""
    n = want.size
    nb = -(-n // 256)
    s64 = np.array([T.scale_of(np.abs(want[b * 256:(b + 1) * 256]).max()) for b in range(nb)])
    assert np.array_equal(scales, s64)
    y = want / np.repeat(s64, 256)[:n]
    got = T.e4m3_values()[codes]
    sure = (got != 0) & (np.abs(want) > error)                              # (a sum that cancels may have either sign)
    assert np.array_equal(np.sign(got)[sure], np.sign(y)[sure])
    least = np.where(y > 0, 2.0 ** -9, 0.0) if floor_one else 0.0
    assert between(np.abs(got), np.abs(y), error / np.repeat(s64, 256)[:n], T.spacing, (bits16.astype(np.float64) + 0.5) / 65536, least).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["float32", "bfloat16"])
@pytest.mark.parametrize("param", ["float32", "bfloat16", "master"])
@pytest.mark.parametrize("sizes,offset", [(SIZES[0], 0), (SIZES[1], 0), (SIZES[2], 0), (SIZES[2], 1), (SIZES[3], 2)])
def test_adamw(ops, sizes, offset, param, grad, bits):
    """Three steps; every step is checked from the state the kernels themselves left before it."""
    import torch
    from paper_2609_23898_b200 import training as R
    rng = np.random.default_rng(sum(sizes) + offset)
    pt = torch.float32 if param == "float32" else torch.bfloat16
    pflat, params = tensors_of(rng, sizes, pt, offset, 0.02)
    mflat, masters = tensors_of(rng, sizes, torch.float32, offset, 0.02) if param == "master" else (None, None)
    gflat, grads = tensors_of(rng, sizes, getattr(torch, grad), offset, 1e-3)
    decay = [0.1 * (i % 2) for i in range(len(sizes))]
    lrs = [1.0 if i % 3 else 0.5 for i in range(len(sizes))]
    s = R.TensorSet(ops, grads=grads, params=params, masters=masters, state_bits=bits, weight_decay=decay, lr_scale=lrs)
    clip = torch.tensor([2.0, 0.5, 1.0], device="cuda")
    for step in range(1, 4):
        seed = (7 << 32) + step
        gflat.copy_(dev(rng.standard_normal(gflat.numel()) * 1e-3))
        before = [f64(t) for t in (masters or params)]
        edges = (pflat[:offset].clone(), pflat[offset + sum(sizes):].clone())
        if bits == 32:
            m0, v0 = f64(s.m), f64(s.v)
        else:
            wide = lambda t: np.repeat(f64(t), 256)  # noqa: E731
            m0, v0 = f64(s.m) * wide(s.m_scale), (f64(s.v) * wide(s.v_scale)) ** 2
        c = clip if step > 1 else None
        s.adamw(lr=HYPER["lr"], betas=(0.9, 0.95), eps=1e-8, step=step, clip=c, seed=seed)
        assert torch.equal(edges[0], pflat[:offset]) and torch.equal(edges[1], pflat[offset + sum(sizes):])
        for i, n in enumerate(sizes):
            if n == 0:
                continue
            at = s.state_offsets[i]
            g = f64(grads[i])
            lr = HYPER["lr"] * lrs[i]
            p64, m64, v64, _ = T.adamw(before[i], g, m0[at:at + n], v0[at:at + n], lr=lr, beta1=0.9, beta2=0.95, eps=1e-8,
                                        decay=np.float64(np.float32(decay[i])), step=step, coef=0.5 if c is not None else 1.0)
            gs = 0.5 * g if c is not None else g
            terms = np.abs(0.9 * m0[at:at + n]) + np.abs(0.1 * gs)
            up = lr / (1 - 0.9 ** step) * terms / (np.sqrt(v64 / (1 - 0.95 ** step)) + 1e-8)
            bound = 3 * U * np.abs(before[i]) + 24 * U * up + U * np.abs(p64)
            got = f64((masters or params)[i])
            if param != "bfloat16":
                assert (np.abs(got - p64) <= bound).all()
                if param == "master":
                    assert torch.equal(params[i], masters[i].bfloat16())
            else:
                h = T.random_bits(at // 256, n, seed, 1) >> np.uint64(16)
                spacing = lambda x: 2.0 ** (np.floor(np.log2(np.maximum(x, 1e-37))) - 7)  # noqa: E731
                assert between(np.abs(got), np.abs(p64), bound, spacing, h.astype(np.float64) / 65536).all()
            if bits == 32:
                assert (np.abs(f64(s.m)[at:at + n] - m64) <= 4 * U * terms).all()
                assert (np.abs(f64(s.v)[at:at + n] - v64) <= 5 * U * (0.95 * v0[at:at + n] + 0.05 * gs * gs)).all()
            else:
                h = T.random_bits(at // 256, n, seed, 0)
                blk = slice(at // 256, at // 256 + -(-n // 256))
                check_state8(s.m.view(torch.uint8)[at:at + n].cpu().numpy(), f64(s.m_scale)[blk], m64, 4 * U * terms, h >> np.uint64(16), False)
                check_state8(s.v.view(torch.uint8)[at:at + n].cpu().numpy(), f64(s.v_scale)[blk], np.sqrt(v64), 4 * U * np.sqrt(v64), h & np.uint64(0xFFFF), True)


def small_set(ops, bits=8, param="bfloat16", n=3000):
    import torch
    from paper_2609_23898_b200 import training as R
    torch.manual_seed(0)
    p = torch.randn(n, device="cuda").to(torch.bfloat16 if param != "float32" else torch.float32)
    g = torch.randn(n, device="cuda")
    return R.TensorSet(ops, grads=[g[:1000], g[1000:]], params=[p[:1000], p[1000:]], state_bits=bits), p, g


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_skips_a_step_whose_norm_is_not_finite(ops, bits):
    import torch
    s, p, g = small_set(ops, bits)
    s.adamw(lr=1e-2, step=1, seed=1)
    keep = [t.clone() for t in (p, s.m.view(torch.uint8), s.v.view(torch.uint8))]
    g[5] = float("nan")
    s.adamw(lr=1e-2, step=2, seed=2, clip=s.grad_norm(1.0))
    for a, b in zip(keep, (p, s.m.view(torch.uint8), s.v.view(torch.uint8))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("param", ["float32", "bfloat16"])
def test_adamw_nan_stays_in_its_element(ops, bits, param):
    import torch
    s, p, g = small_set(ops, bits, param)
    g[5], g[2000] = float("nan"), float("inf")
    for step in (1, 2):
        s.adamw(lr=1e-2, step=step, seed=step)
        g.normal_()
    bad = torch.isnan(p)
    assert bad.sum() == 2 and bad[5] and bad[2000]
    m = s.m.float()
    off = s.state_offsets[1] - 1000
    assert (~torch.isfinite(m)).nonzero().squeeze(1).tolist() == [5, 2000 + off]


def test_adamw_is_reproducible_and_capturable(ops):
    import torch
    out = []
    for run in range(3):
        s, p, g = small_set(ops)
        if run < 2:
            s.adamw(lr=1e-2, step=1, seed=9, clip=s.grad_norm(1.0))
        else:
            clip = torch.empty(3, device="cuda")
            s.grad_norm(1.0, out=clip)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                s.grad_norm(1.0, out=clip)
                s.adamw(lr=1e-2, step=1, seed=9, clip=clip)
            graph.replay()
        out.append((p.clone(), s.m.view(torch.uint8).clone(), s.v.view(torch.uint8).clone()))
    for other in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(out[0], other))


def test_adamw_8_bit_states_hold_a_small_constant_gradient(ops):
    """Rounding to nearest would stop the first moment at about 0.6 of a constant gradient; at random it gets there: mean over
    64 blocks x 256 elements after 60 steps within 1 % (noise of one element 9 %, of the mean 0.1 %)."""
    import torch
    from paper_2609_23898_b200 import training as R
    n = 64 * 256
    g = torch.full((n,), 1e-3, device="cuda")
    p = torch.zeros(n, device="cuda")
    s = R.TensorSet(ops, grads=[g], params=[p], state_bits=8)
    for step in range(1, 61):
        s.adamw(lr=1e-3, step=step, seed=step)
    m = (s.m.float().view(-1, 256) * s.m_scale[:, None]).mean().item()
    assert abs(m / (1e-3 * (1 - 0.9 ** 60)) - 1) < 0.01


# ---------------------------------------------------------------------------------------------------- long tensors

def test_more_than_32_bits_of_elements(ops):
    """A tensor of more than 2^31 elements: norm, 8-bit states, stochastic bfloat16 and conversion at its far end."""
    import torch
    from paper_2609_23898_b200 import training as R
    n, tail = (1 << 31) + 1000, 700
    g = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    g[-tail:].normal_(std=1e-3)
    p = torch.zeros_like(g)
    p[-tail:].normal_(std=0.02)
    s = R.TensorSet(ops, grads=[g], params=[p], state_bits=8)
    gt, pt = f64(g[-tail:]), f64(p[-tail:])
    n64 = np.sqrt((gt ** 2).sum())
    assert abs(f64(s.grad_norm(1.0))[0] - n64) <= 12 * U * n64
    s.adamw(lr=1e-3, step=1, seed=3)
    p64, m64, v64, up = T.adamw(pt, gt, 0.0, 0.0, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, decay=0.0, step=1)
    first = (n - tail) // 256 * 256                                          # the block of the first of them, and what is before it there
    pad = n - tail - first
    h1 = T.random_bits(first // 256, tail + pad, 3, 1)[pad:] >> np.uint64(16)
    h0 = T.random_bits(first // 256, tail + pad, 3, 0)[pad:]
    spacing = lambda x: 2.0 ** (np.floor(np.log2(np.maximum(x, 1e-37))) - 7)  # noqa: E731
    assert between(np.abs(f64(p[-tail:])), np.abs(p64), 3 * U * np.abs(pt) + 24 * U * np.abs(up) + U * np.abs(p64), spacing, h1.astype(np.float64) / 65536).all()
    full = np.concatenate([np.zeros(pad), m64])
    bits = np.concatenate([np.zeros(pad, np.uint64), h0])
    codes = s.m.view(torch.uint8)[first:n].cpu().numpy()
    check_state8(codes, f64(s.m_scale)[first // 256:], full, 4 * U * np.abs(full), bits >> np.uint64(16), False)
    assert not bool(p[:1 << 20].any()) and not bool(s.m.view(torch.uint8)[(1 << 31) - (1 << 20):1 << 31].any())
    del s, p
    x = g[:(n // 4096) * 4096].view(-1, 4096)
    x[-3:].normal_()
    want = f64(x[-3:])
    q, = ops.quantize(x, 0)
    qc, qs = T.quantize(want, 1, 128)
    assert np.array_equal(f64(q.codes[-3:]), qc) and np.array_equal(f64(q.scales[:, -3:]).T, qs)


# ---------------------------------------------------------------------------------------------------- together

@pytest.mark.parametrize("bits", [8, 32])
def test_step_of_all_workers(bits):
    """The example: products, ring, clip and optimizer together.  The decoded mean is the workers' mean gradient up to the design's
    error, the gradient that enters the ring is the layers' own (64-bit products of the same 8-bit operands), the loss falls."""
    import torch
    from paper_2609_23898_b200 import example, training as R
    job = example.Job(workers=4, tokens=160, width=200, hidden=328, state_bits=bits)
    losses = [job.step().item() for _ in range(40)]
    job.check()
    exact = job.grads.double().mean(0)
    # eps = 1e-2: the design's error is of that order (below 10 eps); binary32 adds about kappa 2^-24 = 1e-3 of it
    for i in range(4):
        assert ((job.means[i].double() - exact).norm() / exact.norm()).item() < 0.1
    n64 = float(job.means[0][:sum(p.numel() for p in job.params)].double().norm())
    assert abs(job.clip[0].item() - n64) <= 12 * U * n64 and job.clip[2].item() == 1
    assert losses[-1] < 0.7 * losses[0]
    x = torch.randn(160, 200, device="cuda", dtype=torch.bfloat16)
    w, = job.ops.quantize(job.params[0], R.BY_BLOCK)
    y, xc = R.linear(job.ops, x, w)
    dy = torch.randn_like(y)
    dw = torch.zeros(328, 200, device="cuda")
    R.linear_backward(job.ops, dy, xc, w, dw)
    dc, = job.ops.quantize(dy, R.BY_COLUMN)
    a, b = f64(dc.dequantize()).T, f64(xc.dequantize())
    assert (np.abs(f64(dw) - a @ b) <= product_bound(a, b, 2, a @ b, False)).all()


# ---------------------------------------------------------------------------------------------------- refusals

def test_refusals(ops):
    import torch
    from paper_2609_23898_b200 import cerar, training as R
    x = torch.randn(64, 64, device="cuda")
    q0, q1, q2 = ops.quantize(x, 0, 1, 2)
    n0 = ops.launch_count()

    def refused(status, call, *a, **k):
        with pytest.raises(cerar.CerarError) as e:
            call(*a, **k)
        assert e.value.status == status, e.value

    refused(1, ops.quantize, x)                                            # no output
    refused(1, ops.quantize, x, 0, 0)                                      # the same scaling twice
    refused(1, ops.matmul, q1, q0, trans_b=True)                           # scales across the sum
    refused(1, ops.matmul, q0, q0)
    refused(2, ops.matmul, q0, ops.quantize(x[:, :32].contiguous(), 0)[0], trans_b=True)
    n0 += 1
    for bad in (x.half(), x.to(torch.float64)):
        with pytest.raises(TypeError):
            ops.quantize(bad, 0)
    for bad in (x.t(), x[0], x.cpu(), x[:, ::2]):
        with pytest.raises(ValueError):
            ops.quantize(bad, 0)
    with pytest.raises(ValueError):
        ops.matmul(q0, q0, trans_b=True, accumulate=True)
    with pytest.raises(ValueError):
        ops.matmul(q0, q0, trans_b=True, out=torch.empty(64, 63, device="cuda"))
    with pytest.raises(ValueError):
        R.Quantized(q0.codes, q0.scales[:, :10], 0)

    def raw(d, status, cols=64):
        s = cerar.lib.cerar_fp8_quantize(ops._h, x.data_ptr(), 0, 64, C.addressof(d), 1, 0)
        assert s == status and cerar.lib.cerar_last_error()

    c, s = q0.codes.data_ptr(), q0.scales.data_ptr()
    raw(cerar.Fp8Matrix(c + 8, s, 32, 64, 64, 64, 0), 1)                   # codes off a 16-byte boundary
    raw(cerar.Fp8Matrix(c, s, 64, 64, 72, 64, 0), 2)                       # ld not a multiple of 16
    raw(cerar.Fp8Matrix(c, s, 64, 64, 48, 64, 0), 2)                       # ld below cols
    raw(cerar.Fp8Matrix(c, s, 64, 64, 64, 63, 0), 2)                       # lds too small
    raw(cerar.Fp8Matrix(c, s, -1, 64, 64, 64, 0), 2)
    raw(cerar.Fp8Matrix(c, s, 64, 64, 64, 64, 3), 1)
    raw(cerar.Fp8Matrix(None, s, 64, 64, 64, 64, 0), 1)
    raw(cerar.Fp8Matrix(c, s, 64, 65, 80, 64, 0), 2)                       # ldx below cols

    g = [torch.randn(10, device="cuda")]
    p = [torch.randn(10, device="cuda")]
    refused(5, R.TensorSet(ops, grads=g).adamw, lr=0.1, step=1)            # a set without states
    t = R.TensorSet(ops, grads=g, params=p)
    refused(1, t.adamw, lr=0.1, step=0)
    refused(1, t.adamw, lr=float("nan"), step=1)
    refused(1, t.adamw, lr=0.1, step=1, betas=(0.9, 1.0))
    refused(1, t.adamw, lr=0.1, step=1, eps=-1.0)
    refused(1, t.grad_norm, float("nan"))
    with pytest.raises(ValueError):
        t.adamw(lr=0.1, step=1, clip=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        t.adamw(lr=0.1, step=1, clip=torch.ones(3))
    with pytest.raises(ValueError):
        t.grad_norm(1.0, out=torch.ones(3))
    with pytest.raises(ValueError):
        ops.matmul(q0, q0, trans_b=True, out=torch.empty(64, 64))
    with pytest.raises(ValueError):
        R.TensorSet(ops, grads=[torch.ones(3)])
    refused(1, R.TensorSet, ops, grads=g, params=p, masters=[torch.randn(10, device="cuda")])   # master of a float32 parameter
    with pytest.raises(ValueError):
        R.TensorSet(ops, grads=g, params=[torch.randn(9, device="cuda")])
    with pytest.raises(ValueError):
        R.TensorSet(ops, grads=g, params=p, state_bits=16)
    with pytest.raises(ValueError):
        R.TensorSet(ops, grads=g, params=p, m=torch.zeros(10, device="cuda"))
    with pytest.raises(TypeError):
        R.TensorSet(ops, grads=[g[0].half()])
    assert ops.launch_count() == n0                                        # nothing was launched by a refused call
