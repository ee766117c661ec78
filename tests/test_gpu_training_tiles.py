"""8-bit products of more tiles than the GPU has SMs, on the GPU against 64 bits: the 256-column tiles (pairs of blocks where the scales
are powers of two) and blocks that go through several tiles, with remainders on every side.

Tolerance, as in test_gpu_training.py (u = 2^-24): |C - C64| <= 2 u (128 + blocks + 4) sum |A||B| (+ 2 u (|C0| + |C64|) where C0 is added to, + half
the distance of two bfloat16 numbers at C64).
"""
import ctypes as C

import pytest

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


def tile(m, n, k, pow2):
    import torch
    from paper_2609_23898_b200 import cerar
    split = C.c_int()
    cols = cerar.lib.cerar_fp8_matmul_tile(m, n, k, int(pow2), torch.cuda.get_device_properties(0).multi_processor_count, C.byref(split))
    return cols, split.value


def operand(gen, rows, cols, scaling, pow2):
    """A Quantized of codes over the whole format with NaN between its rows and its scales' rows, and its values in 64 bits."""
    import torch
    from paper_2609_23898_b200 import training as R
    ld = -(-cols // 16) * 16 + 16
    buf = torch.full((rows, ld), 0x7F, dtype=torch.uint8, device="cuda")
    codes = torch.randint(0, 256, (rows, cols), generator=gen, device="cuda", dtype=torch.int32)
    codes = torch.where(codes % 128 == 127, codes - 1, codes)                 # (no NaN)
    codes = torch.where(torch.rand(rows, cols, generator=gen, device="cuda") < 0.5, codes & 0xBF, codes)   # more of the smaller values
    buf[:, :cols] = codes.to(torch.uint8)
    nr, nc = -(-rows // 128), -(-cols // 128)
    shape = {0: (nc, rows), 1: (nr, cols), 2: (nr, nc)}[scaling]
    e = torch.rand(shape, generator=gen, device="cuda") * 9 - 6
    wide = torch.full((shape[0], shape[1] + 3), float("nan"), device="cuda")
    wide[:, :shape[1]] = torch.exp2(e.floor()) if pow2 else torch.exp2(e)
    q = R.Quantized(buf[:, :cols], wide[:, :shape[1]], scaling)
    assert q.desc.pow2 == int(pow2)
    s = q.scales.double().t() if scaling == 0 else q.scales.double()
    if scaling != 0:
        s = s.repeat_interleave(128, 0)[:rows]
    if scaling != 1:
        s = s.repeat_interleave(128, 1)[:, :cols]
    return q, q.codes.view(torch.float8_e4m3fn).double() * s


def bound(a, b, k, c64, bf16):
    import torch
    half = torch.exp2(torch.floor(torch.log2(c64.abs().clamp(min=1e-37))) - 8) if bf16 else 0.0
    return 2 * U * (128 + -(-k // 128) + 4) * (a.abs() @ b.abs()) * (1 + bf16 * 2.0 ** -7) + half + 1e-30


# Every kernel with tiles of either width, in one turn of the GPU and in several (test_training_host.py holds the rule to it).
# (m, n, k): tile columns and the turns a GPU of 148 SMs takes, (any scales, powers of two)
SIZES = {(2601, 2499, 2300): ((128, 3), (256, 2)),
         (3700, 2555, 2300): ((256, 2), (128, 4)),
         (1800, 2180, 300): ((256, 1), (256, 1)),
         (2450, 2600, 130): ((128, 3), (128, 3)),
         (1300, 2300, 4300): ((256, 1), (256, 1))}


@pytest.mark.parametrize("m,n,k", list(SIZES))
@pytest.mark.parametrize("trans_a,trans_b", [(False, True), (False, False), (True, False), (True, True)])
@pytest.mark.parametrize("pow2", [False, True])
def test_product_of_many_tiles(ops, m, n, k, trans_a, trans_b, pow2):
    import torch
    assert tile(m, n, k, pow2) == (SIZES[m, n, k][pow2][0], 1)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + n + k + 2 * trans_a + trans_b)
    for a_block, b_block in ((False, False), (False, True), (True, False)):
        A, a = operand(gen, *((k, m) if trans_a else (m, k)), 2 if a_block else int(trans_a), pow2)
        B, b = operand(gen, *((n, k) if trans_b else (k, n)), 2 if b_block else int(not trans_b), pow2)
        a, b = (a.t() if trans_a else a), (b.t() if trans_b else b)
        c64 = a @ b
        for dtype in (torch.float32, torch.bfloat16):
            err = bound(a, b, k, c64, dtype == torch.bfloat16)
            # rows 16 bytes apart and not, a column of guards on either side, and twice the same bits
            for ldc, first in ((-(-n // 8) * 8 + 8, 0), (n + 2, 2), (n + 1, 1)):
                start = torch.full((m * ldc + 16,), -3.0, device="cuda", dtype=dtype)
                runs = []
                for _ in range(2):
                    buf = start.clone()
                    ops.matmul(A, B, trans_a=trans_a, trans_b=trans_b, out=buf.as_strided((m, n), (ldc, 1), first))
                    runs.append(buf)
                got = runs[0].as_strided((m, n), (ldc, 1), first)
                assert bool(((got.double() - c64).abs() <= err).all()), (a_block, b_block, dtype, ldc)
                assert torch.equal(runs[0], runs[1])
                got.fill_(-3.0)
                assert torch.equal(runs[0], start)


@pytest.mark.parametrize("m,n,k", list(SIZES))
@pytest.mark.parametrize("pow2", [False, True])
def test_product_of_many_tiles_accumulates(ops, m, n, k, pow2):
    """The weight gradient's form, dw += dy^T x, into both types, aligned rows and any."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m * 3 + n + k)
    A, a = operand(gen, k, m, 1, pow2)
    B, b = operand(gen, k, n, 1, pow2)
    prod = a.t() @ b
    for dtype in (torch.float32, torch.bfloat16):
        for ldc, first in ((-(-n // 8) * 8, 0), (n + 3, 1)):
            start = (torch.randn(m * ldc + 16, generator=gen, device="cuda") * 100).to(dtype)
            c0 = start.as_strided((m, n), (ldc, 1), first).double()
            runs = []
            for _ in range(2):
                buf = start.clone()
                ops.matmul(A, B, trans_a=True, out=buf.as_strided((m, n), (ldc, 1), first), accumulate=True)
                runs.append(buf)
            c64 = c0 + prod
            got = runs[0].as_strided((m, n), (ldc, 1), first)
            assert bool(((got.double() - c64).abs() <= bound(a.t(), b, k, c64, dtype == torch.bfloat16) + 2 * U * (c0.abs() + c64.abs())).all()), (dtype, ldc)
            assert torch.equal(runs[0], runs[1])
            got.copy_(start.as_strided((m, n), (ldc, 1), first))
            assert torch.equal(runs[0], start)


@pytest.mark.parametrize("pow2", [False, True])
def test_nan_stays_in_its_row_and_column_of_many_tiles(ops, pow2):
    import torch
    m, n, k = 2601, 2499, 2300
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    A, a = operand(gen, m, k, 0, pow2)
    B, b = operand(gen, n, k, 2, pow2)
    for q, places in ((A, [(7, 3), (2600, 2299), (1500, 2100)]), (B, [(300, 250), (2498, 0)])):
        for r, c in places:
            q.codes[r, c] = 0x7F
    want = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    want[[7, 2600, 1500], :] = True
    want[:, [300, 2498]] = True
    assert torch.equal(torch.isnan(ops.matmul(A, B, trans_b=True, dtype=torch.float32)), want)


def test_a_layer_of_many_tiles(ops):
    """The sizes of a layer's three products together: forward, input gradient, accumulated weight gradient, against 64-bit products of
    the same 8-bit operands."""
    import torch
    from paper_2609_23898_b200 import training as R
    torch.manual_seed(0)
    t, n, k = 4100, 2312, 1544
    x, w, dy = (torch.randn(s, device="cuda").bfloat16() for s in ((t, k), (n, k), (t, n)))
    wq, = ops.quantize(w, R.BY_BLOCK)
    y, xc = R.linear(ops, x, wq)
    dw = torch.randn(n, k, device="cuda")
    c0 = dw.double()
    dx = R.linear_backward(ops, dy, xc, wq, dw)
    xr, = ops.quantize(x, R.BY_ROW)
    dr, dc = ops.quantize(dy, R.BY_ROW, R.BY_COLUMN)
    xr, xc, dr, dc, wd = (q.dequantize().double() for q in (xr, xc, dr, dc, wq))
    for got, a, b, s, start in ((y, xr, wd.t(), k, None), (dx, dr, wd, n, None), (dw, dc.t(), xc, t, c0)):
        assert tile(got.size(0), got.size(1), s, True)[1] == 1
        c64 = a @ b if start is None else start + a @ b
        err = bound(a, b, s, c64, got.dtype == torch.bfloat16) + (0.0 if start is None else 2 * U * (start.abs() + c64.abs()))
        assert bool(((got.double() - c64).abs() <= err).all())
