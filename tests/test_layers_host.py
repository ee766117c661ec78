"""Host side of the layers' operators without a device: which calls layers_api.cu refuses, with which status, and what a call that fails leaves behind
(against fake_cuda.cpp and fake_layers.cpp); the declarations and the binding; the products' choice of tiles; sizes of workspaces."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_23898_b200 import build, cerar

HERE = os.path.dirname(os.path.abspath(__file__))
F32, BF16 = 0, 1
OK, ARG, SHAPE, CUDA = 0, 1, 2, 6
P = 4096                     # an address that looks like device memory; the fakes do not touch it


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    gxx, nvcc = shutil.which("g++"), build._nvcc()
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    assert gxx, "g++ is needed"
    out = str(tmp_path_factory.mktemp("fake") / "libfake.so")
    subprocess.run([gxx, "-std=c++17", "-shared", "-fPIC", "-O1", "-w", "-I", include, "-I", build.CSRC, "-x", "c++", "-Wl,-Bsymbolic",
                    os.path.join(HERE, "fake_cuda.cpp"), os.path.join(HERE, "fake_layers.cpp"), os.path.join(build.CSRC, "ops_api.cu"),
                    os.path.join(build.CSRC, "layers_api.cu"), "-o", out], check=True)
    lib = C.CDLL(out)
    lib.fake_log.restype = lib.fake_error.restype = lib.fake_launches.restype = C.c_char_p
    lib.fake_reset.argtypes = [C.c_char_p]
    for name in ("cerar_ops_create", "cerar_ops_destroy", "cerar_ops_status", "cerar_embed", "cerar_embed_grad", "cerar_rotation_table", "cerar_head_norm",
                 "cerar_head_norm_grad", "cerar_matmul_bf16", "cerar_align_bf16", "cerar_gated_forward", "cerar_gated_backward", "cerar_gated_workspace"):
        getattr(lib, name).argtypes = getattr(cerar.lib, name).argtypes
    lib.cerar_gated_workspace.restype = C.c_size_t
    lib.fake_reset(b"")
    return lib


@pytest.fixture
def ops(fake):
    h = C.c_void_p()
    fake.fake_reset(b"")
    fake.fake_launches_reset(0)
    assert fake.cerar_ops_create(C.byref(h)) == 0
    yield h
    fake.cerar_ops_destroy(h)


def launched(fake):
    out = fake.fake_launches().decode().split("\n")[:-1]
    fake.fake_launches_reset(0)
    return out


def with_changes(good, changes):
    """good with one argument changed at a time: (arguments, wanted status)."""
    yield list(good), OK
    for at, value, status in changes:
        a = list(good)
        a[at] = value
        yield a, status


def check(fake, call, good, changes, name):
    for args, status in with_changes(good, changes):
        got = call(*args)
        assert got == status, (name, args, got, fake.fake_error())
        assert launched(fake) == ([name] if status == OK else [])


def test_embed(fake, ops):
    #       ops table type vocab width ld ids bytes tokens scale y ytype ldy stream
    good = (ops, P, F32, 10, 16, 16, P, 8, 5, 1.0, P, BF16, 16, None)
    check(fake, fake.cerar_embed, good, [(1, None, ARG), (1, P + 2, ARG), (2, 7, ARG), (3, -1, SHAPE), (3, 2 ** 31, SHAPE), (4, -1, SHAPE), (5, 15, SHAPE), (6, None, ARG),
                                         (6, P + 4, ARG), (7, 2, ARG), (8, -1, SHAPE), (8, 2 ** 31, SHAPE), (10, None, ARG), (10, P + 1, ARG), (11, 2, ARG), (12, 8, SHAPE),
                                         (0, None, ARG)], "embed")
    for at, value in ((8, 0), (4, 0)):
        a = list(good)
        a[at] = value
        assert fake.cerar_embed(*a) == OK and launched(fake) == []


def test_embed_grad(fake, ops):
    #       ops dy type lddy ids bytes tokens scale dtable dtype vocab width ld acc ws bytes stream
    good = (ops, P, BF16, 16, P, 4, 5, 1.0, P, F32, 10, 16, 16, 0, P, 1024, None)
    check(fake, fake.cerar_embed_grad, good, [(1, None, ARG), (1, P + 1, ARG), (2, 3, ARG), (3, 15, SHAPE), (4, None, ARG), (4, P + 2, ARG), (5, 3, ARG), (6, -1, SHAPE),
                                              (8, None, ARG), (8, P + 2, ARG), (9, 2, ARG), (10, -2, SHAPE), (11, -1, SHAPE), (12, 7, SHAPE), (14, None, ARG), (14, P + 8, ARG),
                                              (15, 1023, SHAPE)], "embed_grad")
    a = list(good)
    a[6] = 0                                             # no tokens: all rows become zero, without a workspace
    a[14], a[15] = None, 0
    assert fake.cerar_embed_grad(*a) == OK and launched(fake) == ["embed_grad"]
    a[13] = 1                                            # ... and nothing is added
    assert fake.cerar_embed_grad(*a) == OK and launched(fake) == []


def heads(**changes):
    d = dict(x=P, y=P, w=P, dy=P, dw=P, x_token=512, x_head=64, y_token=256, y_head=64, dy_token=256, dy_head=64, heads=4)
    d.update(changes)
    return cerar.Heads(**d)


def rotation(**changes):
    d = dict(table=P, rows=100, positions=P, period=7, position_bytes=8, rotated=64, neighbours=0)
    d.update(changes)
    return cerar.Rotation(**d)


def test_head_norm(fake, ops):
    def call(h=None, r=None, kind=BF16, count=2, w_type=BF16, tokens=7, dim=64, eps=1e-6, grad=False, dw_type=F32, ws=P, size=512, second=None):
        parts = (cerar.Heads * 2)(h or heads(), second or heads())
        rot = r or rotation()
        if grad:
            st = fake.cerar_head_norm_grad(ops, kind, C.addressof(parts), count, w_type, dw_type, 0, tokens, dim, eps, C.addressof(rot), ws, size, None)
        else:
            st = fake.cerar_head_norm(ops, kind, C.addressof(parts), count, w_type, tokens, dim, eps, C.addressof(rot), None)
        return st, launched(fake)

    for grad, name in ((False, "head_norm"), (True, "head_norm_grad")):
        assert call(grad=grad) == (OK, [name])
        for status, kw in ((ARG, dict(kind=2)), (ARG, dict(count=0)), (ARG, dict(count=3)), (ARG, dict(w_type=9)), (SHAPE, dict(tokens=-1)), (SHAPE, dict(tokens=2 ** 31)),
                           (SHAPE, dict(dim=63)), (SHAPE, dict(dim=0)), (SHAPE, dict(dim=514)), (ARG, dict(eps=0.0)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))),
                           (ARG, dict(eps=float("inf"))), (ARG, dict(h=heads(x=None))), (ARG, dict(h=heads(x=P + 1))), (ARG, dict(h=heads(y=None))),
                           (ARG, dict(h=heads(w=P + 1))), (SHAPE, dict(h=heads(heads=-1))), (SHAPE, dict(h=heads(heads=70000))), (ARG, dict(h=heads(x_token=2 ** 40))),
                           (SHAPE, dict(h=heads(y_head=63))), (SHAPE, dict(h=heads(y_token=255))), (SHAPE, dict(h=heads(y_token=0))), (ARG, dict(second=heads(x=None))),
                           (SHAPE, dict(r=rotation(rotated=66))), (SHAPE, dict(r=rotation(rotated=3))), (SHAPE, dict(r=rotation(rotated=-2))), (ARG, dict(r=rotation(table=None))),
                           (ARG, dict(r=rotation(table=P + 4))), (ARG, dict(r=rotation(rows=-1))), (SHAPE, dict(r=rotation(period=0))), (ARG, dict(r=rotation(position_bytes=2))),
                           (ARG, dict(r=rotation(positions=P + 4)))):
            assert call(grad=grad, **kw) == (status, []), (grad, kw)
        for kw in (dict(h=heads(y_head=512, y_token=64), tokens=8), dict(r=rotation(table=None, rotated=0)), dict(r=rotation(positions=None)),
                   dict(h=heads(w=None)), dict(h=heads(heads=0, x=None, y=None, dy=None)), dict(count=1, second=heads(x=None)), dict(h=heads(x_token=0, x_head=0)),
                   dict(h=heads(y_token=-256, y_head=64))):
            assert call(grad=grad, **kw) == (OK, [name]), (grad, kw)
    assert call(tokens=0) == (OK, [])
    for status, kw in ((ARG, dict(h=heads(dy=None))), (ARG, dict(dw_type=5)), (ARG, dict(h=heads(dw=P + 2))), (ARG, dict(ws=None)), (ARG, dict(ws=P + 8)), (SHAPE, dict(size=511))):
        assert call(grad=True, **kw) == (status, []), kw
    for gap, w_type, status in ((16, F32, SHAPE), (127, BF16, ARG), (126, BF16, SHAPE), (128, BF16, OK), (128, F32, SHAPE), (256, F32, OK)):        # dw of both groups
        for a, b in ((P, P + gap), (P + gap, P)):
            assert call(grad=True, h=heads(dw=a), second=heads(dw=b), dw_type=w_type)[0] == status, (gap, w_type)
    assert fake.cerar_head_norm(ops, BF16, None, 1, BF16, 1, 64, 1e-6, C.addressof(rotation()), None) == ARG
    assert fake.cerar_head_norm(ops, BF16, C.addressof((cerar.Heads * 1)(heads())), 1, BF16, 1, 64, 1e-6, None, None) == ARG


def test_rotation_table(fake, ops):
    f = (C.c_double * 4)(1.0, 0.5, 0.25, 0.125)
    bad = (C.c_double * 4)(1.0, float("inf"), 0.25, 0.125)
    check(fake, fake.cerar_rotation_table, (ops, f, 4, 0, 10, P, None), [(1, None, ARG), (1, bad, ARG), (2, 257, SHAPE), (2, -1, SHAPE), (4, -1, SHAPE), (5, None, ARG),
                                                                         (5, P + 4, ARG)], "rotation")


def test_products(fake, ops):
    #       ops A lda ta B ldb tb M N K C type ldc acc stream
    good = (ops, P, 72, 0, P, 72, 1, 30, 50, 70, P, F32, 50, 0, None)
    check(fake, fake.cerar_matmul_bf16, good, [(1, None, ARG), (1, P + 8, ARG), (2, 70, SHAPE), (2, 64, SHAPE), (2, 2 ** 39, SHAPE), (4, P + 2, ARG), (5, 76, SHAPE), (7, -1, SHAPE),
                                               (8, 2 ** 31, SHAPE), (9, -1, SHAPE), (10, None, ARG), (10, P + 2, ARG), (11, 2, ARG), (12, 49, SHAPE), (3, 1, OK)], "matmul")
    check(fake, fake.cerar_matmul_bf16, (ops, P, 32, 1, P, 56, 0, 30, 50, 70, P, BF16, 50, 1, None), [(2, 24, SHAPE), (5, 48, SHAPE)], "matmul")
    fake.fake_reset(b"")
    host = (C.c_float * 64)(*([3.0] * 64))                # an empty sum: zeros, or nothing added; what lies between rows stays
    assert fake.cerar_matmul_bf16(ops, P, 8, 0, P, 8, 1, 4, 5, 0, C.addressof(host), F32, 8, 1, None) == OK and list(host) == [3.0] * 64
    assert fake.cerar_matmul_bf16(ops, P, 8, 0, P, 8, 1, 4, 5, 0, C.addressof(host), F32, 8, 0, None) == OK and launched(fake) == []
    assert [host[8 * r + c] for r in range(4) for c in range(5)] == [0.0] * 20 and [host[8 * r + 6] for r in range(4)] == [3.0] * 4
    for m, n in ((0, 5), (5, 0)):
        assert fake.cerar_matmul_bf16(ops, P, 8, 0, P, 8, 1, m, n, 8, P, F32, 8, 0, None) == OK and launched(fake) == []


def test_row_copies(fake, ops):
    class Rows(C.Structure):
        _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("ldd", C.c_int64)]

    def call(count=1, **kw):
        d = dict(src=P + 2, dst=P, rows=3, cols=5, ld=5, ldd=8)
        d.update(kw)
        r = (Rows * 5)(*[Rows(**d)] * 5)
        return fake.cerar_align_bf16(ops, C.addressof(r), count, None), launched(fake)

    assert call() == (OK, ["align"]) and call(4) == (OK, ["align"]) and call(rows=0, src=None, dst=None) == (OK, ["align"])
    for status, kw in ((ARG, dict(count=0)), (ARG, dict(count=5)), (ARG, dict(src=None)), (ARG, dict(src=P + 1)), (ARG, dict(dst=P + 8)), (ARG, dict(dst=None)), (SHAPE, dict(ldd=4)),
                       (SHAPE, dict(ldd=12)), (SHAPE, dict(ld=4)), (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=2 ** 31))):
        assert call(**kw) == (status, []), kw
    assert fake.cerar_align_bf16(ops, None, 1, None) == ARG


def block(**changes):
    d = dict(tokens=10, width=40, hidden=24, outputs=32, activation=0, accumulate=0, x=P, ldx=40, w_in=P, ldw_in=40, w_out=P, ldw_out=24, kept=P, y=P, ldy=32,
             dy=P, lddy=32, dx=P, lddx=40, dw_in=P, lddw_in=40, dw_in_type=F32, dw_out=P, lddw_out=24, dw_out_type=BF16)
    d.update(changes)
    return cerar.GatedBlock(**d)


def test_gated(fake, ops):
    def call(backward=False, ws=P, size=None, **kw):
        b = block(**kw)
        need = fake.cerar_gated_workspace(C.addressof(b), backward)
        st = (fake.cerar_gated_backward if backward else fake.cerar_gated_forward)(ops, C.addressof(b), ws, need if size is None else size, None)
        return st, launched(fake), need

    def padded(rows, cols):
        return (rows * ((cols + 7) // 8 * 8) * 2 + 255) // 256 * 256

    forward, backward = ["align", "gated_in", "matmul"], ["align", "gated_grad", "matmul", "matmul", "matmul"]
    assert call() == (OK, forward, padded(10, 24)) and call(True) == (OK, backward, padded(10, 48) + padded(10, 24))
    # operands off 16-byte boundaries are copied, each into rows of its own
    assert call(x=P + 2)[2] == padded(10, 24) + padded(10, 40) and call(ldw_in=41)[2] == padded(10, 24) + padded(48, 40)
    assert call(x=P + 2, w_in=P + 2, w_out=P + 4)[2] == padded(10, 24) + padded(10, 40) + padded(48, 40) + padded(32, 24)
    assert call(True, x=P + 2, w_in=P + 2, w_out=P + 4, dy=P + 6)[2] == padded(10, 48) + padded(10, 24) + padded(10, 40) + padded(48, 40) + padded(32, 24) + padded(10, 32)
    assert call(tokens=1, ldx=39)[2] == padded(1, 24)                             # one row may carry any stride
    # what is not wanted is not made, and its operands are not looked at
    assert call(True, dw_out=None) == (OK, backward[:-1], padded(10, 48))
    assert call(True, dx=None, w_in=None)[:2] == (OK, backward[:-1]) and call(True, dw_in=None, x=None)[:2] == (OK, backward[:-1])
    assert call(True, dx=None, dw_in=None, dw_out=None)[:2] == (OK, backward[:2]) and call(kept=None)[:2] == (OK, forward)
    for status, kw in ((SHAPE, dict(tokens=-1)), (SHAPE, dict(tokens=2 ** 31)), (SHAPE, dict(width=-1)), (SHAPE, dict(hidden=-1)), (SHAPE, dict(hidden=2 ** 30)),
                       (SHAPE, dict(outputs=-1)), (ARG, dict(activation=4)), (ARG, dict(activation=-1)), (ARG, dict(x=None)), (ARG, dict(x=P + 1)), (SHAPE, dict(ldx=39)),
                       (ARG, dict(w_in=None)), (SHAPE, dict(ldw_in=39)), (ARG, dict(w_out=P + 1)), (SHAPE, dict(ldw_out=23)), (SHAPE, dict(ldw_out=2 ** 41)),
                       (ARG, dict(kept=P + 8))):
        assert call(**kw) == (status, [], 0) and call(True, **kw) == (status, [], 0), kw
    for status, kw in ((ARG, dict(y=None)), (ARG, dict(y=P + 1)), (SHAPE, dict(ldy=31))):
        assert call(**kw) == (status, [], 0), kw
    for status, kw in ((ARG, dict(kept=None)), (ARG, dict(dy=None)), (SHAPE, dict(lddy=31)), (ARG, dict(dx=P + 1)), (SHAPE, dict(lddx=39)), (ARG, dict(dw_in=P + 2)),
                       (SHAPE, dict(lddw_in=39)), (ARG, dict(dw_in_type=2)), (ARG, dict(dw_out=P + 1)), (SHAPE, dict(lddw_out=23)), (ARG, dict(dw_out_type=-1))):
        assert call(True, **kw) == (status, [], 0), kw
    for back in (False, True):
        good = call(back)[2]
        assert call(back, ws=None)[:2] == (ARG, []) and call(back, ws=P + 8)[:2] == (ARG, []) and call(back, size=good - 1)[:2] == (SHAPE, [])
    assert fake.cerar_gated_workspace(None, 0) == 0 and fake.cerar_gated_forward(ops, None, P, 10 ** 6, None) == ARG and fake.cerar_gated_backward(ops, None, P, 10 ** 6, None) == ARG
    # nothing to do; empty sums are zero, or nothing is added
    assert call(tokens=0)[:2] == (OK, []) and call(outputs=0)[:2] == (OK, [])
    for back, changes in ((False, dict(hidden=0)), (True, dict(tokens=0)), (True, dict(outputs=0)), (True, dict(hidden=0))):
        host = (C.c_uint16 * 4096)(*([7] * 4096))
        at = C.addressof(host)
        sizes = dict(tokens=3, width=4, hidden=2, outputs=5, ldx=8, ldw_in=8, ldw_out=8, ldy=8, lddy=8, lddx=8, lddw_in=8, lddw_out=8, dw_in_type=BF16, dw_out_type=BF16)
        sizes.update(changes)
        where = dict(y=at, dx=at + 1000, dw_in=at + 2000, dw_out=at + 3000)
        assert call(back, accumulate=1, **sizes, **where)[0] == OK
        if back:
            assert [host[1000 + 8 * r] for r in range(2 * sizes["hidden"])] == [7] * (2 * sizes["hidden"])
            assert call(back, **sizes, **where)[0] == OK
            n, f = sizes["outputs"], sizes["hidden"]
            assert [host[1000 + 8 * r + c] for r in range(2 * f) for c in range(4)] == [0] * (8 * f) and [host[1500 + 8 * r + c] for r in range(n) for c in range(f)] == [0] * (n * f)
            assert [host[500 + 8 * r + c] for r in range(sizes["tokens"]) for c in range(4)] == [0] * (4 * sizes["tokens"])
            assert host[1004] == 7 and host[504] == 7
        else:
            assert [host[8 * r + c] for r in range(3) for c in range(5)] == [0] * 15 and host[5] == 7
        launched(fake)
    # no inputs: g = u = 0, h = 0, y = 0; what is kept says so
    space, kept = (C.c_uint8 * 2048)(*([7] * 2048)), (C.c_uint8 * 8192)(*([7] * 8192))
    ws, k = (C.addressof(space) + 15) & -16, (C.addressof(kept) + 15) & -16
    assert call(ws=ws, width=0, kept=k, hidden=3, ldw_out=8)[:2] == (OK, ["align", "matmul"])
    assert sum(kept) == 7 * (8192 - 180) and sum(space) == 7 * (2048 - 160)


def test_calls_that_fail_report_it_and_leave_no_error_behind(fake, ops):
    f = (C.c_double * 1)(1.0)
    part, rot, gated = (cerar.Heads * 1)(heads()), rotation(), block()
    calls = [lambda: fake.cerar_embed(ops, P, F32, 10, 16, 16, P, 8, 5, 1.0, P, BF16, 16, None),
             lambda: fake.cerar_embed_grad(ops, P, BF16, 16, P, 4, 5, 1.0, P, F32, 10, 16, 16, 0, P, 1024, None),
             lambda: fake.cerar_rotation_table(ops, f, 1, 0, 10, P, None),
             lambda: fake.cerar_head_norm(ops, BF16, C.addressof(part), 1, BF16, 7, 64, 1e-6, C.addressof(rot), None),
             lambda: fake.cerar_head_norm_grad(ops, BF16, C.addressof(part), 1, BF16, F32, 0, 7, 64, 1e-6, C.addressof(rot), P, 256, None),
             lambda: fake.cerar_matmul_bf16(ops, P, 72, 0, P, 72, 1, 30, 50, 70, P, F32, 50, 0, None),
             lambda: fake.cerar_gated_forward(ops, C.addressof(gated), P, 10 ** 6, None),
             lambda: fake.cerar_gated_backward(ops, C.addressof(gated), P, 10 ** 6, None)]
    for call in calls:
        fake.fake_launches_reset(1)
        assert call() == CUDA and b"launch: " in fake.fake_error() and fake.fake_last() == 0
    fake.fake_launches_reset(0)


def test_the_header_declares_what_the_binding_uses():
    text = open(os.path.join(build.PKG_DIR, "..", "include", "cerar.h")).read()
    names = set(re.findall(r"\b(cerar_(?:embed|head_norm|rotation|matmul_bf16|align|gated)\w*)\s*\(", text))
    assert {"cerar_embed", "cerar_embed_grad", "cerar_embed_grad_workspace", "cerar_head_norm", "cerar_head_norm_grad", "cerar_rotation_table", "cerar_matmul_bf16",
            "cerar_matmul_bf16_tile", "cerar_align_bf16", "cerar_gated_forward", "cerar_gated_backward", "cerar_gated_workspace", "cerar_gated_kept_bytes"} <= names
    for name in names:
        assert getattr(cerar.lib, name).argtypes is not None, name


def test_structures_are_the_headers():
    """Sizes and offsets as a C compiler sees them."""
    gcc = shutil.which("gcc")
    assert gcc, "gcc is needed"
    source = '#include <stdio.h>\n#include <stddef.h>\n#include "cerar.h"\nint main(void) {\n'
    for t, cls in (("cerar_heads_t", cerar.Heads), ("cerar_rotation_t", cerar.Rotation), ("cerar_gated_t", cerar.GatedBlock)):
        source += f'printf("%zu ", sizeof({t}));\n' + "".join(f'printf("%zu ", offsetof({t}, {f[0]}));\n' for f in cls._fields_)
    import tempfile
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "a.c"), "w") as f:
            f.write(source + "return 0; }\n")
        subprocess.run([gcc, "-I", os.path.join(build.PKG_DIR, "..", "include"), os.path.join(d, "a.c"), "-o", os.path.join(d, "a")], check=True)
        got = [int(v) for v in subprocess.run([os.path.join(d, "a")], capture_output=True, text=True, check=True).stdout.split()]
    want = [v for cls in (cerar.Heads, cerar.Rotation, cerar.GatedBlock) for v in [C.sizeof(cls)] + [getattr(cls, f[0]).offset for f in cls._fields_]]
    assert got == want


def test_without_a_device_calls_are_refused():
    lib = cerar.lib
    assert lib.cerar_embed(None, P, F32, 10, 16, 16, P, 8, 5, 1.0, P, BF16, 16, None) == ARG
    assert lib.cerar_matmul_bf16(None, P, 72, 0, P, 72, 1, 30, 50, 70, P, F32, 50, 0, None) == ARG
    assert lib.cerar_gated_forward(None, None, P, 10 ** 6, None) == ARG


def test_workspaces():
    lib = cerar.lib
    for bad in ((-1, 5, 5), (5, -1, 5), (5, 5, -1), (2 ** 31, 5, 5)):
        assert lib.cerar_embed_grad_workspace(*bad) == 0
    assert lib.cerar_embed_grad_workspace(0, 5, 5) >= 0
    for n in (1, 100, 8192, 8193, 100000, 10 ** 7):                  # keys and numbers of all tokens, twice where they are sorted by digits
        assert lib.cerar_embed_grad_workspace(n, 1000, 64) >= (8 if n <= 8192 else 16) * n
    assert lib.cerar_embed_grad_workspace(2 ** 31 - 256, 2 ** 31 - 256, 512) > 2 ** 33           # (no overflow on the way)
    assert lib.cerar_head_norm_grad_workspace(0, 64) == 0 and lib.cerar_head_norm_grad_workspace(2, 64) == 2 * lib.cerar_head_norm_grad_workspace(1, 64)
    assert lib.cerar_gated_kept_bytes(-1, 5) == 0 and lib.cerar_gated_kept_bytes(32, 32) == 6144 and lib.cerar_gated_kept_bytes(33, 1) == 2 * 6144
    assert lib.cerar_gated_kept_bytes(2 ** 20, 2 ** 20) == 6 * 2 ** 40


@pytest.mark.parametrize("sms", [1, 2, 100, 132, 148, 160])
def test_products_fit_their_launch(sms):
    """Every choice is one the launch can make: a cluster of at most eight blocks, no more parts of a sum than it has blocks of 64, and split tiles
    that run at the same time."""
    split = C.c_int()
    for m in (1, 7, 128, 129, 1000, 4096, 30000):
        for n in (1, 64, 500, 2048, 50000):
            for k in (1, 64, 65, 1000, 8192, 100000):
                form = cerar.lib.cerar_matmul_bf16_tile(m, n, k, sms, C.byref(split))
                blocks = 1 if form == 2 else 2
                rows, cols = (128, 128) if form == 2 else (256, 128) if form == 1 else (256, 256)
                assert form in (0, 1, 2) and 1 <= split.value * blocks <= 8 and split.value <= -(-k // 64)
                assert blocks <= sms
                if split.value > 1:
                    assert -(-m // rows) * -(-n // cols) * split.value * blocks <= sms
    assert cerar.lib.cerar_matmul_bf16_tile(0, 1, 1, 148, C.byref(split)) == -1
    assert cerar.lib.cerar_matmul_bf16_tile(1, 1, 1, 148, None) == -1
