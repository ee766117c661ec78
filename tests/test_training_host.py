"""Host side of the training-step operators: what the binding and the argument checks do without a device."""
import ctypes as C
import os
import re

import pytest

from paper_2609_23898_b200 import cerar

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_call_is_exported_and_bound():
    text = open(os.path.join(ROOT, "include", "cerar.h")).read()
    names = set(re.findall(r"\b(cerar_(?:ops|fp8_quantize|fp8_matmul|tensors|grad|adamw)\w*)\s*\(", text))
    assert {"cerar_ops_create", "cerar_fp8_quantize", "cerar_fp8_matmul", "cerar_grad_norm", "cerar_adamw_step"} <= names
    for n in names:
        assert getattr(cerar.lib, n).argtypes is not None, n


def test_structures_have_the_header_s_layout():
    # pointers and 64-bit numbers first, the 32-bit ones behind them: no padding but at the end
    assert C.sizeof(cerar.Fp8Matrix) == 2 * 8 + 4 * 8 + 2 * 4
    assert C.sizeof(cerar.TensorDesc) == 8 * 8 + 4 * 4
    assert C.sizeof(cerar.AdamwOptions) == 6 * 8
    text = open(os.path.join(ROOT, "include", "cerar.h")).read()
    for struct, end in ((cerar.Fp8Matrix, "cerar_fp8_matrix_t"), (cerar.TensorDesc, "cerar_tensor_t"), (cerar.AdamwOptions, "cerar_adamw_options_t")):
        body = re.sub(r"/\*.*?\*/", "", text[:text.index("} " + end)].rsplit("typedef struct {", 1)[1], flags=re.S)
        fields = [f.strip(" *") for line in body.split(";") if line.strip() for f in re.sub(r"^\s*(const\s+)?\w+", "", line.strip()).split(",")]
        assert fields == [f for f, _ in struct._fields_], end


def test_without_a_handle_every_call_is_refused():
    lib = cerar.lib
    d, o = cerar.Fp8Matrix(), cerar.AdamwOptions()
    assert lib.cerar_ops_create(None) == 1
    assert lib.cerar_ops_status(None, None) == 1
    assert lib.cerar_ops_launch_count(None) == 0
    assert lib.cerar_fp8_quantize(None, 16, 0, 1, C.addressof(d), 1, None) == 1
    assert lib.cerar_fp8_matmul(None, C.addressof(d), 0, C.addressof(d), 1, 16, 0, 1, 0, None) == 1
    out = C.c_void_p(7)
    assert lib.cerar_tensors_create(None, 0, None, 32, C.byref(out)) == 1 and not out.value
    assert lib.cerar_tensors_set_grads(None, None, None) == 1
    assert lib.cerar_grad_norm(None, 1.0, 16, None) == 1
    assert lib.cerar_adamw_step(None, C.addressof(o), None, None) == 1
    lib.cerar_ops_destroy(None)
    lib.cerar_tensors_destroy(None)
    assert b"NULL" in lib.cerar_last_error()


def test_without_a_device_there_is_no_handle():
    import torch
    from paper_2609_23898_b200 import training
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    with pytest.raises(cerar.CerarError) as e:
        training.Ops()
    assert e.value.status == 6


def test_matrices_that_are_refused_before_any_call():
    import torch
    from paper_2609_23898_b200 import training as R
    codes, scales = torch.zeros(4, 16, dtype=torch.uint8), torch.ones(1, 4)
    with pytest.raises(ValueError):
        R.Quantized(codes, scales, R.BY_ROW)                    # not on a device
    with pytest.raises(TypeError):
        R.Quantized(codes.float(), scales, R.BY_ROW)
    with pytest.raises(ValueError):
        R.Quantized._sizes(4, 16, 3)
    assert R.Quantized._sizes(130, 300, R.BY_ROW) == (304, 3, 130)
    assert R.Quantized._sizes(130, 300, R.BY_COLUMN) == (304, 2, 300)
    assert R.Quantized._sizes(130, 300, R.BY_BLOCK) == (304, 2, 3)


def test_an_ops_destroys_its_sets_first(monkeypatch):
    """A set keeps the address of the handle it was made with: calls on it after Ops.destroy() would read freed memory."""
    import torch
    from paper_2609_23898_b200 import training as R

    class Lib:
        def __init__(self):
            self.alive, self.log = {}, []

        def make(self, what, out):
            C.cast(out, C.POINTER(C.c_void_p))[0] = len(self.log) + 16
            self.log.append(what)
            return 0

        def cerar_ops_create(self, out):
            return self.make("ops", out)

        def cerar_tensors_create(self, ops, count, desc, bits, out):
            return self.make("set", out)

        def cerar_ops_destroy(self, h):
            self.log.append("ops gone")

        def cerar_tensors_destroy(self, h):
            self.log.append("set gone")

    lib = Lib()
    monkeypatch.setattr(R, "lib", lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    ops = R.Ops()
    a, b = R.TensorSet(ops, grads=[]), R.TensorSet(ops, grads=[])
    b.destroy()
    ops.destroy()
    assert lib.log == ["ops", "set", "set", "set gone", "set gone", "ops gone"] and not a._h
    ops.destroy()
    del a, b
    assert lib.log[-1] == "ops gone"
    ops, log = R.Ops(), len(lib.log)
    R.TensorSet(ops, grads=[])
    ops.destroy()
    assert lib.log[log:] == ["set", "set gone", "ops gone"]


LONG_MESSAGE = """
import ctypes as C, resource
from paper_2609_23898_b200 import cerar
lib = cerar.lib
lib.cerar_internal_set_error.argtypes = [C.c_char_p]
lib.cerar_internal_set_error.restype = None
message = b"x" * (64 << 20)
now = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (now + (8 << 20), resource.RLIM_INFINITY))
lib.cerar_internal_set_error(message)
assert lib.cerar_last_error() == b""
lib.cerar_internal_set_error(b"short")
assert lib.cerar_last_error() == b"short"
"""


def test_an_error_text_without_memory_for_it():
    """No C++ exception leaves a C entry: a text that cannot be kept is dropped."""
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", LONG_MESSAGE], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stderr)


def tile(m, n, k, pow2, sms=148):
    split = C.c_int(-7)
    return cerar.lib.cerar_fp8_matmul_tile(m, n, k, pow2, sms, C.byref(split)), split.value


def test_products_of_the_gpu_tests_reach_every_kernel():
    """What the comparison with 64 bits at these sizes is worth hangs on the tiles the rule takes there."""
    from tests.test_gpu_training_tiles import SIZES
    for (m, n, k), want in SIZES.items():
        for pow2 in (0, 1):
            cols, turns = want[pow2]
            assert tile(m, n, k, pow2) == (cols, 1)
            rows = 256 if pow2 and cols == 256 else 128
            slots = 74 if rows == 256 else 148
            assert -(-(-(-m // rows) * -(-n // cols)) // slots) == turns, (m, n, k, pow2)
    reached = {(pow2, want[pow2][0], want[pow2][1] > 1) for want in SIZES.values() for pow2 in (0, 1)}
    assert reached >= {(p, c, True) for p in (0, 1) for c in (128, 256)} | {(p, 256, False) for p in (0, 1)}


def test_tiles_of_small_and_large_products():
    assert tile(1, 8192, 2048, 1)[0] == 128 and tile(8192, 8192, 8192, 1) == (256, 1) and tile(8192, 8192, 8192, 0) == (256, 1)
    assert tile(16, 16, 20000, 1)[1] > 1                                   # few tiles, a long sum: shared by a cluster
    for m, n, k in ((1, 1, 1), (129, 1, 128), (1000, 1000, 100000), (0x7FFFFF00, 0x7FFFFF00, 0x7FFFFF00)):
        for pow2 in (0, 1):
            cols, split = tile(m, n, k, pow2)
            assert cols in (128, 256) and 1 <= split <= min(8, -(-k // 128)) and (cols == 128 or split == 1)
    for bad in ((0, 1, 1, 0), (1, -1, 1, 0), (1, 1, 0, 0), (1 << 31, 1, 1, 0), (1, 1, 1, 0, 0)):
        assert tile(*bad) == (-1, -7)
    assert cerar.lib.cerar_fp8_matmul_tile(1, 1, 1, 0, 148, None) == -1
