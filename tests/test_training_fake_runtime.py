"""Host side of the training-step operators (ops_api.cu) against a CUDA runtime that writes its calls down and can be made to
fail (fake_cuda.cpp): what has to be waited for, and what is left behind after an error."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2609_23898_b200 import build, cerar

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    gxx = shutil.which("g++")
    nvcc = build._nvcc()
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    assert gxx, "g++ is needed"
    out = str(tmp_path_factory.mktemp("fake") / "libfake.so")
    subprocess.run([gxx, "-std=c++17", "-shared", "-fPIC", "-O1", "-w", "-I", include, "-I", build.CSRC, "-x", "c++", "-Wl,-Bsymbolic",
                    os.path.join(HERE, "fake_cuda.cpp"), os.path.join(build.CSRC, "ops_api.cu"), "-o", out], check=True)
    lib = C.CDLL(out)
    vp = C.c_void_p
    lib.fake_log.restype = lib.fake_error.restype = C.c_char_p
    lib.fake_reset.argtypes = [C.c_char_p]
    lib.cerar_ops_create.argtypes = [C.POINTER(vp)]
    lib.cerar_ops_status.argtypes = [vp, vp]
    lib.cerar_ops_destroy.argtypes = lib.cerar_tensors_destroy.argtypes = [vp]
    lib.cerar_tensors_create.argtypes = [vp, C.c_int64, C.POINTER(cerar.TensorDesc), C.c_int, C.POINTER(vp)]
    lib.cerar_fp8_quantize.argtypes = [vp, vp, C.c_int, C.c_int64, vp, C.c_int, vp]
    lib.cerar_fp8_matmul.argtypes = [vp, vp, C.c_int, vp, C.c_int, vp, C.c_int, C.c_int64, C.c_int, vp]
    lib.cerar_grad_norm.argtypes = [vp, C.c_float, vp, vp]
    lib.fake_reset(b"")
    return lib


def log(lib):
    return lib.fake_log().decode().split("\n")[:-1]


@pytest.fixture
def ops(fake):
    h = C.c_void_p()
    fake.fake_reset(b"")
    assert fake.cerar_ops_create(C.byref(h)) == 0
    yield h
    fake.cerar_ops_destroy(h)


def make_set(fake, ops):
    d = (cerar.TensorDesc * 1)()
    d[0].numel, d[0].grad = 5000, 4096
    s = C.c_void_p()
    return fake.cerar_tensors_create(ops, 1, d, 0, C.byref(s)), s


# Copies from pageable memory and memsets may return before the device has them, and a non-blocking stream does not wait for the
# stream they run on: whatever a handle needs has to be on the device when the handle is handed out.

def test_a_handle_is_complete_when_it_is_handed_out(fake):
    h = C.c_void_p()
    fake.fake_reset(b"")
    assert fake.cerar_ops_create(C.byref(h)) == 0
    assert log(fake) == ["malloc", "memset", "synchronize"]
    fake.cerar_ops_destroy(h)


def test_a_set_is_complete_when_it_is_handed_out(fake, ops):
    fake.fake_reset(b"")
    st, s = make_set(fake, ops)
    assert st == 0
    calls = log(fake)
    last = max(i for i, c in enumerate(calls) if c in ("memset", "memcpy"))
    assert "synchronize" in calls[last + 1:]
    fake.cerar_tensors_destroy(s)


@pytest.mark.parametrize("call,status", [("malloc", 7), ("memset", 7), ("memcpy", 7), ("synchronize", 6)])
def test_a_set_that_fails_is_no_set(fake, ops, call, status):
    fake.fake_reset(call.encode())
    st, s = make_set(fake, ops)
    assert st == status and not s.value and b"made to fail" in fake.fake_error()
    fake.fake_reset(b"")


# The runtime keeps the last error until it is asked for, and torch asks after each of its own launches: an error that a call here
# has reported must not be found there as well.

@pytest.mark.parametrize("call", ["malloc", "memset", "memcpy"])
def test_a_set_that_fails_leaves_no_error_behind(fake, ops, call):
    fake.fake_reset(call.encode())
    assert make_set(fake, ops)[0] != 0
    assert fake.fake_last() == 0
    fake.fake_reset(b"")


def test_calls_that_fail_leave_no_error_behind(fake, ops):
    st, s = make_set(fake, ops)
    q = cerar.Fp8Matrix(4096, 4096, 16, 16, 16, 16, 0, 1)
    fake.fake_reset(b"launch")
    assert fake.cerar_grad_norm(s, 1.0, 4096, None) == 6 and fake.fake_last() == 0
    assert fake.cerar_fp8_quantize(ops, 4096, 0, 16, C.addressof(q), 1, None) == 6 and fake.fake_last() == 0
    assert fake.cerar_fp8_matmul(ops, C.addressof(q), 0, C.addressof(q), 1, 4096, 0, 16, 0, None) == 6 and fake.fake_last() == 0
    fake.fake_reset(b"memcpy async")
    assert fake.cerar_ops_status(ops, None) != 0 and fake.fake_last() == 0
    h = C.c_void_p()
    fake.fake_reset(b"malloc")
    assert fake.cerar_ops_create(C.byref(h)) == 7 and not h.value and fake.fake_last() == 0
    fake.fake_reset(b"")
    fake.cerar_tensors_destroy(s)
