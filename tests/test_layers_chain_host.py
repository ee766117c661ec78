"""Which of the gated block's gradient products begin beside the one in front (`after`) and let the one behind begin (`followed`), without a device: for every
choice of results, for empty sums, and where results lie over what another product reads or writes."""
import ctypes as C
import itertools
import os
import shutil
import subprocess

import pytest

from paper_2609_23898_b200 import build, cerar

HERE = os.path.dirname(os.path.abspath(__file__))
F32, BF16 = 0, 1
FAR = 1 << 32                # between operands, so that none of them meet


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    gxx, nvcc = shutil.which("g++"), build._nvcc()
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    assert gxx, "g++ is needed"
    out = str(tmp_path_factory.mktemp("fake") / "libfake.so")
    subprocess.run([gxx, "-std=c++17", "-shared", "-fPIC", "-O1", "-w", "-I", include, "-I", build.CSRC, "-x", "c++", "-Wl,-Bsymbolic",
                    os.path.join(HERE, "fake_cuda.cpp"), os.path.join(HERE, "fake_products.cpp"), os.path.join(build.CSRC, "ops_api.cu"),
                    os.path.join(build.CSRC, "layers_api.cu"), "-o", out], check=True)
    lib = C.CDLL(out)
    lib.fake_products.restype = C.c_char_p
    lib.fake_reset.argtypes = [C.c_char_p]
    for name in ("cerar_ops_create", "cerar_ops_destroy", "cerar_gated_backward", "cerar_gated_workspace"):
        getattr(lib, name).argtypes = getattr(cerar.lib, name).argtypes
    lib.cerar_gated_workspace.restype = C.c_size_t
    lib.fake_reset(b"")
    return lib


@pytest.fixture
def products(fake):
    h = C.c_void_p()
    fake.fake_reset(b"")
    fake.fake_launches_reset(0)
    assert fake.cerar_ops_create(C.byref(h)) == 0

    def call(**changes):
        """(after, followed) of every product of a gradient."""
        d = dict(tokens=10, width=40, hidden=24, outputs=32, activation=0, accumulate=0, x=FAR, ldx=40, w_in=2 * FAR, ldw_in=40, w_out=3 * FAR, ldw_out=24, kept=4 * FAR,
                 dy=5 * FAR, lddy=32, dx=6 * FAR, lddx=40, dw_in=7 * FAR, lddw_in=40, dw_in_type=F32, dw_out=8 * FAR, lddw_out=24, dw_out_type=BF16)
        d.update(changes)
        b = cerar.GatedBlock(**d)
        fake.fake_products_reset()
        assert fake.cerar_gated_backward(h, C.addressof(b), 9 * FAR, fake.cerar_gated_workspace(C.addressof(b), 1), None) == 0
        return [tuple(int(v) for v in line.split()) for line in fake.fake_products().decode().split("\n")[:-1]]

    yield call
    fake.cerar_ops_destroy(h)


def sound(flags):
    """The first one waits for the gate's gradient; one that begins early stands behind one that lets it."""
    return all(not after if i == 0 else not after or flags[i - 1][1] for i, (after, _) in enumerate(flags))


CHOICES = [c for n in range(4) for c in itertools.combinations(("dw_out", "dx", "dw_in"), n)]


@pytest.mark.parametrize("wanted", CHOICES, ids=str)
def test_every_choice_of_results(products, wanted):
    absent = {name: None for name in ("dw_out", "dx", "dw_in") if name not in wanted}
    n = len(wanted)
    full = [(int(i > 0), int(i + 1 < n)) for i in range(n)]
    assert products(**absent) == full
    assert products(**absent, x=FAR + 2, w_in=2 * FAR + 2, dy=5 * FAR + 2, lddy=33) == full              # operands that are copied
    flags = products(**absent, width=0)                                                                  # no inputs: dw_out alone
    assert len(flags) == int("dw_out" in wanted) and sound(flags)
    if "dx" not in wanted:                                                                               # empty sums, nothing added: no products
        for sizes in (dict(tokens=0), dict(hidden=0), dict(outputs=0)):
            assert products(**absent, **sizes, accumulate=1) == []


DY = 10 * 32 * 2             # bytes of dy


@pytest.mark.parametrize("changes,early", [
    (dict(width=32, lddx=32, dx=5 * FAR), (0, 0, 1)),                             # dx is dy: written when dw_out has read it
    (dict(dx=5 * FAR + 64), (0, 0, 1)), (dict(dx=5 * FAR + DY - 16), (0, 0, 1)), (dict(dx=5 * FAR + DY), (0, 1, 1)),
    (dict(dx=5 * FAR - 10 * 40 * 2), (0, 1, 1)), (dict(dx=5 * FAR - 10 * 40 * 2 + 16), (0, 0, 1)),
    (dict(dw_in=5 * FAR), (0, 1, 0)),                                             # dw_in over dy, over the weights that dx is made with, over the other results
    (dict(dw_in=2 * FAR, dw_in_type=BF16), (0, 1, 0)), (dict(dw_in=6 * FAR), (0, 1, 0)), (dict(dw_in=8 * FAR), (0, 1, 0)), (dict(dx=8 * FAR), (0, 0, 1)),
    (dict(dx=FAR), (0, 1, 0)),                                                    # dx over x: the order is kept, not dw_in
    (dict(width=32, lddx=32, dx=5 * FAR, dw_in=5 * FAR + 64), (0, 0, 0)),
    (dict(width=32, lddx=32, dx=5 * FAR, dw_out=None), (0, 1)),                   # nobody reads dy any more
    (dict(width=32, lddx=32, ldx=32, dx=5 * FAR + 2, dy=5 * FAR + 2), (0, 1, 1)),  # read from a copy
    (dict(dx=4 * FAR), (0, 1, 1)), (dict(dx=3 * FAR), (0, 1, 1)),                 # over what the gate's gradient alone reads
], ids=str)
def test_results_over_one_another_and_over_operands_keep_the_order(products, changes, early):
    flags = products(**changes)
    assert tuple(a for a, _ in flags) == early and sound(flags)
