"""The tensor-map encoder's look-up (tensor_map.hpp) by several host threads, against a driver of our own (fake_driver.cpp)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2609_23898_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    assert gxx, "g++ is needed"
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    out = str(tmp_path_factory.mktemp("driver") / "libfakedriver.so")
    subprocess.run([gxx, "-std=c++17", "-shared", "-fPIC", "-O1", "-pthread", "-w", "-Wl,-Bsymbolic", "-I", include, "-I", build.CSRC,
                    os.path.join(HERE, "fake_driver.cpp"), "-o", out], check=True)
    return C.CDLL(out)


def test_threads_that_start_together_all_find_the_encoder(driver):
    assert driver.found_by(8) == 8
    assert driver.lookups() == 1


def test_the_first_map_of_a_thread(driver):
    """The encoder refuses a thread without a current device."""
    assert driver.first_map_of_a_thread() == 1
