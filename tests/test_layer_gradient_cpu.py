"""What the calls over a list of gradients name in memory, without a GPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2407_04480_b200 import build as loco_build
from paper_2407_04480_b200 import loco


@pytest.fixture(scope="module")
def addresses(tmp_path_factory):
    here, lib = os.path.dirname(os.path.abspath(__file__)), str(tmp_path_factory.mktemp("lib") / "addresses.so")
    subprocess.check_call([loco_build.nvcc_path(), *loco_build.NVCC_FLAGS, "-shared", "-cudart", "static", "-o", lib, os.path.join(here, "gradient_addresses.cu")])
    L = C.CDLL(lib)
    L.check_addresses.argtypes = [C.c_int32, C.c_size_t, C.c_uint64, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
    return L.check_addresses


@pytest.mark.parametrize("dtype,size", [(loco.BF16, 2), (loco.F32, 4)])
def test_every_copy_names_a_boundary(addresses, dtype, size):
    """Also where nothing is read: a span that ends before its first boundary has no vector, and a copy's address has to be one."""
    lengths = [*range(1, 40), 16379, 16384, 16385, 32768 // size, 32768 // size + 1, 100003]
    for off in range(0, 16, size):
        for n in lengths:
            read, rest = C.c_uint64(), C.c_uint64()
            assert addresses(dtype, (1 << 20) + off, n, C.byref(read), C.byref(rest)) == 0, (off, n)
            assert read.value + rest.value == n, (off, n)
