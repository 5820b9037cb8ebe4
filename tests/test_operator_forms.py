"""Which form of its kernels a row sort takes by its sizes, and that the GPU tests reach every form (CPU only;
operator_forms.cpp compiles the library's own rules for the host)."""

import ctypes
import os
import subprocess

import pytest

from paper_2511_02302_amd import build as ff8_build

import test_gpu_forms
import test_gpu_rows

SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "operator_forms.cpp")
ONE_LAUNCH, COUNTED, ROUTED_FIRST = range(3)


@pytest.fixture(scope="module")
def host_lib(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("forms") / "forms.so")
    cmd = [ff8_build.hipcc()] + ff8_build.COMMON + ["-x", "hip", "--cuda-host-only", "-shared", SRC, "-o", lib]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(lib)


def _sort_form(host_lib, T, k, E, row_bytes):
    row16 = ctypes.c_int64(row_bytes // 16)
    return host_lib.sort_form(ctypes.c_int64(T), k, E, row16), bool(host_lib.sort_narrow(row16))


@pytest.mark.parametrize("T,k,E,row_bytes,form,narrow", [
    (512, 8, 64, 14336, ONE_LAUNCH, False), (513, 8, 64, 14336, COUNTED, False),
    (4096, 1, 1024, 512, ONE_LAUNCH, True),      # us, so / routed first: 10.4 / 12.7
    (8192, 1, 8, 512, COUNTED, True),
    (5001, 8, 32, 7168, COUNTED, False),         # 60 / 64
    (6144, 8, 32, 14336, COUNTED, False), (8192, 8, 32, 14336, ROUTED_FIRST, False),  # 211 / 207
    (16384, 2, 8, 1280, COUNTED, False),         # 19.1 / 18.1
    (20480, 2, 8, 1280, ROUTED_FIRST, False),    # 22.3 / 20.5
    (12288, 2, 8, 1024, COUNTED, True),
    (32768, 2, 8, 256, COUNTED, True), (32769, 2, 8, 256, ROUTED_FIRST, True),
    (4096, 2, 1024, 512, COUNTED, True),         # 21.3 / 23.3
    (6000, 2, 1024, 512, ROUTED_FIRST, True),    # 28.2 / 25.2
    (6000, 2, 1024, 2048, ROUTED_FIRST, False)]) # 33.7 / 30.0
def test_sort_form(host_lib, T, k, E, row_bytes, form, narrow):
    assert _sort_form(host_lib, T, k, E, row_bytes) == (form, narrow)


@pytest.mark.parametrize("element", [2, 1])  # bf16 rows, FP8 rows
def test_sorts_of_the_gpu_tests_take_every_form(host_lib, element):
    """Every form with narrow rows and with wide ones, by cases that end inside a workgroup's pairs too (8 a
    workgroup in one launch, 16 wide or 64 narrow ones behind counts)."""
    seen, ragged = set(), set()
    for T, H, E, k, _, _ in test_gpu_rows.CASES + test_gpu_forms.SORTS:
        f = _sort_form(host_lib, T, k, E, H * element)
        seen.add(f)
        if T * k % 8:
            ragged.add(f)
    want = {(form, narrow) for form in (ONE_LAUNCH, COUNTED, ROUTED_FIRST) for narrow in (False, True)}
    assert seen == want and ragged == want
