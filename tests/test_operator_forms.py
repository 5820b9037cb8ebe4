"""Which form of its kernels a row sort or a 4-bit product takes by its sizes, and that the GPU tests reach every form
(CPU only; operator_forms.cpp compiles the library's own rules for the host)."""

import ctypes
import os
import subprocess

import pytest

from paper_2511_02302_amd import build as ff8_build

import test_gpu_forms
import test_gpu_mxfp4
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


MANY = 1  # blocks of up to 96 rows; otherwise the waves of a 16-row workgroup, negative where its weights are kept


def _mxfp4_form(host_lib, x_rows, top_k, M_cap, E, N, K, swiglu, cus=256):
    a = [ctypes.c_int64(v) for v in (M_cap, N, K, cus)]
    return host_lib.mxfp4_form(ctypes.c_int64(x_rows), top_k, a[0], E, a[1], a[2], int(swiglu), a[3])


# Measured on one MI355X: us, as chosen / the other way.  T > 0: gathered tokens, M_cap 0; T = 0: grouped rows.
@pytest.mark.parametrize("T,k,M_cap,E,N,K,swiglu,form", [
    (1, 8, 0, 32, 4096, 7168, True, 4),           # 22.4 / 25.2 kept
    (8, 8, 0, 32, 4096, 7168, True, 4),           # 8 rows an expert are 64 here: 66 / 74 kept
    (32, 8, 0, 32, 4096, 7168, True, 4),          # 8 rows an expert: 81 / 83
    (48, 8, 0, 32, 4096, 7168, True, MANY),       # 12: 84 / 92
    (256, 8, 0, 32, 4096, 7168, True, MANY),
    (408, 2, 0, 4, 1024, 6528, True, -4),         # 204 rows each, 48 items: 25.6 / 29.6 not kept
    (0, 0, 512, 32, 7168, 2048, False, 4),        # one token of k = 8: 14.6 / 17.4
    (0, 0, 1024, 32, 7168, 2048, False, MANY),    # the same with 32-row padding: 17.6 / 18.6
    (0, 0, 4096, 32, 7168, 2048, False, MANY),    # with 128: 19.8 / 43.8
    (0, 0, 640, 32, 7168, 2048, False, 4),        # 4 tokens: 30.1 / 41.5
    (0, 0, 128, 4, 7168, 2048, False, -4),        # one token of k = 2: 6.4 / 6.6 not kept
    (0, 0, 1024, 64, 2048, 1408, False, 2)])      # 7 tokens of k = 6: 11.0 / 11.4 kept
def test_mxfp4_form(host_lib, T, k, M_cap, E, N, K, swiglu, form):
    assert _mxfp4_form(host_lib, T or M_cap, k, M_cap or 128, E, N, K, swiglu) == form


def _parameters(test):
    return [m for m in test.pytestmark if m.name == "parametrize"][0].args[1]


def test_mxfp4_products_of_the_gpu_tests_take_every_form(host_lib):
    seen = set()
    for swiglu, n_out, K, align, counts, form in test_gpu_forms.GROUPED:
        _, _, M_cap = test_gpu_mxfp4._groups(counts, align, extra=200)
        N = 2 * n_out if swiglu else n_out
        assert _mxfp4_form(host_lib, M_cap, 0, M_cap, len(counts), N, K, swiglu) == form, (swiglu, n_out, K)
        seen.add((swiglu, form))
    for T, E, k, I, K, form in test_gpu_forms.GATHERED:
        assert _mxfp4_form(host_lib, T, k, 128, E, 2 * I, K, True) == form, (T, E, k)
        seen.add((True, form))
    assert seen == {(s, f) for s in (False, True) for f in (MANY, 2, -2, 4, -4)}


def test_many_rows_of_the_gpu_tests_are_many(host_lib):
    many = test_gpu_mxfp4.MANY
    for N, K, align, copies in _parameters(test_gpu_mxfp4.test_many_rows_product):
        _, _, M_cap = test_gpu_mxfp4._groups(many * copies, align, seed=1, extra=300)
        assert _mxfp4_form(host_lib, M_cap, 0, M_cap, len(many) * copies, N, K, False) == MANY
    for I, K, T, k, _, copies in _parameters(test_gpu_mxfp4.test_many_rows_swiglu_of_gathered_tokens):
        E = len(many) * copies
        assert _mxfp4_form(host_lib, max(T, 12 * E // k + 1), k, 128, E, 2 * I, K, True) == MANY
