"""Which kernel a call takes, without a GPU: the cases of the GPU tests that are meant for a form go there, by the rules that the launches follow (256 compute units)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2211_13939_amd import binding
from tests import test_gpu_cross_many, test_gpu_linear8_forms
from tests.test_operators_host import Made, lib  # noqa: F401  (a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FORMS = ("few", "split", "64x64", "64x128", "128x128", "256x128")
N_CU = 256


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("plans") / "libplans.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "operator_plans.cpp"), "-o", out],
                   check=True)
    return C.CDLL(out)


def _ints(v):
    return (C.c_int * len(v))(*v)


@pytest.mark.parametrize("shape", test_gpu_linear8_forms.SHAPES)
def test_shapes_of_the_products_forms(plans, shape):
    rows, k, n = shape
    assert tuple(FORMS[plans.plan_linear8(rows, k, n, two, N_CU)] for two in (1, 0)) == test_gpu_linear8_forms.SHAPES[shape]


def test_every_form_of_the_product_has_its_shapes(plans):
    for i in range(2):
        assert {f[i] for f in test_gpu_linear8_forms.SHAPES.values()} == set(FORMS)
        assert {FORMS[plans.plan_linear8(*s, 1 - i, N_CU)] for s in test_gpu_linear8_forms.LARGE} == set(FORMS[2:])


@pytest.mark.parametrize("tiles", [1, 7, 8, 9, 1000, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, (1 << 20) + 9, 3 * (1 << 20) + 5, (1 << 24) - 3, 1 << 24, (1 << 25) + 13, 1 << 28])
def test_the_products_grid_has_a_workgroup_for_every_tile(plans, tiles):
    """Up to 2^24 rows and 65536 channels in tiles of 64 x 64: each side of the grid is one that can be launched, and workgroups of a row of it stay in turn with the XCDs."""
    across, down = C.c_int(), C.c_int()
    assert plans.plan_linear8_grid(tiles, C.byref(across), C.byref(down)) == 0
    assert across.value % 8 == 0 and across.value * 256 < 1 << 32 and down.value < 1 << 16
    assert across.value * down.value < tiles + 8 * down.value + 8


def _launches(lib, heads, kv, d, q_len, mem):      # noqa: F811
    """(launches, those for many queries, requests in all of them) of a call of the library's host code."""
    lib.fake_reset()
    m = Made(lib, "cross", binding.make_cross_config(heads, kv, d, True))
    b = binding.CrossBatch(q_len, [0] * len(q_len), mem)
    t = binding.TtsCrossTensors(q=1 << 20, k=2 << 20, v=3 << 20, out=4 << 20)
    assert lib.tts_cross_run(m.h, C.byref(b.c), C.byref(t)) == 0
    m.close()
    return lib.fake_launches(), lib.fake_many(), lib.fake_requests_seen()


CROSS = list(test_gpu_cross_many.CASES.values()) + [(h, kv, d, test_gpu_cross_many.mask_queries(name, mem), [mem, 60], large)
                                                    for name, (h, kv, d, _, large) in test_gpu_cross_many.MASKS.items() for mem in test_gpu_cross_many.MASK_LENGTHS]


@pytest.mark.parametrize("case", CROSS)
def test_cases_of_many_queries_are(lib, plans, case):      # noqa: F811
    heads, kv, d, q_len, mem, large = case
    assert _launches(lib, heads, kv, d, q_len, mem) == (1, 1, len(q_len))
    assert bool(plans.plan_cross_large(_ints(q_len), _ints(mem), len(mem), heads // kv, kv, N_CU)) == large


def test_the_mixed_call_is_of_both_kinds(lib, plans):      # noqa: F811
    heads, kv, d, q_len, mem = test_gpu_cross_many.mixed()
    launches, many, seen = _launches(lib, heads, kv, d, q_len, mem)
    few = sum(0 < q * heads // kv < plans.plan_cross_many_rows() for q in q_len)
    of_many = sum(q * heads // kv >= plans.plan_cross_many_rows() for q in q_len)
    assert few and of_many and seen == few + of_many and many == -(-of_many // 128) and launches - many == -(-few // 128)
    # and the same frames among fewer tiles are not worth a launch of their own
    assert _launches(lib, heads, kv, d, q_len[:30], mem[:30])[1] == 0
