"""Which kernel a call takes, without a GPU: the cases of the GPU tests that are meant for a form go there, by the rules that the launches follow (256 compute units)."""
import ctypes as C
import os
import subprocess

import pytest

from tests import test_gpu_linear8_forms

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FORMS = ("few", "split", "64x64", "64x128", "128x128", "256x128")
N_CU = 256


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("plans") / "libplans.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "operator_plans.cpp"), "-o", out],
                   check=True)
    return C.CDLL(out)


@pytest.mark.parametrize("shape", test_gpu_linear8_forms.SHAPES)
def test_shapes_of_the_products_forms(plans, shape):
    rows, k, n = shape
    assert tuple(FORMS[plans.plan_linear8(rows, k, n, two, N_CU)] for two in (1, 0)) == test_gpu_linear8_forms.SHAPES[shape]


def test_every_form_of_the_product_has_its_shapes(plans):
    for i in range(2):
        assert {f[i] for f in test_gpu_linear8_forms.SHAPES.values()} == set(FORMS)
        assert {FORMS[plans.plan_linear8(*s, 1 - i, N_CU)] for s in test_gpu_linear8_forms.LARGE} == set(FORMS[2:])
