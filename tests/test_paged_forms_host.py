"""The calls of test_gpu_paged_forms.py without a GPU: each is taken the way that it is there for, and their reference is the definition."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import past_ref as ref
from tests.paged_cases import CASES, plan
from tests.test_operators_host import Made
from tests.test_past_host import _paged, lib  # noqa: F401


@pytest.mark.parametrize("name", CASES)
def test_how_the_cases_are_taken(lib, name):  # noqa: F811
    c, want = CASES[name], plan(name)
    m = Made(lib, "paged", binding.make_paged_config(c["heads"], c["kv"], c["d"], c["page"], c.get("bf16", True), c["causal"]))
    lib.past_reset()
    assert _paged(lib, m, c["q_len"], c["own_len"], [0] * len(c["q_len"]), c["prefix"], c["prefix_len"], [1] * len(c["prefix_len"]), table_cols=3000) == 0
    assert {k: getattr(lib, f"past_{k}")() for k in want} == want
    m.close()


@pytest.mark.parametrize("causal", [False, True])
def test_the_reference_is_the_definition(causal):
    import torch
    from tests import paged_torch_ref
    rng = np.random.default_rng(4)
    q_len, own, table_row, prefix, lens, at = [3, 1, 0, 40, 2], [10, 0, 5, 33, 1], [0, 1, 2, 3, 4], [1, -1, 0, 0, 1], [20, 35], [5, 6]
    table = rng.permutation(40)[:28].reshape(7, 4).astype(np.int32)
    table[3, 1], table[5, 0], table[0, 0] = -1, 99, 40
    q = rng.standard_normal((sum(q_len), 4, 8)).astype(np.float32)
    k, v = (rng.standard_normal((40, 2, 16, 8)).astype(np.float32) for _ in range(2))
    args = (q_len, own, table_row, prefix, lens, at)
    want = ref.paged(q, k, v, table, 16, *args, causal=causal, scale=0.3)
    got = paged_torch_ref.paged(*[torch.from_numpy(x) for x in (q, k, v, table)], 16, *args, causal=causal, scale=0.3)
    for a, b in zip(got, want):
        assert (np.isfinite(a) == np.isfinite(b)).all() and np.abs(np.nan_to_num(a, neginf=0) - np.nan_to_num(b, neginf=0)).max() < 1e-12
