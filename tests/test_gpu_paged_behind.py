"""tts_paged: keys that lie behind the last one any row of a tile sees, in the same step of keys, may hold anything.  Tiles whose rows all end at one key are those of one query (groups of 16 heads and
more), and those of queries that see nothing of their own."""
import numpy as np
import pytest

from tests.helpers import say
from tests.test_gpu_paged import Case, _check

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _check_rows(c, out, lse, want, rows):
    at = c.torch.from_numpy(np.flatnonzero(rows)).to("cuda:0")
    _check(out[at], lse[at], [w[rows] for w in want], c.shape[2], c.longest, c.bf16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads,kv,d", [(16, 1, 64), (32, 1, 40), (32, 2, 128), (32, 2, 64)])
@pytest.mark.parametrize("past", [0, 3, 29, 45])
def test_a_query_by_itself(heads, kv, d, past, bf16):
    """A tile is one query's heads: the rows behind its own hold infinities and NaN."""
    say(f"case paged behind {heads}/{kv} heads of {d} past {past} {'bf16' if bf16 else 'fp32'}")
    q_len = [2, 5, 1, 3]
    own = [q + past + 7 * i for i, q in enumerate(q_len)]
    c = Case(_torch(), heads, kv, d, 16, bf16, q_len, own, [0, -1, 0, -1], [21], seed=heads + past)
    ends = np.cumsum(q_len) - 1
    others = np.ones(sum(q_len), bool)
    others[ends] = False
    want = c.want()
    for what in (float("nan"), float("inf"), -float("inf")):
        for t in (c.v, c.k):
            keep = t.clone()
            for i, m in enumerate(own):
                t[int(c.table_np[i, (m - 1) // 16]), :, (m - 1) % 16] = what
            out, lse = c.run()
            assert not bool(c.torch.isfinite(out[c.torch.from_numpy(ends).to("cuda:0")]).any()), what
            _check_rows(c, out, lse, want, others)
            t.copy_(keep)
    c.check(want=want)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads,kv", [(4, 4), (4, 2), (16, 1)])
@pytest.mark.parametrize("prefix,own,q", [(10, 5, 40), (48, 20, 37), (0, 3, 50)])
def test_queries_that_see_nothing_of_their_own(prefix, own, q, heads, kv, bf16):
    """More queries than rows: the first see the prefix alone, which ends in the middle of a step, and rows of their request behind it hold infinities and NaN."""
    say(f"case paged behind prefix {prefix} own {own} q {q} {heads}/{kv} heads {'bf16' if bf16 else 'fp32'}")
    c = Case(_torch(), heads, kv, 64, 16, bf16, [q], [own], [0] if prefix else None, [prefix] if prefix else [], seed=prefix + q)
    want, none = c.want(), np.arange(q) < q - own
    for what in (float("nan"), float("inf"), -float("inf")):
        for t in (c.v, c.k):
            keep = t.clone()
            for j in range(own):
                t[int(c.table_np[0, j // 16]), :, j % 16] = what
            out, lse = c.run()
            _check_rows(c, out, lse, want, none)
            t.copy_(keep)
    c.check(want=want)
