"""tts_cross in its form for many queries (two-byte requests of enough rows, in calls of enough of them): masks, what hidden and foreign positions hold, masks longer than are looked at at once, heads
of every width, both sizes of a workgroup, loud scores, strides, addresses past 32 bits, graphs, calls that are part few and part many.  That a case goes there the rule itself
says (tests/test_operator_plans.py, for 256 compute units)."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import operator_ref as ref
from tests.helpers import say
from tests.test_gpu_cross import _check, _make, _np, _packed, _run

pytestmark = pytest.mark.gpu

# name: (heads, kv, head_dim, q_len, mem_len, workgroups of 256 rows)
CASES = {
    "heads of 64": (32, 32, 64, [150, 33, 130, 257], [270, 65, 64, 129], False),
    "heads of 128": (32, 32, 128, [150, 33, 130, 257], [63, 200, 1, 1000], False),
    "heads of 24": (32, 32, 24, [200, 33, 128, 140], [300, 64, 70, 31], False),
    "heads of 40": (32, 32, 40, [200, 33, 129, 140], [130, 64, 70, 0], False),
    "heads of 72": (64, 16, 72, [90, 9, 65, 40], [32, 500, 70, 129], False),
    "heads of 96": (64, 16, 96, [90, 9, 65, 40], [33, 128, 0, 70], False),
    "narrow heads of 8": (40, 40, 8, [150, 130], [260, 97], False),
    "one key head": (64, 1, 64, [150, 33, 9], [190, 64, 33], False),
    "long, heads of 64": (64, 64, 64, [257, 33, 100, 300], [1100, 64, 1025, 1], True),
    "long, heads of 128": (64, 64, 128, [257, 33, 100, 260], [1025, 127, 0, 1090], True),
    "long, heads of 40": (64, 64, 40, [257, 33, 100, 300], [1090, 64, 1025, 31], True),
    "long, heads of 96": (64, 64, 96, [257, 33, 100, 260], [1033, 65, 1, 1089], True),
    "long, shared heads": (64, 16, 128, [257, 1000], [1024, 1500], True),
    "as long, too few tiles": (24, 24, 64, [257, 300, 100], [1100, 1025, 64], False),
    "as many tiles, too short": (64, 64, 64, [257, 33, 100, 300], [1023, 64, 1000, 1], False),
}


@pytest.mark.parametrize("name", CASES)
def test_ragged_lengths(name):
    heads, kv, d, q_len, mem, _ = CASES[name]
    say(f"case cross many {name}")
    _run(__import__("torch"), heads, kv, d, True, q_len, _packed(mem), mem, seed=d)


@pytest.mark.parametrize("name", CASES)
def test_hidden_and_foreign_positions(name):
    """A third of the positions hidden, all of one request's, whole tiles of another's in front, in the middle and behind; those and what lies behind a memory in its slot hold NaN or infinities."""
    import torch
    say(f"case cross many hidden {name}")
    heads, kv, d, q_len, mem, _ = CASES[name]
    rng = np.random.default_rng(d)
    slot = -(-max(mem) // 8) * 8 + 8
    n = len(mem)
    row = [slot * i for i in rng.permutation(n)]
    rows = slot * n
    keep = (rng.random(rows) > 0.3).astype(np.uint8) * 3
    longest, other = int(np.argmax(mem)), int(np.argsort(mem)[-2])
    keep[row[other]: row[other] + mem[other]] = 0
    r, m = row[longest], mem[longest]
    keep[r: r + min(70, m // 2)] = 0
    keep[r + m // 2: r + m // 2 + min(130, m // 4)] = 0
    keep[r + m - m // 8: r + m] = 0
    unseen = keep == 0
    for r, m in zip(row, mem):
        unseen[r + m: r + slot] = True
    q, k, v = _make(torch, rng, sum(q_len), heads, d, True, size=1.5), _make(torch, rng, rows, kv, d, True), _make(torch, rng, rows, kv, d, True)
    want = ref.cross(_np(q), _np(k), _np(v), q_len, row, mem, keep)
    at, keep_d = torch.from_numpy(np.flatnonzero(unseen)).to("cuda:0"), torch.from_numpy(keep).to("cuda:0")
    none = np.repeat(np.array([m == 0 or not keep[r: r + m].any() for r, m in zip(row, mem)]), q_len)
    assert none.any()
    op = binding.CrossAttention(binding.make_cross_config(heads, kv, d, True), stream=torch.cuda.current_stream())
    first = None
    for what in (0.0, float("nan"), float("inf"), float("-inf")):
        k[at], v[at] = what, what
        out, lse = torch.full_like(q, 3), torch.full(q.shape[:2], 3.0, device="cuda:0")
        op.run_device(op.batch(q_len, row, mem), q, k, v, out, keep=keep_d, lse=lse)
        torch.cuda.synchronize()
        if first is None:
            _check(out, lse, want, d, max(mem), True)
            assert (out.cpu()[torch.from_numpy(none)] == 0).all() and torch.isneginf(lse.cpu()[torch.from_numpy(none)]).all()
            first = (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), what
    op.close()


@pytest.mark.parametrize("name", ["heads of 64", "heads of 128", "long, heads of 40", "long, heads of 128"])
def test_what_lies_behind_a_memory_without_a_mask(name):
    import torch
    heads, kv, d, q_len, mem, _ = CASES[name]
    rng = np.random.default_rng(d)
    slot = -(-max(mem) // 8) * 8 + 72
    row, rows = [slot * i + 8 for i in range(len(mem))], slot * len(mem)
    q, k, v = _make(torch, rng, sum(q_len), heads, d, True, size=1.5), _make(torch, rng, rows, kv, d, True), _make(torch, rng, rows, kv, d, True)
    want = ref.cross(_np(q), _np(k), _np(v), q_len, row, mem)
    there = np.zeros(rows, bool)
    for r, m in zip(row, mem):
        there[r: r + m] = True
    at = torch.from_numpy(np.flatnonzero(~there)).to("cuda:0")
    k[at], v[at] = float("nan"), float("inf")
    op = binding.CrossAttention(binding.make_cross_config(heads, kv, d, True), stream=torch.cuda.current_stream())
    out = torch.empty_like(q)
    op.run_device(op.batch(q_len, row, mem), q, k, v, out)
    torch.cuda.synchronize()
    _check(out, None, want, d, max(mem), True)
    op.close()


# (heads, kv, head_dim, queries of two requests): of 128 and of 256 rows a workgroup
MASKS = {"128 rows": (48, 48, 64, [150, 73], False), "128 rows of 128": (48, 48, 128, [150, 73], False), "256 rows": (100, 100, 64, [257, 33], True), "256 rows of 128": (100, 100, 128, [150, 33], True)}


MASK_LENGTHS = (4097, 12300)


def mask_queries(name, mem):
    """(of 128 rows and over a long memory, those of the first request are few: the numpy side goes over them all)"""
    return [60, 150] if not MASKS[name][4] and mem > 5000 else MASKS[name][3]


@pytest.mark.parametrize("name", MASKS)
@pytest.mark.parametrize("mem", MASK_LENGTHS)
def test_masks_longer_than_are_looked_at_at_once(name, mem):
    """4096 positions at a time: the first of them hidden, some in the middle, and a request of its own with few."""
    import torch
    say(f"case cross many mask {name} {mem}")
    heads, kv, d, _, _ = MASKS[name]
    q_len = mask_queries(name, mem)
    rng = np.random.default_rng(mem)
    keep = rng.random(mem + 60) > 0.5
    keep[:4095] = False
    keep[4160:8190] = False
    keep[8256:] = True
    keep = torch.from_numpy(keep.astype(np.uint8)).to("cuda:0")
    _run(torch, heads, kv, d, True, q_len, [0, mem], [mem, 60], keep=keep, seed=mem)


@pytest.mark.parametrize("name", ["heads of 64", "heads of 128", "long, heads of 64", "long, heads of 128"])
def test_loud_scores(name):
    """Scores of hundreds, growing from key to key: sums are rescaled again and again, and one key takes all."""
    import torch
    heads, kv, d, q_len, mem, _ = CASES[name]
    rng = np.random.default_rng(7)
    mem = [max(m, 100) for m in mem]
    q, k, v = _make(torch, rng, sum(q_len), heads, d, True, size=20), _make(torch, rng, sum(mem), kv, d, True, size=5), _make(torch, rng, sum(mem), kv, d, True)
    k *= torch.linspace(0.01, 1, sum(mem), device="cuda:0")[:, None, None].bfloat16()
    op = binding.CrossAttention(binding.make_cross_config(heads, kv, d, True), stream=torch.cuda.current_stream())
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda:0")
    op.run_device(op.batch(q_len, _packed(mem), mem), q, k, v, out, lse=lse)
    torch.cuda.synchronize()
    _check(out, lse, ref.cross(_np(q), _np(k), _np(v), q_len, _packed(mem), mem), d, max(mem), True)
    op.close()


@pytest.mark.parametrize("name", ["heads of 64", "heads of 72", "long, shared heads"])
def test_rows_apart_shared_and_overlapping_memories_and_a_scale(name):
    import torch
    heads, kv, d, q_len, mem, _ = CASES[name]
    most = max(mem)
    _run(torch, heads, kv, d, True, q_len, [0, 0, 20, 7][:len(mem)], [most, most, most - 20, 1][:len(mem)], rows=most + 30, pad=16, scale=0.3, seed=11)


def mixed():
    """Steps between frames, requests without queries, more requests than a launch takes of either."""
    n = 400
    return 16, 4, 64, [(0, 1, 5, 64, 9)[i % 5] for i in range(n)], [(7 * i) % 150 for i in range(n)]


def test_part_few_and_part_many():
    import torch
    heads, kv, d, q, mem = mixed()
    keep = torch.from_numpy((np.random.default_rng(1).random(sum(mem)) > 0.3).astype(np.uint8)).to("cuda:0")
    for mask in (None, keep):
        _run(torch, heads, kv, d, True, q, _packed(mem), mem, keep=mask, seed=300)


@pytest.mark.parametrize("name", ["heads of 128", "long, shared heads"])
def test_addresses_past_32_bits(name):
    """Memories that begin more than 2^32 bytes, and 2^31 elements, into their array."""
    import torch
    heads, kv, d, q_len, mem, _ = CASES[name]
    rng = np.random.default_rng(8)
    used = sum(mem)
    rows = (1 << 31) // (kv * d) + used + 500
    big_k, big_v = (torch.empty(rows, kv, d, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    keep = torch.ones(rows, dtype=torch.uint8, device="cuda:0")
    k, v, q = _make(torch, rng, used, kv, d, True), _make(torch, rng, used, kv, d, True), _make(torch, rng, sum(q_len), heads, d, True, size=1.5)
    first = rows - used
    big_k[first:], big_v[first:] = k, v
    want = ref.cross(_np(q), _np(k), _np(v), q_len, _packed(mem), mem)
    op = binding.CrossAttention(binding.make_cross_config(heads, kv, d, True), stream=torch.cuda.current_stream())
    for mask in (None, keep):
        out = torch.empty_like(q)
        op.run_device(op.batch(q_len, [first + r for r in _packed(mem)], mem), q, big_k, big_v, out, keep=mask)
        torch.cuda.synchronize()
        _check(out, None, want, d, max(mem), True)
    op.close()


@pytest.mark.parametrize("name", ["heads of 64", "heads of 128", "long, heads of 64", "long, heads of 128"])
def test_a_graph_on_a_stream_of_its_own(name):
    import torch
    heads, kv, d, q_len, mem, _ = CASES[name]
    rng = np.random.default_rng(12)
    op = binding.CrossAttention(binding.make_cross_config(heads, kv, d, True))
    k, v = _make(torch, rng, sum(mem), kv, d, True), _make(torch, rng, sum(mem), kv, d, True)
    qs = [_make(torch, rng, sum(q_len), heads, d, True) for _ in range(3)]
    keeps = [torch.from_numpy((rng.random(sum(mem)) > 0.2 * i).astype(np.uint8)).to("cuda:0") for i in range(3)]
    q, keep, out = qs[0].clone(), keeps[0].clone(), torch.empty_like(qs[0])
    batch = op.batch(q_len, _packed(mem), mem)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=op.stream):
        op.run_device(batch, q, k, v, out, keep=keep)
    for i in range(3):
        q.copy_(qs[i])
        keep.copy_(keeps[i])
        torch.cuda.synchronize()
        with torch.cuda.stream(op.stream):
            g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        op.run_device(batch, q, k, v, out, keep=keep)
        torch.cuda.synchronize()
        assert torch.equal(got, out), i
    op.close()
