"""tts_cross against its definition in 64 bits: lengths from none to thousands, heads that share keys, head widths, hidden and foreign positions, slots, strides,
long memories in parts, addresses past 32 bits, graphs."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import operator_ref as ref
from tests.helpers import say

pytestmark = pytest.mark.gpu


def _make(torch, rng, rows, heads, d, bf16, pad=0, size=1.0):
    t = torch.from_numpy((size * rng.standard_normal((rows, heads * d + pad))).astype(np.float32)).to("cuda:0")
    t = t.bfloat16() if bf16 else t
    return t[:, : heads * d].unflatten(1, (heads, d))


def _np(t):
    return t.double().cpu().numpy()


def _check(got, lse, want, d, longest, bf16):
    """Scores: d products summed in fp32, the scale's and the exponent's rounding (8 half steps of the score), so that a weight is off by twice that; sums over at most
    `longest` keys in fp32; bf16: weights and the result rounded once each."""
    out, want_lse, mass, size = want
    off = 2 * (d + 4 + 8) * ref.EPS32 * size + (longest + 64) * ref.EPS32
    tol = (off[:, :, None] + (ref.EPS_BF16 if bf16 else 0)) * mass + (ref.EPS_BF16 if bf16 else ref.EPS32) * np.abs(out)
    g = _np(got)
    assert np.isfinite(g).all()
    assert (np.abs(g - out) <= tol).all(), float(np.max(np.abs(g - out) - tol))
    if lse is not None:
        l, there = lse.cpu().numpy().astype(np.float64), np.isfinite(want_lse)
        assert (np.isneginf(l) == ~there).all()
        assert (np.abs(l[there] - want_lse[there]) <= (off + 8 * ref.EPS32 * (np.abs(want_lse) + size))[there]).all()


def _run(torch, heads, kv, d, bf16, q_len, mem_row, mem_len, rows=None, keep=None, seed=0, pad=0, lse=True, scale=0.0):
    rng = np.random.default_rng(seed)
    rows = max([r + m for r, m in zip(mem_row, mem_len)] + [1]) if rows is None else rows
    nq = sum(q_len)
    q, k, v = _make(torch, rng, nq, heads, d, bf16, pad, 1.5), _make(torch, rng, rows, kv, d, bf16, pad), _make(torch, rng, rows, kv, d, bf16, pad)
    op = binding.CrossAttention(binding.make_cross_config(heads, kv, d, bf16), stream=torch.cuda.current_stream())
    whole = torch.full((nq + 2, heads * d + pad), 3.0, dtype=q.dtype, device="cuda:0")
    out = whole[1:-1, : heads * d].unflatten(1, (heads, d))
    l = torch.full((nq, heads), 3.0, device="cuda:0") if lse else None
    op.run_device(op.batch(q_len, mem_row, mem_len), q, k, v, out, keep=keep, lse=l, scale=scale)
    torch.cuda.synchronize()
    kp = None if keep is None else keep.cpu().numpy()
    want = ref.cross(_np(q), _np(k), _np(v), q_len, mem_row, mem_len, kp, scale or None)
    _check(out, l, want, d, max(mem_len), bf16)
    whole[1:-1, : heads * d] = 3.0
    assert (whole == 3.0).all()                         # nothing around the rows was written
    op.close()


def _packed(mem_len):
    return [int(x) for x in np.cumsum([0] + list(mem_len))[:-1]]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads,kv,d", [(1, 1, 64), (8, 8, 64), (8, 2, 128), (6, 1, 96), (4, 4, 8), (3, 3, 40), (32, 2, 72), (5, 5, 128)])
def test_steps_of_ragged_memories(heads, kv, d, bf16):
    import torch
    say(f"case cross step {heads}/{kv} heads of {d} {'bf16' if bf16 else 'fp32'}")
    mem = [1, 0, 31, 32, 33, 250, 16, 129, 65, 2]
    _run(torch, heads, kv, d, bf16, [1] * len(mem), _packed(mem), mem, seed=heads * d)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 2, 128), (4, 1, 96), (2, 2, 24)])
def test_many_queries_of_ragged_lengths(heads, kv, d, bf16):
    import torch
    say(f"case cross frames {heads}/{kv} heads of {d} {'bf16' if bf16 else 'fp32'}")
    q, mem = [1, 127, 0, 128, 129, 17, 64, 300, 33], [63, 64, 5, 65, 1, 0, 200, 127, 520]
    _run(torch, heads, kv, d, bf16, q, _packed(mem), mem, seed=d)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("q_hi", [1, 150])
def test_hidden_positions_slots_and_what_they_hold(bf16, q_hi):
    """Positions hidden at random, all of a request's, and those behind its memory: what they hold, infinities and NaN among it, is not used."""
    import torch
    rng = np.random.default_rng(5)
    heads, kv, d, slot = 8, 4, 64, 264
    mem = [250, 1, 40, 0, 264, 77]
    q_len = [1 + (37 * i) % q_hi for i in range(6)]
    row = [slot * i for i in (5, 0, 3, 1, 2, 4)]        # slots in any order
    rows = slot * 6
    keep = (rng.random(rows) > 0.3).astype(np.uint8) * 255
    keep[row[2]: row[2] + 40] = 0                       # a request with nothing left
    keep[row[0]: row[0] + 100] = 0                      # whole tiles hidden in front ...
    keep[row[4] + 64: row[4] + 264] = 0                 # ... and behind
    q, k, v = _make(torch, rng, sum(q_len), heads, d, bf16, size=1.5), _make(torch, rng, rows, kv, d, bf16), _make(torch, rng, rows, kv, d, bf16)
    unseen = keep == 0
    for r, m, i in zip(row, mem, range(6)):
        unseen[r + m: r + slot] = True
    at = torch.from_numpy(np.flatnonzero(unseen)).to("cuda:0")
    want = ref.cross(_np(q), _np(k), _np(v), q_len, row, mem, keep)
    for what in (float("nan"), float("inf"), float("-inf")):
        k[at], v[at] = what, what
        op = binding.CrossAttention(binding.make_cross_config(heads, kv, d, bf16), stream=torch.cuda.current_stream())
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda:0")
        op.run_device(op.batch(q_len, row, mem), q, k, v, out, keep=torch.from_numpy(keep).to("cuda:0"), lse=lse)
        torch.cuda.synchronize()
        _check(out, lse, want, d, max(mem), bf16)
        none = np.repeat(np.array([m == 0 or not keep[r: r + m].any() for r, m in zip(row, mem)]), q_len)
        assert (out.cpu()[torch.from_numpy(none)] == 0).all() and none.any()
        op.close()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("q_len", [[1, 1], [1, 3], [200, 130]])
def test_what_lies_behind_a_memory_without_a_mask(bf16, q_len):
    import torch
    rng = np.random.default_rng(6)
    heads, kv, d = 4, 2, 128
    mem, row, rows = [70, 33], [8, 120], 200
    q, k, v = _make(torch, rng, sum(q_len), heads, d, bf16, size=1.5), _make(torch, rng, rows, kv, d, bf16), _make(torch, rng, rows, kv, d, bf16)
    want = ref.cross(_np(q), _np(k), _np(v), q_len, row, mem)
    there = np.zeros(rows, bool)
    for r, m in zip(row, mem):
        there[r: r + m] = True
    at = torch.from_numpy(np.flatnonzero(~there)).to("cuda:0")
    k[at], v[at] = float("nan"), float("inf")
    op = binding.CrossAttention(binding.make_cross_config(heads, kv, d, bf16), stream=torch.cuda.current_stream())
    out = torch.empty_like(q)
    op.run_device(op.batch(q_len, row, mem), q, k, v, out)
    torch.cuda.synchronize()
    _check(out, None, want, d, max(mem), bf16)
    op.close()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,heads,kv,d,mem", [(1, 2, 1, 64, 5000), (2, 8, 2, 128, 3001), (1, 1, 1, 64, 513), (3, 4, 4, 40, 1024)])
def test_long_memories_in_parts(n, heads, kv, d, mem, bf16):
    """Few queries over long memories: parts meet; a request without any and one that is shorter than a part among them."""
    import torch
    lens = ([mem, 0, 3][:n]) if n > 1 else [mem]
    _run(torch, heads, kv, d, bf16, [1] * n, _packed(lens), lens, seed=mem)
    keep = torch.ones(sum(lens), dtype=torch.uint8, device="cuda:0")
    keep[: mem // 2 + 7] = 0                            # whole parts hidden
    _run(torch, heads, kv, d, bf16, [2] * n, _packed(lens), lens, keep=keep, seed=mem + 1)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,heads,kv,d,q", [(70, 8, 4, 40, 1), (70, 4, 4, 64, 3), (90, 6, 2, 64, 12), (64, 4, 4, 128, 1), (128, 8, 8, 96, 1), (140, 4, 2, 64, 1)])
def test_parts_of_many_requests(n, heads, kv, d, q, bf16):
    """A few long memories among many short ones and absent ones: requests of several row tiles, or without queries, and of as many parts as their lengths give."""
    import torch
    say(f"case parts {n} x {q}, {heads}/{kv} heads of {d} {'bf16' if bf16 else 'fp32'}")
    mem = [(37 * i) % 90 for i in range(n)]
    mem[3], mem[n - 1], mem[n // 2] = 9001, 6000, 4096
    q_len = [(q * (i % 4 + 1)) // 2 if q > 1 else 1 for i in range(n)]
    keep = torch.from_numpy((np.random.default_rng(n + d).random(sum(mem)) > 0.3).astype(np.uint8)).to("cuda:0")
    for mask in (None, keep):
        _run(torch, heads, kv, d, bf16, q_len, _packed(mem), mem, keep=mask, seed=n + q)


@pytest.mark.parametrize("heads,kv,d,mem", [(2, 1, 64, 9000), (2, 2, 128, 8193)])
def test_many_queries_over_long_hidden_memories(heads, kv, d, mem):
    """More than the 4096 keys whose mask is looked at at once, whole stretches hidden."""
    import torch
    rng = np.random.default_rng(mem)
    keep = rng.random(mem + 60) > 0.5
    keep[:4200] = False
    keep[5000:8190] = False
    keep = torch.from_numpy(keep.astype(np.uint8)).to("cuda:0")
    _run(torch, heads, kv, d, True, [150, 33], [0, mem], [mem, 60], keep=keep, seed=mem)
    _run(torch, heads, kv, d, True, [150, 33], [0, mem], [mem, 60], seed=mem)


@pytest.mark.parametrize("n,q,mem,d", [(20, 600, 70, 64), (40, 300, 130, 128)])
def test_many_large_tiles(n, q, mem, d):
    """Enough rows for 256 a workgroup, ragged, shares of the XCDs of different sizes."""
    import torch
    q_len = [(q * (i % 5 + 1)) // 3 for i in range(n)]
    lens = [(mem * (i % 4)) for i in range(n)]
    _run(torch, 8, 4, d, True, q_len, _packed(lens), lens, seed=n)


@pytest.mark.parametrize("bf16", [False, True])
def test_strides_a_shared_memory_and_a_scale(bf16):
    """Rows apart (as of a projection to keys and values together), two requests over one memory, overlapping memories, another scale."""
    import torch
    _run(torch, 4, 2, 64, bf16, [3, 150, 1], [0, 0, 20], [90, 90, 60], pad=16, scale=0.3, seed=11)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("q", [1, 40])
def test_loud_scores(bf16, q):
    """Scores of hundreds: the running maximum carries them; one key takes all."""
    import torch
    rng = np.random.default_rng(7)
    qq, k, v = _make(torch, rng, q, 2, 64, bf16, size=30), _make(torch, rng, 300, 2, 64, bf16, size=10), _make(torch, rng, 300, 2, 64, bf16)
    op = binding.CrossAttention(binding.make_cross_config(2, 2, 64, bf16), stream=torch.cuda.current_stream())
    out, lse = torch.empty_like(qq), torch.empty(qq.shape[:2], device="cuda:0")
    op.run_device(op.batch([q], [0], [300]), qq, k, v, out, lse=lse)
    torch.cuda.synchronize()
    _check(out, lse, ref.cross(_np(qq), _np(k), _np(v), [q], [0], [300]), 64, 300, bf16)
    op.close()


def test_more_requests_than_a_launch_takes():
    import torch
    n = 300
    mem = [(7 * i) % 41 for i in range(n)]
    q = [(i * 5) % 4 for i in range(n)]
    _run(torch, 2, 1, 64, True, q, _packed(mem), mem, seed=300)


@pytest.mark.parametrize("q", [1, 140])
def test_addresses_past_32_bits(q):
    """A memory that begins more than 2^32 bytes, and 2^31 elements, into its array."""
    import torch
    rng = np.random.default_rng(8)
    kv, d, mem = 8, 128, 100
    rows = (1 << 31) // (kv * d) + 500
    big_k, big_v = (torch.empty(rows, kv, d, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    k, v, qq = _make(torch, rng, mem, kv, d, True), _make(torch, rng, mem, kv, d, True), _make(torch, rng, q, 8, d, True, size=1.5)
    first = rows - mem
    big_k[first:], big_v[first:] = k, v
    op = binding.CrossAttention(binding.make_cross_config(8, kv, d, True), stream=torch.cuda.current_stream())
    out = torch.empty_like(qq)
    op.run_device(op.batch([q], [first], [mem]), qq, big_k, big_v, out)
    torch.cuda.synchronize()
    _check(out, None, ref.cross(_np(qq), _np(k), _np(v), [q], [0], [mem]), d, mem, True)
    op.close()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("q_len,mem", [([1, 1], [3000, 2000]), ([1, 200], [50, 90])])
def test_a_graph_on_a_stream_of_its_own(q_len, mem, bf16):
    import torch
    rng = np.random.default_rng(12)
    op = binding.CrossAttention(binding.make_cross_config(4, 2, 64, bf16))
    q, k, v = _make(torch, rng, sum(q_len), 4, 64, bf16), _make(torch, rng, sum(mem), 2, 64, bf16), _make(torch, rng, sum(mem), 2, 64, bf16)
    out = torch.empty_like(q)
    batch = op.batch(q_len, _packed(mem), mem)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=op.stream):
        op.run_device(batch, q, k, v, out)
    for i in range(3):
        q.copy_(_make(torch, rng, sum(q_len), 4, 64, bf16))
        torch.cuda.synchronize()
        with torch.cuda.stream(op.stream):
            g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        op.run_device(batch, q, k, v, out)
        torch.cuda.synchronize()
        assert torch.equal(got, out), i
    op.close()


def test_no_queries_and_no_memory():
    import torch
    op = binding.CrossAttention(binding.make_cross_config(2, 2, 64, True), stream=torch.cuda.current_stream())
    none, q = (torch.ones(n, 2, 64, dtype=torch.bfloat16, device="cuda:0") for n in (0, 3))
    op.run_device(op.batch([0, 0], [0, 0], [0, 0]), none, none, none, none)
    out, lse = torch.ones_like(q), torch.ones(3, 2, device="cuda:0")
    op.run_device(op.batch([1, 2], [0, 0], [0, 0]), q, none, none, out, lse=lse)
    torch.cuda.synchronize()
    assert (out == 0).all() and torch.isneginf(lse).all()
    op.close()
