"""tts_cache against its definition in 64 bits: ragged new rows into pages in any order, types, strides, pages that there are not, what stays as it was, queries beside them, graphs."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import past_ref as ref
from tests.helpers import say

pytestmark = pytest.mark.gpu


def _rand(torch, rng, shape, bf16):
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to("cuda:0")
    return t.bfloat16() if bf16 else t


def _rows(torch, rng, rows, heads, d, bf16, pad=0):
    return _rand(torch, rng, (rows, heads * d + pad), bf16)[:, : heads * d].unflatten(1, (heads, d))


def _np(t):
    return t.double().cpu().numpy()


def _table(rng, lengths, page, spare=3, cols=None):
    """(table [sequences, pages], pages in all): numbers in any order, -1 behind a sequence's."""
    counts = [-(-n // page) for n in lengths]
    total = sum(counts) + spare
    order, table = rng.permutation(total), np.full((len(lengths), cols or max(counts + [1])), -1, np.int32)
    at = 0
    for i, c in enumerate(counts):
        table[i, :c] = order[at: at + c]
        at += c
    return table, total


def _run(torch, kv, heads, d, page, rot, pairs, x_bf16, bf16, length, row, table_row=None, position=None, gone=(), pad=0, page_pad=0, seed=0, **angles):
    rng = np.random.default_rng(seed)
    n, rows = len(length), sum(length)
    table_row = list(range(n)) if table_row is None else table_row
    lengths = [0] * (max(table_row) + 1)
    for t, r, m in zip(table_row, row, length):
        lengths[t] = max(lengths[t], r + m)
    table, pages = _table(rng, lengths, page)
    for t, c in gone:
        table[t, c] = [-1, pages, 1 << 30, -(1 << 31)][(t + c) % 4]
    k, v = _rows(torch, rng, rows, kv, d, x_bf16, pad), _rows(torch, rng, rows, kv, d, x_bf16, pad)
    q = _rows(torch, rng, rows, heads, d, x_bf16, pad) if heads else None
    wide = kv * page * d
    kp, vp = (_rand(torch, rng, (pages, wide + page_pad), bf16) for _ in range(2))
    before = [_np(kp), _np(vp)]
    kp_, vp_ = (t[:, :wide].unflatten(1, (kv, page, d)) for t in (kp, vp))
    q_out = _rows(torch, rng, rows, heads, d, bf16, pad) if heads else None
    op = binding.Cache(binding.make_cache_config(kv, d, page, binding.make_rotary_angles(rot, pairs, **angles) if rot else None, n_heads=heads, bf16=bf16, x_bf16=x_bf16),
                       stream=torch.cuda.current_stream())
    op.run_device(op.batch(length, row, table_row, position), k, v, kp_, vp_, torch.from_numpy(table).to("cuda:0"), q=q, q_out=q_out)
    torch.cuda.synchronize()
    p = np.concatenate([np.arange(m) + f for m, f in zip(length, position or row)] + [np.zeros(0, int)])

    def turned(t):
        return ref.rotary(_np(t), p, rot, pairs, **angles) if rot else (_np(t), np.zeros(t.shape))

    (k_want, k_size), v_want = turned(k), _np(v)
    want, tol = [b.copy() for b in before], [np.zeros(b.shape) for b in before]
    # (views of the pages, which may lie apart)
    wide_views = [np.lib.stride_tricks.as_strided(a, (pages, kv, page, d), (a.strides[0], page * d * 8, d * 8, 8)) for a in want + tol]
    at = 0
    for t, r, m in zip(table_row, row, length):
        pg, off = ref.places(table, t, r, m, page)
        there = (pg >= 0) & (pg < pages)
        i = np.arange(at, at + m)[there]
        wide_views[0][pg[there], :, off[there]] = k_want[i]
        wide_views[1][pg[there], :, off[there]] = v_want[i]
        wide_views[2][pg[there], :, off[there]] = ref.rotary_tolerance(k_want[i], k_size[i], bf16)
        wide_views[3][pg[there], :, off[there]] = (ref.EPS_BF16 if bf16 and not x_bf16 else 0) * np.abs(v_want[i])
        at += m
    # all of both arrays: what no new row goes to has a tolerance of 0
    for got, w, o in zip((kp, vp), want, tol):
        assert (np.abs(_np(got) - w) <= o).all(), float(np.max(np.abs(_np(got) - w) - o))
    if heads:
        w, size = turned(q)
        assert (np.abs(_np(q_out) - w) <= ref.rotary_tolerance(w, size, bf16)).all()
    op.close()


@pytest.mark.parametrize("x_bf16,bf16", [(True, True), (False, False), (True, False), (False, True)])
@pytest.mark.parametrize("kv,heads,d,page,rot,pairs", [(1, 0, 64, 16, 64, False), (2, 8, 64, 16, 64, True), (8, 8, 128, 64, 128, False), (3, 6, 40, 32, 40, False), (4, 4, 96, 128, 36, True),
                                                      (2, 2, 8, 1024, 6, False), (5, 0, 128, 32, 0, False), (1, 1, 72, 16, 70, False)])
def test_ragged_rows(kv, heads, d, page, rot, pairs, x_bf16, bf16):
    import torch
    say(f"case append {kv}/{heads} heads of {d}, pages of {page}, {rot} turn {x_bf16} {bf16}")
    length, row = [1, 0, 17, 33, 1, 64, 5, 130], [0, 3, 15, 31, 200, 0, 77, 1]
    _run(torch, kv, heads, d, page, rot, pairs, x_bf16, bf16, length, row, seed=d + page)


@pytest.mark.parametrize("bf16", [False, True])
def test_pages_that_there_are_not(bf16):
    """Numbers outside the cache: their rows are not kept, all others are, and queries of all rows come back."""
    import torch
    _run(torch, 2, 4, 64, 16, 64, False, bf16, bf16, [50, 3, 40], [10, 0, 0], gone=[(0, 1), (0, 3), (1, 0), (2, 2)], seed=2)


@pytest.mark.parametrize("bf16", [False, True])
def test_strides_positions_and_table_rows(bf16):
    """Rows of a joint projection, pages apart, positions other than the rows, one sequence in two pieces, table rows in another order."""
    import torch
    _run(torch, 2, 4, 64, 16, 32, True, bf16, bf16, [5, 20, 9], [40, 3, 10], table_row=[4, 1, 4], position=[1000000, -3, 0], pad=24, page_pad=40, seed=3, scaling=1, factor=4.0)


def test_more_requests_than_a_launch_takes():
    import torch
    n = 300
    _run(torch, 2, 2, 64, 16, 64, False, True, True, [(7 * i) % 5 for i in range(n)], [(13 * i) % 90 for i in range(n)], seed=4)
    _run(torch, 2, 2, 64, 16, 64, False, True, True, [1] * 129, [(13 * i) % 90 for i in range(129)], seed=5)


def test_many_rows():
    import torch
    _run(torch, 4, 16, 64, 64, 64, False, True, True, [3000, 1, 2500], [5, 100, 64], seed=6)


@pytest.mark.parametrize("bf16", [False, True])
def test_queries_in_place_and_none(bf16):
    import torch
    rng = np.random.default_rng(7)
    kv, heads, d, page = 2, 4, 64, 16
    cfg = binding.make_cache_config(kv, d, page, binding.make_rotary_angles(d), n_heads=heads, bf16=bf16, x_bf16=bf16)
    op = binding.Cache(cfg, stream=torch.cuda.current_stream())
    k, v, q = _rows(torch, rng, 9, kv, d, bf16), _rows(torch, rng, 9, kv, d, bf16), _rows(torch, rng, 9, heads, d, bf16)
    table = torch.arange(2, dtype=torch.int32, device="cuda:0").view(1, 2)
    pages = [torch.zeros(2, kv, page, d, dtype=k.dtype, device="cuda:0") for _ in range(4)]
    out = torch.empty_like(q)
    batch = op.batch([9], [4], [0])
    op.run_device(batch, k, v, pages[0], pages[1], table, q=q, q_out=out)
    op.run_device(batch, k, v, pages[2], pages[3], table)
    torch.cuda.synchronize()
    assert torch.equal(pages[0], pages[2]) and torch.equal(pages[1], pages[3])
    op.run_device(batch, k, v, pages[2], pages[3], table, q=q, q_out=q)
    torch.cuda.synchronize()
    assert torch.equal(q, out)
    op.close()


def test_addresses_past_32_bits():
    """A page more than 2^32 bytes, and 2^31 elements, into its array."""
    import torch
    rng = np.random.default_rng(8)
    kv, d, page = 8, 128, 64
    n = (1 << 31) // (kv * d * page) + 3
    kp, vp = (torch.empty(n, kv, page, d, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    kp[n - 1], vp[n - 1] = 0, 0
    k, v = _rows(torch, rng, 20, kv, d, True), _rows(torch, rng, 20, kv, d, True)
    op = binding.Cache(binding.make_cache_config(kv, d, page, bf16=True, x_bf16=True), stream=torch.cuda.current_stream())
    op.run_device(op.batch([20], [30], [0]), k, v, kp, vp, torch.tensor([[n - 1]], dtype=torch.int32, device="cuda:0"))
    torch.cuda.synchronize()
    for got, want in ((kp, k), (vp, v)):
        assert torch.equal(got[n - 1, :, 30:50].transpose(0, 1), want)
        assert (got[n - 1, :, :30] == 0).all() and (got[n - 1, :, 50:] == 0).all()
    op.close()


def test_a_graph_reads_its_table_anew():
    import torch
    rng = np.random.default_rng(9)
    kv, d, page = 2, 64, 16
    op = binding.Cache(binding.make_cache_config(kv, d, page, binding.make_rotary_angles(d), bf16=True, x_bf16=True))
    k, v = _rows(torch, rng, 12, kv, d, True), _rows(torch, rng, 12, kv, d, True)
    kp, vp, ke, ve = (torch.zeros(6, kv, page, d, dtype=torch.bfloat16, device="cuda:0") for _ in range(4))
    table = torch.zeros(2, 2, dtype=torch.int32, device="cuda:0")
    batch = op.batch([2, 10], [3, 14], [0, 1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=op.stream):
        op.run_device(batch, k, v, kp, vp, table)
    for i in range(3):
        table.copy_(torch.from_numpy(rng.permutation(6)[:4].reshape(2, 2).astype(np.int32)))
        k.copy_(_rows(torch, rng, 12, kv, d, True))
        torch.cuda.synchronize()
        with torch.cuda.stream(op.stream):
            g.replay()
        op.run_device(batch, k, v, ke, ve, table)
        torch.cuda.synchronize()
        assert torch.equal(kp, ke) and torch.equal(vp, ve), i
    op.close()


def test_no_rows():
    import torch
    op = binding.Cache(binding.make_cache_config(2, 64, 16, binding.make_rotary_angles(64), n_heads=2), stream=torch.cuda.current_stream())
    none = torch.empty(0, 2, 64, device="cuda:0")
    pages = torch.ones(1, 2, 16, 64, device="cuda:0")
    op.run_device(op.batch([0, 0], [0, 5], [0, 0]), none, none, pages, pages.clone(), torch.zeros(1, 1, dtype=torch.int32, device="cuda:0"), q=none, q_out=none)
    torch.cuda.synchronize()
    assert (pages == 1).all()
    op.close()


@pytest.mark.parametrize("x_bf16,bf16", [(True, True), (False, True), (False, False)])
@pytest.mark.parametrize("n,each", [(20, 5), (130, 1), (7, 64), (128, 3), (1, 300), (200, 2)])
def test_requests_of_as_many_rows_each(n, each, x_bf16, bf16):
    import torch
    say(f"case append {n} requests of {each} rows {x_bf16} {bf16}")
    _run(torch, 2, 4, 96, 16, 26, False, x_bf16, bf16, [each] * n, [(13 * i) % 50 for i in range(n)], seed=n)
