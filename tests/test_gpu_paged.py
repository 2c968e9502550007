"""tts_paged against its definition in 64 bits: steps, chunks and prompts of ragged requests, prefixes that they share, pages in any order and pages that there are not, what is not seen and what it
holds, heads that share keys, head widths, strides, long sequences in parts, addresses past 32 bits, graphs."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import past_ref as ref
from tests.helpers import say
from tests.test_gpu_cache import _np, _rand, _rows, _table

pytestmark = pytest.mark.gpu


def _check(got, lse, want, d, longest, bf16):
    """Scores: d products summed in fp32, the scale's and the exponent's rounding (8 half steps of the score), so that a weight is off by twice that; sums over at most `longest` keys in fp32, in
    parts that meet (8 roundings more each); bf16: weights and the result rounded once each."""
    out, want_lse, mass, size = want
    off = 2 * (d + 4 + 8) * ref.EPS32 * size + (longest + 64 + 8 * 257) * ref.EPS32
    tol = (off[:, :, None] + (ref.EPS_BF16 if bf16 else 0)) * mass + (ref.EPS_BF16 if bf16 else ref.EPS32) * np.abs(out)
    g = _np(got)
    assert np.isfinite(g).all()
    assert (np.abs(g - out) <= tol).all(), float(np.max(np.abs(g - out) - tol))
    if lse is not None:
        l, there = lse.cpu().numpy().astype(np.float64), np.isfinite(want_lse)
        assert (np.isneginf(l) == ~there).all()
        assert (np.abs(l[there] - want_lse[there]) <= (off + 8 * ref.EPS32 * (np.abs(want_lse) + size))[there]).all()


class Case:
    """A cache with its sequences (the requests' first, then the prefixes'), queries, and what they see."""

    def __init__(self, torch, heads, kv, d, page, bf16, q_len, own_len, prefix=None, prefix_len=(), gone=(), seed=0, pad=0, page_pad=0, size=1.0, causal=True, scale=0.0):
        rng = np.random.default_rng(seed)
        self.torch, self.shape, self.bf16, self.causal, self.scale = torch, (heads, kv, d, page), bf16, causal, scale
        n = len(q_len)
        self.table_np, pages = _table(rng, list(own_len) + list(prefix_len), page)
        for t, c in gone:
            self.table_np[t, c] = [-1, pages, 1 << 30, -(1 << 31)][(t + c) % 4]
        self.args = (q_len, own_len, list(range(n)), prefix, list(prefix_len), list(range(n, n + len(prefix_len))))
        wide = kv * page * d
        self.q = _rows(torch, rng, sum(q_len), heads, d, bf16, pad)
        self.q *= 1.5 * size
        self.k, self.v = (_rand(torch, rng, (pages, wide + page_pad), bf16)[:, :wide].unflatten(1, (kv, page, d)) for _ in range(2))
        self.k *= size
        self.table = torch.from_numpy(self.table_np).to("cuda:0")
        self.longest = max(list(own_len) + [0]) + max(list(prefix_len) + [0])

    def want(self):
        return ref.paged(_np(self.q), _np(self.k), _np(self.v), self.table_np, self.shape[3], *self.args, causal=self.causal, scale=self.scale or None)

    def op(self, stream=None):
        return binding.PagedAttention(binding.make_paged_config(*self.shape, self.bf16, self.causal), stream=stream or self.torch.cuda.current_stream())

    def run(self, lse=True):
        torch, op = self.torch, self.op()
        out = torch.full_like(self.q, 7.0)
        lse = torch.full(self.q.shape[:2], 7.0, device="cuda:0") if lse else None
        for i in range(2):
            op.run_device(op.batch(*self.args), self.q, self.k, self.v, self.table, out, lse=lse, scale=self.scale)
            torch.cuda.synchronize()
            if i == 0:
                first = out.clone()
        bits = torch.int16 if self.bf16 else torch.int32
        assert torch.equal(first.view(bits), out.view(bits))
        op.close()
        return out, lse

    def check(self, lse=True, want=None):
        out, l = self.run(lse)
        _check(out, l, want or self.want(), self.shape[2], self.longest, self.bf16)
        return out


HEADS = [(1, 1, 64), (8, 8, 64), (8, 2, 128), (6, 1, 96), (4, 4, 8), (3, 3, 40), (32, 2, 72), (5, 5, 128)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("heads,kv,d", HEADS)
def test_steps_of_ragged_requests(heads, kv, d, page, bf16):
    import torch
    say(f"case paged step {heads}/{kv} heads of {d}, pages of {page} {'bf16' if bf16 else 'fp32'}")
    own = [1, 0, 31, 32, 33, 250, 16, 129, 65, 2]
    Case(torch, heads, kv, d, page, bf16, [1] * len(own), own, seed=heads * d).check()
    Case(torch, heads, kv, d, page, bf16, [1] * len(own), own, [0, 0, -1, 1, 2, 0, 0, 2, 1, -1], [77, 16, 500], seed=heads * d + 1).check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,d,page", [(4, 4, 64, 16), (8, 2, 128, 64), (4, 1, 96, 32), (2, 2, 24, 16)])
def test_chunks_of_ragged_requests(heads, kv, d, page, causal, bf16):
    """From one query to hundreds, over pasts from none to long ones; more queries than rows; no own rows at all, with a prefix and without."""
    import torch
    say(f"case paged chunks {heads}/{kv} heads of {d}, pages of {page} {'bf16' if bf16 else 'fp32'} causal {causal}")
    q, own = [1, 127, 0, 128, 129, 17, 64, 300, 33, 5, 40, 2], [63, 127, 5, 400, 129, 30, 500, 300, 33, 3, 0, 0]
    Case(torch, heads, kv, d, page, bf16, q, own, seed=d, causal=causal).check()
    Case(torch, heads, kv, d, page, bf16, q, own, [0, 0, 0, 1, -1, 1, 1, 0, -1, 2, 0, -1], [100, 65, 0], seed=d + 1, causal=causal).check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,d,page,q", [(8, 8, 64, 16, 150), (8, 2, 128, 64, 70), (8, 4, 40, 32, 130), (4, 1, 96, 16, 300), (16, 16, 128, 128, 200)])
def test_many_rows(heads, kv, d, page, q, causal):
    """Enough rows for the tiles of 128."""
    import torch
    n = 24
    q_len, past = [1 + (q * (i % 7)) // 4 for i in range(n)], [(53 * i) % 260 for i in range(n)]
    own = [a + b for a, b in zip(q_len, past)]
    Case(torch, heads, kv, d, page, True, q_len, own, seed=q, causal=causal).check()
    Case(torch, heads, kv, d, page, True, q_len, own, [i % 4 - 1 for i in range(n)], [130, 64, 17], seed=q + 1, causal=causal).check()


@pytest.mark.parametrize("heads,kv,d,q,past,prefix", [(8, 8, 64, 1300, 0, 70), (16, 4, 128, 1100, 300, 1000)])
def test_large_tiles(heads, kv, d, q, past, prefix):
    """Enough rows for 256 a workgroup, more tiles than are looked up at once."""
    import torch
    n = 6
    q_len = [q + 37 * i for i in range(n)]
    own = [a + past for a in q_len]
    own[3] += 4300
    Case(torch, heads, kv, d, 16, True, q_len, own, [0, -1, 0, 0, -1, 0], [prefix], seed=q).check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,heads,kv,d", [(64, 8, 8, 64), (128, 16, 2, 128), (100, 4, 4, 40), (40, 32, 8, 96)])
def test_steps_over_a_shared_prefix(n, heads, kv, d, bf16):
    import torch
    own = [1 + (29 * i) % 150 for i in range(n)]
    Case(torch, heads, kv, d, 32, bf16, [1] * n, own, [0] * n, [1203], seed=n).check()
    Case(torch, heads, kv, d, 32, bf16, [1 + i % 3 for i in range(n)], [3 + o for o in own], [i % 3 - 1 for i in range(n)], [700, 65], seed=n + 1).check(lse=False)


@pytest.mark.parametrize("bf16", [False, True])
def test_more_requests_and_prefixes_than_a_launch_takes(bf16):
    import torch
    n = 300
    q_len, own = [(i * 5) % 4 for i in range(n)], [(7 * i) % 41 for i in range(n)]
    Case(torch, 2, 1, 64, 16, bf16, q_len, own, [(i * 11) % 41 - 1 for i in range(n)], [(13 * g) % 70 for g in range(40)], seed=300).check()
    Case(torch, 2, 2, 64, 16, bf16, [1] * 200, own[:200], [0] * 200, [333], seed=301).check()


def test_more_parts_than_there_is_room_for():
    """Requests whose own parts and prefix's would not all fit in the arena: several launches, the prefix read in each."""
    import torch
    n, heads = 40, 256
    Case(torch, heads, heads, 8, 16, True, [32] * n, [40 + i for i in range(n)], [0] * n, [50], seed=5).check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("q", [1, 20, 150])
def test_pages_that_there_are_not(q, bf16):
    """Pages given back: early ones, the last, a prefix's, all of a request's; a request with nothing left."""
    import torch
    n = 6
    q_len, own, page = [q, 1, q, q, 2, q], [q + 130, 40, q + 200, q, 90, q + 10], 16
    prefix, lens = [0, -1, 1, -1, 0, -1], [100, 33]
    gone = [(0, 1), (0, 2), (2, (q + 199) // page), (n, 0), (n, 5), (n + 1, 1)] + [(r, c) for r in (1, 3) for c in range(-(-own[r] // page))] + [(4, c) for c in range(6)]
    c = Case(torch, 8, 4, 64, page, bf16, q_len, own, prefix, lens, gone=gone, seed=q)
    out = c.check()
    first = sum(q_len[:3])
    assert (out[q_len[0]: q_len[0] + 1] == 0).all() and (out[first: first + q] == 0).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d", [64, 128, 40])
@pytest.mark.parametrize("q", [1, 5, 30, 150])
def test_what_is_not_seen_holds_anything(q, d, bf16):
    """Rows of a page behind a sequence's last, pages of nobody, pages that were given back and, for a query, the rows behind its own: infinities and NaN there are not used."""
    import torch
    page, n = 32, 4
    q_len, own, lens = [q] * n, [q + 50, q, q + 131, q + 31], [45]
    c = Case(torch, 4, 2, d, page, bf16, q_len, own, [0, -1, 0, -1], lens, gone=[(2, 1)], seed=q + d)
    seen = np.zeros(c.k.shape[:1] + (page,), bool)
    for row, m in enumerate(own + lens):
        for j in range(m):
            if c.table_np[row, j // page] in range(len(seen)):
                seen[c.table_np[row, j // page], j % page] = True
    want = c.want()
    k, v = c.k.clone(), c.v.clone()
    at = torch.from_numpy(np.argwhere(~seen)).to("cuda:0")
    for what in (float("nan"), float("inf"), -float("inf")):
        for t in (c.k, c.v):
            t[at[:, 0], :, at[:, 1]] = what
        c.check(want=want)
    # the last row of each request: its last query alone sees it
    last = [(int(c.table_np[i, (m - 1) // page]), (m - 1) % page) for i, m in enumerate(own)]
    ends = np.cumsum(q_len) - 1
    others = torch.ones(sum(q_len), dtype=torch.bool)
    others[torch.from_numpy(ends)] = False
    for what in (float("nan"), float("inf")):
        for pg, off in last:
            c.v[pg, :, off, :: 3] = what
        out, lse = c.run()
        for x in (out, lse):
            assert torch.isfinite(x[others.to("cuda:0")]).all()
        bad = ~torch.isfinite(out[torch.from_numpy(ends).to("cuda:0")])
        assert bad[:, :, ::3].all() and not bad[:, :, 1::3].any() and not bad[:, :, 2::3].any()
        for pg, off in last:
            c.v[pg, :, off] = v[pg, :, off]
        for pg, off in last:
            c.k[pg, :, off] = what
        out, _ = c.run()
        assert torch.isfinite(out[others.to("cuda:0")]).all()
        for pg, off in last:
            c.k[pg, :, off] = k[pg, :, off]
    c.check(want=want)


@pytest.mark.parametrize("q", [2, 150])
@pytest.mark.parametrize("bf16", [False, True])
def test_values_that_are_no_numbers_for_those_that_see_them(q, bf16):
    """An infinity that a query sees is its result's, with its sign; two of both signs, or a NaN, make NaN."""
    import torch
    c = Case(torch, 4, 2, 64, 16, bf16, [q, q], [q + 3, q + 40], seed=q)
    for i, m in enumerate((q + 3, q + 40)):
        at = lambda j: (int(c.table_np[i, j // 16]), slice(None), j % 16)       # noqa: E731
        c.v[at(m - 1)][:, 0], c.v[at(m - 1)][:, 1] = float("inf"), -float("inf")
        c.v[at(m - 2)][:, 0], c.v[at(m - 2)][:, 2] = -float("inf"), float("nan")
        c.v[at(0)][:, 3] = float("inf")
    out, _ = c.run()
    want = c.want()[0]
    got = _np(out)
    assert (np.isnan(got) == np.isnan(want)).all() and (got[np.isinf(want)] == want[np.isinf(want)]).all() and (np.isfinite(got) == np.isfinite(want)).all()
    assert np.isnan(got[q - 1, :, 0]).all() and (got[q - 2, :, 0] == -np.inf).all() and (got[:, :, 3] == np.inf).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,heads,kv,d,own", [(1, 2, 1, 64, 5000), (2, 8, 2, 128, 3001), (1, 1, 1, 64, 513), (3, 4, 4, 40, 1024), (1, 8, 8, 128, 20000)])
def test_long_sequences_in_parts(n, heads, kv, d, own, bf16):
    import torch
    lens = ([own, 0, 3][:n]) if n > 1 else [own]
    Case(torch, heads, kv, d, 64, bf16, [1] * n, lens, seed=own).check()
    Case(torch, heads, kv, d, 64, bf16, [3] * n, lens, [0] * n, [own // 2 + 5], gone=[(0, c) for c in range(own // 128)], seed=own + 1).check()


@pytest.mark.parametrize("n,heads,kv,d,q", [(70, 8, 4, 40, 1), (90, 6, 2, 64, 12), (64, 4, 4, 128, 1), (140, 4, 2, 64, 1)])
@pytest.mark.parametrize("bf16", [False, True])
def test_parts_of_many_requests(n, heads, kv, d, q, bf16):
    """A few long pasts among many short ones and absent ones."""
    import torch
    own = [(37 * i) % 90 for i in range(n)]
    own[3], own[n - 1], own[n // 2] = 9001, 6000, 4096
    q_len = [(q * (i % 4 + 1)) // 2 if q > 1 else 1 for i in range(n)]
    Case(torch, heads, kv, d, 32, bf16, q_len, own, seed=n + q).check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("q", [1, 140])
def test_strides_and_a_scale(q, bf16):
    """Rows apart (queries of a joint projection), pages apart (keys and values in one array), another scale."""
    import torch
    Case(torch, 4, 2, 64, 16, bf16, [q, 3, q], [q + 90, 30, q], [0, 0, -1], [50], pad=16, page_pad=72, scale=0.3, seed=11).check()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("q", [1, 40])
def test_loud_scores(q, bf16):
    """Scores of hundreds: the running maximum carries them, across parts too; one key takes all."""
    import torch
    Case(torch, 2, 2, 64, 16, bf16, [q] * 3, [q + 300] * 3, [0, 0, -1], [400], size=12, seed=7).check()


@pytest.mark.parametrize("q", [1, 140])
def test_addresses_past_32_bits(q):
    """Pages more than 2^32 bytes, and 2^31 elements, into their arrays."""
    import torch
    kv, d, page = 8, 128, 64
    c = Case(torch, 8, kv, d, page, True, [q], [q + 100], seed=8)
    want, extra = c.want(), (1 << 31) // (kv * d * page) + 3
    n = c.k.shape[0]
    big = [torch.empty(extra + n, kv, page, d, dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    big[0][extra:], big[1][extra:] = c.k, c.v
    c.k, c.v, c.table = big[0], big[1], c.table + extra
    c.check(want=want)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("q_len,own,prefix", [([1, 1], [3000, 2000], None), ([1, 1, 2], [50, 90, 8], [0, 0, 0]), ([200, 130], [400, 130], [0, -1]), ([1] * 30, [20] * 30, [0] * 30)])
def test_a_graph_on_a_stream_of_its_own(q_len, own, prefix, bf16):
    """Replays read queries, pages and the table anew; two graphs of one object in turn, whose parts share the arena."""
    import torch
    c = Case(torch, 4, 2, 64, 16, bf16, q_len, own, prefix, [300] if prefix else [], seed=12)
    op = c.op(torch.cuda.Stream())
    outs = [torch.empty_like(c.q) for _ in range(3)]
    batch, half = op.batch(*c.args), op.batch([1], [own[0] // 2 + 1], [0])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0], stream=op.stream):
        op.run_device(batch, c.q, c.k, c.v, c.table, outs[0])
    with torch.cuda.graph(graphs[1], stream=op.stream):
        op.run_device(half, c.q[:1], c.k, c.v, c.table, outs[1][:1])
    rng = np.random.default_rng(1)
    for i in range(4):
        c.q.copy_(_rows(torch, rng, sum(q_len), 4, 64, bf16))
        c.table[0] = c.table[0].flip(0) if (c.table[0] >= 0).all() else c.table[0]
        torch.cuda.synchronize()
        with torch.cuda.stream(op.stream):
            graphs[0].replay()
            graphs[1].replay()
            graphs[0].replay()
        torch.cuda.synchronize()
        op.run_device(batch, c.q, c.k, c.v, c.table, outs[2])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2]), i
        op.run_device(half, c.q[:1], c.k, c.v, c.table, outs[2][:1])
        torch.cuda.synchronize()
        assert torch.equal(outs[1][:1], outs[2][:1]), i
    op.close()


def test_nothing_to_do_and_nothing_to_see():
    import torch
    op = binding.PagedAttention(binding.make_paged_config(2, 2, 64, 16, True), stream=torch.cuda.current_stream())
    pages, table = torch.full((1, 2, 16, 64), float("nan"), dtype=torch.bfloat16, device="cuda:0"), torch.zeros(1, 1, dtype=torch.int32, device="cuda:0")
    none, q = (torch.ones(n, 2, 64, dtype=torch.bfloat16, device="cuda:0") for n in (0, 3))
    op.run_device(op.batch([0, 0], [0, 5], [0, 0]), none, pages, pages, table, none)
    out, lse = torch.ones_like(q), torch.ones(3, 2, device="cuda:0")
    for args in (([1, 2], [0, 0], [7, -1]), ([1, 2], [0, 0], [0, 0], [0, -1], [0], [9])):
        op.run_device(op.batch(*args), q, pages, pages, table, out, lse=lse)
        torch.cuda.synchronize()
        assert (out == 0).all() and torch.isneginf(lse).all()
        out.fill_(1)
    op.close()


@pytest.mark.parametrize("n,heads,kv,d,page,q,past,causal", [(1, 8, 2, 128, 16, 128, 3000, True), (1, 4, 1, 64, 64, 300, 1500, True), (2, 8, 8, 40, 16, 150, 2000, False), (3, 16, 2, 72, 32, 40, 2500, True),
                                                            (1, 4, 4, 128, 128, 700, 900, False)])
def test_parts_of_many_rows(n, heads, kv, d, page, q, past, causal):
    """Tiles of many rows over parts of their sequences, of which some see nothing of the last ones; prefixes ahead; pages that there are not; joined by a launch behind them."""
    import torch
    q_len, prefix = [max(1, q - 31 * i) for i in range(n)], [0] * n if n > 1 else None
    own = [past + a - 17 * i for i, a in enumerate(q_len)]
    Case(torch, heads, kv, d, page, True, q_len, own, prefix, [100] if prefix else [], gone=[(0, 3), (0, 0)], seed=d + q, causal=causal).check()
