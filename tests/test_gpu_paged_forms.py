"""tts_paged in each way that a call of many rows, or over long prefixes, can be taken (paged_cases.py; that the calls are taken so is held by test_paged_forms_host.py): whole requests, parts of their keys,
prefixes in tiles of 64 and 128, requests of both kinds in one call; heads of every width, pages that there are not, what is not seen and what it holds, values that are no numbers, strides, addresses past 32 bits, graphs."""
import numpy as np
import pytest

from tests import paged_torch_ref
from tests.helpers import say
from tests.paged_cases import CASES
from tests.test_gpu_cache import _np, _rows
from tests.test_gpu_paged import Case, _check

pytestmark = pytest.mark.gpu


def _case(name, **more):
    import torch
    c = CASES[name]
    say(f"case paged form {name} {more if 'gone' not in more else 'pages gone'}")
    return Case(torch, c["heads"], c["kv"], c["d"], c["page"], c.get("bf16", True), c["q_len"], c["own_len"], c["prefix"], c["prefix_len"], causal=c["causal"], **{"seed": len(name), **more})


def _want(c):
    return paged_torch_ref.paged(c.q, c.k, c.v, c.table, c.shape[3], *c.args, causal=c.causal, scale=c.scale or None)


def _check_rows(c, out, lse, want, rows):
    at = c.torch.from_numpy(np.flatnonzero(rows)).to("cuda:0")
    _check(out[at], lse[at], [w[rows] for w in want], c.shape[2], c.longest, c.bf16)


@pytest.mark.parametrize("name", CASES)
def test_form(name):
    c = _case(name)
    want = _want(c)
    c.check(want=want)
    out, _ = c.run(lse=False)
    _check(out, None, want, c.shape[2], c.longest, c.bf16)


def _gone(name):
    """Pages of requests (all of one's) and of prefixes, first, last and between."""
    c = CASES[name]
    pages = lambda m: -(-m // c["page"])                                         # noqa: E731
    n, got = len(c["q_len"]), []
    for i, m in enumerate(c["own_len"]):
        got += [(i, j) for j in range(pages(m)) if (i == 2 or (i % 3 == 0 and j % 5 == 1) or (i % 4 == 1 and j == pages(m) - 1))]
    for g, m in enumerate(c["prefix_len"]):
        got += [(n + g, j) for j in range(pages(m)) if j in (0, pages(m) - 1) or j % 7 == 3]
    return got


@pytest.mark.parametrize("name", ["many_64", "many_40", "many_72", "many_128", "many_64_all", "parts_128", "parts_64", "parts_40", "parts_128_own", "parts_64_own", "parts_128_short", "parts_64_short",
                                  "parts_64_all", "prefix_128_of_128", "prefix_128_of_40", "prefix_64_of_128", "prefix_64_of_40", "chunks_64", "chunks_64_long", "chunks_40_fp32", "chunks_128_fp32",
                                  "chunks_128_fp32_long"])
def test_what_is_not_seen_holds_anything(name):
    """Rows behind a sequence's last, pages of nobody, pages that are gone and, for a query, the rows behind its own: infinities and NaN there are not used."""
    c = _case(name, gone=_gone(name))
    torch, page = c.torch, c.shape[3]
    q_len, own, lens = c.args[0], c.args[1], c.args[4]
    want = _want(c)
    c.check(want=want)
    seen = np.zeros((c.k.shape[0], page), bool)
    for row, m in enumerate(list(own) + list(lens)):
        j = np.arange(m)
        at = c.table_np[row, j // page] if m else j
        there = (at >= 0) & (at < len(seen))
        seen[at[there], j[there] % page] = True
    at = torch.from_numpy(np.argwhere(~seen)).to("cuda:0")
    for what in (float("nan"), float("inf"), -float("inf")):
        for t in (c.k, c.v):
            t[at[:, 0], :, at[:, 1]] = what
        c.check(want=want)
    if not c.causal:
        return
    # rows that later queries of their request see: the last of each, and one that a third of its queries see
    places, others, first = [], np.ones(sum(q_len), bool), 0
    for i, (n, m) in enumerate(zip(q_len, own)):
        for behind in {0, min(n, m) // 3}:
            if 0 <= m - 1 - behind and 0 <= c.table_np[i, (m - 1 - behind) // page] < len(seen):
                places.append((int(c.table_np[i, (m - 1 - behind) // page]), (m - 1 - behind) % page))
                others[first + n - 1 - behind: first + n] = False
        first += n
    at, none = torch.tensor(places, device="cuda:0"), torch.from_numpy(np.flatnonzero(~others)).to("cuda:0")
    assert len(places) and others.any()
    for t in (c.v, c.k):
        keep = t[at[:, 0], :, at[:, 1]].clone()
        for what in (float("nan"), float("inf")):
            t[at[:, 0], :, at[:, 1]] = what
            out, lse = c.run()
            _check_rows(c, out, lse, want, others)
            assert not bool(torch.isfinite(out[none]).any())
        t[at[:, 0], :, at[:, 1]] = keep
    c.check(want=want)


@pytest.mark.parametrize("name", ["many_64", "many_40", "many_128", "many_64_all", "parts_64", "parts_128_own", "prefix_128_of_128", "chunks_64", "chunks_128_fp32"])
def test_values_that_are_no_numbers_for_those_that_see_them(name):
    """An infinity that a query sees is its result's, with its sign; two of both signs, or a NaN, make NaN."""
    c = _case(name)
    q_len, own = c.args[0], c.args[1]
    for i, (n, m) in enumerate(zip(q_len, own)):
        at = lambda j: (int(c.table_np[i, j // c.shape[3]]), slice(None), j % c.shape[3])       # noqa: E731
        if m > 2:
            c.v[at(m - 1)][:, 0], c.v[at(m - 1)][:, 1] = float("inf"), -float("inf")
            c.v[at(m - 2)][:, 0], c.v[at(m - 2)][:, 2] = -float("inf"), float("nan")
            c.v[at(0)][:, 3] = float("inf")
    out, _ = c.run()
    got, first = _np(out), 0
    for i, (n, m) in enumerate(zip(q_len, own)):
        last = m - n + np.arange(n) if c.causal else np.full(n, m - 1)         # the last row that a query sees
        rows, first = got[first: first + n], first + n
        if m <= 2:
            assert np.isfinite(rows).all()
            continue
        sees = [last >= m - 1, last >= m - 2, last >= 0]
        assert np.isfinite(rows[:, :, 4:]).all()
        assert (np.isnan(rows[:, :, 0]) == (sees[0])[:, None]).all() and (rows[:, :, 0][sees[1] & ~sees[0]] == -np.inf).all() and np.isfinite(rows[:, :, 0][~sees[1]]).all()
        assert ((rows[:, :, 1] == -np.inf) == sees[0][:, None]).all() and np.isfinite(rows[:, :, 1][~sees[0]]).all()
        assert (np.isnan(rows[:, :, 2]) == sees[1][:, None]).all() and np.isfinite(rows[:, :, 2][~sees[1]]).all()
        assert ((rows[:, :, 3] == np.inf) == sees[2][:, None]).all() and np.isfinite(rows[:, :, 3][~sees[2]]).all()


@pytest.mark.parametrize("name", ["many_96", "many_40", "many_64_all", "parts_72", "parts_64", "prefix_128_of_96", "prefix_64_of_40"])
def test_strides_and_a_scale(name):
    """Rows apart, pages apart, another scale."""
    c = _case(name, pad=16, page_pad=72, scale=0.3)
    c.check(want=_want(c))


@pytest.mark.parametrize("name", ["many_64", "many_128", "parts_64", "parts_128_own", "prefix_128_of_128", "prefix_64_of_128", "chunks_64_long", "chunks_40_fp32"])
def test_loud_scores(name):
    """Scores of hundreds: the running maximum carries them, across parts too; one key takes all."""
    c = _case(name, size=12)
    c.check(want=_want(c))


@pytest.mark.parametrize("name", ["many_128", "parts_128", "prefix_128_of_128"])
def test_addresses_past_32_bits(name):
    """Pages more than 2^32 bytes, and 2^31 elements, into their arrays."""
    c = _case(name)
    torch, want = c.torch, _want(c)
    shape = c.k.shape
    extra = (1 << 31) // (shape[1] * shape[2] * shape[3]) + 3
    for which in ("k", "v"):
        big = torch.empty(extra + shape[0], *shape[1:], dtype=torch.bfloat16, device="cuda:0")
        big[extra:] = getattr(c, which)
        setattr(c, which, big)
    c.table = c.table + extra * (c.table >= 0).int()
    c.check(want=want)


@pytest.mark.parametrize("name", ["many_72", "parts_64", "parts_128_own", "prefix_128_of_128", "prefix_64_of_128"])
def test_a_graph_on_a_stream_of_its_own(name):
    """Replays read queries, pages and the table anew; two graphs of one object in turn, whose parts share the arena."""
    c = _case(name)
    torch, page = c.torch, c.shape[3]
    op = c.op(torch.cuda.Stream())
    outs = [torch.empty_like(c.q) for _ in range(3)]
    own = c.args[1]
    batch, half = op.batch(*c.args), op.batch([1], [own[0] // 2 + 1], [0])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0], stream=op.stream):
        op.run_device(batch, c.q, c.k, c.v, c.table, outs[0])
    with torch.cuda.graph(graphs[1], stream=op.stream):
        op.run_device(half, c.q[:1], c.k, c.v, c.table, outs[1][:1])
    rng, before, pages = np.random.default_rng(1), None, -(-own[0] // page)
    for i in range(4):
        c.q.copy_(_rows(torch, rng, c.q.shape[0], c.shape[0], c.shape[2], c.bf16))
        c.table[0, :pages] = c.table[0, :pages].flip(0).clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(op.stream):
            graphs[0].replay()
            graphs[1].replay()
            graphs[0].replay()
        torch.cuda.synchronize()
        op.run_device(batch, c.q, c.k, c.v, c.table, outs[2])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2]) and (before is None or not torch.equal(before, outs[0])), i
        before = outs[0].clone()
        op.run_device(half, c.q[:1], c.k, c.v, c.table, outs[2][:1])
        torch.cuda.synchronize()
        assert torch.equal(outs[1][:1], outs[2][:1]), i
    op.close()
