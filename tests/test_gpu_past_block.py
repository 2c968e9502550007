"""What a decoder block does with its own past, one call behind the other: norm and codes (tts_norm), one product for queries, keys and values (tts_linear8), rotary positions and new rows into
pages (tts_cache), attention to them (tts_paged): a prefix that requests share, their prompts behind it, steps of one token each.  Every stage against its definition in 64 bits."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import past_ref as ref
from tests.test_gpu_cache import _np
from tests.test_gpu_paged import _check

pytestmark = pytest.mark.gpu


class Block:
    def __init__(self, torch, heads, kv, d, page, bf16, pairs, stream):
        rng = np.random.default_rng(d)
        self.torch, self.shape, self.bf16, self.pairs, self.stream, self.dim = torch, (heads, kv, d, page), bf16, pairs, stream, 256
        wide = (heads + 2 * kv) * d
        self.rot = d // 2 if pairs else d
        self.norm = binding.Norm(binding.make_norm_config(self.dim, True), np.ones(self.dim, np.float32), stream=stream)
        self.linear = binding.Linear8(binding.make_linear8_config(self.dim, wide, bf16), rng.standard_normal((wide, self.dim)).astype(np.float32) / 16, stream=stream)
        self.cache = binding.Cache(binding.make_cache_config(kv, d, page, binding.make_rotary_angles(self.rot, pairs), n_heads=heads, bf16=bf16, x_bf16=bf16), stream=stream)
        self.attend = binding.PagedAttention(binding.make_paged_config(heads, kv, d, page, bf16), stream=stream)
        self.type = torch.bfloat16 if bf16 else torch.float32

    def buffers(self, rows):
        torch, (heads, _, d, _) = self.torch, self.shape
        e = lambda shape, t: torch.empty(shape, dtype=t, device="cuda:0")               # noqa: E731
        return dict(x=e((rows, self.dim), torch.bfloat16), x8=e((rows, binding.width8(self.dim)), torch.float8_e4m3fn), s8=e((rows, binding.scale_columns(self.dim)), torch.float8_e8m0fnu),
                    qkv=e((rows, self.linear._widths[2]), self.type), q=e((rows, heads, d), self.type), out=e((rows, heads, d), self.type), lse=e((rows, heads), torch.float32))

    def parts(self, qkv):
        heads, kv, d, _ = self.shape
        return (t.unflatten(1, (-1, d)) for t in qkv.split([heads * d, kv * d, kv * d], 1))

    def run(self, b, new, batch, pages):
        """New rows of sequences 0 .. (a request's table row is its number)."""
        self.norm.run_device(b["x"], y8=b["x8"], scales=b["s8"])
        self.linear.run_device(b["x8"], b["s8"], b["qkv"])
        q, k, v = self.parts(b["qkv"])
        self.cache.run_device(new, k, v, *pages, q=q, q_out=b["q"])
        self.attend.run_device(batch, b["q"], *pages, b["out"], lse=b["lse"])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads,kv,d,page,pairs,prefix,prompts,steps", [
    (8, 8, 64, 16, False, 100, [37, 1, 60], 3),
    (8, 2, 128, 64, False, 700, [3, 300, 64, 129], 2),
    (4, 4, 40, 32, True, 33, [0, 5], 2),
    (16, 4, 64, 16, True, 1500, [1] * 20, 2),
])
def test_a_block_over_its_past(heads, kv, d, page, pairs, prefix, prompts, steps, bf16):
    """Each call's pages and queries against 64 bits of the product's own rows, its attention against 64 bits of the pages; on a stream of the test's own."""
    import torch
    rng = np.random.default_rng(heads)
    stream = torch.cuda.Stream()
    block = Block(torch, heads, kv, d, page, bf16, pairs, stream)
    n = len(prompts)
    lengths = [m + steps for m in prompts] + [prefix]
    counts = [-(-m // page) for m in lengths]
    table_np = np.full((n + 1, max(counts)), -1, np.int32)
    order, at = rng.permutation(sum(counts)), 0
    for i, c in enumerate(counts):
        table_np[i, :c] = order[at: at + c]
        at += c
    table = torch.from_numpy(table_np).to("cuda:0")
    kp, vp = (torch.full((sum(counts), kv, page, d), float("nan"), dtype=block.type, device="cuda:0") for _ in range(2))      # (nothing of it is used before it is written)
    want = [np.full(kp.shape, np.nan) for _ in range(2)]
    # (a request's rows, of them those that are there before, its table row and its positions' first) of each call
    calls = [([prefix], [0], [n], [0])] + [(prompts, [0] * n, list(range(n)), [prefix] * n)] + [([1] * n, [m + s for m in prompts], list(range(n)), [prefix + m + s for m in prompts]) for s in range(steps)]
    for length, row, table_row, position in calls:
        b = block.buffers(sum(length))
        b["x"].copy_(torch.from_numpy(rng.standard_normal(b["x"].shape).astype(np.float32)))
        own = [r + m for r, m in zip(row, length)]
        shares = table_row != [n]
        batch = block.attend.batch(length, own, table_row, [0] * n, [prefix], [n]) if shares else block.attend.batch(length, own, table_row)
        torch.cuda.synchronize()
        block.run(b, block.cache.batch(length, row, table_row, position), batch, (kp, vp, table))
        torch.cuda.synchronize()
        q, k, v = (_np(t) for t in block.parts(b["qkv"]))
        assert np.isfinite(q).all()
        p = np.concatenate([f + np.arange(m) for f, m in zip(position, length)])
        (q_want, q_size), (k_want, k_size) = ref.rotary(q, p, block.rot, pairs), ref.rotary(k, p, block.rot, pairs)
        assert (np.abs(_np(b["q"]) - q_want) <= ref.rotary_tolerance(q_want, q_size, bf16)).all()
        at = 0
        got_k, got_v = _np(kp), _np(vp)
        for t, r, m in zip(table_row, row, length):
            pg, off = ref.places(table_np, t, r, m, page)
            assert (np.abs(got_k[pg, :, off] - k_want[at: at + m]) <= ref.rotary_tolerance(k_want[at: at + m], k_size[at: at + m], bf16)).all()
            assert (got_v[pg, :, off] == v[at: at + m]).all()
            want[0][pg, :, off], want[1][pg, :, off] = got_k[pg, :, off], v[at: at + m]
            at += m
        for got, kept in zip((got_k, got_v), want):                                    # what was there stays, and nothing else comes
            assert np.array_equal(got, kept, equal_nan=True)
        args = (length, own, table_row, [0] * n, [prefix], [n]) if shares else (length, own, table_row)
        _check(b["out"], b["lse"], ref.paged(_np(b["q"]), got_k, got_v, table_np, page, *args), d, max(own) + prefix, bf16)


@pytest.mark.parametrize("bf16", [False, True])
def test_a_step_in_a_graph(bf16):
    """The four calls of a step captured, replayed with other inputs and tables between eager calls of the same objects: the same bits."""
    import torch
    rng = np.random.default_rng(3)
    heads, kv, d, page, n = 8, 2, 64, 16, 12
    block = Block(torch, heads, kv, d, page, bf16, False, torch.cuda.Stream())
    own = [17 * i + 1 for i in range(n)]
    cols = -(-max(own) // page)
    pages = n * cols
    kp, vp = (torch.randn((pages, kv, page, d), device="cuda:0").to(block.type) for _ in range(2))
    table = torch.arange(pages, dtype=torch.int32, device="cuda:0").reshape(n, cols)
    b, e = block.buffers(n), block.buffers(n)
    new, batch = block.cache.batch([1] * n, [m - 1 for m in own], list(range(n))), block.attend.batch([1] * n, own, list(range(n)))
    for t in (b, e):
        t["x"].zero_()
    torch.cuda.synchronize()
    block.run(b, new, batch, (kp, vp, table))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=block.stream):
        block.run(b, new, batch, (kp, vp, table))
    for i in range(4):
        x = torch.from_numpy(rng.standard_normal(b["x"].shape).astype(np.float32)).to("cuda:0")
        b["x"].copy_(x)
        e["x"].copy_(x)
        table.copy_(torch.from_numpy(rng.permutation(pages).reshape(n, cols).astype(np.int32)))
        torch.cuda.synchronize()
        with torch.cuda.stream(block.stream):
            graph.replay()
        torch.cuda.synchronize()
        got_k, got_v = kp.clone(), vp.clone()
        block.run(e, new, batch, (kp, vp, table))
        torch.cuda.synchronize()
        assert torch.equal(b["out"], e["out"]) and torch.equal(b["lse"], e["lse"]) and torch.equal(b["q"], e["q"]), i
        assert torch.equal(got_k, kp) and torch.equal(got_v, vp), i


def test_tensors_that_do_not_fit_are_refused():
    """Another device, type or number of elements, rows that do not lie back to back, arrays that come together: before anything is queued."""
    import torch
    heads, kv, d, page = 4, 2, 64, 16
    cache = binding.Cache(binding.make_cache_config(kv, d, page, binding.make_rotary_angles(d), n_heads=heads, bf16=True, x_bf16=True))
    attend = binding.PagedAttention(binding.make_paged_config(heads, kv, d, page, True))
    rotary = binding.Rotary(binding.make_rotary_config(heads, d, binding.make_rotary_angles(d), True, True))
    z = lambda *shape, **k: torch.zeros(shape, **{"dtype": torch.bfloat16, "device": "cuda:0", **k})             # noqa: E731
    good = dict(k=z(3, kv, d), v=z(3, kv, d), k_pages=z(2, kv, page, d), v_pages=z(2, kv, page, d), table=z(1, 2, dtype=torch.int32), q=z(3, heads, d), q_out=z(3, heads, d))
    bad = [dict(k=z(3, kv, d, device="cpu")), dict(k=z(3, kv, d, device="meta")), dict(v=z(3, kv, d, dtype=torch.float32)), dict(k=z(2, kv, d)), dict(k=z(3, d, kv).transpose(1, 2)), dict(q=None),
           dict(q_out=z(3, heads, d, dtype=torch.float32)), dict(k_pages=z(2, kv, page, d, dtype=torch.float16)), dict(v_pages=z(1, kv, page, d)), dict(k_pages=z(2, page, kv, d).transpose(1, 2)),
           dict(k_pages=z(3, kv, page, d + 8)[:, :, :, :d]), dict(table=z(1, 2, dtype=torch.int64)), dict(table=z(2, dtype=torch.int32)), dict(table=z(1, 4, dtype=torch.int32)[:, ::2]),
           dict(v_pages=z(4, kv, page, d)[::2])]
    batch = cache.batch([3], [0], [0])
    cache.run_device(batch, **good)
    for change in bad:
        with pytest.raises(ValueError):
            cache.run_device(batch, **{**good, **change})
    good = dict(q=z(3, heads, d), k_pages=good["k_pages"], v_pages=good["v_pages"], table=good["table"], out=z(3, heads, d), lse=z(3, heads, dtype=torch.float32))
    batch = attend.batch([3], [3], [0])
    attend.run_device(batch, **good)
    for change in [dict(q=z(3, heads, d, device="cpu")), dict(out=z(3, heads, d, dtype=torch.float32)), dict(out=z(4, heads, d)), dict(q=z(heads, 3, d).transpose(0, 1)), dict(lse=z(3, heads)),
                   dict(lse=z(2, heads, dtype=torch.float32)), dict(table=z(1, 2, dtype=torch.int32, device="cpu")), dict(scale=1e-60)] + [b for b in bad if set(b) & {"k_pages", "v_pages", "table"}]:
        with pytest.raises(ValueError):
            attend.run_device(batch, **{**good, **change})
    for scale in (-1.0, float("nan"), float("inf")):
        with pytest.raises(binding.TtsError):
            attend.run_device(batch, **good, scale=scale)
    x = z(3, heads, d)
    rotary.run_device(x, x)
    for args in ((z(3, heads, d, device="cpu"), x), (x, z(2, heads, d)), (x, z(3, heads, d, dtype=torch.float32)), (z(3, heads, 40), x), (z(3, d, heads).transpose(1, 2), x)):
        with pytest.raises(ValueError):
            rotary.run_device(*args)
    for more in (dict(positions=z(2, dtype=torch.int32)), dict(positions=z(3, dtype=torch.int64)), dict(positions=z(6, dtype=torch.int32)[::2]), dict(first=1 << 31)):
        with pytest.raises(ValueError):
            rotary.run_device(x, x, **more)
    torch.cuda.synchronize()


def test_streams_that_wait_for_each_other():
    """Objects on streams of their own, tensors of the default one, and an event between them, as the headers ask: what is queued later on a stream sees what was ahead."""
    import torch
    heads, kv, d, page, n = 4, 2, 64, 16, 400
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    cache = binding.Cache(binding.make_cache_config(kv, d, page, binding.make_rotary_angles(d), n_heads=heads), stream=one)
    attend = binding.PagedAttention(binding.make_paged_config(heads, kv, d, page), stream=two)
    table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda:0")[None]
    kp, vp = (torch.zeros(table.shape[1], kv, page, d, device="cuda:0") for _ in range(2))
    q_out, out = (torch.zeros(n, heads, d, device="cuda:0") for _ in range(2))
    new, batch = cache.batch([n], [0], [0]), attend.batch([n], [n], [0])
    want = None
    for i in range(3):
        g = torch.Generator(device="cuda:0").manual_seed(5)
        k, v, q = (torch.randn(n, h, d, generator=g, device="cuda:0") for h in (kv, kv, heads))
        one.wait_stream(torch.cuda.current_stream())
        cache.run_device(new, k, v, kp, vp, table, q=q, q_out=q_out)
        two.wait_stream(one)
        attend.run_device(batch, q_out, kp, vp, table, out)
        torch.cuda.current_stream().wait_stream(two)
        got = out.clone()
        for t in (kp, vp, q_out, out):
            t.zero_()
        torch.cuda.synchronize()
        assert bool(torch.isfinite(got).all()) and float(got.abs().max()) > 0.1
        want = got if want is None else want
        assert torch.equal(got, want), i
