"""The operators as an attention block uses them: the encoder's F_enc rounded to 8 bits and projected to keys and values once, then a pool's steps -- residual and
norm to 8 bits, query projection, attention to each request's own positions, its output rounded and projected back into the stream.  Every stage is held to its definition in
64 bits on what the stage before it left, so that each tolerance is that stage's own; the steps run eagerly and as a replayed graph, bit for bit the same."""
import numpy as np
import pytest

from paper_2211_13939_amd import binding, synth
from tests import operator_ref as ref

pytestmark = pytest.mark.gpu

DIM, HEADS, KV, D = 512, 8, 2, 64
LENS = [37, 1, 120, 64]


def _bytes(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def _np(t):
    return t.double().cpu().numpy()


def _held8(b, s, y, slack):
    """8-bit rows hold y to half a step (tests/test_gpu_norm.py)."""
    scale = np.repeat(2.0 ** (s[:, : b.shape[1] // 128].astype(np.float64) - 127), 128, axis=1)
    assert (np.abs(ref.TABLE[b] * scale - y) <= np.maximum(np.abs(y) * (2.0 ** -4 + slack), scale * 2.0 ** -10) + np.abs(y) * slack).all()


def _held_product(y, b, s, w, bias):
    """bf16 results of 8-bit rows (tests/test_gpu_linear8.py)."""
    x, ww = ref.values8(b, s), ref.values8(*ref.round8(w.astype(np.float64)))
    want = x @ ww.T + bias
    tol = (x.shape[1] + 16) * ref.EPS32 * (np.abs(x) @ np.abs(ww).T + np.abs(bias)) + ref.EPS_BF16 * np.abs(want)
    for k in range(0, x.shape[1], 128):
        tol += 128 * 2.0 ** -16 * np.abs(x[:, k:k + 128]).max(1)[:, None] * np.abs(ww[:, k:k + 128]).max(1)[None, :]
    assert (np.abs(_np(y) - want) <= tol).all()


def test_an_attention_block_over_the_encoders_states():
    import torch
    rng = np.random.default_rng(21)
    stream = torch.cuda.Stream()
    n, tokens = len(LENS), sum(LENS)
    enc = binding.Encoder(binding.make_encoder_config(max_tokens=256, max_len=128), synth.make_encoder_weights(), stream=stream)
    weight = lambda out, k: (rng.standard_normal((out, k)) / np.sqrt(k)).astype(np.float32)   # noqa: E731
    w_kv, w_q, w_o = weight(2 * KV * D, DIM), weight(HEADS * D, DIM), weight(DIM, HEADS * D)
    b_kv, b_q, b_o = (0.1 * rng.standard_normal(w.shape[0]).astype(np.float32) for w in (w_kv, w_q, w_o))
    gain = (1 + 0.1 * rng.standard_normal(DIM)).astype(np.float32)
    plain32 = binding.Norm(binding.make_norm_config(DIM, kind=binding.NORM_NONE), stream=stream)
    plain16 = binding.Norm(binding.make_norm_config(HEADS * D, x_bf16=True, kind=binding.NORM_NONE), stream=stream)
    norm = binding.Norm(binding.make_norm_config(DIM, x_bf16=True), gain, stream=stream)
    kv_proj = binding.Linear8(binding.make_linear8_config(DIM, 2 * KV * D, True), w_kv, b_kv, stream=stream)
    q_proj = binding.Linear8(binding.make_linear8_config(DIM, HEADS * D, True), w_q, b_q, stream=stream)
    o_proj = binding.Linear8(binding.make_linear8_config(HEADS * D, DIM, True), w_o, b_o, stream=stream)
    att = binding.CrossAttention(binding.make_cross_config(HEADS, KV, D, True), stream=stream)
    with torch.cuda.stream(stream):
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda:0")   # noqa: E731
        f = new(tokens, DIM, dtype=torch.float32)
        f8, fs = new(tokens, DIM, dtype=torch.float8_e4m3fn), new(tokens, 4, dtype=torch.float8_e8m0fnu)
        kv = new(tokens, 2 * KV * D)
        delta = torch.from_numpy(rng.standard_normal((n, DIM)).astype(np.float32)).to("cuda:0").bfloat16()
        h = torch.from_numpy(rng.standard_normal((n, DIM)).astype(np.float32)).to("cuda:0")
        first = (delta.clone(), h.clone())
        x8, xs, a8, a_s = new(n, DIM, dtype=torch.float8_e4m3fn), new(n, 4, dtype=torch.float8_e8m0fnu), new(n, HEADS * D, dtype=torch.float8_e4m3fn), new(n, 4, dtype=torch.float8_e8m0fnu)
        q, o = new(n, HEADS * D), new(n, HEADS, D)
    # the requests join: keys and values, side by side in a row
    enc.run_device([synth.encoder_ids(L, 7 + i) for i, L in enumerate(LENS)], f)
    plain32.run_device(f, y8=f8, scales=fs)
    kv_proj.run_device(f8, fs, kv)
    rows = kv.unflatten(1, (2 * KV, D))
    k, v = rows[:, :KV], rows[:, KV:]
    start = [int(x) for x in np.cumsum([0] + LENS)[:-1]]
    batch = att.batch([1] * n, start, LENS)

    def step():
        norm.run_device(delta, res=h, total=h, y8=x8, scales=xs)
        q_proj.run_device(x8, xs, q)
        att.run_device(batch, q.view(n, HEADS, D), k, v, o)
        plain16.run_device(o.view(n, HEADS * D), y8=a8, scales=a_s)
        o_proj.run_device(a8, a_s, delta)

    stream.synchronize()
    _held8(_bytes(f8), _bytes(fs), _np(f), 0)
    _held_product(kv, _bytes(f8), _bytes(fs), w_kv, b_kv)
    trail = []
    for _ in range(3):
        before = (_np(delta), _np(h))
        step()
        stream.synchronize()
        total, y = ref.norm(before[0], before[1], gain, np.float32(1e-5))
        assert (np.abs(_np(h) - total) <= ref.EPS32 * np.abs(total)).all()
        _held8(_bytes(x8), _bytes(xs), y, (0.5 * (DIM / 64 + 20) + 8) * ref.EPS32)
        _held_product(q, _bytes(x8), _bytes(xs), w_q, b_q)
        want, _, mass, size = ref.cross(_np(q).reshape(n, HEADS, D), _np(k), _np(v), [1] * n, start, LENS)
        off = 2 * (D + 12) * ref.EPS32 * size + (max(LENS) + 64) * ref.EPS32
        assert (np.abs(_np(o) - want) <= (off[:, :, None] + ref.EPS_BF16) * mass + ref.EPS_BF16 * np.abs(want)).all()
        _held8(_bytes(a8), _bytes(a_s), _np(o).reshape(n, -1), 0)
        _held_product(delta, _bytes(a8), _bytes(a_s), w_o, b_o)
        trail.append((delta.clone(), h.clone()))
    stream.synchronize()
    # the same steps as a graph's replays
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    with torch.cuda.stream(stream):
        delta.copy_(first[0])
        h.copy_(first[1])
    for d_want, h_want in trail:
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        assert torch.equal(delta, d_want) and torch.equal(h, h_want)
    for op in (plain32, plain16, norm, kv_proj, q_proj, o_proj, att, enc):
        op.close()


def test_two_streams_at_once():
    """Objects of two streams, their calls in flight together: each has an arena of its own."""
    import torch
    rng = np.random.default_rng(2)
    made = []
    for i in range(2):
        st = torch.cuda.Stream()
        att = binding.CrossAttention(binding.make_cross_config(2, 1, 64, True), stream=st)
        t = [torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to("cuda:0").bfloat16() for s in ((1, 2, 64), (6000, 1, 64), (6000, 1, 64))]
        made.append((st, att, t, [torch.empty_like(t[0]) for _ in range(20)], att.batch([1], [0], [6000])))
    torch.cuda.synchronize()
    for r in range(20):
        for st, att, (q, k, v), outs, batch in made:
            att.run_device(batch, q, k, v, outs[r])
    torch.cuda.synchronize()
    for st, att, (q, k, v), outs, batch in made:
        want, _, mass, size = ref.cross(_np(q), _np(k), _np(v), [1], [0], [6000])
        off = 2 * (64 + 12) * ref.EPS32 * size + (6000 + 64) * ref.EPS32
        assert (np.abs(_np(outs[0]) - want) <= (off[:, :, None] + ref.EPS_BF16) * mass + ref.EPS_BF16 * np.abs(want)).all()
        assert all(torch.equal(outs[0], x) for x in outs)
        att.close()


def test_tensors_that_do_not_fit_are_refused():
    import torch
    norm = binding.Norm(binding.make_norm_config(64), np.ones(64, np.float32))
    lin = binding.Linear8(binding.make_linear8_config(64, 32), np.ones((32, 64), np.float32))
    att = binding.CrossAttention(binding.make_cross_config(2, 1, 64))
    new = lambda *shape, dtype=torch.float32, device="cuda:0": torch.empty(shape, dtype=dtype, device=device)   # noqa: E731
    x = new(4, 64)
    for call in (lambda: norm.run_device(new(4, 64, device="cpu"), y=x), lambda: norm.run_device(x, y=new(4, 63)), lambda: norm.run_device(x, y=new(3, 64)), lambda: norm.run_device(x.bfloat16(), y=x),
                 lambda: norm.run_device(x, y=new(64, 4).t()), lambda: norm.run_device(x, y8=new(4, 64, dtype=torch.float8_e4m3fn), scales=new(4, 4, dtype=torch.float8_e8m0fnu)),
                 lambda: norm.run_device(x), lambda: norm.run_device(x, y8=new(4, 128, dtype=torch.float8_e4m3fn)), lambda: norm.run_device(x, y=x[:1].expand(4, 64)),
                 lambda: lin.run_device(new(4, 128, dtype=torch.float8_e4m3fn), new(4, 4, dtype=torch.float8_e8m0fnu), new(4, 32, dtype=torch.bfloat16)),
                 lambda: lin.run_device(new(4, 64, dtype=torch.float8_e4m3fn), new(4, 4, dtype=torch.float8_e8m0fnu), new(4, 32)),
                 lambda: att.run_device(att.batch([4], [0], [9]), new(4, 2, 64), new(8, 1, 64), new(8, 1, 64), new(4, 2, 64)),
                 lambda: att.run_device(att.batch([4], [0], [8]), new(3, 2, 64), new(8, 1, 64), new(8, 1, 64), new(4, 2, 64)),
                 lambda: att.run_device(att.batch([4], [0], [8]), new(4, 2, 64), new(8, 1, 68)[:, :, :64], new(8, 1, 64), new(4, 2, 64)),
                 lambda: att.run_device(att.batch([4], [0], [8]), new(4, 2, 64), new(8, 1, 64), new(8, 1, 64), new(4, 2, 64), keep=new(8)),
                 lambda: att.batch([1, 2], [0], [1, 2]), lambda: binding.Norm(binding.make_norm_config(64), np.ones(63, np.float32)),
                 lambda: binding.Linear8(binding.make_linear8_config(64, 32), np.ones((64, 32), np.float32)), lambda: binding.CrossAttention(binding.make_cross_config(2, 1, 136))):
        with pytest.raises((ValueError, binding.TtsError)):
            call()
    for op in (norm, lin, att):
        op.close()
