"""The operators of an attention block over the encoder's states, as measurable cases: the root-mean-square norm with the
residual's addition and 8-bit outputs, the 8-bit product with a scale for each block of 128, and cross attention to memories of
another length than the queries'.

A case's state holds the inputs of one pass, the buffers that its results go to and the handle that a program keeps.  Lengths
follow from the case, values from the seed.  8-bit values are e4m3 with a power of two (e8m0) for each 128 of a row; they come back as
the tensors of those two types."""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
BLOCK = 128                # columns under one scale
SCALE_PAD = 4              # a row's scales come in whole words


def listed():
    return [
        # One request's step: what the block's product before it gave joins the residual stream; the next product's 8-bit rows.
        dict(name="norm_step_1", kind="norm", rows=1, dim=512, x="bf16", res="f32", total=True, y="", y8=True),
        # A call in full precision, a width that is no multiple of anything, norm alone.
        dict(name="norm_300_odd", kind="norm", rows=300, dim=1001, x="f32", res="", total=False, y="f32", y8=False),
        # Many frames at once, a wide stream in two bytes.
        dict(name="norm_16384", kind="norm", rows=16384, dim=4096, x="bf16", res="bf16", total=True, y="", y8=True),
        # One request's step through a projection: the weights are what there is to read.
        dict(name="product_step_1", kind="product", rows=1, dim=1024, out=4096, y="bf16", bias=True),
        # A full pool's step (64 requests).
        dict(name="product_step_64", kind="product", rows=64, dim=2048, out=2048, y="bf16", bias=True),
        # Ragged in all three directions, results in full precision.
        dict(name="product_odd", kind="product", rows=777, dim=1000, out=1111, y="f32", bias=True),
        # All frames of a large batch.
        dict(name="product_16384", kind="product", rows=16384, dim=4096, out=4096, y="bf16", bias=False),
        # One request's step in full precision: one query a head, a short text.
        dict(name="cross_step_1", kind="cross", type="f32", n=1, heads=8, kv=8, head=64, q=1, q_hi=1, mem=120, mem_hi=120, slots=False, mask=False, lse=False, empty=False),
        # A pool's step: 64 requests of 20 to 250 tokens in slots of 400, positions hidden here and there, one request with none left.
        dict(name="cross_step_64", kind="cross", type="bf16", n=64, heads=8, kv=8, head=64, q=1, q_hi=1, mem=20, mem_hi=250, slots=True, mask=True, lse=False, empty=True),
        # Four requests over long memories, four query heads to a key head.
        dict(name="cross_step_long", kind="cross", type="bf16", n=4, heads=32, kv=8, head=128, q=1, q_hi=1, mem=24001, mem_hi=30000, slots=False, mask=False, lse=True, empty=False),
        # Sixteen requests' frames at once over their texts.
        dict(name="cross_frames_16", kind="cross", type="bf16", n=16, heads=8, kv=8, head=64, q=200, q_hi=1000, mem=20, mem_hi=250, slots=False, mask=True, lse=False, empty=False),
        # Long frames over long memories, heads that share keys.
        dict(name="cross_frames_long", kind="cross", type="bf16", n=8, heads=16, kv=4, head=128, q=2000, q_hi=4000, mem=2000, mem_hi=4000, slots=False, mask=False, lse=True, empty=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["norm", "product", "cross"])
    if kind == "norm":
        dim = _log_int(rng, 100, 8192)
        if rng.random() < 0.6:
            dim = max(128, dim // 64 * 64)
        y8 = rng.random() < 0.6
        return dict(kind=kind, rows=_log_int(rng, 1, max(2, min(16384, 16384 * 4096 // dim))), dim=dim, x=rng.choice(["bf16", "f32"]),
                    res=rng.choice(["", "bf16", "f32"]), total=rng.random() < 0.6, y=rng.choice(["bf16", "f32"]) if not y8 or rng.random() < 0.3 else "", y8=y8)
    if kind == "product":
        dim, out = _log_int(rng, 100, 4096), _log_int(rng, 64, 4096)
        if rng.random() < 0.6:
            dim, out = max(128, dim // 64 * 64), max(64, out // 64 * 64)
        return dict(kind=kind, rows=_log_int(rng, 1, 16384), dim=dim, out=out, y=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.5)
    bf16 = rng.random() < 0.7
    kv = rng.choice([1, 2, 4, 8])
    case = dict(kind=kind, type="bf16" if bf16 else "f32", heads=kv * rng.choice([1, 1, 2, 4]), kv=kv, head=rng.choice([64, 64, 128, 128, 40, 96]))
    if rng.random() < 0.5:          # a step
        case["n"] = _log_int(rng, 1, 128)
        case["q"], case["q_hi"] = 1, 1
        case["mem_hi"] = _log_int(rng, 1, min(30000, 1 + 200000 // case["n"]))
    else:
        case["n"] = _log_int(rng, 1, 24)
        case["q_hi"] = _log_int(rng, 2, 2000 if bf16 else 800)
        case["q"] = rng.randint(1, case["q_hi"])
        case["mem_hi"] = _log_int(rng, 1, 2000 if bf16 else 600)
    case["mem"] = rng.randint(1, case["mem_hi"])
    case.update(slots=rng.random() < 0.5, mask=rng.random() < 0.4, lse=rng.random() < 0.4, empty=rng.random() < 0.3)
    return case


# ---- what follows from a case alone

def _dtype(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _bytes(name):
    return {"bf16": 2, "f32": 4, "": 0}[name]


def _up(x, m):
    return -(-x // m) * m


def _spread(n, lo, hi, phase):
    """n lengths from lo to hi, evenly mixed (multiples of the golden ratio); the last is the longest."""
    got = [lo + int((hi - lo + 1) * ((i + 1) * 0.6180339887498949 + phase) % (hi - lo + 1)) for i in range(n)]
    got[-1] = hi
    return got


def _lengths(case):
    """(queries, first memory row, memory length) of every request, and the rows of the memory."""
    n = case["n"]
    q, mem = _spread(n, case["q"], case["q_hi"], 0.25), _spread(n, case["mem"], case["mem_hi"], 0.5)
    if case["empty"] and n > 1:
        mem[0] = 0
    room = [_up(case["mem_hi"], 8) if case["slots"] else m for m in mem]
    first = [0] * n
    for i in range(1, n):
        first[i] = first[i - 1] + room[i - 1]
    return q, first, mem, first[-1] + room[-1]


def work(case):
    if case["kind"] == "norm":
        r, d = case["rows"], case["dim"]
        b = r * d * (_bytes(case["x"]) + _bytes(case["res"]) + (_bytes(case["res"] or case["x"]) if case["total"] else 0) + _bytes(case["y"]))
        b += r * (_up(d, BLOCK) + _up(d, BLOCK) // BLOCK) if case["y8"] else 0
        return {"bytes": b + 4 * d, "flops": 6 * r * d}
    if case["kind"] == "product":
        r, k, n = case["rows"], case["dim"], case["out"]
        return {"bytes": (r + n) * (k + k / BLOCK) + r * n * _bytes(case["y"]) + (4 * n if case["bias"] else 0), "flops": 2 * r * k * n}
    q, _, mem, _ = _lengths(case)
    size = _bytes(case["type"])
    b = size * case["head"] * (2 * case["heads"] * sum(q) + 2 * case["kv"] * sum(mem))
    b += sum(mem) * case["mask"] + 4 * case["heads"] * sum(q) * case["lse"]
    return {"bytes": b, "flops": 4 * case["heads"] * case["head"] * sum(a * m for a, m in zip(q, mem))}


# ---- a pass's inputs

def _rounded(v):
    """fp32 [rows, any width] -> (e4m3 [rows, width in whole blocks], e8m0 [rows, blocks in whole words]): each block's scale is the least power
    of two that brings its largest magnitude to 448 at most, 1 where all are zero."""
    rows, dim = v.shape
    v = torch.nn.functional.pad(v, (0, _up(dim, BLOCK) - dim)).view(rows, -1, BLOCK)
    m, e = torch.frexp(v.abs().amax(2))
    k = torch.where(m == 0, 0, torch.where(m <= 0.875, e - 9, e - 8)).clamp(min=-127)
    v8 = torch.ldexp(v, -k[:, :, None]).to(torch.float8_e4m3fn).view(rows, -1)
    words = torch.nn.functional.pad(k + 127, (0, _up(k.shape[1], SCALE_PAD) - k.shape[1]), value=127)
    return v8, words.to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(v8, scales):
    """What 8-bit rows and their scales stand for, in fp32."""
    rows, width = v8.shape
    s = scales.float()[:, : width // BLOCK]
    return (v8.float().view(rows, -1, BLOCK) * s[:, :, None]).view(rows, width)


def _norm_inputs(case, g):
    r, d = case["rows"], case["dim"]
    loud = 1 + 15 * (torch.rand(d, generator=g, device=DEVICE) < 0.01)          # a few channels of a stream are loud
    x = (torch.randn(r, d, generator=g, device=DEVICE) * loud).to(_dtype(case["x"]))
    res = (3 * torch.randn(r, d, generator=g, device=DEVICE) * loud).to(_dtype(case["res"])) if case["res"] else None
    gain = 1 + 0.2 * torch.randn(d, generator=g, device=DEVICE)
    return x, res, gain


def _product_inputs(case, g):
    r, k, n = case["rows"], case["dim"], case["out"]
    x8, sx = _rounded(torch.randn(r, k, generator=g, device=DEVICE) * torch.exp(torch.randn(r, 1, generator=g, device=DEVICE)))
    w = torch.randn(n, k, generator=g, device=DEVICE) / math.sqrt(k)
    bias = torch.randn(n, generator=g, device=DEVICE) if case["bias"] else None
    return x8, sx, w, bias


def _cross_inputs(case, g):
    q_len, first, mem, rows = _lengths(case)
    t, d = _dtype(case["type"]), case["head"]
    q = (1.5 * torch.randn(sum(q_len), case["heads"], d, generator=g, device=DEVICE)).to(t)
    k = torch.randn(rows, case["kv"], d, generator=g, device=DEVICE).to(t)
    v = torch.randn(rows, case["kv"], d, generator=g, device=DEVICE).to(t)
    keep = None
    if case["mask"]:
        keep = (torch.rand(rows, generator=g, device=DEVICE) >= 0.1).to(torch.uint8)
        if case["empty"]:                                                       # one request's positions are hidden, all of them
            i = case["n"] // 2
            keep[first[i]: first[i] + mem[i]] = 0
    return q, k, v, keep


EPS = 1e-5


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    s = dict(case=case)
    if case["kind"] == "norm":
        s["x"], s["res"], s["gain"] = _norm_inputs(case, g)
    elif case["kind"] == "product":
        s["x8"], s["sx"], s["w"], s["bias"] = _product_inputs(case, g)
        s["w8"], s["sw"] = _rounded(s["w"])                                     # a program rounds its weights once
    else:
        s["q"], s["k"], s["v"], s["keep"] = _cross_inputs(case, g)
        q_len, first, mem, rows = _lengths(case)
        s["lengths"] = (q_len, first, mem)
        # the plain form's plan: rows of a padded batch and back
        at = lambda v: torch.tensor(v, device=DEVICE)                           # noqa: E731
        ql, f, m = at(q_len), at(first), at(mem)
        j = torch.arange(max(1, max(mem)), device=DEVICE)
        i = torch.arange(max(q_len), device=DEVICE)
        q0 = ql.cumsum(0) - ql
        s["there"] = j < m[:, None]
        s["mem_at"] = (f[:, None] + j).clamp(max=rows - 1)
        s["q_at"] = (q0[:, None] + i).clamp(max=sum(q_len) - 1)
        s["q_there"] = i < ql[:, None]
    if own:
        _own_prepare(s)
    return s


# ---- the framework's calls

def _own_prepare(s):
    """The handle of a case, and the buffers that a program has its results in."""
    from paper_2211_13939_amd import binding
    case, here = s["case"], torch.cuda.current_stream()
    new = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device=DEVICE)   # noqa: E731
    if case["kind"] == "norm":
        r, d = case["rows"], case["dim"]
        cfg = binding.make_norm_config(d, x_bf16=case["x"] == "bf16", res_bf16=(case["res"] or case["x"]) == "bf16", y_bf16=case["y"] == "bf16", eps=EPS)
        s["op"] = binding.Norm(cfg, s["gain"].cpu().numpy(), stream=here)
        s["total"] = new(r, d, dtype=_dtype(case["res"] or case["x"])) if case["total"] else None
        s["y"] = new(r, d, dtype=_dtype(case["y"])) if case["y"] else None
        s["y8"] = new(r, binding.width8(d), dtype=torch.float8_e4m3fn) if case["y8"] else None
        s["sy"] = new(r, binding.scale_columns(d), dtype=torch.float8_e8m0fnu) if case["y8"] else None
    elif case["kind"] == "product":
        cfg = binding.make_linear8_config(case["dim"], case["out"], bf16=case["y"] == "bf16")
        bias = s["bias"].cpu().numpy() if case["bias"] else None
        s["op"] = binding.Linear8(cfg, s["w"].cpu().numpy(), bias, stream=here)
        s["y"] = new(case["rows"], case["out"], dtype=_dtype(case["y"]))
    else:
        cfg = binding.make_cross_config(case["heads"], case["kv"], case["head"], bf16=case["type"] == "bf16")
        s["op"] = binding.CrossAttention(cfg, stream=here)
        s["batch"] = s["op"].batch(*s["lengths"])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = new(s["q"].shape[0], case["heads"], dtype=torch.float32) if case["lse"] else None


def _own_run(s):
    kind = s["case"]["kind"]
    if kind == "norm":
        s["op"].run_device(s["x"], res=s["res"], total=s["total"], y=s["y"], y8=s["y8"], scales=s["sy"])
        return {k: s[k] for k in ("total", "y", "y8", "sy") if s[k] is not None}
    if kind == "product":
        s["op"].run_device(s["x8"], s["sx"], s["y"])
        return s["y"]
    s["op"].run_device(s["batch"], s["q"], s["k"], s["v"], s["out"], keep=s["keep"], lse=s["lse"])
    return (s["out"], s["lse"]) if s["lse"] is not None else s["out"]


# ---- the plain forms

def _plain_norm(s):
    case = s["case"]
    t = s["x"].float() if s["res"] is None else s["x"].float() + s["res"].float()
    y = t * torch.rsqrt((t * t).mean(1, keepdim=True) + EPS) * s["gain"]
    got = {}
    if case["total"]:
        got["total"] = t.to(_dtype(case["res"] or case["x"]))
    if case["y"]:
        got["y"] = y.to(_dtype(case["y"]))
    if case["y8"]:
        got["y8"], got["sy"] = _rounded(y)
    return got


def _plain_product(s):
    y = _values(s["x8"], s["sx"]) @ _values(s["w8"], s["sw"]).t()
    return (y if s["bias"] is None else y + s["bias"]).to(_dtype(s["case"]["y"]))


def _plain_cross(s):
    case = s["case"]
    n, d, kv, group = case["n"], case["head"], case["kv"], case["heads"] // case["kv"]
    there = s["there"] if s["keep"] is None else s["there"] & (s["keep"][s["mem_at"]] != 0)
    q = s["q"].float()[s["q_at"]]                                               # [n, queries, heads, d]
    most = q.shape[1]
    q = q.view(n, most, kv, group, d).permute(0, 2, 1, 3, 4).reshape(n, kv, most * group, d)
    k = s["k"].float()[s["mem_at"]].permute(0, 2, 3, 1).contiguous()            # [n, kv, d, memory]
    v = torch.where(there[:, :, None, None], s["v"].float()[s["mem_at"]], 0).permute(0, 2, 1, 3).contiguous()
    score = (q @ k).mul_(1 / math.sqrt(d)).masked_fill_(~there[:, None, None, :], -math.inf)
    top = score.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    e = score.sub_(top).exp_()
    total = e.sum(3, keepdim=True)
    out = (e @ v) / torch.where(total == 0, 1, total)
    back = lambda a: a.view(n, kv, most, group, -1).permute(0, 2, 1, 3, 4)[s["q_there"]].flatten(1, 2)   # noqa: E731
    got = back(out).to(_dtype(case["type"]))
    return (got, back(top + total.log()).squeeze(2)) if case["lse"] else got


def run(state):
    if own:
        return _own_run(state)
    return {"norm": _plain_norm, "product": _plain_product, "cross": _plain_cross}[state["case"]["kind"]](state)


# ---- the definitions in 64 bits

def _exact_rounded(v):
    """As values of e4m3 and powers of two, all in 64 bits."""
    rows, dim = v.shape
    width = _up(dim, BLOCK)
    b = torch.zeros(rows, width, dtype=torch.float64, device=v.device)
    b[:, :dim] = v
    b = b.view(rows, -1, BLOCK)
    top = b.abs().max(2).values
    scale = torch.exp2(torch.ceil(torch.log2(top / 448)))
    scale[top == 0] = 1
    a = b / scale[:, :, None]
    step = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)   # e4m3: three bits behind the first, exponents from -6
    words = torch.ones(rows, _up(scale.shape[1], SCALE_PAD), dtype=torch.float64, device=v.device)
    words[:, : scale.shape[1]] = scale
    return ((a / step).round() * step).view(rows, width), words


def exact(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    if case["kind"] == "norm":
        x, res, gain = _norm_inputs(case, g)
        t = x.double() + (0 if res is None else res.double())
        y = gain.double() * t / torch.sqrt(t.pow(2).sum(1, keepdim=True) / case["dim"] + EPS)
        got = {}
        if case["total"]:
            got["total"] = t
        if case["y"]:
            got["y"] = y
        if case["y8"]:
            got["y8"], got["sy"] = _exact_rounded(y)
        return got
    if case["kind"] == "product":
        x8, sx, w, bias = _product_inputs(case, g)
        w8, sw = _exact_rounded(w.double())
        spread = lambda s, width: s.double()[:, : width // BLOCK].repeat_interleave(BLOCK, 1)   # noqa: E731
        y = (x8.double() * spread(sx, x8.shape[1])) @ (w8 * spread(sw, w8.shape[1])).T
        return y if bias is None else y + bias.double()
    q, k, v, keep = _cross_inputs(case, g)
    q_len, first, mem, _ = _lengths(case)
    group = case["heads"] // case["kv"]
    outs, lses, at = [], [], 0
    for n, f, m in zip(q_len, first, mem):
        rows = torch.arange(f, f + m, device=DEVICE)
        if keep is not None:
            rows = rows[keep[f: f + m] != 0]
        qi = q[at: at + n].double().transpose(0, 1)                             # [heads, queries, d]
        at += n
        if not len(rows):
            outs.append(torch.zeros(n, case["heads"], case["head"], dtype=torch.float64, device=DEVICE))
            lses.append(torch.full((n, case["heads"]), -math.inf, dtype=torch.float64, device=DEVICE))
            continue
        o, l = [], []
        for h in range(case["heads"]):
            sc = qi[h] @ k[rows, h // group].double().T / math.sqrt(case["head"])
            l.append(torch.logsumexp(sc, 1))
            o.append(torch.softmax(sc, 1) @ v[rows, h // group].double())
        outs.append(torch.stack(o, 1))
        lses.append(torch.stack(l, 1))
    out = torch.cat(outs)
    return (out, torch.cat(lses)) if case["lse"] else out
