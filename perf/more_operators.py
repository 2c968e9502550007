"""The operators of a decoder block's own past, as measurable cases: rotary positions, keys and values on their way to a paged cache (rotated), and
attention of a dynamic batch to that cache, with prefixes that requests share.

A case's state holds the inputs of one pass, the buffers that its results go to and the handle that a program keeps.  Lengths follow from the case, values and the
order of the pages from the seed.  A cache's pages are [pages, heads, rows of a page, head_dim], keys' and values' apart; a table of page numbers has a row for each
request and each prefix, and a number below zero where there is no page."""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
BASE, FACTOR, TRAINED, LOW, HIGH, MAGNITUDE = 10000.0, 8.0, 4096, 1.0, 32.0, 1.2       # MAGNITUDE: of positions scaled by parts


def listed():
    return [
        # One request's step: queries and keys of one frame take their position.
        dict(name="rotary_step_1", kind="rotary", rows=1, heads=16, head=64, rot=64, pairs=False, x="bf16", y="bf16", scaling="plain", each=True, far=2000, back=False),
        # Full precision, neighbouring columns as pairs, part of a head, positions far behind what was trained on.
        dict(name="rotary_odd", kind="rotary", rows=777, heads=12, head=96, rot=56, pairs=True, x="f32", y="f32", scaling="parts", each=True, far=500000, back=False),
        # All frames of a large batch.
        dict(name="rotary_16384", kind="rotary", rows=16384, heads=40, head=128, rot=128, pairs=False, x="bf16", y="bf16", scaling="plain", each=True, far=30000, back=False),
        # A pool's step: 64 requests, a frame each, queries on the way.
        dict(name="append_step_64", kind="append", cache="bf16", x="bf16", n=64, kv=8, heads=8, head=64, rot=64, pairs=False, scaling="plain", rows=1, rows_hi=1, past=20, past_hi=600, page=16),
        # Requests join with recordings of their own: ragged, from full precision, part of a head, pages of 32.
        dict(name="append_ragged", kind="append", cache="bf16", x="f32", n=7, kv=4, heads=0, head=96, rot=48, pairs=True, scaling="linear", rows=1, rows_hi=501, past=0, past_hi=77, page=32),
        # Long prompts of a batch.
        dict(name="append_16000", kind="append", cache="bf16", x="bf16", n=8, kv=8, heads=32, head=128, rot=128, pairs=False, scaling="base", rows=1200, rows_hi=2800, past=0, past_hi=0, page=64),
        # One request's step in full precision.
        dict(name="attend_step_1", kind="attend", type="f32", n=1, heads=8, kv=8, head=64, q=1, q_hi=1, past=299, past_hi=299, prefixes=0, prefix=0, prefix_hi=0, page=16, lse=False, gone=False, empty=False),
        # A pool's step: 64 requests of one voice, whose recording all of them attend.
        dict(name="attend_step_64", kind="attend", type="bf16", n=64, heads=8, kv=8, head=64, q=1, q_hi=1, past=20, past_hi=600, prefixes=1, prefix=2000, prefix_hi=2000, page=16, lse=False, gone=False, empty=False),
        # A large pool's step: heads that share keys, a long prefix.
        dict(name="attend_step_prefix", kind="attend", type="bf16", n=128, heads=32, kv=8, head=128, q=1, q_hi=1, past=10, past_hi=400, prefixes=1, prefix=16001, prefix_hi=16001, page=64, lse=False, gone=False, empty=False),
        # Long pasts of their own, three short prefixes, pages given back, one request with none left.
        dict(name="attend_step_long", kind="attend", type="bf16", n=16, heads=16, kv=4, head=128, q=1, q_hi=1, past=3001, past_hi=9000, prefixes=3, prefix=100, prefix_hi=300, page=64, lse=True, gone=True, empty=True),
        # A chunk of 40 frames of each of 32 requests, two voices.
        dict(name="attend_chunk", kind="attend", type="bf16", n=32, heads=8, kv=8, head=64, q=40, q_hi=40, past=0, past_hi=900, prefixes=2, prefix=700, prefix_hi=1500, page=16, lse=False, gone=False, empty=False),
        # Long prompts of a batch over a prefix that is there.
        dict(name="attend_prompts", kind="attend", type="bf16", n=8, heads=16, kv=4, head=128, q=1500, q_hi=4000, past=0, past_hi=0, prefixes=1, prefix=500, prefix_hi=500, page=64, lse=True, gone=False, empty=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _angles_of(rng, head):
    rot = rng.choice([head, head, head // 2, 2 * rng.randint(1, head // 2)])
    return dict(rot=max(4, rot // 2 * 2), pairs=rng.random() < 0.5, scaling=rng.choice(["plain", "plain", "linear", "base", "parts"]))


def draw(rng):
    kind = rng.choice(["rotary", "append", "attend", "attend"])
    if kind == "rotary":
        head, heads = rng.choice([64, 64, 128, 128, 40, 96]), rng.randint(1, 48)
        x = rng.choice(["bf16", "f32"])
        case = dict(kind=kind, rows=_log_int(rng, 1, 16384 * 40 * 128 // (2 * heads * head)), heads=heads, head=head, x=x, y=x if rng.random() < 0.7 else rng.choice(["bf16", "f32"]))
        case.update(_angles_of(rng, head), each=rng.random() < 0.7, far=_log_int(rng, 100, 1000000), back=rng.random() < 0.2)
        return case
    if kind == "append":
        kv, head = rng.choice([1, 2, 4, 8]), rng.choice([64, 64, 128, 128, 40, 96])
        cache = rng.choice(["bf16", "bf16", "f32"])
        case = dict(kind=kind, cache=cache, x=cache if rng.random() < 0.6 else "f32", kv=kv, heads=rng.choice([0, 1, 2, 4]) * kv, head=head, page=rng.choice([16, 32, 64, 128]))
        case.update(_angles_of(rng, head), n=_log_int(rng, 1, 128))
        case["rows_hi"] = 1 if rng.random() < 0.4 else _log_int(rng, 1, min(3000, 1 + 8000 // case["n"]))
        case["rows"] = rng.randint(1, case["rows_hi"])
        case["past_hi"] = _log_int(rng, 1, min(4000, 1 + 30000 // case["n"])) - 1
        case["past"] = rng.randint(0, case["past_hi"])
        return case
    bf16 = rng.random() < 0.7
    kv = rng.choice([1, 2, 4, 8])
    case = dict(kind=kind, type="bf16" if bf16 else "f32", heads=kv * rng.choice([1, 1, 2, 4]), kv=kv, head=rng.choice([64, 64, 128, 128, 40, 96]), page=rng.choice([16, 32, 64, 128]))
    step = rng.random() < 0.5
    if step:
        case["n"] = _log_int(rng, 1, 128)
        case["q"], case["q_hi"] = 1, 1
        case["past_hi"] = _log_int(rng, 1, min(20000, 1 + 100000 // case["n"])) - 1
    else:
        case["n"] = _log_int(rng, 1, 32)
        case["q_hi"] = _log_int(rng, 2, (30000 if bf16 else 8000) // case["n"] // 10)
        case["q"] = rng.randint(1, case["q_hi"])
        case["past_hi"] = _log_int(rng, 1, 1500 if bf16 else 600) - 1
    case["past"] = rng.randint(0, case["past_hi"])
    case["prefixes"] = rng.choice([0, 1, 1, 2, 5]) if case["n"] >= 5 else rng.choice([0, 1])
    case["prefix_hi"] = _log_int(rng, 16, 8000 if step else 1500) if case["prefixes"] else 0
    case["prefix"] = rng.randint(1, case["prefix_hi"]) if case["prefixes"] else 0
    case.update(lse=rng.random() < 0.4, gone=rng.random() < 0.3, empty=rng.random() < 0.2)
    return case


# ---- what follows from a case alone

def _dtype(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _bytes(name):
    return {"bf16": 2, "f32": 4}[name]


def _spread(n, lo, hi, phase):
    """n lengths from lo to hi, evenly mixed (multiples of the golden ratio); the last is the longest."""
    got = [lo + int((hi - lo + 1) * ((i + 1) * 0.6180339887498949 + phase) % (hi - lo + 1)) for i in range(n)]
    if n:
        got[-1] = hi
    return got


def _lengths(case):
    """(queries or new rows, rows of its own with them) of every request."""
    new = _spread(case["n"], case["q" if case["kind"] == "attend" else "rows"], case["q_hi" if case["kind"] == "attend" else "rows_hi"], 0.25)
    past = _spread(case["n"], case["past"], case["past_hi"], 0.5)
    return new, [a + b for a, b in zip(new, past)]


def _prefixes(case):
    """(each request's prefix or -1, each prefix's length); one request in five has none."""
    p = case["prefixes"]
    return [i % p if p and i % 5 != 4 else -1 for i in range(case["n"])], _spread(p, case["prefix"], case["prefix_hi"], 0.75)


def _no_page(case):
    """For every request the numbers of its pages that were given back, from and to: early ones of long pasts, all of one request's."""
    new, mem = _lengths(case)
    got = []
    for i in range(case["n"]):
        pages = -(-mem[i] // case["page"])
        kept = -(-new[i] // case["page"]) + 1
        got.append((1, max(1, (pages - kept) // 2)) if case["gone"] and pages - kept >= 4 and i % 2 == 0 else (0, 0))
    if case["empty"] and case["n"] > 1:
        got[case["n"] // 2] = (0, 1 << 30)
    return got


def _freqs(rot, scaling):
    """Turns of each pair of columns in radians a position, in 64 bits."""
    base = BASE * FACTOR ** (rot / (rot - 2)) if scaling == "base" else BASE
    f = [base ** (-2 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        f = [v / FACTOR for v in f]
    if scaling == "parts":
        keep = [min(1.0, max(0.0, (TRAINED * v / (2 * math.pi) - LOW) / (HIGH - LOW))) for v in f]
        f = [v * (k + (1 - k) / FACTOR) for v, k in zip(f, keep)]
    return f


def work(case):
    if case["kind"] == "rotary":
        n = case["rows"] * case["heads"] * case["head"]
        return {"bytes": n * (_bytes(case["x"]) + _bytes(case["y"])) + 4 * case["rows"] * case["each"], "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    new, mem = _lengths(case)
    if case["kind"] == "append":
        wide = 2 * case["kv"] + case["heads"]
        turned = case["kv"] + case["heads"]
        return {"bytes": sum(new) * wide * case["head"] * (_bytes(case["x"]) + _bytes(case["cache"])), "flops": 3 * sum(new) * turned * case["rot"]}
    size, page = _bytes(case["type"]), case["page"]
    of, lengths = _prefixes(case)
    rows, pairs = sum(lengths), 0
    for i, (a, b) in enumerate(_no_page(case)):
        there = [j for j in range(-(-mem[i] // page)) if not a <= j < b]
        rows += sum(min(page, mem[i] - j * page) for j in there)
        # query t sees the rows up to mem - new + t
        first = mem[i] - new[i] + 1
        for j in there:
            lo, hi = j * page, min(mem[i], (j + 1) * page)
            full = max(0, mem[i] - max(first, hi) + 1)                          # queries that see all of the page's rows
            pairs += full * (hi - lo)
            part = range(max(first, lo + 1), min(mem[i] + 1, hi))               # rows up to here are seen by one query each
            pairs += sum(r - lo for r in part)
        pairs += new[i] * (lengths[of[i]] if of[i] >= 0 else 0)
    b = size * case["head"] * (2 * case["heads"] * sum(new) + 2 * case["kv"] * rows) + 4 * case["heads"] * sum(new) * case["lse"]
    return {"bytes": b, "flops": 4 * case["heads"] * case["head"] * pairs}


# ---- a pass's inputs

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _rotary_inputs(case, g):
    x = (1.5 * torch.randn(case["rows"], case["heads"], case["head"], generator=g, device=DEVICE)).to(_dtype(case["x"]))
    if case["each"]:
        return x, torch.randint(0, case["far"] + 1, (case["rows"],), generator=g, device=DEVICE, dtype=torch.int32)
    return x, torch.arange(case["far"], case["far"] + case["rows"], dtype=torch.int32, device=DEVICE)


def _table(case, mem, g):
    """Page numbers [requests and prefixes, most pages] and how many pages there are: in any order, some of them nobody's."""
    lengths = mem + (_prefixes(case)[1] if case["kind"] == "attend" else [])
    counts = [-(-m // case["page"]) for m in lengths]
    pages = sum(counts) + 3
    order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
    c = torch.tensor(counts, device=DEVICE)
    j = torch.arange(max(1, max(counts)), device=DEVICE)
    at = ((c.cumsum(0) - c)[:, None] + j).clamp(max=pages - 1)
    there = j < c[:, None]
    if case["kind"] == "attend":
        cut = torch.tensor(_no_page(case) + [(0, 0)] * (len(lengths) - case["n"]), device=DEVICE)
        there = there & ~((j >= cut[:, :1]) & (j < cut[:, 1:]))
    return torch.where(there, order[at], -1).to(torch.int32), pages


def _append_inputs(case, g):
    new, mem = _lengths(case)
    t, n, d = _dtype(case["x"]), sum(new), case["head"]
    make = lambda heads: torch.randn(n, heads, d, generator=g, device=DEVICE).to(t)   # noqa: E731
    k, v = make(case["kv"]), make(case["kv"])
    q = make(case["heads"]) if case["heads"] else None
    table, pages = _table(case, mem, g)
    shape = (pages, case["kv"], case["page"], d)
    kp, vp = (torch.randn(shape, generator=g, device=DEVICE).to(_dtype(case["cache"])) for _ in range(2))
    return k, v, q, kp, vp, table


def _attend_inputs(case, g):
    new, mem = _lengths(case)
    t, d = _dtype(case["type"]), case["head"]
    table, pages = _table(case, mem, g)
    q = (1.5 * torch.randn(sum(new), case["heads"], d, generator=g, device=DEVICE)).to(t)
    kp, vp = (torch.randn(pages, case["kv"], case["page"], d, generator=g, device=DEVICE).to(t) for _ in range(2))
    return q, kp, vp, table


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case=case)
    at = lambda v: torch.tensor(v, device=DEVICE)                               # noqa: E731
    if case["kind"] != "attend":
        s["freqs"] = torch.tensor(_freqs(case["rot"], case["scaling"]), dtype=torch.float64, device=DEVICE)
        s["magnitude"] = MAGNITUDE if case["scaling"] == "parts" else 1.0
    if case["kind"] == "rotary":
        s["x"], s["positions"] = _rotary_inputs(case, g)
    elif case["kind"] == "append":
        s["k"], s["v"], s["q"], s["kp"], s["vp"], s["table"] = _append_inputs(case, g)
        new, mem = s["lengths"] = _lengths(case)
        # the plain form's plan: request and cache row of every new row
        n = at(new)
        s["request"] = torch.arange(case["n"], device=DEVICE).repeat_interleave(n)
        s["row"] = torch.arange(sum(new), device=DEVICE) - (n.cumsum(0) - n)[s["request"]] + at([m - a for a, m in zip(new, mem)])[s["request"]]
    else:
        s["q"], s["kp"], s["vp"], s["table"] = _attend_inputs(case, g)
        new, mem = s["lengths"] = _lengths(case)
        of, lengths = s["prefixes"] = _prefixes(case)
        # the plain form's plan: rows of a padded batch and back, a prefix's requests side by side and back
        n, m, page = at(new), at(mem), case["page"]
        i, j = torch.arange(max(new), device=DEVICE), torch.arange(max(mem), device=DEVICE)
        s["q_at"] = ((n.cumsum(0) - n)[:, None] + i).clamp(max=sum(new) - 1)
        s["q_there"] = i < n[:, None]
        s["own_page"], s["own_row"] = s["table"][:case["n"]][:, j // page].clamp(min=0).long(), j % page
        s["own_there"] = (j < m[:, None]) & (s["table"][:case["n"]][:, j // page] >= 0)
        s["seen"] = j <= (m - n)[:, None, None] + i[:, None]                    # [requests, queries, rows]
        if lengths:
            j = torch.arange(max(lengths), device=DEVICE)
            s["pre_page"], s["pre_row"] = s["table"][case["n"]:][:, j // page].clamp(min=0).long(), j % page
            s["pre_there"] = j < at(lengths)[:, None]
            slot = [of[:r].count(of[r]) for r in range(case["n"])]
            most = 1 + max(x for x, o in zip(slot, of) if o >= 0)
            members = [[0] * most for _ in lengths]
            for r in range(case["n"]):
                if of[r] >= 0:
                    members[of[r]][slot[r]] = r
            s["members"], s["of"], s["slot"], s["has"] = at(members), at([max(0, o) for o in of]), at([x if o >= 0 else 0 for x, o in zip(slot, of)]), at([o >= 0 for o in of])
    if own:
        _own_prepare(s)
    return s


# ---- the framework's calls

def _own_angles(binding, case):
    kinds = dict(plain=binding.ROTARY_PLAIN, linear=binding.ROTARY_LINEAR, base=binding.ROTARY_BASE, parts=binding.ROTARY_PARTS)
    return binding.make_rotary_angles(case["rot"], pairs=case["pairs"], base=BASE, scaling=kinds[case["scaling"]], factor=FACTOR, trained_len=TRAINED, low=LOW, high=HIGH,
                                      magnitude=MAGNITUDE if case["scaling"] == "parts" else 1.0)


def _own_prepare(s):
    """The handle of a case, its batch's lengths, and the buffers that a program has its results in."""
    from paper_2211_13939_amd import binding
    case, here = s["case"], torch.cuda.current_stream()
    if case["kind"] == "rotary":
        cfg = binding.make_rotary_config(case["heads"], case["head"], _own_angles(binding, case), x_bf16=case["x"] == "bf16", y_bf16=case["y"] == "bf16")
        s["op"] = binding.Rotary(cfg, stream=here)
        s["y"] = torch.empty_like(s["x"], dtype=_dtype(case["y"]))
    elif case["kind"] == "append":
        cfg = binding.make_cache_config(case["kv"], case["head"], case["page"], _own_angles(binding, case), n_heads=case["heads"], bf16=case["cache"] == "bf16", x_bf16=case["x"] == "bf16")
        s["op"] = binding.Cache(cfg, stream=here)
        new, mem = s["lengths"]
        s["batch"] = s["op"].batch(new, [m - n for n, m in zip(new, mem)], list(range(case["n"])))
        s["q_out"] = torch.empty_like(s["q"], dtype=_dtype(case["cache"])) if case["heads"] else None
    else:
        cfg = binding.make_paged_config(case["heads"], case["kv"], case["head"], case["page"], bf16=case["type"] == "bf16")
        s["op"] = binding.PagedAttention(cfg, stream=here)
        new, mem = s["lengths"]
        of, lengths = s["prefixes"]
        s["batch"] = s["op"].batch(new, mem, list(range(case["n"])), prefix=of, prefix_len=lengths, prefix_table_row=[case["n"] + p for p in range(len(lengths))])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEVICE) if case["lse"] else None


def _own_run(s):
    case = s["case"]
    if case["kind"] == "rotary":
        if case["each"]:
            s["op"].run_device(s["x"], s["y"], positions=s["positions"], back=case["back"])
        else:
            s["op"].run_device(s["x"], s["y"], first=case["far"], back=case["back"])
        return s["y"]
    if case["kind"] == "append":
        s["op"].run_device(s["batch"], s["k"], s["v"], s["kp"], s["vp"], s["table"], q=s["q"], q_out=s["q_out"])
        return {"k": s["kp"], "v": s["vp"], "q": s["q_out"]} if case["heads"] else {"k": s["kp"], "v": s["vp"]}
    s["op"].run_device(s["batch"], s["q"], s["kp"], s["vp"], s["table"], s["out"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]} if case["lse"] else {"out": s["out"]}


# ---- the plain forms

def _plain_turn(x, positions, s, back=False):
    """Rows of heads at their positions, in 32 bits; the angles in 64."""
    case, half = s["case"], s["case"]["rot"] // 2
    a = positions.double()[:, None] * s["freqs"]
    c, n = (a.cos() * s["magnitude"]).float()[:, None], (a.sin() * (-s["magnitude"] if back else s["magnitude"])).float()[:, None]
    x = x.float()
    turned = x[..., :2 * half]
    u, w = (turned[..., 0::2], turned[..., 1::2]) if case["pairs"] else (turned[..., :half], turned[..., half:])
    p, r = u * c - w * n, w * c + u * n
    return torch.cat([torch.stack([p, r], 3).flatten(2) if case["pairs"] else torch.cat([p, r], 2), x[..., 2 * half:]], 2)


def _plain_append(s):
    case = s["case"]
    to = _dtype(case["cache"])
    page, row = s["table"][s["request"], s["row"] // case["page"]].long(), s["row"] % case["page"]
    s["kp"][page, :, row] = _plain_turn(s["k"], s["row"], s).to(to)
    s["vp"][page, :, row] = s["v"].to(to)
    got = {"k": s["kp"], "v": s["vp"]}
    if case["heads"]:
        got["q"] = _plain_turn(s["q"], s["row"], s).to(to)
    return got


def _plain_attend(s):
    case = s["case"]
    n, d, kv, group = case["n"], case["head"], case["kv"], case["heads"] // case["kv"]
    most = s["q_at"].shape[1]
    q = s["q"].float()[s["q_at"]].view(n, most, kv, group, d).permute(0, 2, 1, 3, 4).reshape(n, kv, most * group, d) * (1 / math.sqrt(d))
    k = s["kp"][s["own_page"], :, s["own_row"]].float().permute(0, 2, 3, 1).contiguous()                  # [n, kv, d, rows]
    v = torch.where(s["own_there"][:, :, None, None], s["vp"][s["own_page"], :, s["own_row"]].float(), 0).permute(0, 2, 1, 3).contiguous()
    hidden = ~(s["own_there"][:, None] & s["seen"]).repeat_interleave(group, 1)
    score = (q @ k).masked_fill_(hidden[:, None], -math.inf)
    rows = score.shape[3]
    if case["prefixes"]:
        # a prefix's requests as rows of one product
        p, slots = s["members"].shape
        side = lambda x: x[s["members"]].permute(0, 2, 1, 3, 4).reshape(p, kv, slots * most * group, -1)   # noqa: E731
        back = lambda x: x.view(p, kv, slots, most * group, -1)[s["of"], :, s["slot"]]                      # noqa: E731
        k = s["kp"][s["pre_page"], :, s["pre_row"]].float().permute(0, 2, 3, 1).contiguous()
        v_pre = torch.where(s["pre_there"][:, :, None, None], s["vp"][s["pre_page"], :, s["pre_row"]].float(), 0).permute(0, 2, 1, 3).contiguous()
        hidden = ~(s["pre_there"][s["of"]] & s["has"][:, None])
        score = torch.cat([score, back(side(q) @ k).masked_fill_(hidden[:, None, None], -math.inf)], 3)
    top = score.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    e = score.sub_(top).exp_()
    total = e.sum(3, keepdim=True)
    out = e[..., :rows].contiguous() @ v
    if case["prefixes"]:
        out += torch.where(s["has"][:, None, None, None], back(side(e[..., rows:]) @ v_pre), 0)
    out /= torch.where(total == 0, 1, total)
    rows_of = lambda a: a.view(n, kv, most, group, -1).permute(0, 2, 1, 3, 4)[s["q_there"]].flatten(1, 2)   # noqa: E731
    got = {"out": rows_of(out).to(_dtype(case["type"]))}
    if case["lse"]:
        got["lse"] = rows_of(top + total.log()).squeeze(2)
    return got


def run(state):
    if own:
        return _own_run(state)
    if state["case"]["kind"] == "rotary":
        return _plain_turn(state["x"], state["positions"], state, state["case"]["back"]).to(_dtype(state["case"]["y"]))
    return _plain_append(state) if state["case"]["kind"] == "append" else _plain_attend(state)


# ---- the definitions in 64 bits

def _exact_turn(case, x, positions, back=False):
    """Pairs of columns as complex numbers."""
    half = case["rot"] // 2
    a = positions.double()[:, None] * torch.tensor(_freqs(case["rot"], case["scaling"]), dtype=torch.float64, device=DEVICE)
    y = x.double().clone()
    at = torch.arange(half, device=DEVICE)
    first, second = (2 * at, 2 * at + 1) if case["pairs"] else (at, at + half)
    size = torch.full_like(a, MAGNITUDE if case["scaling"] == "parts" else 1.0)
    z = torch.complex(y[:, :, first], y[:, :, second]) * torch.polar(size, -a if back else a)[:, None]
    y[:, :, first], y[:, :, second] = z.real, z.imag
    return y


def exact(case, seed):
    g = _generator(seed)
    if case["kind"] == "rotary":
        return _exact_turn(case, *_rotary_inputs(case, g), back=case["back"])
    new, mem = _lengths(case)
    if case["kind"] == "append":
        k, v, q, kp, vp, table = _append_inputs(case, g)
        got = {"k": kp.double(), "v": vp.double()}
        positions, at = torch.cat([torch.arange(m - n, m, device=DEVICE) for n, m in zip(new, mem)]), 0
        k = _exact_turn(case, k, positions)
        for i, (n, m) in enumerate(zip(new, mem)):
            rows = torch.arange(m - n, m, device=DEVICE)
            pages = table[i].long()[rows // case["page"]]
            got["k"][pages, :, rows % case["page"]] = k[at: at + n]
            got["v"][pages, :, rows % case["page"]] = v[at: at + n].double()
            at += n
        if q is not None:
            got["q"] = _exact_turn(case, q, positions)
        return got
    q, kp, vp, table = _attend_inputs(case, g)
    of, lengths = _prefixes(case)
    group, page = case["heads"] // case["kv"], case["page"]

    def rows_of(table_row, length):
        """(page, row in it, number) of the rows that there are."""
        j = torch.arange(length, device=DEVICE)
        pages = table[table_row].long()[j // page]
        j = j[pages >= 0]
        return table[table_row].long()[j // page], j % page, j

    outs, lses, at = [], [], 0
    for i, (n, m) in enumerate(zip(new, mem)):
        qi = q[at: at + n].double()
        at += n
        pages, row, j = rows_of(i, m)
        seen = j <= m - n + torch.arange(n, device=DEVICE)[:, None]
        if of[i] >= 0:
            more_pages, more_row, more = rows_of(case["n"] + of[i], lengths[of[i]])
            pages, row, seen = torch.cat([more_pages, pages]), torch.cat([more_row, row]), torch.cat([torch.ones(n, len(more), dtype=torch.bool, device=DEVICE), seen], 1)
        o, l = [], []
        for h in range(case["heads"]):
            sc = (qi[:, h] @ kp[pages, h // group, row].double().T / math.sqrt(case["head"])).masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(sc, 1) if sc.shape[1] else torch.full((n,), -math.inf, dtype=torch.float64, device=DEVICE)
            w = torch.exp(sc - torch.where(lse == -math.inf, 0, lse)[:, None])
            o.append(w @ vp[pages, h // group, row].double())
            l.append(lse)
        outs.append(torch.stack(o, 1))
        lses.append(torch.stack(l, 1))
    got = {"out": torch.cat(outs)}
    if case["lse"]:
        got["lse"] = torch.cat(lses)
    return got
