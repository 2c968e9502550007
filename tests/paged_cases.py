"""Calls of attention to a paged cache for each way that they can be taken (256 compute units), with what the plan has to say of them: the tests of the kernels run these calls, a test of the host's
code holds the plan against them."""


def _many(heads, kv, d, page, n=24, causal=True):
    """Requests of 33 rows and more, of different lengths, half of them behind a prefix, one with more queries than rows."""
    q = [170 - 11 * (i % 7) for i in range(n)]
    own = [a + (53 * i) % 300 for i, a in enumerate(q)]
    own[1] = 90
    return dict(heads=heads, kv=kv, d=d, page=page, causal=causal, q_len=q, own_len=own, prefix=[i % 2 - 1 for i in range(n)], prefix_len=[70])


def _parts(heads, kv, d, page, q, own, prefix=0, causal=True):
    """Few requests of many rows over long sequences."""
    return dict(heads=heads, kv=kv, d=d, page=page, causal=causal, q_len=q, own_len=own, prefix=[0] * len(q) if prefix else None, prefix_len=[prefix] if prefix else [])


def _steps(heads, kv, d, page, n, lens, q=lambda i: 1):
    """Steps over prefixes: requests of every prefix, some of none, some that have no rows of their own."""
    q_len = [q(i) for i in range(n)]
    own = [0 if i % 17 == 5 else 1 + (29 * i) % 150 + a for i, a in enumerate(q_len)]
    return dict(heads=heads, kv=kv, d=d, page=page, causal=True, q_len=q_len, own_len=own, prefix=[-1 if i % 31 == 7 else i % len(lens) for i in range(n)], prefix_len=lens)


MANY = {
    "many_64": _many(16, 8, 64, 16), "many_40": _many(16, 8, 40, 16), "many_8": _many(32, 32, 8, 16, n=12), "many_72": _many(16, 8, 72, 32), "many_96": _many(16, 4, 96, 32),
    "many_128": _many(16, 8, 128, 64), "many_64_all": _many(16, 8, 64, 64, causal=False), "many_40_all": _many(16, 8, 40, 32, causal=False), "many_128_all": _many(16, 8, 128, 16, causal=False),
}
PARTS = {
    "parts_128": _parts(32, 8, 128, 64, [128], [4224]), "parts_72": _parts(32, 8, 72, 16, [128], [4224]), "parts_64": _parts(16, 4, 64, 16, [300, 290], [4300, 4270], 100),
    "parts_40": _parts(32, 8, 40, 32, [300], [4300]), "parts_96": _parts(16, 4, 96, 16, [300, 290], [4300, 4270]),
    # causal, from the beginning: the first rows see nothing of the last parts
    "parts_128_own": _parts(4, 1, 128, 16, [1500], [1500]), "parts_64_own": _parts(8, 1, 64, 16, [1500], [1500]),
    # more queries than rows: the first see their prefix alone
    "parts_128_short": _parts(4, 1, 128, 16, [1000], [333], 1500), "parts_64_short": _parts(8, 2, 64, 32, [1000], [333], 1500),
    "parts_128_all": _parts(32, 8, 128, 16, [128], [4224], causal=False), "parts_64_all": _parts(16, 4, 64, 16, [300, 290], [4300, 4270], 100, causal=False),
}
PREFIX = {
    "prefix_128_of_128": _steps(32, 8, 128, 64, 64, [4000, 3993]), "prefix_128_of_64": _steps(16, 4, 64, 16, 128, [16000, 15993]), "prefix_128_of_96": _steps(8, 1, 96, 16, 128, [16000, 15993]),
    "prefix_128_of_40": _steps(16, 2, 40, 32, 128, [16000, 15993]), "prefix_128_of_96_queries": _steps(16, 4, 96, 16, 64, [4000, 3993, 3986, 3979], lambda i: 1 + i % 4),
    "prefix_64_of_128": _steps(32, 8, 128, 64, 32, [16000, 15993]), "prefix_64_of_64": _steps(32, 16, 64, 16, 128, [16000, 15993, 15986, 15979]),
    "prefix_64_of_96": _steps(16, 8, 96, 16, 128, [16000, 15993, 15986, 15979]), "prefix_64_of_40": _steps(32, 32, 40, 32, 64, [32000]),
}


def _chunks(heads, kv, d, page, n, q, lens, bf16=True):
    """Chunks of many requests, some of them half as long, most behind a prefix."""
    q_len = [q if i % 5 else q // 2 for i in range(n)]
    return dict(heads=heads, kv=kv, d=d, page=page, bf16=bf16, causal=True, q_len=q_len, own_len=[a + (53 * i) % 300 for i, a in enumerate(q_len)],
                prefix=[i % len(lens) if i % 5 != 4 else -1 for i in range(n)], prefix_len=lens)


# Requests of both kinds in one call, and of many rows that tiles of 16 take, in fp32 always: with the plan of each
CHUNKS = {
    "chunks_64": (_chunks(8, 8, 64, 16, 32, 40, [700, 1500]), dict(few=2, many=0, joins=2, pools=4, split=5, height=0)),
    "chunks_64_long": (_chunks(8, 8, 64, 64, 32, 40, [4000, 3993]), dict(few=2, many=1, joins=2, pools=4, split=4, height=128)),
    "chunks_128_long": (_chunks(16, 4, 128, 64, 32, 40, [16000, 15993]), dict(few=1, many=1, joins=1, pools=2, split=2, height=128)),
    "chunks_40_long": (_chunks(16, 8, 40, 32, 32, 40, [16000, 15993]), dict(few=1, many=1, joins=1, pools=2, split=2, height=128)),
    "chunks_40_ahead": (_chunks(16, 8, 40, 16, 32, 40, [700, 1500]), dict(few=1, many=0, joins=0, pools=0, split=0, height=0)),
    "chunks_40_fp32": (_chunks(16, 8, 40, 32, 64, 20, [4000, 3993], False), dict(few=2, many=0, joins=1, pools=2, split=2, height=0)),
    "chunks_128_fp32": (_chunks(16, 4, 128, 64, 24, 150, [500, 400], False), dict(few=1, many=0, joins=0, pools=0, split=0, height=0)),
    "chunks_128_fp32_long": (_chunks(16, 4, 128, 64, 32, 40, [16000, 15993], False), dict(few=1, many=0, joins=1, pools=0, split=26, height=0)),
    "chunks_64_fp32": (_chunks(8, 8, 64, 16, 24, 150, [4000], False), dict(few=1, many=0, joins=0, pools=0, split=0, height=0)),
}
CASES = {**MANY, **PARTS, **PREFIX, **{name: case for name, (case, _) in CHUNKS.items()}}


def plan(name):
    """Launches of few and of many rows, of what joins parts, prefixes read apart, and the height of the tiles of many rows."""
    if name in CHUNKS:
        return CHUNKS[name][1]
    if name in MANY:
        return dict(few=0, many=1, joins=0, pools=0, split=0, height=128)
    if name in PARTS:
        return dict(few=0, many=1, joins=1, pools=0, split=len(CASES[name]["q_len"]), height=128)
    n = len(CASES[name]["prefix_len"])
    return dict(few=1, many=1, joins=1, pools=n, split=n, height=int(name.split("_")[1]))
