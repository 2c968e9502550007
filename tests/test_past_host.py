"""The host code of a decoder block's own past (tts_rotary, tts_cache, tts_paged) without a GPU: what the headers declare is exported, what they do not allow is refused before anything is
launched, failing HIP calls come back as errors, frequencies hold what the definition says."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import past_ref as ref
from tests.test_operators_host import HIP, INVAL, ROOT, UNSUPPORTED, Made

OPS = ("rotary", "cache", "paged")


def test_library_exports_every_declared_operator():
    names = set()
    for op in OPS:
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", f"tts_{op}.h")).read(), flags=re.S)
        names |= set(re.findall(rf"\b(tts_{op}_(?!angles|config|rows|batch|tensors)\w+)\s*\(", text))
    assert names == set(binding.PAST_EXPORTS)
    for n in names:
        assert hasattr(binding.lib(), n), n


def _angles(**change):
    a = binding.make_rotary_angles(64)
    for k, v in change.items():
        setattr(a, k, v)
    return a


BAD_ANGLES = (dict(rot_dim=1), dict(rot_dim=66), dict(rot_dim=7), dict(rot_dim=-2), dict(layout=2), dict(layout=-1), dict(scaling=4), dict(scaling=-1), dict(base=0.5), dict(base=float("nan")),
              dict(base=2.0 ** 61), dict(magnitude=0.0), dict(magnitude=-1.0), dict(magnitude=float("inf")), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")), dict(scaling=2, rot_dim=2),
              dict(scaling=2, factor=2.0 ** 31), dict(scaling=3, trained_len=0), dict(scaling=3, trained_len=9, low=2.0, high=2.0), dict(scaling=3, trained_len=9, low=-1.0),
              dict(scaling=3, trained_len=9, high=float("nan")))


def test_configurations_without_gpu():
    L = binding.lib()
    assert L.tts_rotary_workspace_bytes(C.byref(binding.make_rotary_config(4, 64, _angles()))) >= 32 * 8
    assert L.tts_cache_workspace_bytes(C.byref(binding.make_cache_config(4, 64, 16, _angles()))) >= 32 * 8
    assert L.tts_cache_workspace_bytes(C.byref(binding.make_cache_config(4, 64, 16))) > 0
    for change in (dict(n_heads=0), dict(n_heads=1025), dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(x_dtype=2), dict(y_dtype=-1)):
        c = binding.make_rotary_config(4, 64, _angles())
        for k, v in change.items():
            setattr(c, k, v)
        assert L.tts_rotary_workspace_bytes(C.byref(c)) == 0 and L.tts_last_error(), change
    for change in BAD_ANGLES:
        assert L.tts_rotary_workspace_bytes(C.byref(binding.make_rotary_config(4, 64, _angles(**change)))) == 0, change
        assert L.tts_cache_workspace_bytes(C.byref(binding.make_cache_config(4, 64, 16, _angles(**change)))) == 0, change
    assert L.tts_rotary_workspace_bytes(C.byref(binding.make_rotary_config(4, 64, _angles(rot_dim=0)))) == 0
    for change in (dict(n_kv_heads=0), dict(n_kv_heads=257), dict(n_heads=-1), dict(n_heads=257), dict(head_dim=0), dict(head_dim=20), dict(head_dim=136), dict(page_rows=8), dict(page_rows=0),
                   dict(page_rows=48), dict(page_rows=2048), dict(x_dtype=2), dict(dtype=2)):
        c = binding.make_cache_config(4, 64, 16, _angles())
        for k, v in change.items():
            setattr(c, k, v)
        assert L.tts_cache_workspace_bytes(C.byref(c)) == 0 and L.tts_last_error(), change
    assert L.tts_paged_workspace_bytes(C.byref(binding.make_paged_config(8, 2, 64, 16))) > 0
    for change in (dict(n_heads=0), dict(n_heads=257), dict(n_kv_heads=0), dict(n_kv_heads=3), dict(n_kv_heads=16), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136), dict(page_rows=8),
                   dict(page_rows=24), dict(page_rows=2048), dict(dtype=2), dict(causal=2)):
        c = binding.make_paged_config(8, 2, 64, 16)
        for k, v in change.items():
            setattr(c, k, v)
        assert L.tts_paged_workspace_bytes(C.byref(c)) == 0 and L.tts_last_error(), change
    for op in OPS:
        assert getattr(L, f"tts_{op}_workspace_bytes")(None) == 0


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libpast.so")
    csrc = os.path.join(ROOT, "paper_2211_13939_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-Wno-unused-result",
                    os.path.join(ROOT, "tests", "fake_past.cpp")] + [os.path.join(csrc, f"{op}.cpp") for op in OPS] + ["-o", out], check=True)
    L = C.CDLL(out)
    L.tts_last_error.restype = C.c_char_p
    L.past_append_k.restype = L.past_rows.restype = C.c_longlong
    L.past_wrong.restype = C.c_char_p
    for op in OPS:
        getattr(L, f"tts_{op}_workspace_bytes").restype = C.c_size_t
        f = getattr(L, f"tts_{op}_destroy")
        f.restype, f.argtypes = None, [C.c_void_p]
    return L


@pytest.mark.parametrize("angles", [dict(), dict(scaling=1, factor=8.0), dict(scaling=2, factor=4.0), dict(scaling=3, factor=8.0, trained_len=4096), dict(base=1.0), dict(base=2.0 ** 60)])
@pytest.mark.parametrize("rot", [4, 64, 38])
def test_frequencies(lib, rot, angles):
    """Turns a position, times 2^64.  Long double on both sides: some ten roundings of 2^-64 each; by parts, g (at most 33 / 31, of three roundings) is off by 4 * 2^-64 on either side,
    which is (1 - 1 / factor) * factor = 7 times that where g is 0: 2 * (28 + 10) * 2^-64 < 2^-57."""
    lib.past_reset()
    for m in (Made(lib, "rotary", binding.make_rotary_config(2, 64, binding.make_rotary_angles(rot, **angles))),
              Made(lib, "cache", binding.make_cache_config(2, 64, 16, binding.make_rotary_angles(rot, **angles)))):
        got = m.arena[: rot * 4].view(np.uint64).astype(np.longdouble)
        want = ref.freqs(rot, **angles) / (2 * ref.PI) * np.longdouble(2) ** 64
        assert (np.abs(got - want) <= 1 + want * np.longdouble(2) ** -57).all()
        m.close()


def test_rotary_refuses(lib):
    lib.past_reset()
    m = Made(lib, "rotary", binding.make_rotary_config(3, 40, binding.make_rotary_angles(40), True, False))
    same = Made(lib, "rotary", binding.make_rotary_config(3, 40, binding.make_rotary_angles(40), True, True))
    wide = binding.make_rotary_config(3, 264, binding.make_rotary_angles(40))
    assert lib.tts_rotary_create(C.byref(wide), None, C.c_size_t(0), None, C.byref(C.c_void_p())) == UNSUPPORTED

    def run(op=m, **change):
        r = binding.TtsRotaryRows(rows=3, x=1 << 20, y=2 << 20, positions=3 << 20)
        for k, v in change.items():
            setattr(r, k, v)
        n = lib.fake_launches()
        rc = lib.tts_rotary_run(op.h, C.byref(r))
        assert (lib.fake_launches() > n) == (rc == 0 and r.rows > 0)
        return rc

    assert run() == 0 and run(rows=0, x=None, y=None) == 0 and run(rows=1 << 24) == 0 and run(back=1) == 0
    assert run(positions=None, first=-(1 << 31)) == 0 and lib.past_rotary_first() == -(1 << 31)
    assert run(positions=None, first=(1 << 31) - 3) == 0 and run(first=(1 << 31) - 1) == 0 and lib.past_rotary_first() == 0
    assert run(x_stride=128, y_stride=1 << 40) == 0 and run(op=same, y=1 << 20) == 0
    for change in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(x=None), dict(y=None), dict(x=(1 << 20) + 8), dict(y=(2 << 20) + 4), dict(positions=(3 << 20) + 2), dict(x_stride=112), dict(x_stride=124),
                   dict(y_stride=-120), dict(y_stride=(1 << 40) + 8), dict(back=2), dict(back=-1), dict(positions=None, first=(1 << 31) - 2), dict(y=1 << 20), dict(op=same, y=1 << 20, y_stride=128)):
        assert run(**change) == INVAL, change
        assert lib.tts_last_error()
    assert lib.tts_rotary_run(None, None) == INVAL and lib.tts_rotary_run(m.h, None) == INVAL
    lib.fake_fail(b"launch")
    r = binding.TtsRotaryRows(rows=3, x=1 << 20, y=2 << 20)
    assert lib.tts_rotary_run(m.h, C.byref(r)) == HIP
    lib.past_reset()
    lib.fake_device(3)                       # another device is current: the object's is while it launches, and the other again afterwards
    assert run() == 0 and lib.fake_seen() == 0 and lib.fake_current() == 3
    m.close()
    same.close()


def test_cache_refuses(lib):
    lib.past_reset()
    m = Made(lib, "cache", binding.make_cache_config(2, 40, 32, binding.make_rotary_angles(40), n_heads=4, bf16=True, x_bf16=True))
    none = Made(lib, "cache", binding.make_cache_config(2, 40, 32, bf16=True))
    wide = binding.make_cache_config(2, 136, 32)
    assert lib.tts_cache_create(C.byref(wide), None, C.c_size_t(0), None, C.byref(C.c_void_p())) == UNSUPPORTED

    def run(length=(2, 0, 3), row=(0, 5, 9), table_row=(0, 1, 2), position=None, op=m, n=None, null=None, **change):
        b = binding.CacheBatch(list(length), list(row), list(table_row), position)
        if n is not None:
            b.c.n = n
        if null:
            setattr(b.c, null, C.POINTER(C.c_int)())
        t = binding.TtsCacheTensors(k=1 << 20, v=2 << 20, k_pages=3 << 20, v_pages=4 << 20, table=5 << 20, n_pages=7, table_rows=3, table_cols=4)
        if op is m:
            t.q, t.q_out = 6 << 20, 7 << 20
        for key, v in change.items():
            setattr(t, key, v)
        before = lib.fake_launches()
        rc = lib.tts_cache_run(op.h, C.byref(b.c), C.byref(t))
        assert (lib.fake_launches() > before) == (rc == 0 and sum(length) > 0)
        return rc

    assert run() == 0 and lib.fake_requests() == 2 and lib.past_append_rows() == 5 and (lib.past_append_first(1), lib.past_append_position(1)) == (2, 9)
    assert run(position=[7, 0, -4]) == 0 and (lib.past_append_position(0), lib.past_append_position(1)) == (7, -4)
    assert run(length=(0, 0, 0), k=None, v=None, table_row=(9, -1, 9)) == 0              # (a request without rows has no sequence to be right)
    assert run(q=None, q_out=None) == 0 and run(op=none) == 0 and run(q_out=6 << 20) == 0
    assert run(length=(127, 1, 1), row=(0, 0, 127), table_row=(0, 1, 0)) == 0
    assert run(page_stride=2 * 32 * 40 + 8, k_stride=88, q_stride=168, q_out_stride=1 << 40) == 0
    # more requests than a launch takes: the second launch's rows begin where the first's end
    lib.past_reset()
    assert run([1, 2] * 150, [0] * 300, list(range(300)), table_rows=300) == 0
    assert lib.fake_launches() == 3 and lib.past_append_rows() == 450 and lib.fake_requests_seen() == 300 and lib.past_append_k() == (1 << 20) + 2 * 80 * 384
    for change in (dict(n=0), dict(n=-1), dict(null="len"), dict(null="row"), dict(null="table_row"), dict(length=(-1, 0, 0)), dict(length=((1 << 24) + 1, 0, 0)), dict(row=(-1, 0, 0)), dict(row=(127, 0, 0)),
                   dict(row=(1 << 24, 0, 0)), dict(row=((1 << 31) - 1, 0, 0)), dict(table_row=(3, 1, 2)), dict(table_row=(-1, 1, 2)), dict(position=[(1 << 31) - 1, 0, 0]), dict(k=None), dict(v=None),
                   dict(k_pages=None), dict(v_pages=None), dict(table=None), dict(q=None), dict(q_out=None), dict(n_pages=0), dict(table_rows=0), dict(table_cols=0), dict(k_stride=79), dict(v_stride=84),
                   dict(q_stride=152), dict(q_out_stride=-160), dict(page_stride=2552), dict(page_stride=2564), dict(page_stride=(1 << 40) + 8), dict(k=(1 << 20) + 8), dict(v=(2 << 20) + 4),
                   dict(k_pages=(3 << 20) + 8), dict(v_pages=(4 << 20) + 8), dict(q=(6 << 20) + 2), dict(q_out=(7 << 20) + 8), dict(table=(5 << 20) + 2), dict(q_out=6 << 20, q_out_stride=168),
                   dict(op=none, q=6 << 20, q_out=7 << 20), dict(length=[1] * 1025, row=[0] * 1025, table_row=list(range(1025)), table_rows=2000),
                   dict(length=[1 << 24, 1], row=[0, 0], table_row=[0, 1], table_cols=1 << 20)):
        assert run(**change) == INVAL, change
        assert lib.tts_last_error()
    # one place twice
    for length, row, table_row in (((2, 2, 1), (0, 1, 0), (0, 0, 1)), ((1, 5, 1), (3, 0, 9), (2, 2, 0)), ((3, 1, 2), (4, 0, 5), (1, 0, 1)), ((1, 1, 1), (0, 7, 0), (0, 1, 0))):
        assert run(length, row, table_row) == INVAL, (length, row, table_row)
    assert run((2, 3, 1), (0, 2, 5), (0, 0, 0)) == 0 and run((2, 0, 1), (0, 1, 2), (0, 0, 0)) == 0
    assert lib.tts_cache_run(None, None, None) == INVAL and lib.tts_cache_run(m.h, None, None) == INVAL
    lib.fake_fail(b"launch")
    b = binding.CacheBatch([1], [0], [0])
    t = binding.TtsCacheTensors(k=1 << 20, v=2 << 20, k_pages=3 << 20, v_pages=4 << 20, table=5 << 20, n_pages=7, table_rows=3, table_cols=4)
    assert lib.tts_cache_run(m.h, C.byref(b.c), C.byref(t)) == HIP
    lib.past_reset()
    m.close()
    none.close()


def _paged(lib, m, q_len=(2, 0, 3), own=(5, 4, 0), table_row=(0, 1, 2), prefix=(0, -1, 1), lens=(7, 9), rows=(3, 4), n=None, null=None, **change):
    b = binding.PagedBatch(list(q_len), list(own), list(table_row), None if prefix is None else list(prefix), list(lens), list(rows))
    if n is not None:
        b.c.n = n
    if null:
        setattr(b.c, null, C.POINTER(C.c_int)())
    t = binding.TtsPagedTensors(q=1 << 20, k_pages=2 << 20, v_pages=3 << 20, out=4 << 20, table=5 << 20, lse=6 << 20, n_pages=7, table_rows=5, table_cols=4)
    for key, v in change.items():
        setattr(b.c if key == "n_prefixes" else t, key, v)
    before = lib.fake_launches()
    rc = lib.tts_paged_run(m.h, C.byref(b.c), C.byref(t))
    assert (lib.fake_launches() > before) == (rc == 0 and sum(q_len) > 0)
    assert lib.past_wrong() == b""
    return rc


def test_paged_refuses(lib):
    lib.past_reset()
    m = Made(lib, "paged", binding.make_paged_config(8, 2, 40, 32, True))
    wide = binding.make_paged_config(8, 2, 136, 32)
    assert lib.tts_paged_create(C.byref(wide), None, C.c_size_t(0), None, C.byref(C.c_void_p())) == UNSUPPORTED

    def run(**change):
        return _paged(lib, m, **change)

    assert run() == 0 and lib.fake_requests_seen() == 2 and lib.past_rows() == 20                # a request without queries is left out
    assert run(prefix=None) == 0 and run(prefix=(-1, 0, -1)) == 0
    assert run(q_len=(0, 0, 0), q=None, out=None, k_pages=None, v_pages=None, table=None) == 0
    assert run(own=(0, 0, 0), table_row=(9, -1, 5), lens=(0, 0), rows=(-1, 99), k_pages=None, v_pages=None, table=None) == 0
    assert run(prefix=None, lens=(), rows=()) == 0 and run(lse=None) == 0 and run(own=(128, 1, 97)) == 0 and run(scale=0.5) == 0
    assert run(page_stride=2 * 32 * 40 + 8, q_stride=328, out_stride=1 << 40) == 0
    for change in (dict(n=0), dict(n=-1), dict(null="q_len"), dict(null="own_len"), dict(null="table_row"), dict(null="prefix_len"), dict(null="prefix_table_row"), dict(q_len=(-1, 0, 0)),
                   dict(q_len=((1 << 24) + 1, 0, 0)), dict(own=(-1, 0, 0)), dict(own=((1 << 24) + 1, 0, 0)), dict(own=(129, 0, 0)), dict(table_row=(5, 1, 2)), dict(table_row=(-1, 1, 2)),
                   dict(prefix=(2, 0, 0)), dict(prefix=(-2, 0, 0)), dict(lens=(-1, 9)), dict(lens=(7, 129)), dict(lens=(7, (1 << 24) + 1)), dict(rows=(3, 5)), dict(rows=(-1, 4)),
                   dict(n_prefixes=-1), dict(n_prefixes=1025), dict(n_prefixes=0), dict(q=None), dict(out=None), dict(k_pages=None), dict(v_pages=None), dict(table=None), dict(n_pages=0), dict(table_rows=0),
                   dict(table_cols=0), dict(q_stride=319), dict(q_stride=312), dict(out_stride=-320), dict(out_stride=(1 << 40) + 8), dict(page_stride=2552), dict(page_stride=2564), dict(q=(1 << 20) + 8),
                   dict(k_pages=(2 << 20) + 8), dict(v_pages=(3 << 20) + 4), dict(out=(4 << 20) + 8), dict(table=(5 << 20) + 2), dict(lse=(6 << 20) + 2), dict(scale=-1.0), dict(scale=float("nan")),
                   dict(scale=float("inf")), dict(scale=2.4e38), dict(q_len=[1] * 1025, own=[0] * 1025, table_row=[0] * 1025, prefix=None),
                   dict(q_len=[1 << 24] * 129, own=[0] * 129, table_row=[0] * 129, prefix=None), dict(q_len=[1 << 24, 1], own=[0] * 2, table_row=[0] * 2, prefix=None)):
        assert run(**change) == INVAL, change
        assert lib.tts_last_error()
    assert run(scale=2.3e38) == 0 and run(q_len=[1 << 24], own=[1], table_row=[0], prefix=None) == 0
    assert lib.tts_paged_run(None, None, None) == INVAL and lib.tts_paged_run(m.h, None, None) == INVAL
    lib.fake_fail(b"launch")
    assert _paged(lib, m, q_len=(0, 0, 0)) == 0
    b, t = binding.PagedBatch([1], [1], [0]), binding.TtsPagedTensors(q=1 << 20, k_pages=2 << 20, v_pages=3 << 20, out=4 << 20, table=5 << 20, n_pages=7, table_rows=5, table_cols=4)
    assert lib.tts_paged_run(m.h, C.byref(b.c), C.byref(t)) == HIP
    lib.past_reset()
    m.close()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads,kv,d", [(1, 1, 64), (8, 8, 64), (32, 8, 128), (16, 4, 128), (256, 256, 8), (256, 1, 128)])
def test_plans_of_attention(lib, heads, kv, d, bf16):
    """Launches of all kinds of batches: every request in one of them, parts that cover their sequences, parts that fit in the arena and are joined ahead of the next launch."""
    rng = np.random.default_rng(heads + d)
    m = Made(lib, "paged", binding.make_paged_config(heads, kv, d, 16, bf16))
    for n in (1, 2, 16, 17, 64, 128, 129, 500, 1024):
        for q_hi in (1, 3, 40, 700):
            for own_hi in (0, 30, 500, 20000):
                for prefixes, pre_hi in ((0, 0), (1, 100), (1, 16000), (3, 1000), (50, 300)):
                    q_len = [int(v) for v in rng.integers(0 if n > 4 else 1, q_hi + 1, n)]
                    if sum((q * (heads // kv) + 15) // 16 * kv for q in q_len) > 1 << 23:
                        continue
                    own = [int(v) for v in rng.integers(0, own_hi + 1, n)]
                    prefix = [int(v) for v in rng.integers(-1, prefixes, n)]
                    lens = [int(v) for v in rng.integers(0, pre_hi + 1, prefixes)]
                    lib.past_reset()
                    assert _paged(lib, m, q_len, own, [0] * n, prefix, lens, [1] * prefixes, table_cols=2000) == 0
                    assert lib.fake_requests_seen() == sum(q > 0 for q in q_len) and lib.past_rows() == sum(q_len) * (heads // kv), (n, q_hi, own_hi, prefixes)
    m.close()


@pytest.mark.parametrize("shape,q_len,own,prefix,lens,want", [
    ((8, 8, 64), [1] * 64, 300, [0] * 64, [2000], dict(few=1, many=0, pools=1, joins=1)),                # a prefix in tiles of its own beside the requests', joined by their last parts
    ((32, 8, 128), [1] * 128, 200, [0] * 128, [16001], dict(few=1, many=1, pools=1, joins=1)),           # larger tiles, a launch for them and one that joins
    ((8, 8, 64), [1, 2], 30, [0, 0], [41], dict(few=1, many=0, pools=0, joins=0)),                       # a short one ahead of each request's own rows
    ((8, 8, 64), [1] * 64, 300, [-1] * 64, [2000], dict(few=1, many=0, pools=0, joins=0)),               # nobody's prefix is not read
    ((4, 4, 64), [1], 9000, [-1], [], dict(few=1, many=0, pools=0, joins=1)),                            # a long sequence in parts
    ((16, 4, 128), [2000] * 8, 2000, [0] * 8, [500], dict(few=0, many=1, pools=0, joins=0)),             # many rows
    ((32, 8, 128), [128], 4224, [-1], [], dict(few=0, many=1, pools=0, joins=1, split=1)),               # many rows of one request over parts of its keys
    ((8, 2, 64), [40], 40, [-1], [], dict(few=1, many=0, pools=0, joins=0)),                             # many, but soon done
])
def test_how_calls_are_taken(lib, shape, q_len, own, prefix, lens, want):
    lib.past_reset()
    m = Made(lib, "paged", binding.make_paged_config(*shape, 16, True))
    n = len(q_len)
    assert _paged(lib, m, q_len, [own] * n, [0] * n, prefix, lens, [1] * len(lens), table_cols=2000) == 0
    assert {k: getattr(lib, f"past_{k}")() for k in want} == want
    m.close()


def test_numbers_that_their_types_do_not_hold():
    for args in (([1], [1 << 32], [0]), ([1 << 32], [1], [0]), ([1], [1], [-(1 << 32)]), ([1], [1], [0], [1 << 31]), ([1], [1], [0], [0], [1 << 32], [0]), ([1], [1], [0], [0], [1, 2], [0]),
                 ([1], [1, 2], [0]), ([1], [1], [0], [0, 1], [1], [1])):
        with pytest.raises(ValueError):
            binding.PagedBatch(*args)
    assert binding.PagedBatch([1, 2], [3, 4], [0, 1], [0, -1], [5], [2]).queries == 3
    with pytest.raises(ValueError):
        binding.CacheBatch([1], [1 << 32], [0])
    with pytest.raises(ValueError):
        binding.CacheBatch([1], [0], [0], [1 << 31])
    with pytest.raises(ValueError):
        binding.CacheBatch([1, 2], [0], [0, 0])
    assert binding.CacheBatch([1, 2], [0, 5], [0, 1]).rows == 3
