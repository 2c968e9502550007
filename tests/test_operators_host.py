"""The operators' host code without a GPU: the library exports what the headers declare, configurations and calls outside what the headers allow are refused before
anything is launched, failing HIP calls come back as errors, and the weights' 8-bit layout holds what the definition says."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2211_13939_amd import binding
from tests import operator_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVAL, HIP, UNSUPPORTED = binding.TTS_E_INVAL, binding.TTS_E_HIP, binding.TTS_E_UNSUPPORTED
_fp, _ip = C.POINTER(C.c_float), C.POINTER(C.c_int)


def test_library_exports_every_declared_operator():
    names = set()
    for header in ("tts_norm.h", "tts_linear8.h", "tts_cross.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names |= set(re.findall(r"\b(tts_(?:norm|linear8|cross)_\w+)\s*\(", text))
    assert names == set(binding.OPERATOR_EXPORTS)
    for n in names:
        assert hasattr(binding.lib(), n), n


def test_configurations_without_gpu():
    L = binding.lib()
    assert L.tts_norm_workspace_bytes(C.byref(binding.make_norm_config(513))) >= 513 * 4
    for change in (dict(dim=0), dict(dim=16385), dict(kind=2), dict(x_dtype=2), dict(res_dtype=-1), dict(y_dtype=3), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        c = binding.make_norm_config(64)
        for k, v in change.items():
            setattr(c, k, v)
        assert L.tts_norm_workspace_bytes(C.byref(c)) == 0 and L.tts_last_error(), change
    assert L.tts_linear8_workspace_bytes(C.byref(binding.make_linear8_config(1000, 100))) >= 1024 * 112
    for change in (dict(in_dim=0), dict(in_dim=65537), dict(out_dim=0), dict(out_dim=65537), dict(y_dtype=2)):
        c = binding.make_linear8_config(64, 64)
        for k, v in change.items():
            setattr(c, k, v)
        assert L.tts_linear8_workspace_bytes(C.byref(c)) == 0 and L.tts_last_error(), change
    assert L.tts_cross_workspace_bytes(C.byref(binding.make_cross_config(8, 2, 96))) > 0
    for change in (dict(n_heads=0), dict(n_heads=257), dict(n_kv_heads=0), dict(n_kv_heads=3), dict(n_kv_heads=16), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136), dict(dtype=2)):
        c = binding.make_cross_config(8, 8, 64)
        for k, v in change.items():
            setattr(c, k, v)
        assert L.tts_cross_workspace_bytes(C.byref(c)) == 0 and L.tts_last_error(), change
    for f in (L.tts_norm_workspace_bytes, L.tts_linear8_workspace_bytes, L.tts_cross_workspace_bytes):
        assert f(None) == 0


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "liboperators.so")
    csrc = os.path.join(ROOT, "paper_2211_13939_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-Wno-unused-result",
                    os.path.join(ROOT, "tests", "fake_operators.cpp")] + [os.path.join(csrc, f) for f in ("norm.cpp", "linear8.cpp", "cross.cpp")] + ["-o", out], check=True)
    L = C.CDLL(out)
    L.tts_last_error.restype = C.c_char_p
    for op in ("norm", "linear8", "cross"):
        getattr(L, f"tts_{op}_workspace_bytes").restype = C.c_size_t
        f = getattr(L, f"tts_{op}_destroy")
        f.restype, f.argtypes = None, [C.c_void_p]
    return L


class Made:
    """An object of the fake library, with its arena."""

    def __init__(self, lib, op, cfg, *weights, want=0):
        self.lib, self.op = lib, op
        n = int(getattr(lib, f"tts_{op}_workspace_bytes")(C.byref(cfg)))
        self.raw = np.zeros(n + 512, np.uint8)
        self.skip = (-self.raw.ctypes.data) % 256
        self.arena = self.raw[self.skip: self.skip + n]
        self.h = C.c_void_p()
        create = getattr(lib, f"tts_{op}_create")
        args = (C.byref(cfg), *weights)
        assert create(*args, None, C.c_size_t(n), None, C.byref(self.h)) == INVAL
        assert create(*args, C.c_void_p(self.arena.ctypes.data + 4), C.c_size_t(n + 256), None, C.byref(self.h)) == INVAL
        assert create(*args, C.c_void_p(self.arena.ctypes.data), C.c_size_t(n - 1), None, C.byref(self.h)) == INVAL
        assert create(*args, C.c_void_p(self.arena.ctypes.data), C.c_size_t(n), None, None) == INVAL
        for name in ("hipPointerGetAttributes", "hipGetDevice", "hipDeviceGetAttribute", "hipMemcpy"):
            lib.fake_fail(name.encode())
            rc = create(*args, C.c_void_p(self.arena.ctypes.data), C.c_size_t(n), None, C.byref(self.h))
            if rc == 0:                                    # (a call that this object does not make)
                getattr(lib, f"tts_{op}_destroy")(self.h)
            else:
                assert rc in (INVAL, HIP) and not self.h
        lib.fake_reset()
        assert create(*args, C.c_void_p(self.arena.ctypes.data), C.c_size_t(n), None, C.byref(self.h)) == 0, lib.tts_last_error()

    def close(self):
        getattr(self.lib, f"tts_{self.op}_destroy")(self.h)
        getattr(self.lib, f"tts_{self.op}_destroy")(None)


def _floats(a):
    return np.ascontiguousarray(a, np.float32).ctypes.data_as(_fp)


def test_norm_refuses(lib):
    lib.fake_reset()
    gain = np.ones(100, np.float32)
    bad = C.c_void_p()
    cfg = binding.make_norm_config(100, True, False, True)
    arena = np.zeros(1 << 12, np.uint8)
    at = C.c_void_p(arena.ctypes.data + (-arena.ctypes.data) % 256)
    assert lib.tts_norm_create(C.byref(cfg), None, at, C.c_size_t(1024), None, C.byref(bad)) == INVAL
    none = binding.make_norm_config(100, kind=binding.NORM_NONE)
    assert lib.tts_norm_create(C.byref(none), _floats(gain), at, C.c_size_t(1024), None, C.byref(bad)) == INVAL
    m = Made(lib, "norm", cfg, _floats(gain))
    np.testing.assert_array_equal(m.arena[:400].view(np.float32), gain)

    def run(**change):
        r = binding.TtsNormRows(rows=3, x=1 << 20, y=2 << 20, total=3 << 20, res=4 << 20, y8=5 << 20, scales=6 << 20)
        for k, v in change.items():
            setattr(r, k, v)
        n = lib.fake_launches()
        rc = lib.tts_norm_run(m.h, C.byref(r))
        assert (lib.fake_launches() > n) == (rc == 0 and r.rows > 0)
        return rc

    assert run() == 0 and lib.fake_rows() == 3
    assert run(rows=0, x=None) == 0
    assert run(rows=1 << 24) == 0
    for change in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(x=None), dict(y=None, total=None, y8=None, scales=None), dict(y8=None), dict(scales=None), dict(x_stride=99), dict(x_stride=-100),
                   dict(res_stride=99), dict(total_stride=1), dict(y_stride=(1 << 40) + 1), dict(x=(1 << 20) + 1), dict(res=(4 << 20) + 2), dict(total=(3 << 20) + 2), dict(y=(2 << 20) + 1),
                   dict(y8=(5 << 20) + 8), dict(scales=(6 << 20) + 2)):
        assert run(**change) == INVAL, change
        assert lib.tts_last_error()
    # what an absent array has for a stride does not matter; elements need no more than their own alignment
    assert run(res=None, res_stride=1) == 0 and run(x=(1 << 20) + 2, y=(2 << 20) + 2, x_stride=101) == 0
    assert lib.tts_norm_run(None, None) == INVAL and lib.tts_norm_run(m.h, None) == INVAL
    lib.fake_fail(b"launch")
    r = binding.TtsNormRows(rows=1, x=1 << 20, y=2 << 20)
    assert lib.tts_norm_run(m.h, C.byref(r)) == HIP
    lib.fake_reset()
    # another device is current: the object's is while it launches, and the other again afterwards
    lib.fake_device(3)
    assert run() == 0 and lib.fake_seen() == 0 and lib.fake_current() == 3
    m.close()


def test_linear8_refuses(lib):
    lib.fake_reset()
    w, bias = np.ones((70, 300), np.float32), np.ones(70, np.float32)
    bad = C.c_void_p()
    cfg = binding.make_linear8_config(300, 70, True)
    arena = np.zeros(1 << 16, np.uint8)
    assert lib.tts_linear8_create(C.byref(cfg), None, None, C.c_void_p(arena.ctypes.data + (-arena.ctypes.data) % 256), C.c_size_t(60000), None, C.byref(bad)) == INVAL
    m = Made(lib, "linear8", cfg, _floats(w), _floats(bias))

    def run(x8=1 << 20, sx=2 << 20, rows=3, y=3 << 20, stride=0):
        n = lib.fake_launches()
        rc = lib.tts_linear8_run(m.h, C.c_void_p(x8), C.c_void_p(sx), rows, C.c_void_p(y), C.c_longlong(stride))
        assert (lib.fake_launches() > n) == (rc == 0 and rows > 0)
        return rc

    assert run() == 0 and run(rows=0, x8=None, y=None) == 0 and run(y=(3 << 20) + 2, stride=71) == 0 and run(rows=1 << 24) == 0
    for change in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(x8=None), dict(sx=None), dict(y=None), dict(x8=(1 << 20) + 8), dict(sx=(2 << 20) + 2), dict(y=(3 << 20) + 1), dict(stride=69),
                   dict(stride=-70), dict(stride=(1 << 40) + 1)):
        assert run(**change) == INVAL, change
        assert lib.tts_last_error()
    assert lib.tts_linear8_run(None, None, None, 1, None, C.c_longlong(0)) == INVAL
    lib.fake_fail(b"launch")
    assert lib.tts_linear8_run(m.h, C.c_void_p(1 << 20), C.c_void_p(2 << 20), 3, C.c_void_p(3 << 20), C.c_longlong(0)) == HIP
    lib.fake_reset()
    m.close()


@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (70, 300), (33, 1100)])
def test_linear8_weights_are_rounded_and_laid_out(lib, n, k):
    """The arena against the definition: [units of 32 channels][steps of 64 columns][2][64 lanes] 16 bytes, the c-th of lane l of row l % 32 from column
    32 * (l / 32) + 16 * c on; then scales [units][words][32 rows], then the bias.  Row 8 a + 4 h + j of the t-th of two units is channel 32 h + 16 t + 4 a + j."""
    lib.fake_reset()
    rng = np.random.default_rng(n + k)
    w = (rng.standard_normal((n, k)) * 2.0 ** rng.integers(-30, 30, (n, 1))).astype(np.float32)
    w[0, : min(k, 64)] = (np.arange(min(k, 64)) + 0.5) / 8        # ties
    w[-1, -1] = 2.0 ** -140
    if n > 3:
        w[3] = 0
    bias = rng.standard_normal(n).astype(np.float32)
    m = Made(lib, "linear8", binding.make_linear8_config(k, n), _floats(w), _floats(bias))
    want, want_s = ref.round8(w.astype(np.float64))
    units, blocks, words = -(-n // 64) * 2, ref.blocks_of(k), want_s.shape[1] // 4
    size = units * blocks * 4096
    c = np.arange(units * 32)
    row = (c // 64 * 2 + c // 16 % 2) * 32 + c // 4 % 4 * 8 + c // 32 % 2 * 4 + c % 4        # where channel c lies
    got = m.arena[:size].reshape(units, 2 * blocks, 2, 2, 32, 16)           # unit, step, c, l / 32, row, byte
    got = got.transpose(0, 4, 1, 3, 2, 5).reshape(units * 32, blocks * 128)[row]
    np.testing.assert_array_equal(got[:n], want)
    assert (got[n:] == 0).all()
    at = -(-size // 256) * 256
    s = m.arena[at: at + units * words * 128].reshape(units, words, 32, 4).transpose(0, 2, 1, 3).reshape(units * 32, words * 4)[row]
    np.testing.assert_array_equal(s[:n], want_s)
    assert (s[n:] == 127).all()
    at += -(-units * words * 128 // 256) * 256
    np.testing.assert_array_equal(m.arena[at: at + 4 * n].view(np.float32), bias)
    m.close()


def test_cross_refuses(lib):
    lib.fake_reset()
    m = Made(lib, "cross", binding.make_cross_config(8, 2, 40, True))
    wide = binding.make_cross_config(8, 2, 136)
    assert lib.tts_cross_create(C.byref(wide), None, C.c_size_t(0), None, C.byref(C.c_void_p())) == UNSUPPORTED

    def run(q_len=(2, 0, 3), row=(0, 5, 9), mem=(5, 4, 0), n=None, null=None, **change):
        b = binding.CrossBatch(list(q_len), list(row), list(mem))
        if n is not None:
            b.c.n = n
        if null:
            setattr(b.c, null, {"q_len": _ip(), "mem_row": C.POINTER(C.c_longlong)(), "mem_len": _ip()}[null])
        t = binding.TtsCrossTensors(q=1 << 20, k=2 << 20, v=3 << 20, out=4 << 20, keep=(5 << 20) + 1, lse=6 << 20)
        for key, v in change.items():
            setattr(t, key, v)
        before = lib.fake_launches()
        rc = lib.tts_cross_run(m.h, C.byref(b.c), C.byref(t))
        assert (lib.fake_launches() > before) == (rc == 0 and sum(q_len) > 0)
        return rc

    assert run() == 0 and lib.fake_requests() == 2 and lib.fake_rows() == 5        # a request without queries is left out
    assert run(q_len=(0, 0, 0), q=None, out=None, k=None, v=None) == 0
    assert run(mem=(0, 0, 0), k=None, v=None) == 0
    assert run(q_len=[1] * 300, row=[0] * 300, mem=[1] * 300) == 0 and lib.fake_requests() == 300 % 128 and lib.fake_rows() == 300
    # requests of many rows go by themselves (8 / 2 heads: 4 rows a query); every request once
    lib.fake_reset()
    assert run(q_len=[1, 500] * 70, row=[0] * 140, mem=[1] * 140) == 0
    assert lib.fake_launches() == 2 and lib.fake_many() == 1 and lib.fake_requests_seen() == 140 and lib.fake_rows() == 70 * 501
    lib.fake_reset()
    assert run(q_len=[500] * 300, row=[0] * 300, mem=[1] * 300) == 0 and lib.fake_launches() == lib.fake_many() == 3 and lib.fake_requests_seen() == 300
    assert run(q_len=[1 << 24], row=[0], mem=[1]) == 0                # 2^23 tiles of 16 rows
    assert run(scale=0.5) == 0 and run(k_stride=1 << 24, q_stride=328, row=(1 << 40, 0, 0)) == 0
    for change in (dict(n=0), dict(n=-1), dict(null="q_len"), dict(null="mem_row"), dict(null="mem_len"), dict(q_len=(-1, 0, 0)), dict(q_len=((1 << 24) + 1, 0, 0)), dict(mem=(-1, 0, 0)),
                   dict(mem=((1 << 24) + 1, 0, 0)), dict(row=(-1, 0, 0)), dict(row=((1 << 40) + 1, 0, 0)), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q_stride=319), dict(q_stride=321),
                   dict(k_stride=72), dict(v_stride=-80), dict(out_stride=(1 << 24) + 8), dict(q=(1 << 20) + 8), dict(k=(2 << 20) + 2), dict(v=(3 << 20) + 4), dict(out=(4 << 20) + 8),
                   dict(lse=(6 << 20) + 2), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_len=[1 << 24] * 129, row=[0] * 129, mem=[1] * 129),
                   dict(q_len=[1 << 24, 1], row=[0] * 2, mem=[1] * 2), dict(q_len=[1] * 1025, row=[0] * 1025, mem=[1] * 1025)):
        assert run(**change) == INVAL, change
        assert lib.tts_last_error()
    assert lib.tts_cross_run(None, None, None) == INVAL and lib.tts_cross_run(m.h, None, None) == INVAL
    lib.fake_fail(b"launch")
    b, t = binding.CrossBatch([1], [0], [1]), binding.TtsCrossTensors(q=1 << 20, k=2 << 20, v=3 << 20, out=4 << 20)
    assert lib.tts_cross_run(m.h, C.byref(b.c), C.byref(t)) == HIP
    lib.fake_reset()
    m.close()
