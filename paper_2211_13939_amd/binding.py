"""Thin ctypes binding of the C-ABI library declared in include/tts_pool.h.

Argument marshalling only: every step of the decoder path runs in the HIP
kernels of libtts_pool.so.  PyTorch is used for the device arena and the
stream, nothing else.  If the library has not been built this module raises;
there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtts_pool.so")

TTS_OK = 0
TTS_E_INVAL, TTS_E_FULL, TTS_E_NOTFOUND, TTS_E_HIP, TTS_E_ARENA, TTS_E_UNSUPPORTED, TTS_E_LOST = -1, -2, -3, -4, -5, -6, -7
DTYPE_F32, DTYPE_BF16 = 0, 1
STATE = dict(m=0, a=1, w_last=2, w_acc=3, h_att=4, c_att=5, h_dec=6, c_dec=7)

_CFG_INT_FIELDS = ("n_mel", "prenet_dim", "enc_dim", "att_rnn_dim", "dec_rnn_dim", "att_dim",
                   "loc_filters", "loc_kernel", "loc_in_channels",
                   "max_pool", "max_enc_len", "max_steps", "chunk_frames",
                   "weight_dtype", "memory_dtype", "use_graph")
WEIGHT_FIELDS = ("prenet1", "prenet2", "att_w_ih", "att_w_hh", "att_b", "q_w", "mem_w", "loc_conv",
                 "loc_w", "v", "dec_w_ih", "dec_w_hh", "dec_b", "mel_w", "mel_b", "stop_w", "stop_b")

# every symbol include/tts_pool.h declares
EXPORTS = (
    "tts_pool_workspace_bytes", "tts_pool_create", "tts_pool_add_request", "tts_pool_add_requests", "tts_pool_step",
    "tts_pool_step_n", "tts_pool_drain_chunk", "tts_pool_get_stop_logits", "tts_pool_retire",
    "tts_pool_get_state", "tts_pool_set_state", "tts_pool_frames", "tts_pool_size", "tts_pool_n_active",
    "tts_pool_span", "tts_pool_moves", "tts_pool_segments", "tts_pool_fp32_segments",
    "tts_pool_sync", "tts_pool_lost", "tts_pool_set_wait_polls", "tts_pool_timing", "tts_pool_elapsed_ms", "tts_pool_kernel_times", "tts_pool_destroy",
    "tts_last_error",
    "tts_book_create", "tts_book_add", "tts_book_step", "tts_book_drain", "tts_book_retire",
    "tts_book_slot", "tts_book_compact", "tts_book_destroy",
    "tts_pool_chunk_window", "tts_pool_chunk_windows",
    "tts_postnet_workspace_bytes", "tts_postnet_create", "tts_postnet_run", "tts_postnet_run_static", "tts_postnet_set_wait_polls",
    "tts_postnet_one_launch_calls", "tts_postnet_elapsed_ms",
    "tts_postnet_destroy",
    "tts_vocoder_workspace_bytes", "tts_vocoder_create", "tts_vocoder_run", "tts_vocoder_elapsed_ms",
    "tts_vocoder_destroy",
    "tts_encoder_workspace_bytes", "tts_encoder_create", "tts_encoder_run", "tts_encoder_set_wait_polls",
    "tts_encoder_one_launch_calls", "tts_encoder_elapsed_ms",
    "tts_encoder_destroy",
)

# every symbol include/tts_norm.h, tts_linear8.h and tts_cross.h declare
OPERATOR_EXPORTS = tuple(f"tts_{op}_{call}" for op in ("norm", "linear8", "cross") for call in ("workspace_bytes", "create", "run", "destroy"))

# every symbol include/tts_rotary.h, tts_cache.h and tts_paged.h declare
PAST_EXPORTS = tuple(f"tts_{op}_{call}" for op in ("rotary", "cache", "paged") for call in ("workspace_bytes", "create", "run", "destroy"))

_fp = C.POINTER(C.c_float)
_ip = C.POINTER(C.c_int)
_i64p = C.POINTER(C.c_int64)


class TtsConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in _CFG_INT_FIELDS] + [("stop_threshold", C.c_float)]


class TtsWeights(C.Structure):
    _fields_ = [(n, _fp) for n in WEIGHT_FIELDS]


class TtsPostnetConfig(C.Structure):
    _fields_ = [("n_mel", C.c_int), ("channels", C.c_int), ("max_columns", C.c_int), ("weight_dtype", C.c_int)]


class TtsPostnetWeights(C.Structure):
    _fields_ = [("conv_w", C.POINTER(C.c_float) * 5), ("conv_b", C.POINTER(C.c_float) * 5)]


class TtsVocoderConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_mel", "c0", "overlap", "max_chunk", "max_requests", "max_batch", "weight_dtype")]


class TtsVocoderWeights(C.Structure):
    _fields_ = [("pre_w", _fp), ("pre_b", _fp), ("up_w", _fp * 4), ("up_b", _fp * 4),
                ("res_w", _fp * 6 * 3 * 4), ("res_b", _fp * 6 * 3 * 4), ("post_w", _fp), ("post_b", _fp)]


class TtsEncoderConfig(C.Structure):
    _fields_ = [("dim", C.c_int), ("hid", C.c_int), ("vocab", C.c_int * 4), ("max_tokens", C.c_int), ("max_len", C.c_int),
                ("weight_dtype", C.c_int)]


class TtsEncoderWeights(C.Structure):
    _fields_ = [("tables", _fp * 4), ("conv_w", _fp * 3), ("conv_b", _fp * 3), ("w_ih", _fp * 2), ("w_hh", _fp * 2), ("b", _fp * 2)]


class TtsNormConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("dim", "kind", "x_dtype", "res_dtype", "y_dtype")] + [("eps", C.c_float)]


class TtsNormRows(C.Structure):
    _fields_ = [("rows", C.c_int), ("x", C.c_void_p), ("x_stride", C.c_longlong), ("res", C.c_void_p), ("res_stride", C.c_longlong),
                ("total", C.c_void_p), ("total_stride", C.c_longlong), ("y", C.c_void_p), ("y_stride", C.c_longlong),
                ("y8", C.c_void_p), ("scales", C.c_void_p)]


class TtsLinear8Config(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("in_dim", "out_dim", "y_dtype")]


class TtsCrossConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_heads", "n_kv_heads", "head_dim", "dtype")]


class TtsCrossBatch(C.Structure):
    _fields_ = [("n", C.c_int), ("q_len", _ip), ("mem_row", C.POINTER(C.c_longlong)), ("mem_len", _ip)]


class TtsCrossTensors(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_stride", C.c_longlong), ("k", C.c_void_p), ("k_stride", C.c_longlong),
                ("v", C.c_void_p), ("v_stride", C.c_longlong), ("out", C.c_void_p), ("out_stride", C.c_longlong),
                ("keep", C.c_void_p), ("lse", C.c_void_p), ("scale", C.c_float)]


class TtsRotaryAngles(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("rot_dim", "layout", "scaling", "trained_len")] + [(n, C.c_double) for n in ("base", "factor", "low", "high", "magnitude")]


class TtsRotaryConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_heads", "head_dim", "x_dtype", "y_dtype")] + [("angles", TtsRotaryAngles)]


class TtsRotaryRows(C.Structure):
    _fields_ = [("rows", C.c_int), ("x", C.c_void_p), ("x_stride", C.c_longlong), ("y", C.c_void_p), ("y_stride", C.c_longlong),
                ("positions", C.c_void_p), ("first", C.c_int), ("back", C.c_int)]


class TtsCacheConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_kv_heads", "n_heads", "head_dim", "page_rows", "x_dtype", "dtype")] + [("angles", TtsRotaryAngles)]


class TtsCacheBatch(C.Structure):
    _fields_ = [("n", C.c_int), ("len", _ip), ("row", _ip), ("table_row", _ip), ("position", _ip)]


class TtsCacheTensors(C.Structure):
    _fields_ = [("k", C.c_void_p), ("k_stride", C.c_longlong), ("v", C.c_void_p), ("v_stride", C.c_longlong), ("q", C.c_void_p), ("q_stride", C.c_longlong),
                ("q_out", C.c_void_p), ("q_out_stride", C.c_longlong), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("page_stride", C.c_longlong),
                ("n_pages", C.c_int), ("table", C.c_void_p), ("table_rows", C.c_int), ("table_cols", C.c_int)]


class TtsPagedConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_heads", "n_kv_heads", "head_dim", "page_rows", "dtype", "causal")]


class TtsPagedBatch(C.Structure):
    _fields_ = [("n", C.c_int), ("q_len", _ip), ("own_len", _ip), ("table_row", _ip), ("prefix", _ip), ("n_prefixes", C.c_int), ("prefix_len", _ip), ("prefix_table_row", _ip)]


class TtsPagedTensors(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_stride", C.c_longlong), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("page_stride", C.c_longlong), ("n_pages", C.c_int),
                ("table", C.c_void_p), ("table_rows", C.c_int), ("table_cols", C.c_int), ("out", C.c_void_p), ("out_stride", C.c_longlong), ("lse", C.c_void_p), ("scale", C.c_float)]


VOCODER_HOP = 256
VOCODER_FIRST, VOCODER_LAST = 1, 2
POSTNET_CONTEXT = 10      # frames in front of a chunk that can influence it (2 per layer)
TTS_POSTNET_STATIC_MAX_COLUMNS = 4096   # most frames one tts_postnet_run_static call may carry


class TtsError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"tts_pool error {code}: {text}")
        self.code = code
        self.text = text


_lib = None


def lib() -> C.CDLL:
    """Load libtts_pool.so (built beforehand by paper_2211_13939_amd/build.py)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2211_13939_amd.build` "
                           "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    vp = C.c_void_p
    L.tts_pool_workspace_bytes.restype = C.c_size_t
    L.tts_pool_workspace_bytes.argtypes = [C.POINTER(TtsConfig)]
    L.tts_pool_create.argtypes = [C.POINTER(TtsConfig), C.POINTER(TtsWeights), vp, C.c_size_t, vp, C.POINTER(vp)]
    L.tts_pool_add_request.argtypes = [vp, vp, C.c_int, C.c_int, _i64p]
    L.tts_pool_add_requests.argtypes = [vp, C.c_int, C.POINTER(vp), _ip, _ip, _i64p]
    L.tts_pool_step.argtypes = [vp, _ip]
    L.tts_pool_step_n.argtypes = [vp, C.c_int, _i64p]
    L.tts_pool_drain_chunk.argtypes = [vp, C.c_int64, vp, vp, vp]
    L.tts_pool_get_stop_logits.argtypes = [vp, C.c_int64, C.c_int, C.c_int, _fp]
    L.tts_pool_retire.argtypes = [vp, C.c_int64]
    L.tts_pool_get_state.argtypes = [vp, C.c_int64, C.c_int, _fp, C.c_int, _ip]
    L.tts_pool_set_state.argtypes = [vp, C.c_int64, C.c_int, _fp, C.c_int]
    L.tts_pool_frames.argtypes = [vp, C.c_int64, _ip, _ip]
    L.tts_pool_size.argtypes = [vp]
    L.tts_pool_n_active.argtypes = [vp]
    L.tts_pool_span.argtypes = [vp]
    for f in (L.tts_pool_moves, L.tts_pool_segments, L.tts_pool_fp32_segments, L.tts_postnet_one_launch_calls, L.tts_encoder_one_launch_calls):
        f.restype = C.c_longlong
        f.argtypes = [vp]
    L.tts_pool_sync.argtypes = [vp]
    L.tts_pool_lost.argtypes = [vp, C.c_int64, _ip]
    L.tts_pool_set_wait_polls.argtypes = [vp, C.c_int]
    L.tts_pool_timing.argtypes = [vp, C.c_int]
    L.tts_pool_elapsed_ms.argtypes = [vp, _fp]
    L.tts_pool_kernel_times.argtypes = [vp, C.c_int, _fp, C.c_int, _ip]
    L.tts_pool_destroy.restype = None
    L.tts_pool_destroy.argtypes = [vp]
    L.tts_last_error.restype = C.c_char_p
    L.tts_last_error.argtypes = []
    L.tts_book_create.restype = vp
    L.tts_book_create.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int]
    L.tts_book_add.argtypes = [vp, C.c_int, C.c_int, _i64p]
    L.tts_book_step.argtypes = [vp, _i64p, _ip]
    L.tts_book_drain.argtypes = [vp, C.c_int64, _ip, _ip, _ip]
    L.tts_book_retire.argtypes = [vp, C.c_int64]
    L.tts_book_slot.argtypes = [vp, C.c_int64]
    L.tts_book_compact.argtypes = [vp, C.c_int, _ip, _ip, C.c_int]
    L.tts_book_destroy.restype = None
    L.tts_book_destroy.argtypes = [vp]
    L.tts_pool_chunk_window.argtypes = [vp, C.c_int64, C.c_int, vp, _ip, _ip, _ip]
    L.tts_pool_chunk_windows.argtypes = [vp, C.c_int, C.POINTER(C.c_int64), C.c_int, vp, _ip, _ip, _ip]
    L.tts_postnet_workspace_bytes.restype = C.c_size_t
    L.tts_postnet_workspace_bytes.argtypes = [C.POINTER(TtsPostnetConfig)]
    L.tts_postnet_create.argtypes = [C.POINTER(TtsPostnetConfig), C.POINTER(TtsPostnetWeights), vp, C.c_size_t, vp,
                                     C.POINTER(vp)]
    L.tts_postnet_run.argtypes = [vp, vp, _ip, _ip, C.c_int, vp]
    L.tts_postnet_run_static.argtypes = [vp, vp, _ip, _ip, C.c_int, vp]
    L.tts_postnet_set_wait_polls.argtypes = [vp, C.c_int]
    L.tts_postnet_elapsed_ms.argtypes = [vp, _fp]
    L.tts_postnet_destroy.restype = None
    L.tts_postnet_destroy.argtypes = [vp]
    L.tts_vocoder_workspace_bytes.restype = C.c_size_t
    L.tts_vocoder_workspace_bytes.argtypes = [C.POINTER(TtsVocoderConfig)]
    L.tts_vocoder_create.argtypes = [C.POINTER(TtsVocoderConfig), C.POINTER(TtsVocoderWeights), vp, C.c_size_t, vp,
                                     C.POINTER(vp)]
    L.tts_vocoder_run.argtypes = [vp, vp, _ip, _ip, _ip, C.c_int, vp, _ip]
    L.tts_vocoder_elapsed_ms.argtypes = [vp, _fp]
    L.tts_vocoder_destroy.restype = None
    L.tts_vocoder_destroy.argtypes = [vp]
    L.tts_encoder_workspace_bytes.restype = C.c_size_t
    L.tts_encoder_workspace_bytes.argtypes = [C.POINTER(TtsEncoderConfig)]
    L.tts_encoder_create.argtypes = [C.POINTER(TtsEncoderConfig), C.POINTER(TtsEncoderWeights), vp, C.c_size_t, vp,
                                     C.POINTER(vp)]
    L.tts_encoder_run.argtypes = [vp, _ip, _ip, C.c_int, vp]
    L.tts_encoder_set_wait_polls.argtypes = [vp, C.c_int]
    L.tts_encoder_elapsed_ms.argtypes = [vp, _fp]
    L.tts_encoder_destroy.restype = None
    L.tts_encoder_destroy.argtypes = [vp]
    L.tts_norm_workspace_bytes.restype = C.c_size_t
    L.tts_norm_workspace_bytes.argtypes = [C.POINTER(TtsNormConfig)]
    L.tts_norm_create.argtypes = [C.POINTER(TtsNormConfig), _fp, vp, C.c_size_t, vp, C.POINTER(vp)]
    L.tts_norm_run.argtypes = [vp, C.POINTER(TtsNormRows)]
    L.tts_linear8_workspace_bytes.restype = C.c_size_t
    L.tts_linear8_workspace_bytes.argtypes = [C.POINTER(TtsLinear8Config)]
    L.tts_linear8_create.argtypes = [C.POINTER(TtsLinear8Config), _fp, _fp, vp, C.c_size_t, vp, C.POINTER(vp)]
    L.tts_linear8_run.argtypes = [vp, vp, vp, C.c_int, vp, C.c_longlong]
    L.tts_cross_workspace_bytes.restype = C.c_size_t
    L.tts_cross_workspace_bytes.argtypes = [C.POINTER(TtsCrossConfig)]
    L.tts_cross_create.argtypes = [C.POINTER(TtsCrossConfig), vp, C.c_size_t, vp, C.POINTER(vp)]
    L.tts_cross_run.argtypes = [vp, C.POINTER(TtsCrossBatch), C.POINTER(TtsCrossTensors)]
    for op, config, *args in (("rotary", TtsRotaryConfig, C.POINTER(TtsRotaryRows)), ("cache", TtsCacheConfig, C.POINTER(TtsCacheBatch), C.POINTER(TtsCacheTensors)),
                             ("paged", TtsPagedConfig, C.POINTER(TtsPagedBatch), C.POINTER(TtsPagedTensors))):
        f = getattr(L, f"tts_{op}_workspace_bytes")
        f.restype, f.argtypes = C.c_size_t, [C.POINTER(config)]
        getattr(L, f"tts_{op}_create").argtypes = [C.POINTER(config), vp, C.c_size_t, vp, C.POINTER(vp)]
        getattr(L, f"tts_{op}_run").argtypes = [vp, *args]
    for f in (L.tts_norm_destroy, L.tts_linear8_destroy, L.tts_cross_destroy, L.tts_rotary_destroy, L.tts_cache_destroy, L.tts_paged_destroy):
        f.restype = None
        f.argtypes = [vp]
    _lib = L
    return L


def _check(rc: int) -> None:
    if rc != TTS_OK:
        raise TtsError(rc, lib().tts_last_error().decode("utf-8", "replace"))


def make_config(dims: Dict[str, int], max_pool: int, max_enc_len: int, max_steps: int, chunk_frames: int = 40,
                bf16: bool = False, memory_bf16: Optional[bool] = None, use_graph: bool = True,
                stop_threshold: float = -1.0) -> TtsConfig:
    if memory_bf16 is None:
        memory_bf16 = bf16
    c = TtsConfig()
    for k, v in dims.items():
        setattr(c, k, int(v))
    c.max_pool, c.max_enc_len, c.max_steps, c.chunk_frames = int(max_pool), int(max_enc_len), int(max_steps), int(chunk_frames)
    c.weight_dtype = DTYPE_BF16 if bf16 else DTYPE_F32
    c.memory_dtype = DTYPE_BF16 if memory_bf16 else DTYPE_F32
    c.use_graph = int(bool(use_graph))
    c.stop_threshold = float(stop_threshold)
    return c


def workspace_bytes(cfg: TtsConfig) -> int:
    return int(lib().tts_pool_workspace_bytes(C.byref(cfg)))


class Pool:
    """tts_pool_* calls on one pool; owns the torch arena and stream."""

    def __init__(self, cfg: TtsConfig, weights: Dict[str, np.ndarray], device: str = "cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the decoder step has no CPU path")
        self._torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = workspace_bytes(cfg)
        if nbytes == 0:
            _check(TTS_E_INVAL)
        with torch.cuda.device(self.device):
            self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.stream = torch.cuda.Stream(device=self.device)
        self._warr = {n: np.ascontiguousarray(weights[n], dtype=np.float32) for n in WEIGHT_FIELDS}
        w = TtsWeights(*[self._warr[n].ctypes.data_as(_fp) for n in WEIGHT_FIELDS])
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().tts_pool_create(C.byref(cfg), C.byref(w), C.c_void_p(self.arena.data_ptr()), nbytes,
                                         C.c_void_p(self.stream.cuda_stream), C.byref(h)))
        self._h = h
        self.n_mel = cfg.n_mel
        self.chunk = cfg.chunk_frames
        self._drain = lib().tts_pool_drain_chunk
        self._drain_out = (C.c_int(), C.c_int())
        self._chunk_buffer = (C.c_float * (self.chunk * self.n_mel)).from_buffer

    # -- the five pool calls
    def add_request(self, enc_out, n_steps: int) -> int:
        """enc_out: numpy fp32 [L, enc_dim] (host) or a torch CUDA fp32 tensor (device)."""
        rid = C.c_int64()
        if isinstance(enc_out, np.ndarray):
            a = np.ascontiguousarray(enc_out, dtype=np.float32)
            ptr, L = a.ctypes.data, a.shape[0]
        else:
            # read by work queued on the pool's stream after this call returns: a temporary copy could be gone by then
            a = enc_out
            assert a.is_cuda and a.dtype == self._torch.float32 and a.is_contiguous()
            ptr, L = a.data_ptr(), a.shape[0]
        _check(lib().tts_pool_add_request(self._h, C.c_void_p(ptr), int(L), int(n_steps), C.byref(rid)))
        return rid.value

    def add_requests(self, enc_outs, n_steps) -> list:
        """Several requests in one call; each enc_out as in add_request."""
        n = len(enc_outs)
        keep, ptrs, Ls = [], (C.c_void_p * max(n, 1))(), (C.c_int * max(n, 1))()
        for i, e in enumerate(enc_outs):
            if isinstance(e, np.ndarray):
                a = np.ascontiguousarray(e, dtype=np.float32)
                ptrs[i] = a.ctypes.data
            else:
                a = e
                assert a.is_cuda and a.dtype == self._torch.float32 and a.is_contiguous()
                ptrs[i] = a.data_ptr()
            Ls[i] = a.shape[0]
            keep.append(a)
        ns = (C.c_int * max(n, 1))(*[int(x) for x in n_steps])
        ids = (C.c_int64 * max(n, 1))()
        _check(lib().tts_pool_add_requests(self._h, n, ptrs, Ls, ns, ids))
        return [ids[i] for i in range(n)]

    def add_request_raw(self, ptr: int, L: int, n_steps: int) -> int:
        rid = C.c_int64()
        _check(lib().tts_pool_add_request(self._h, C.c_void_p(ptr), int(L), int(n_steps), C.byref(rid)))
        return rid.value

    def step(self) -> int:
        n = C.c_int()
        _check(lib().tts_pool_step(self._h, C.byref(n)))
        return n.value

    def step_n(self, n: int) -> int:
        frames = C.c_int64()
        _check(lib().tts_pool_step_n(self._h, int(n), C.byref(frames)))
        return frames.value

    def drain_chunk(self, rid: int) -> Tuple[np.ndarray, bool]:
        # called once per request and chunk, right between two segments of steps: the pointers are made once (4.2 -> 1.9 us a call)
        buf = np.empty((self.chunk, self.n_mel), np.float32)
        n, fin = self._drain_out
        rc = self._drain(self._h, rid, C.addressof(self._chunk_buffer(buf)), C.addressof(n), C.addressof(fin))
        if rc != TTS_OK:
            _check(rc)
        n = n.value
        return (buf if n == self.chunk else buf[:n]), fin.value != 0

    def retire(self, rid: int) -> None:
        _check(lib().tts_pool_retire(self._h, rid))

    # -- helpers
    def stop_logits(self, rid: int, first: int, count: int) -> np.ndarray:
        buf = np.empty(count, np.float32)
        _check(lib().tts_pool_get_stop_logits(self._h, rid, first, count, buf.ctypes.data_as(_fp)))
        return buf

    def get_state(self, rid: int, name: str) -> np.ndarray:
        buf = np.empty(max(self.cfg.max_enc_len, 1024), np.float32)
        n = C.c_int()
        _check(lib().tts_pool_get_state(self._h, rid, STATE[name], buf.ctypes.data_as(_fp), buf.shape[0], C.byref(n)))
        return buf[: n.value].copy()

    def set_state(self, rid: int, name: str, value) -> None:
        v = np.ascontiguousarray(value, np.float32).ravel()
        _check(lib().tts_pool_set_state(self._h, rid, STATE[name], v.ctypes.data_as(_fp), v.shape[0]))

    def set_wait_polls(self, polls: int) -> None:
        _check(lib().tts_pool_set_wait_polls(self._h, int(polls)))

    def frames(self, rid: int) -> Tuple[int, bool]:
        n, fin = C.c_int(), C.c_int()
        _check(lib().tts_pool_frames(self._h, rid, C.byref(n), C.byref(fin)))
        return n.value, bool(fin.value)

    def size(self) -> int:
        return lib().tts_pool_size(self._h)

    def n_active(self) -> int:
        return lib().tts_pool_n_active(self._h)

    def span(self) -> int:
        return lib().tts_pool_span(self._h)

    def moves(self) -> int:
        return lib().tts_pool_moves(self._h)

    def segments(self) -> int:
        return lib().tts_pool_segments(self._h)

    def fp32_segments(self) -> int:
        return lib().tts_pool_fp32_segments(self._h)

    def lost(self, rid: int) -> bool:
        """True if the device ended the request early because a step could not be completed for it."""
        v = C.c_int()
        _check(lib().tts_pool_lost(self._h, rid, C.byref(v)))
        return bool(v.value)

    def sync(self) -> None:
        _check(lib().tts_pool_sync(self._h))

    def timing(self, on: bool) -> None:
        _check(lib().tts_pool_timing(self._h, int(on)))

    def elapsed_ms(self) -> float:
        ms = C.c_float()
        _check(lib().tts_pool_elapsed_ms(self._h, C.byref(ms)))
        return ms.value

    KERNEL_NAMES = ("k_lstm_att", "k_lsa", "k_lstm_dec", "k_proj")

    def kernel_times_us(self, n_steps: int) -> Dict[str, float]:
        """Average device time of each kernel over n un-graphed, event-bracketed steps."""
        buf = (C.c_float * 8)()
        nk = C.c_int()
        _check(lib().tts_pool_kernel_times(self._h, int(n_steps), buf, 8, C.byref(nk)))
        out = {self.KERNEL_NAMES[i]: float(buf[i]) for i in range(nk.value)}
        out["event_cost"] = float(buf[nk.value])
        if buf[nk.value + 1] > 0:
            out["k_proj_last_step"] = float(buf[nk.value + 1])
        return out

    def drain_all(self, rid: int) -> np.ndarray:
        """Every remaining frame of a finished request (host convenience loop over drain_chunk)."""
        out = []
        while True:
            chunk, fin = self.drain_chunk(rid)
            if chunk.shape[0]:
                out.append(chunk.copy())
            if fin or chunk.shape[0] == 0:
                break
        return np.concatenate(out, axis=0) if out else np.zeros((0, self.n_mel), np.float32)

    def chunk_window(self, rid: int, context: int, d_dst) -> Tuple[int, int, bool]:
        """Next chunk of `rid` preceded by up to `context` earlier frames, into the CUDA fp32 tensor d_dst
        ([>= context + chunk, n_mel]); returns (context frames copied, chunk frames, finished)."""
        assert d_dst.is_cuda and d_dst.dtype == self._torch.float32 and d_dst.is_contiguous()
        assert d_dst.numel() >= (context + self.chunk) * self.n_mel
        c, n, fin = C.c_int(), C.c_int(), C.c_int()
        _check(lib().tts_pool_chunk_window(self._h, rid, int(context), C.c_void_p(d_dst.data_ptr()), C.byref(c),
                                           C.byref(n), C.byref(fin)))
        return c.value, n.value, bool(fin.value)

    def chunk_windows(self, rids, context: int, d_dst) -> list:
        """chunk_window for several requests with one launch, their windows back to back in d_dst
        ([>= len(rids) * (context + chunk), n_mel]): [(context frames, chunk frames, finished)] of each."""
        n = len(rids)
        assert d_dst.is_cuda and d_dst.dtype == self._torch.float32 and d_dst.is_contiguous()
        assert d_dst.numel() >= n * (context + self.chunk) * self.n_mel
        ids, out = (C.c_int64 * n)(*rids), [(C.c_int * n)() for _ in range(3)]
        _check(lib().tts_pool_chunk_windows(self._h, n, ids, int(context), C.c_void_p(d_dst.data_ptr()), *out))
        return [(c, k, bool(f)) for c, k, f in zip(*out)]

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().tts_pool_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Book:
    """Host-only bookkeeping model (tts_book_*): pooling semantics without a device."""

    def __init__(self, max_pool: int, max_enc_len: int, max_steps: int, chunk_frames: int):
        self._h = lib().tts_book_create(max_pool, max_enc_len, max_steps, chunk_frames)
        if not self._h:
            raise ValueError("tts_book_create rejected its arguments")
        self.max_pool = max_pool

    def add(self, L: int, n_steps: int) -> int:
        rid = C.c_int64()
        _check(lib().tts_book_add(self._h, L, n_steps, C.byref(rid)))
        return rid.value

    def step(self):
        ids = (C.c_int64 * self.max_pool)()
        n = C.c_int()
        _check(lib().tts_book_step(self._h, ids, C.byref(n)))
        return [ids[i] for i in range(n.value)]

    def drain(self, rid: int):
        first, n, fin = C.c_int(), C.c_int(), C.c_int()
        _check(lib().tts_book_drain(self._h, rid, C.byref(first), C.byref(n), C.byref(fin)))
        return first.value, n.value, bool(fin.value)

    def retire(self, rid: int) -> None:
        _check(lib().tts_book_retire(self._h, rid))

    def slot(self, rid: int) -> int:
        return lib().tts_book_slot(self._h, rid)

    def compact(self, min_span: int = 16):
        src, dst = (C.c_int * self.max_pool)(), (C.c_int * self.max_pool)()
        n = lib().tts_book_compact(self._h, min_span, src, dst, self.max_pool)
        _check(min(n, 0))
        return [(src[i], dst[i]) for i in range(n)]

    def close(self):
        if self._h:
            lib().tts_book_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def make_postnet_config(max_columns: int, bf16: bool = False, n_mel: int = 80, channels: int = 512) -> TtsPostnetConfig:
    return TtsPostnetConfig(n_mel, channels, int(max_columns), DTYPE_BF16 if bf16 else DTYPE_F32)


def postnet_workspace_bytes(cfg: TtsPostnetConfig) -> int:
    return int(lib().tts_postnet_workspace_bytes(C.byref(cfg)))


class Postnet:
    """tts_postnet_* calls; owns its torch arena.  `stream` is a torch.cuda.Stream (e.g. a Pool's)."""

    def __init__(self, cfg: TtsPostnetConfig, conv_w, conv_b, stream=None, device: str = "cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the PostNet has no CPU path")
        self._torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = postnet_workspace_bytes(cfg)
        if nbytes == 0:
            _check(TTS_E_INVAL)
        with torch.cuda.device(self.device):
            self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
        self._w = [np.ascontiguousarray(a, np.float32) for a in conv_w]
        self._b = [np.ascontiguousarray(a, np.float32) for a in conv_b]
        w = TtsPostnetWeights((_fp * 5)(*[a.ctypes.data_as(_fp) for a in self._w]),
                              (_fp * 5)(*[a.ctypes.data_as(_fp) for a in self._b]))
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().tts_postnet_create(C.byref(cfg), C.byref(w), C.c_void_p(self.arena.data_ptr()), nbytes,
                                            C.c_void_p(self.stream.cuda_stream), C.byref(h)))
        self._h = h

    def run_device(self, d_mel, win_len, keep_from, d_out, static: bool = False) -> None:
        """d_mel / d_out: CUDA fp32 tensors (packed windows in, packed chunks out); queued on the stream.
        static: tts_postnet_run_static, the call that allocates nothing (its scratch is the library's static array)."""
        wl = np.ascontiguousarray(win_len, np.int32)
        kf = np.ascontiguousarray(keep_from, np.int32)
        assert d_mel.is_cuda and d_out.is_cuda and d_mel.is_contiguous() and d_out.is_contiguous()
        assert d_mel.numel() >= int(wl.sum()) * self.cfg.n_mel and d_out.numel() >= int((wl - kf).sum()) * self.cfg.n_mel
        fn = lib().tts_postnet_run_static if static else lib().tts_postnet_run
        with self._torch.cuda.device(self.device):
            _check(fn(self._h, C.c_void_p(d_mel.data_ptr()), wl.ctypes.data_as(_ip),
                      kf.ctypes.data_as(_ip), int(wl.shape[0]), C.c_void_p(d_out.data_ptr())))

    def run(self, windows, keep_from) -> list:
        """windows: list of numpy [T_i, n_mel]; returns the post-processed chunks as numpy arrays."""
        torch = self._torch
        wl = [int(w.shape[0]) for w in windows]
        packed = np.ascontiguousarray(np.concatenate(windows, axis=0), np.float32)
        n_out = sum(t - k for t, k in zip(wl, keep_from))
        with torch.cuda.stream(self.stream):
            d_in = torch.from_numpy(packed).to(self.device, non_blocking=False)
            d_out = torch.empty((n_out, self.cfg.n_mel), dtype=torch.float32, device=self.device)
        self.stream.synchronize()
        self.run_device(d_in, wl, keep_from, d_out)
        self.stream.synchronize()
        out = d_out.cpu().numpy()
        res, r = [], 0
        for t, k in zip(wl, keep_from):
            res.append(out[r:r + t - k])
            r += t - k
        return res

    def set_wait_polls(self, polls: int) -> None:
        _check(lib().tts_postnet_set_wait_polls(self._h, int(polls)))

    def one_launch_calls(self) -> int:
        return lib().tts_postnet_one_launch_calls(self._h)

    def elapsed_ms(self) -> float:
        ms = C.c_float()
        _check(lib().tts_postnet_elapsed_ms(self._h, C.byref(ms)))
        return ms.value

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().tts_postnet_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def make_vocoder_config(overlap: int, max_chunk: int, max_requests: int, max_batch: int, bf16: bool = False,
                        n_mel: int = 80, c0: int = 128) -> TtsVocoderConfig:
    return TtsVocoderConfig(n_mel, c0, int(overlap), int(max_chunk), int(max_requests), int(max_batch),
                            DTYPE_BF16 if bf16 else DTYPE_F32)


def vocoder_workspace_bytes(cfg: TtsVocoderConfig) -> int:
    return int(lib().tts_vocoder_workspace_bytes(C.byref(cfg)))


class Vocoder:
    """tts_vocoder_* calls; owns its torch arena.  `weights` is the dict of synth.make_vocoder_weights."""

    def __init__(self, cfg: TtsVocoderConfig, weights: dict, stream=None, device: str = "cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the vocoder has no CPU path")
        self._torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = vocoder_workspace_bytes(cfg)
        if nbytes == 0:
            _check(TTS_E_INVAL)
        with torch.cuda.device(self.device):
            self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
        keep = []

        def ptr(a):
            a = np.ascontiguousarray(a, np.float32)
            keep.append(a)
            return a.ctypes.data_as(_fp)

        w = TtsVocoderWeights()
        w.pre_w, w.pre_b, w.post_w, w.post_b = ptr(weights["pre_w"]), ptr(weights["pre_b"]), ptr(weights["post_w"]), ptr(weights["post_b"])
        for s_ in range(4):
            w.up_w[s_], w.up_b[s_] = ptr(weights["up_w"][s_]), ptr(weights["up_b"][s_])
            for b_ in range(3):
                for i in range(6):
                    w.res_w[s_][b_][i] = ptr(weights["res_w"][s_][b_][i])
                    w.res_b[s_][b_][i] = ptr(weights["res_b"][s_][b_][i])
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().tts_vocoder_create(C.byref(cfg), C.byref(w), C.c_void_p(self.arena.data_ptr()), nbytes,
                                            C.c_void_p(self.stream.cuda_stream), C.byref(h)))
        self._h = h

    def run_device(self, d_mel, n_frames, state_slot, flags, d_audio) -> list:
        """d_mel: CUDA fp32 [sum n_frames, n_mel] (the chunks back to back); d_audio: CUDA fp32 (or pinned host memory) with room for
        256 * (overlap + n_frames[i]) samples per chunk.  Queued on the stream; returns the responses' lengths.  Both tensors are the
        caller's to keep until the stream has come this far, pinned memory whichever stream it is used on."""
        nf = np.ascontiguousarray(n_frames, np.int32)
        sl = np.ascontiguousarray(state_slot, np.int32)
        fl = np.ascontiguousarray(flags, np.int32)
        n = int(nf.shape[0])
        assert sl.shape[0] == n and fl.shape[0] == n
        assert d_mel.is_cuda and (d_audio.is_cuda or d_audio.is_pinned()) and d_mel.is_contiguous() and d_audio.is_contiguous()
        assert d_mel.dtype == self._torch.float32 and d_audio.dtype == self._torch.float32
        assert d_mel.numel() >= int(nf.sum()) * self.cfg.n_mel
        assert d_audio.numel() >= int((nf + self.cfg.overlap).sum()) * VOCODER_HOP
        out = np.zeros(n, np.int32)
        _check(lib().tts_vocoder_run(self._h, C.c_void_p(d_mel.data_ptr()), nf.ctypes.data_as(_ip), sl.ctypes.data_as(_ip),
                                     fl.ctypes.data_as(_ip), n, C.c_void_p(d_audio.data_ptr()), out.ctypes.data_as(_ip)))
        return [int(x) for x in out]

    def run(self, chunks, state_slot, flags) -> list:
        """chunks: list of numpy [n_i, n_mel]; returns the responses as numpy arrays."""
        torch = self._torch
        nf = [int(c.shape[0]) for c in chunks]
        packed = np.ascontiguousarray(np.concatenate(chunks, axis=0), np.float32)
        with torch.cuda.stream(self.stream):
            d_in = torch.from_numpy(packed).to(self.device, non_blocking=False)
            d_out = torch.empty(sum(n + self.cfg.overlap for n in nf) * VOCODER_HOP, dtype=torch.float32, device=self.device)
        self.stream.synchronize()
        lens = self.run_device(d_in, nf, state_slot, flags, d_out)
        self.stream.synchronize()
        out = d_out.cpu().numpy()
        res, r = [], 0
        for n in lens:
            res.append(out[r:r + n])
            r += n
        return res

    def elapsed_ms(self) -> float:
        ms = C.c_float()
        _check(lib().tts_vocoder_elapsed_ms(self._h, C.byref(ms)))
        return ms.value

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().tts_vocoder_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def make_encoder_config(max_tokens: int, max_len: int, bf16: bool = False, vocab=(128, 4, 4, 4), dim: int = 512,
                        hid: int = 256) -> TtsEncoderConfig:
    return TtsEncoderConfig(dim, hid, (C.c_int * 4)(*vocab), int(max_tokens), int(max_len), DTYPE_BF16 if bf16 else DTYPE_F32)


def encoder_workspace_bytes(cfg: TtsEncoderConfig) -> int:
    return int(lib().tts_encoder_workspace_bytes(C.byref(cfg)))


class Encoder:
    """tts_encoder_* calls; owns its torch arena.  `weights` is the dict of synth.make_encoder_weights."""

    def __init__(self, cfg: TtsEncoderConfig, weights: dict, stream=None, device: str = "cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the encoder has no CPU path")
        self._torch = torch
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = encoder_workspace_bytes(cfg)
        if nbytes == 0:
            _check(TTS_E_INVAL)
        with torch.cuda.device(self.device):
            self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
        keep = []

        def ptr(a):
            a = np.ascontiguousarray(a, np.float32)
            keep.append(a)
            return a.ctypes.data_as(_fp)

        w = TtsEncoderWeights()
        for t in range(4):
            w.tables[t] = ptr(weights["tables"][t])
        for i in range(3):
            w.conv_w[i], w.conv_b[i] = ptr(weights["conv_w"][i]), ptr(weights["conv_b"][i])
        for d, k in enumerate(("f", "b")):
            w.w_ih[d], w.w_hh[d], w.b[d] = ptr(weights["w_ih_" + k]), ptr(weights["w_hh_" + k]), ptr(weights["b_" + k])
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().tts_encoder_create(C.byref(cfg), C.byref(w), C.c_void_p(self.arena.data_ptr()), nbytes,
                                            C.c_void_p(self.stream.cuda_stream), C.byref(h)))
        self._h = h

    def run_device(self, ids_list, d_out) -> list:
        """ids_list: one int array [4, L_i] per request; d_out: CUDA fp32 [>= sum L_i, 2 hid].  Queued on the stream;
        returns the first row of every request in d_out."""
        lens = np.ascontiguousarray([a.shape[1] for a in ids_list], np.int32)
        ids = np.ascontiguousarray(np.concatenate([np.asarray(a, np.int32) for a in ids_list], axis=1))   # [4, total]
        total = int(lens.sum())
        assert ids.shape == (4, total)
        assert d_out.is_cuda and d_out.is_contiguous() and d_out.dtype == self._torch.float32
        assert d_out.numel() >= total * 2 * self.cfg.hid
        _check(lib().tts_encoder_run(self._h, ids.ctypes.data_as(_ip), lens.ctypes.data_as(_ip), int(lens.shape[0]),
                                     C.c_void_p(d_out.data_ptr())))
        return [int(x) for x in np.concatenate([[0], np.cumsum(lens)[:-1]])]

    def set_wait_polls(self, polls: int) -> None:
        _check(lib().tts_encoder_set_wait_polls(self._h, int(polls)))

    def one_launch_calls(self) -> int:
        return lib().tts_encoder_one_launch_calls(self._h)

    def run(self, ids_list) -> list:
        """Returns F_enc of every request as numpy [L_i, 2 hid]."""
        torch = self._torch
        total = sum(a.shape[1] for a in ids_list)
        with torch.cuda.stream(self.stream):
            d_out = torch.empty((max(total, 1), 2 * self.cfg.hid), dtype=torch.float32, device=self.device)
        self.stream.synchronize()
        starts = self.run_device(ids_list, d_out)
        self.stream.synchronize()
        out = d_out.cpu().numpy()
        return [out[s:s + a.shape[1]] for s, a in zip(starts, ids_list)]

    def elapsed_ms(self) -> float:
        ms = C.c_float()
        _check(lib().tts_encoder_elapsed_ms(self._h, C.byref(ms)))
        return ms.value

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().tts_encoder_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


SCALE_BLOCK = 128         # columns of an 8-bit row under one scale
NORM_RMS, NORM_NONE = 0, 1
MAX_ROWS = 1 << 24        # of one call


def width8(dim: int) -> int:
    """Columns of an 8-bit row: whole blocks of 128."""
    return -(-dim // SCALE_BLOCK) * SCALE_BLOCK


def scale_columns(dim: int) -> int:
    """Scales of an 8-bit row: whole words of four."""
    return -(-width8(dim) // (4 * SCALE_BLOCK)) * 4


class _Operator:
    """An object on a stream with an arena of its own, as the modules above have them.  Calls are queued on that stream (None: a new one) whichever is current, and wait for no other: what a call
    reads has to be there in that stream's order, and its tensors are the caller's to keep until the stream has come this far."""

    _name = ""

    def _setup(self, cfg, stream, device):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError(f"no GPU visible: tts_{self._name} has no CPU path")
        self._torch = torch
        self.cfg = cfg
        d = torch.device(device)
        if d.type != "cuda":
            raise ValueError(f"{device}: a GPU is wanted")
        self._index = torch.cuda.current_device() if d.index is None else d.index
        self.device = torch.device("cuda", self._index)
        if stream is not None and stream.device != self.device:
            raise ValueError(f"a stream of {stream.device} for an object on {self.device}")
        nbytes = int(getattr(lib(), f"tts_{self._name}_workspace_bytes")(C.byref(cfg)))
        if nbytes == 0:
            raise TtsError(TTS_E_INVAL, lib().tts_last_error().decode("utf-8", "replace"))
        with torch.cuda.device(self.device):
            self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
            torch.cuda.current_stream().synchronize()      # (the arena's memory may have been in use on this stream)
            self.arena.record_stream(self.stream)          # (an object may go while its last calls are under way: its memory is not handed on before they end)
        self._handle = C.c_void_p()
        self._run = getattr(lib(), f"tts_{self._name}_run")
        return C.c_void_p(self.arena.data_ptr()), nbytes, C.c_void_p(self.stream.cuda_stream), C.byref(self._handle)

    def _type(self, dtype: int):
        return self._torch.bfloat16 if dtype == DTYPE_BF16 else self._torch.float32

    # (the checks of a call's tensors are half of what it costs the host: one function a tensor, cheapest questions first)
    def _at(self, t, name, dtype, count) -> int:
        """Address of a tensor of this device and type with so many elements, back to back."""
        if t.dtype is not dtype or t.get_device() != self._index or t.numel() != count or not t.is_contiguous():
            raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype} on {t.device} where {count} elements, back to back, of {dtype} on {self.device} are wanted")
        return t.data_ptr()

    def _rows(self, t, name, dtype, count, rows):
        """(address, distance of the rows) of one whose rows, along its first dimension, may lie apart; 0: all elements lie back to back."""
        if t.dtype is dtype and t.get_device() == self._index and t.numel() == count:
            if t.is_contiguous():
                return t.data_ptr(), 0
            if t.shape[0] == rows and t.stride(0) > 0 and t[0].is_contiguous():
                return t.data_ptr(), t.stride(0)
        raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype} on {t.device} where {rows} rows, back to back each, of {count} elements in all, {dtype} on {self.device} are wanted")

    def close(self) -> None:
        if getattr(self, "_handle", None):
            getattr(lib(), f"tts_{self._name}_destroy")(self._handle)
            self._handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def make_norm_config(dim: int, x_bf16: bool = False, res_bf16: bool = False, y_bf16: bool = False, eps: float = 1e-5,
                     kind: int = NORM_RMS) -> TtsNormConfig:
    pick = lambda b: DTYPE_BF16 if b else DTYPE_F32   # noqa: E731
    return TtsNormConfig(int(dim), int(kind), pick(x_bf16), pick(res_bf16), pick(y_bf16), float(eps))


class Norm(_Operator):
    """tts_norm_* calls: residual's addition, root-mean-square norm (kind NORM_NONE: none) and output in 8 bits with scales."""

    _name = "norm"

    def __init__(self, cfg: TtsNormConfig, gain=None, stream=None, device: str = "cuda:0"):
        where = self._setup(cfg, stream, device)
        g = None if gain is None else np.ascontiguousarray(gain, np.float32)
        if g is not None and g.shape != (cfg.dim,):
            raise ValueError(f"gain: {g.shape} where ({cfg.dim},) is wanted")
        _check(lib().tts_norm_create(C.byref(cfg), None if g is None else g.ctypes.data_as(_fp), *where))
        self._types = [self._type(t) for t in (cfg.x_dtype, cfg.res_dtype, cfg.y_dtype)]
        self._dim, self._widths, self._types8 = cfg.dim, (width8(cfg.dim), scale_columns(cfg.dim)), (self._torch.float8_e4m3fn, self._torch.float8_e8m0fnu)

    def run_device(self, x, res=None, total=None, y=None, y8=None, scales=None) -> None:
        """x, res, total, y: CUDA [rows, dim] of the configuration's types, rows any distance apart; y8: float8_e4m3fn [rows, width8(dim)],
        scales: float8_e8m0fnu [rows, scale_columns(dim)].  Those that are None are not there.  Queued on the object's stream."""
        x_type, res_type, y_type = self._types
        count = x.numel()
        rows, rest = divmod(count, self._dim)
        if rest or rows > MAX_ROWS:
            raise ValueError(f"x: {tuple(x.shape)} where rows of {self._dim}, {MAX_ROWS} at most, are wanted")
        a = TtsNormRows()
        a.rows = rows
        a.x, a.x_stride = self._rows(x, "x", x_type, count, rows)
        if res is not None:
            a.res, a.res_stride = self._rows(res, "res", res_type, count, rows)
        if total is not None:
            a.total, a.total_stride = self._rows(total, "total", res_type, count, rows)
        if y is not None:
            a.y, a.y_stride = self._rows(y, "y", y_type, count, rows)
        if y8 is not None:
            a.y8 = self._at(y8, "y8", self._types8[0], rows * self._widths[0])
        if scales is not None:
            a.scales = self._at(scales, "scales", self._types8[1], rows * self._widths[1])
        rc = self._run(self._handle, a)
        if rc:
            _check(rc)


def make_linear8_config(in_dim: int, out_dim: int, bf16: bool = False) -> TtsLinear8Config:
    return TtsLinear8Config(int(in_dim), int(out_dim), DTYPE_BF16 if bf16 else DTYPE_F32)


class Linear8(_Operator):
    """tts_linear8_* calls: the product of 8-bit rows with 8-bit weights, a scale for each 128 columns.  w: fp32 [out_dim, in_dim] (host)."""

    _name = "linear8"

    def __init__(self, cfg: TtsLinear8Config, w, bias=None, stream=None, device: str = "cuda:0"):
        where = self._setup(cfg, stream, device)
        w = np.ascontiguousarray(w, np.float32)
        b = None if bias is None else np.ascontiguousarray(bias, np.float32)
        if w.shape != (cfg.out_dim, cfg.in_dim) or (b is not None and b.shape != (cfg.out_dim,)):
            raise ValueError(f"w: {w.shape}, bias: {None if b is None else b.shape} where {(cfg.out_dim, cfg.in_dim)} and {(cfg.out_dim,)} are wanted")
        _check(lib().tts_linear8_create(C.byref(cfg), w.ctypes.data_as(_fp), None if b is None else b.ctypes.data_as(_fp), *where))
        self._y_type = self._type(cfg.y_dtype)
        self._widths, self._types8 = (width8(cfg.in_dim), scale_columns(cfg.in_dim), cfg.out_dim), (self._torch.float8_e4m3fn, self._torch.float8_e8m0fnu)

    def run_device(self, x8, scales, y) -> None:
        """x8: CUDA float8_e4m3fn [rows, width8(in_dim)], zeros past in_dim; scales: float8_e8m0fnu [rows, scale_columns(in_dim)]; y: [rows, out_dim],
        rows any distance apart.  Queued on the object's stream."""
        k, n_scales, n = self._widths
        rows = x8.numel() // k
        at = self._at(x8, "x8", self._types8[0], rows * k)
        sx = self._at(scales, "scales", self._types8[1], rows * n_scales)
        to, apart = self._rows(y, "y", self._y_type, rows * n, rows)
        rc = self._run(self._handle, at, sx, rows, to, apart)
        if rc:
            _check(rc)


def make_cross_config(n_heads: int, n_kv_heads: int, head_dim: int, bf16: bool = False) -> TtsCrossConfig:
    return TtsCrossConfig(int(n_heads), int(n_kv_heads), int(head_dim), DTYPE_BF16 if bf16 else DTYPE_F32)


class CrossBatch:
    """The lengths of a dynamic batch: queries, first memory row and memory rows of every request."""

    def __init__(self, q_len, mem_row, mem_len):
        n = len(q_len)
        if len(mem_row) != n or len(mem_len) != n:
            raise ValueError("q_len, mem_row and mem_len have a value for each request")
        self._keep = tuple(self._array(t, name, v) for t, name, v in ((C.c_int, "q_len", q_len), (C.c_longlong, "mem_row", mem_row), (C.c_int, "mem_len", mem_len)))
        self.queries = sum(self._keep[0])
        self.memory_rows = max((r + m for r, m in zip(self._keep[1], self._keep[2]) if m > 0), default=0)      # that k and v have to have
        self.c = TtsCrossBatch(n, *self._keep)

    @staticmethod
    def _array(ctype, name, values):
        values = [int(v) for v in values]
        a = (ctype * len(values))(*values)
        if list(a) != values:                 # (ctypes takes a number's low bits)
            raise ValueError(f"{name}: a number that {8 * C.sizeof(ctype)} bits do not hold")
        return a


class CrossAttention(_Operator):
    """tts_cross_* calls: attention of a dynamic batch's queries to its requests' memories."""

    _name = "cross"

    def __init__(self, cfg: TtsCrossConfig, stream=None, device: str = "cuda:0"):
        where = self._setup(cfg, stream, device)
        _check(lib().tts_cross_create(C.byref(cfg), *where))
        self._dtype = self._type(cfg.dtype)
        self._widths = (cfg.n_heads, cfg.n_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim)

    def batch(self, q_len, mem_row, mem_len) -> CrossBatch:
        """A batch's lengths, for any number of calls."""
        return CrossBatch(q_len, mem_row, mem_len)

    def run_device(self, batch: CrossBatch, q, k, v, out, keep=None, lse=None, scale: float = 0.0) -> None:
        """q, out: CUDA [queries, n_heads, head_dim]; k, v: [memory rows, n_kv_heads, head_dim], rows any multiple of 8 elements apart, or None where no
        request has a memory; keep: uint8 [memory rows], 0 = hidden; lse: fp32 [queries, n_heads].  Queued on the object's stream; scale 0: 1 / sqrt(head_dim)."""
        t, (heads, of_q, of_k) = self._dtype, self._widths
        if (k is None) != (v is None):
            raise ValueError("k and v come together")
        queries, rows = batch.queries, 0 if k is None else k.numel() // of_k
        if rows < batch.memory_rows:
            raise ValueError(f"k has {rows} rows, the batch's memories end at {batch.memory_rows}")
        a = TtsCrossTensors()
        a.q, a.q_stride = self._rows(q, "q", t, queries * of_q, queries)
        if k is not None:
            a.k, a.k_stride = self._rows(k, "k", t, rows * of_k, rows)
            a.v, a.v_stride = self._rows(v, "v", t, rows * of_k, rows)
        a.out, a.out_stride = self._rows(out, "out", t, queries * of_q, queries)
        if keep is not None:
            a.keep = self._at(keep, "keep", self._torch.uint8, rows)
        if lse is not None:
            a.lse = self._at(lse, "lse", self._torch.float32, queries * heads)
        a.scale = scale
        if scale and not a.scale:
            raise ValueError(f"a scale of {scale} is 0 in fp32")
        rc = self._run(self._handle, batch.c, a)
        if rc:
            _check(rc)


ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS = 0, 1, 2, 3
ROTARY_MAX_ROWS = 1 << 24  # of one call


def make_rotary_angles(rot_dim: int, pairs: bool = False, base: float = 10000.0, scaling: int = ROTARY_PLAIN, factor: float = 1.0, trained_len: int = 0, low: float = 1.0, high: float = 32.0,
                       magnitude: float = 1.0) -> TtsRotaryAngles:
    return TtsRotaryAngles(int(rot_dim), int(bool(pairs)), int(scaling), int(trained_len), float(base), float(factor), float(low), float(high), float(magnitude))


def make_rotary_config(n_heads: int, head_dim: int, angles: TtsRotaryAngles, x_bf16: bool = False, y_bf16: bool = False) -> TtsRotaryConfig:
    pick = lambda b: DTYPE_BF16 if b else DTYPE_F32   # noqa: E731
    return TtsRotaryConfig(int(n_heads), int(head_dim), pick(x_bf16), pick(y_bf16), angles)


class Rotary(_Operator):
    """tts_rotary_* calls: heads' columns turned in pairs to their rows' positions."""

    _name = "rotary"

    def __init__(self, cfg: TtsRotaryConfig, stream=None, device: str = "cuda:0"):
        where = self._setup(cfg, stream, device)
        _check(lib().tts_rotary_create(C.byref(cfg), *where))
        self._types = (self._type(cfg.x_dtype), self._type(cfg.y_dtype), self._torch.int32)
        self._width = cfg.n_heads * cfg.head_dim

    def run_device(self, x, y, positions=None, first: int = 0, back: bool = False) -> None:
        """x, y: CUDA [rows, n_heads, head_dim] of the configuration's types, rows any multiple of 8 elements apart; y may be x.  positions: int32 [rows], or None: row r is at
        first + r.  back: the other way, as the gradient is.  Queued on the object's stream."""
        count = x.numel()
        rows, rest = divmod(count, self._width)
        if rest or rows > ROTARY_MAX_ROWS:
            raise ValueError(f"x: {tuple(x.shape)} where rows of {self._width}, {ROTARY_MAX_ROWS} at most, are wanted")
        a = TtsRotaryRows()
        a.rows = rows
        a.x, a.x_stride = self._rows(x, "x", self._types[0], count, rows)
        a.y, a.y_stride = self._rows(y, "y", self._types[1], count, rows)
        if positions is not None:
            a.positions = self._at(positions, "positions", self._types[2], rows)
        elif not -(1 << 31) <= first < 1 << 31:
            raise ValueError(f"first: {first} is a number that 32 bits do not hold")
        else:
            a.first = first
        a.back = bool(back)
        rc = self._run(self._handle, a)
        if rc:
            _check(rc)


def make_cache_config(n_kv_heads: int, head_dim: int, page_rows: int, angles: Optional[TtsRotaryAngles] = None, n_heads: int = 0, bf16: bool = False, x_bf16: bool = False) -> TtsCacheConfig:
    """angles None: nothing turns; n_heads 0: no queries come along."""
    pick = lambda b: DTYPE_BF16 if b else DTYPE_F32   # noqa: E731
    return TtsCacheConfig(int(n_kv_heads), int(n_heads), int(head_dim), int(page_rows), pick(x_bf16), pick(bf16), angles if angles is not None else TtsRotaryAngles())


class CacheBatch:
    """The numbers of a dynamic batch's new rows: how many, where the first of them goes, the sequence's row of the table, the first one's position (None: where it goes)."""

    def __init__(self, length, row, table_row, position=None):
        n = len(length)
        if len(row) != n or len(table_row) != n or (position is not None and len(position) != n):
            raise ValueError("length, row, table_row and position have a value for each request")
        self._keep = [None if v is None else CrossBatch._array(C.c_int, name, v) for name, v in (("length", length), ("row", row), ("table_row", table_row), ("position", position))]
        self.rows = sum(self._keep[0])
        self.c = TtsCacheBatch(n, *self._keep)


class _Paged(_Operator):
    """An operator on a paged cache."""

    def _setup_pages(self, cfg):
        self._pages_type, self._int = self._type(cfg.dtype), self._torch.int32
        self._page = cfg.n_kv_heads * cfg.page_rows * cfg.head_dim

    def _pages(self, a, k_pages, v_pages, table) -> None:
        n, rest = divmod(k_pages.numel(), self._page)
        if rest or n >= 1 << 31:
            raise ValueError(f"k_pages: {tuple(k_pages.shape)} where pages of {self._page} elements are wanted")
        a.k_pages, a.page_stride = self._rows(k_pages, "k_pages", self._pages_type, n * self._page, n)
        a.v_pages, v_stride = self._rows(v_pages, "v_pages", self._pages_type, n * self._page, n)
        if n > 1 and (a.page_stride or self._page) != (v_stride or self._page):
            raise ValueError(f"pages of keys lie {a.page_stride or self._page} elements apart, those of values {v_stride or self._page}")
        if table.dim() != 2 or table.shape[0] >= 1 << 31 or table.shape[1] >= 1 << 31:
            raise ValueError(f"table: {tuple(table.shape)} where [sequences, pages] is wanted")
        a.n_pages, (a.table_rows, a.table_cols) = n, table.shape
        a.table = self._at(table, "table", self._int, table.numel())


class Cache(_Paged):
    """tts_cache_* calls: new rows of keys (turned to their positions) and values on their way to a paged cache, queries beside them."""

    _name = "cache"

    def __init__(self, cfg: TtsCacheConfig, stream=None, device: str = "cuda:0"):
        where = self._setup(cfg, stream, device)
        _check(lib().tts_cache_create(C.byref(cfg), *where))
        self._setup_pages(cfg)
        self._x_type, self._widths = self._type(cfg.x_dtype), (cfg.n_kv_heads * cfg.head_dim, cfg.n_heads * cfg.head_dim)

    def batch(self, length, row, table_row, position=None) -> CacheBatch:
        """A batch's numbers, for any number of calls."""
        return CacheBatch(length, row, table_row, position)

    def run_device(self, batch: CacheBatch, k, v, k_pages, v_pages, table, q=None, q_out=None) -> None:
        """k, v: CUDA [new rows, n_kv_heads, head_dim], q: [new rows, n_heads, head_dim], rows any multiple of 8 elements apart; q_out: as q, of the cache's type (or q itself);
        k_pages, v_pages: [pages, n_kv_heads, page_rows, head_dim], pages any multiple of 8 elements apart; table: int32 [sequences, pages], other numbers than 0 .. pages - 1 for
        what is no page.  Queued on the object's stream."""
        if (q is None) != (q_out is None):
            raise ValueError("q and q_out come together")
        rows, (of_k, of_q) = batch.rows, self._widths
        a = TtsCacheTensors()
        a.k, a.k_stride = self._rows(k, "k", self._x_type, rows * of_k, rows)
        a.v, a.v_stride = self._rows(v, "v", self._x_type, rows * of_k, rows)
        if q is not None:
            a.q, a.q_stride = self._rows(q, "q", self._x_type, rows * of_q, rows)
            a.q_out, a.q_out_stride = self._rows(q_out, "q_out", self._pages_type, rows * of_q, rows)
        self._pages(a, k_pages, v_pages, table)
        rc = self._run(self._handle, batch.c, a)
        if rc:
            _check(rc)


def make_paged_config(n_heads: int, n_kv_heads: int, head_dim: int, page_rows: int, bf16: bool = False, causal: bool = True) -> TtsPagedConfig:
    return TtsPagedConfig(int(n_heads), int(n_kv_heads), int(head_dim), int(page_rows), DTYPE_BF16 if bf16 else DTYPE_F32, int(bool(causal)))


class PagedBatch:
    """The numbers of a dynamic batch over a paged cache: of every request its queries, its own rows there, its row of the table and its prefix (-1, or None for all: none); of every
    prefix its rows and its row of the table."""

    def __init__(self, q_len, own_len, table_row, prefix=None, prefix_len=(), prefix_table_row=()):
        n = len(q_len)
        if len(own_len) != n or len(table_row) != n or (prefix is not None and len(prefix) != n):
            raise ValueError("q_len, own_len, table_row and prefix have a value for each request")
        if len(prefix_len) != len(prefix_table_row):
            raise ValueError("prefix_len and prefix_table_row have a value for each prefix")
        q, own, row, of, length, at = [None if v is None else CrossBatch._array(C.c_int, name, v) for name, v in (("q_len", q_len), ("own_len", own_len), ("table_row", table_row), ("prefix", prefix),
                                                                                                            ("prefix_len", prefix_len), ("prefix_table_row", prefix_table_row))]
        self.queries = sum(q)
        self.c = TtsPagedBatch(n, q, own, row, of, len(length), length, at)      # (which keeps its arrays)


class PagedAttention(_Paged):
    """tts_paged_* calls: attention of a dynamic batch to its own rows, and to prefixes that requests share, in a paged cache."""

    _name = "paged"

    def __init__(self, cfg: TtsPagedConfig, stream=None, device: str = "cuda:0"):
        where = self._setup(cfg, stream, device)
        _check(lib().tts_paged_create(C.byref(cfg), *where))
        self._setup_pages(cfg)
        self._widths = (cfg.n_heads, cfg.n_heads * cfg.head_dim)

    def batch(self, q_len, own_len, table_row, prefix=None, prefix_len=(), prefix_table_row=()) -> PagedBatch:
        """A batch's numbers, for any number of calls."""
        return PagedBatch(q_len, own_len, table_row, prefix, prefix_len, prefix_table_row)

    def run_device(self, batch: PagedBatch, q, k_pages, v_pages, table, out, lse=None, scale: float = 0.0) -> None:
        """q, out: CUDA [queries, n_heads, head_dim], rows any multiple of 8 elements apart; k_pages, v_pages: [pages, n_kv_heads, page_rows, head_dim], pages any multiple of 8 elements apart;
        table: int32 [sequences, pages], other numbers than 0 .. pages - 1 for what is no page; lse: fp32 [queries, n_heads].  Queued on the object's stream; scale 0:
        1 / sqrt(head_dim)."""
        queries, (heads, of_q) = batch.queries, self._widths
        a = TtsPagedTensors()
        a.q, a.q_stride = self._rows(q, "q", self._pages_type, queries * of_q, queries)
        a.out, a.out_stride = self._rows(out, "out", self._pages_type, queries * of_q, queries)
        self._pages(a, k_pages, v_pages, table)
        if lse is not None:
            a.lse = self._at(lse, "lse", self._torch.float32, queries * heads)
        a.scale = scale
        if scale and not a.scale:
            raise ValueError(f"a scale of {scale} is 0 in fp32")
        rc = self._run(self._handle, batch.c, a)
        if rc:
            _check(rc)
