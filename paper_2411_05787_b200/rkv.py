"""Thin ctypes binding of librkv.so: argument marshalling only.

Every step of the RefreshKV decode path runs inside the CUDA library; this
module turns torch tensors into device pointers and checks status codes.
torch is used for device memory and streams only.  There is no fallback: if
the shared library is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librkv.so")

RKV_OK = 0
AGG_MAX, AGG_MEAN, AGG_FIRST = 0, 1, 2
DEV_APPEND_OVERFLOW, DEV_LEN_CLAMPED, DEV_NONFINITE, DEV_BAD_INDEX, DEV_TIMEOUT = 1, 2, 4, 8, 16
DEV_BAD_LAYOUT = 32

EXPORTS = ["rkv_create", "rkv_destroy", "rkv_workspace_bytes", "rkv_full_step", "rkv_gather_small",
           "rkv_small_step", "rkv_append", "rkv_should_refresh", "rkv_get_device_status",
           "rkv_status_string", "rkv_last_cuda_error", "rkv_launch_count", "rkv_set_profiling", "rkv_get_profile",
           "rkv_set_option", "rkv_small_step_noalloc", "rkv_append_small_step", "rkv_score_step",
           "rkv_gather_small_evict", "rkv_append_small_step_evict", "rkv_full_attention", "rkv_select_topk",
           "rkv_append_full_attention", "rkv_get_option", "rkv_score_keys", "rkv_quant_store",
           "rkv_quant_full_attention", "rkv_quant_score_keys", "rkv_quant_select_topk", "rkv_quant_full_step",
           "rkv_quant_gather_small", "rkv_rope_frequencies", "rkv_rope"]
QUANT_BLOCK = 64
NOALLOC_MAX_PROBLEMS, NOALLOC_MAX_LEN = 32, 65536
OPT_SMALL_MIN_CHUNK, OPT_DEPENDENT_LAUNCH, OPT_SMALL_CLUSTER, OPT_EARLY_CACHE_READ, OPT_INTERLEAVE_TILES = 1, 2, 3, 4, 5
OPT_SELECT_KEYS_PER_CTA = 6
OPT_SCORE_SLICE = 7
KERNEL_NAMES = ["attn_full", "select", "attn_small", "gather", "append", "trigger", "fold", "score", "rope"]


class RkvConfig(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("max_len", ctypes.c_int32), ("max_small", ctypes.c_int32),
                ("agg", ctypes.c_int32), ("pool_kernel", ctypes.c_int32), ("softmax_scale", ctypes.c_float)]


class RkvCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_rows", ctypes.c_int64),
                ("row_offset", ctypes.c_void_p), ("cap", ctypes.c_void_p), ("len", ctypes.c_void_p)]


class RkvQuantCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_rows", ctypes.c_int64), ("row_offset", ctypes.c_void_p), ("cap", ctypes.c_void_p),
                ("len", ctypes.c_void_p)]


class RkvRopeConfig(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("scaling", ctypes.c_int32), ("theta", ctypes.c_double),
                ("factor", ctypes.c_double), ("trained_len", ctypes.c_int32), ("low", ctypes.c_double),
                ("high", ctypes.c_double), ("fast", ctypes.c_double), ("slow", ctypes.c_double)]


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "bands": 2, "ramp": 3}


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it first (python -m paper_2411_05787_b200.build); "
                          "there is no CPU or PyTorch fallback for this library")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    cfgp, cachep = ctypes.POINTER(RkvConfig), ctypes.POINTER(RkvCache)
    lib.rkv_create.argtypes = [cfgp, ctypes.POINTER(vp)]
    lib.rkv_destroy.argtypes = [vp]
    lib.rkv_workspace_bytes.argtypes = [cfgp]
    lib.rkv_workspace_bytes.restype = ctypes.c_size_t
    lib.rkv_full_step.argtypes = [vp, vp, cachep, vp, i32, vp, vp, vp, i64, vp, vp, i32, vp]
    lib.rkv_gather_small_evict.argtypes = [vp, vp, vp, i32, cachep, cachep, vp, vp, vp, i32, vp]
    lib.rkv_gather_small_evict.restype = i32
    lib.rkv_append_small_step_evict.argtypes = [vp, vp, vp, vp, cachep, cachep, vp, vp, vp, vp, vp, i32, i32, vp]
    lib.rkv_append_small_step_evict.restype = i32
    lib.rkv_score_step.argtypes = [vp, vp, cachep, vp, i32, vp, vp, i64, vp, vp, i32, vp]
    lib.rkv_score_step.restype = i32
    lib.rkv_full_attention.argtypes = [vp, vp, cachep, vp, vp, i32, vp]
    lib.rkv_full_attention.restype = i32
    lib.rkv_append_full_attention.argtypes = [vp, vp, vp, vp, cachep, vp, vp, i32, vp]
    lib.rkv_append_full_attention.restype = i32
    lib.rkv_select_topk.argtypes = [vp, vp, cachep, vp, i32, vp, vp, i64, vp, vp, vp]
    lib.rkv_select_topk.restype = i32
    lib.rkv_score_keys.argtypes = [vp, vp, cachep, vp, i32, vp, vp, i64, vp, vp]
    lib.rkv_score_keys.restype = i32
    lib.rkv_gather_small.argtypes = [vp, vp, vp, i32, cachep, cachep, vp, vp]
    lib.rkv_small_step.argtypes = [vp, vp, cachep, vp, vp, i32, vp]
    lib.rkv_append.argtypes = [vp, vp, vp, cachep, cachep, vp]
    lib.rkv_append_small_step.argtypes = [vp, vp, vp, vp, cachep, cachep, vp, vp, i32, vp]
    lib.rkv_append_small_step.restype = i32
    lib.rkv_should_refresh.argtypes = [vp, vp, vp, f32, vp, vp, vp, vp]
    lib.rkv_get_device_status.argtypes = [vp, ctypes.POINTER(i32), vp]
    lib.rkv_status_string.argtypes = [i32]
    lib.rkv_status_string.restype = ctypes.c_char_p
    lib.rkv_last_cuda_error.argtypes = [vp]
    lib.rkv_last_cuda_error.restype = ctypes.c_char_p
    lib.rkv_launch_count.argtypes = [vp]
    lib.rkv_launch_count.restype = i64
    lib.rkv_set_option.argtypes = [vp, i32, i32]
    lib.rkv_set_option.restype = i32
    lib.rkv_get_option.argtypes = [vp, i32, ctypes.POINTER(i32)]
    lib.rkv_get_option.restype = i32
    lib.rkv_set_profiling.argtypes = [vp, i32]
    lib.rkv_set_profiling.restype = i32
    lib.rkv_get_profile.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
    lib.rkv_get_profile.restype = i32
    lib.rkv_small_step_noalloc.argtypes = [cfgp, vp, cachep, vp, vp, i32, vp, vp, ctypes.c_char_p, ctypes.c_size_t]
    lib.rkv_small_step_noalloc.restype = i32
    quantp = ctypes.POINTER(RkvQuantCache)
    lib.rkv_quant_store.argtypes = [vp, vp, i64, i64, vp, i64, i64, i32, vp, vp, quantp, vp]
    lib.rkv_quant_full_attention.argtypes = [vp, vp, quantp, vp, vp, i32, i32, vp]
    lib.rkv_quant_score_keys.argtypes = [vp, vp, quantp, vp, i32, vp, vp, i64, vp, vp]
    lib.rkv_quant_select_topk.argtypes = [vp, vp, quantp, vp, i32, vp, vp, i64, vp, vp, vp]
    lib.rkv_quant_full_step.argtypes = [vp, vp, quantp, vp, i32, vp, vp, vp, i64, vp, vp, i32, vp]
    lib.rkv_quant_gather_small.argtypes = [vp, vp, vp, i32, quantp, cachep, vp, vp]
    lib.rkv_rope_frequencies.argtypes = [ctypes.POINTER(RkvRopeConfig), ctypes.POINTER(ctypes.c_uint64),
                                         ctypes.POINTER(f32)]
    lib.rkv_rope.argtypes = [vp, vp, i32, i64, vp, i32, i32, i32, vp, i32, i32, f32, vp, vp, vp, vp]
    for name in ("rkv_rope_frequencies", "rkv_rope", "rkv_quant_store", "rkv_quant_full_attention", "rkv_quant_score_keys", "rkv_quant_select_topk",
                 "rkv_quant_full_step", "rkv_quant_gather_small"):
        getattr(lib, name).restype = i32
    for name in ("rkv_create", "rkv_destroy", "rkv_full_step", "rkv_gather_small", "rkv_small_step",
                 "rkv_append", "rkv_should_refresh", "rkv_get_device_status"):
        getattr(lib, name).restype = i32
    return lib


lib = _load()


class RkvError(RuntimeError):
    def __init__(self, code: int, detail: str = ""):
        self.code = code
        msg = lib.rkv_status_string(code).decode()
        super().__init__(f"rkv status {code} ({msg}){': ' + detail if detail else ''}")


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("librkv takes device tensors")
    if not t.is_contiguous():
        raise ValueError("librkv takes contiguous tensors")
    return t.data_ptr()


def _current_device() -> int:
    return torch.cuda.current_device()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def cache_struct(k, v, row_offset, cap, length) -> RkvCache:
    """Describe a packed K/V cache (see include/rkv.h).  The caller keeps the tensors alive."""
    assert k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16 and k.shape == v.shape and k.shape[-1] == 128
    assert row_offset.dtype == torch.int64 and cap.dtype == torch.int32 and length.dtype == torch.int32
    c = RkvCache(_ptr(k), _ptr(v), k.numel() // 128, _ptr(row_offset), _ptr(cap), _ptr(length))
    # what the 8-bit cache's rebuild checks: the GPU of all of these tensors (-1: more than one), the sequences they describe
    c.device = k.device.index if all(t.device == k.device for t in (v, row_offset, cap, length)) else -1
    c.n_seq = min(row_offset.numel(), cap.numel(), length.numel())
    return c


def quant_cache_struct(k8, v8, k_scale, v_scale, row_offset, cap, length) -> RkvQuantCache:
    """Describe a packed 8-bit K/V cache (see include/rkv.h).  The caller keeps the tensors alive.

    k8, v8: float8_e4m3fn (or uint8 codes) [n_rows, 128], n_rows a multiple of 64; scales: float32 [n_rows / 64];
    row_offset and cap hold multiples of 64 (checked on the device: DEV_BAD_LAYOUT)."""
    for t in (k8, v8):
        if t.dtype not in (torch.float8_e4m3fn, torch.uint8) or t.dim() != 2 or t.shape[1] != 128:
            raise ValueError("k8 and v8 are float8_e4m3fn or uint8 tensors [n_rows, 128]")
    n_rows = k8.shape[0]
    if v8.shape[0] != n_rows or n_rows == 0 or n_rows % QUANT_BLOCK != 0:
        raise ValueError("k8 and v8 have the same number of rows, a multiple of 64")
    for t in (k_scale, v_scale):
        if t.dtype != torch.float32 or t.numel() != n_rows // QUANT_BLOCK:
            raise ValueError("scales are float32 tensors with one element per 64 rows")
    if row_offset.dtype != torch.int64 or cap.dtype != torch.int32 or length.dtype != torch.int32:
        raise ValueError("row_offset is int64, cap and length are int32")
    c = RkvQuantCache(_ptr(k8), _ptr(v8), _ptr(k_scale), _ptr(v_scale), n_rows, _ptr(row_offset), _ptr(cap), _ptr(length))
    c.device = k8.device.index
    if any(t.device != k8.device for t in (v8, k_scale, v_scale, row_offset, cap, length)):
        raise ValueError("the tensors of a cache are on one device")
    if not row_offset.numel() == cap.numel() == length.numel():
        raise ValueError("row_offset, cap and length have one element per sequence")
    c.n_seq = cap.numel()
    return c


class RopeTable:
    """What rkv_rope needs of a model's rotary positions, laid out once: the frequencies as fixed-point turns on the
    device, the rotated part, the pairs' layout and the amplitude (formulas: include/rkv.h).

    layout: "half" or "interleaved"; scaling: "none", "linear", "bands" (trained_len, low, high) or "ramp" (trained_len,
    fast, slow)."""

    def __init__(self, rot_dim=128, theta=10000.0, layout="half", scaling="none", factor=1.0, trained_len=8192, low=1.0,
                 high=4.0, fast=32.0, slow=1.0, device="cuda"):
        if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
            raise ValueError(f"layout is one of {list(ROPE_LAYOUTS)}, scaling one of {list(ROPE_SCALINGS)}")
        cfg = RkvRopeConfig(rot_dim, ROPE_SCALINGS[scaling], theta, factor, trained_len, low, high, fast, slow)
        turns = (ctypes.c_uint64 * 64)()
        amp = ctypes.c_float(0.0)
        rc = lib.rkv_rope_frequencies(ctypes.byref(cfg), turns, ctypes.byref(amp))
        if rc != RKV_OK:
            raise RkvError(rc, "rotary positions")
        self.rot_dim, self.layout, self.amplitude = rot_dim, ROPE_LAYOUTS[layout], amp.value
        self.turns = [turns[i] for i in range(rot_dim // 2)]          # f_i / 2 pi as a fraction of 2^64
        signed = [t - (1 << 64) if t >> 63 else t for t in self.turns]
        self.freqs = torch.tensor(signed, dtype=torch.int64).to(device)


class _LazyCalls:
    """Stands for the extension until its first call: the bf16 calls need neither it nor a host compiler to build it."""

    def __getattr__(self, name):
        global _calls
        try:
            from . import _rkv_calls     # links the librkv.so loaded above
        except ImportError as e:
            raise ImportError(f"the binding's extension cannot be loaded ({e}): build it first "
                              "(python -m paper_2411_05787_b200.build)") from e
        # what its checks compare with; the last: cudaStream_t of a device's current stream
        raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw_stream is None:
            raw_stream = lambda device: torch.cuda.current_stream(device).cuda_stream
        _rkv_calls.setup(torch.bfloat16, torch.float32, torch.int32, RkvQuantCache, RkvCache, RopeTable, raw_stream)
        _calls = _rkv_calls
        return getattr(_rkv_calls, name)


_calls = _LazyCalls()


def small_step_noalloc(cfg: RkvConfig, q, small: RkvCache, out, active=None, max_len_hint=0, device_status=None,
                       stream=None):
    """Partial step for callers that may not allocate device memory (no context; see include/rkv.h).

    Raises RkvError carrying the library's one-line reason, e.g. when a size exceeds the static scratch."""
    msg = ctypes.create_string_buffer(256)
    rc = lib.rkv_small_step_noalloc(ctypes.byref(cfg), _ptr(q), ctypes.byref(small), _ptr(active), _ptr(out),
                                    max_len_hint, _ptr(device_status), _stream(stream), msg, len(msg))
    if rc != RKV_OK:
        raise RkvError(rc, msg.value.decode())


class Context:
    """Owns one rkv_ctx (its scratch workspace).  Calls on one context share one stream."""

    def __init__(self, n_seq, n_q_heads, n_kv_heads, max_len, max_small, agg=AGG_MAX, pool_kernel=1,
                 softmax_scale=0.0, head_dim=128):
        self.cfg = RkvConfig(n_seq, n_q_heads, n_kv_heads, head_dim, max_len, max_small, agg, pool_kernel,
                             softmax_scale)
        handle = ctypes.c_void_p()
        rc = lib.rkv_create(ctypes.byref(self.cfg), ctypes.byref(handle))
        if rc != RKV_OK:
            raise RkvError(rc)
        self._h = handle
        self.device = torch.cuda.current_device()
        self._key = (handle.value, n_seq, n_q_heads, n_kv_heads, self.device)     # what _rkv_calls knows of the context

    def close(self):
        if getattr(self, "_h", None):
            lib.rkv_destroy(self._h)
            self._h = None
            self._key = (0,) + self._key[1:]

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc != RKV_OK:
            raise RkvError(rc, lib.rkv_last_cuda_error(self._h).decode())

    @property
    def workspace_bytes(self) -> int:
        return lib.rkv_workspace_bytes(ctypes.byref(self.cfg))

    @property
    def launch_count(self) -> int:
        return lib.rkv_launch_count(self._h)

    def full_step(self, q, full: RkvCache, k_small, k_max, out, topk_idx, active=None, scores=None,
                  q_last_full=None, max_len_hint=0, stream=None):
        stride = scores.shape[-1] if scores is not None else 0
        self._check(lib.rkv_full_step(self._h, _ptr(q), ctypes.byref(full), _ptr(k_small), k_max, _ptr(active),
                                      _ptr(out), _ptr(scores), stride, _ptr(topk_idx), _ptr(q_last_full),
                                      max_len_hint, _stream(stream)))

    def score_step(self, q, full: RkvCache, k_small, k_max, topk_idx, active=None, scores=None, q_last_full=None,
                   max_len_hint=0, stream=None):
        stride = scores.shape[-1] if scores is not None else 0
        self._check(lib.rkv_score_step(self._h, _ptr(q), ctypes.byref(full), _ptr(k_small), k_max, _ptr(active),
                                       _ptr(scores), stride, _ptr(topk_idx), _ptr(q_last_full), max_len_hint,
                                       _stream(stream)))

    def full_attention(self, q, full: RkvCache, out, active=None, max_len_hint=0, stream=None):
        self._check(lib.rkv_full_attention(self._h, _ptr(q), ctypes.byref(full), _ptr(active), _ptr(out),
                                           max_len_hint, _stream(stream)))

    def append_full_attention(self, q, k_new, v_new, full: RkvCache, out, active=None, max_len_hint=0, stream=None):
        self._check(lib.rkv_append_full_attention(self._h, _ptr(q), _ptr(k_new), _ptr(v_new), ctypes.byref(full),
                                                  _ptr(active), _ptr(out), max_len_hint, _stream(stream)))

    def select_topk(self, q, full: RkvCache | RkvQuantCache, k_small, k_max, topk_idx, active=None, scores=None,
                    q_last_full=None, stream=None):
        if isinstance(full, RkvQuantCache):
            args = (self._key, q, full, k_small, k_max, topk_idx, active, scores, q_last_full, stream)
            return self._done(_calls.quant_select_topk(*args), _calls.quant_select_topk, *args)
        stride = scores.shape[-1] if scores is not None else 0
        self._check(lib.rkv_select_topk(self._h, _ptr(q), ctypes.byref(full), _ptr(k_small), k_max, _ptr(active),
                                        _ptr(scores), stride, _ptr(topk_idx), _ptr(q_last_full), _stream(stream)))

    def score_keys(self, q, full: RkvCache | RkvQuantCache, k_small, k_max, active=None, scores=None, q_last_full=None,
                   stream=None):
        """The score pass alone; the next select_topk (scores=None, q_last_full=None) launches the selection alone."""
        if isinstance(full, RkvQuantCache):
            rc = _calls.quant_score_keys(self._key, q, full, k_small, k_max, active, scores, q_last_full, stream)
            if rc:
                self._done(rc, _calls.quant_score_keys, self._key, q, full, k_small, k_max, active, scores, q_last_full, stream)
            return
        stride = scores.shape[-1] if scores is not None else 0
        self._check(lib.rkv_score_keys(self._h, _ptr(q), ctypes.byref(full), _ptr(k_small), k_max, _ptr(active),
                                       _ptr(scores), stride, _ptr(q_last_full), _stream(stream)))

    def gather_small(self, topk_idx, k_small, k_max, full: RkvCache, small: RkvCache, active=None, stream=None):
        self._check(lib.rkv_gather_small(self._h, _ptr(topk_idx), _ptr(k_small), k_max, ctypes.byref(full),
                                         ctypes.byref(small), _ptr(active), _stream(stream)))

    def small_step(self, q, small: RkvCache, out, active=None, max_len_hint=0, stream=None):
        self._check(lib.rkv_small_step(self._h, _ptr(q), ctypes.byref(small), _ptr(active), _ptr(out),
                                       max_len_hint, _stream(stream)))

    def append(self, k_new, v_new, full: RkvCache | None, small: RkvCache | None, stream=None):
        self._check(lib.rkv_append(self._h, _ptr(k_new), _ptr(v_new),
                                   ctypes.byref(full) if full is not None else None,
                                   ctypes.byref(small) if small is not None else None, _stream(stream)))

    def append_small_step(self, q, k_new, v_new, full: RkvCache | None, small: RkvCache, out, active=None,
                          max_len_hint=0, stream=None):
        self._check(lib.rkv_append_small_step(self._h, _ptr(q), _ptr(k_new), _ptr(v_new),
                                              ctypes.byref(full) if full is not None else None, ctypes.byref(small),
                                              _ptr(active), _ptr(out), max_len_hint, _stream(stream)))

    def gather_small_evict(self, topk_idx, k_small, k_max, full: RkvCache, small: RkvCache, evict_order, evict_count,
                           active=None, stream=None):
        self._check(lib.rkv_gather_small_evict(self._h, _ptr(topk_idx), _ptr(k_small), k_max, ctypes.byref(full),
                                               ctypes.byref(small), _ptr(active), _ptr(evict_order), _ptr(evict_count),
                                               evict_order.shape[-1], _stream(stream)))

    def append_small_step_evict(self, q, k_new, v_new, full: RkvCache | None, small: RkvCache, k_small, out,
                                evict_order, evict_count, active=None, max_len_hint=0, stream=None):
        self._check(lib.rkv_append_small_step_evict(self._h, _ptr(q), _ptr(k_new), _ptr(v_new),
                                                    ctypes.byref(full) if full is not None else None,
                                                    ctypes.byref(small), _ptr(k_small), _ptr(active), _ptr(out),
                                                    _ptr(evict_order), _ptr(evict_count), evict_order.shape[-1],
                                                    max_len_hint, _stream(stream)))

    # ------------------------------------------------------------------ the full cache in 8 bits, rotary positions
    # These calls run in decode loops, where the host's time per launch counts: _rkv_calls checks their arguments
    # (ValueError for what does not fit) and calls the library with them.
    def _done(self, rc, call, *args):
        """rc of call(*args).  The library refuses to launch unless the context's device is current: then once more there."""
        if rc == RKV_OK:
            return
        if self._key[0] and _current_device() != self.device:
            with torch.cuda.device(self.device):
                rc = call(*args)
        self._check(rc)

    def quant_store(self, k_new, v_new, full: RkvQuantCache, start=None, count=None, stream=None):
        """Append rows to an 8-bit cache.  k_new, v_new: bfloat16 [B, T, Hkv, 128]; sequences and tokens may be strided
        (a slice of a projection's output), the heads of a token lie side by side.  start, count: int32 [B] or None."""
        rc = _calls.quant_store(self._key, k_new, v_new, full, start, count, stream)
        if rc:
            self._done(rc, _calls.quant_store, self._key, k_new, v_new, full, start, count, stream)

    def quant_full_attention(self, q, full: RkvQuantCache, out, active=None, max_len_hint=0, keep_logits=True, stream=None):
        """Attention over an 8-bit cache.  keep_logits: leave what score_keys / select_topk need in the workspace."""
        rc = _calls.quant_full_attention(self._key, q, full, out, active, max_len_hint, keep_logits, stream)
        if rc:
            self._done(rc, _calls.quant_full_attention, self._key, q, full, out, active, max_len_hint, keep_logits, stream)

    def quant_full_step(self, q, full: RkvQuantCache, k_small, k_max, out, topk_idx, active=None, scores=None,
                        q_last_full=None, max_len_hint=0, stream=None):
        args = (self._key, q, full, k_small, k_max, out, topk_idx, active, scores, q_last_full, max_len_hint, stream)
        self._done(_calls.quant_full_step(*args), _calls.quant_full_step, *args)

    def quant_gather_small(self, topk_idx, k_small, k_max, full: RkvQuantCache, small: RkvCache, active=None, stream=None):
        """Rebuild of the bf16 small cache from the selected positions of an 8-bit full cache."""
        rc = _calls.quant_gather_small(self._key, topk_idx, k_small, k_max, full, small, active, stream)
        if rc:
            self._done(rc, _calls.quant_gather_small, self._key, topk_idx, k_small, k_max, full, small, active, stream)

    def rope(self, qkv, pos, table: RopeTable, q, k, v=None, stream=None):
        """Split the fused projection's rows [T, (Hq + 2 Hkv) * 128] (bfloat16 or float32; tokens may be strided) into
        q [T, Hq, 128] and k, v [T, Hkv, 128] (bfloat16), queries and keys turned by their positions.  pos: int32 [T].
        Hq and Hkv are those of q and k, whatever the context's.  v=None: the values are not copied."""
        rc = _calls.rope(self._key, qkv, pos, table, q, k, v, stream)
        if rc:
            self._done(rc, _calls.rope, self._key, qkv, pos, table, q, k, v, stream)

    def should_refresh(self, q_now, q_last_full, threshold, flag, sim=None, keep=None, stream=None):
        self._check(lib.rkv_should_refresh(self._h, _ptr(q_now), _ptr(q_last_full), float(threshold), _ptr(flag),
                                           _ptr(keep), _ptr(sim), _stream(stream)))

    def set_option(self, option: int, value: int):
        self._check(lib.rkv_set_option(self._h, option, value))

    def get_option(self, option: int) -> int:
        value = ctypes.c_int32(0)
        self._check(lib.rkv_get_option(self._h, option, ctypes.byref(value)))
        return value.value

    def set_profiling(self, on: bool):
        self._check(lib.rkv_set_profiling(self._h, 1 if on else 0))

    def get_profile(self) -> dict:
        """{kernel name: (total microseconds, launches)} since the last call; waits for the recorded events."""
        us = (ctypes.c_double * len(KERNEL_NAMES))()
        cnt = (ctypes.c_int64 * len(KERNEL_NAMES))()
        self._check(lib.rkv_get_profile(self._h, us, cnt))
        return {n: (us[i], cnt[i]) for i, n in enumerate(KERNEL_NAMES)}

    def device_status(self, stream=None) -> int:
        """Synchronises the stream; returns and clears the sticky device status bits."""
        bits = ctypes.c_int32(0)
        rc = lib.rkv_get_device_status(self._h, ctypes.byref(bits), _stream(stream))
        if rc not in (RKV_OK, 5):
            raise RkvError(rc, lib.rkv_last_cuda_error(self._h).decode())
        return bits.value
