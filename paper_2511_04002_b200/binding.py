"""Thin binding of the tsq C ABI (include/tsq.h): argument marshalling only.

Every step of encode and decode runs inside the CUDA library; torch is used for device
memory and streams.  Function names mirror the C entry points.  The calls of a decode step,
encode and decode and those of the paged cache, go through the extension module built from
csrc/tsq_torch.cpp (5 us less host time per call than ctypes); everything else goes through ctypes.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

import torch

F16, BF16 = 0, 1
STATUS = {0: "TSQ_OK", 1: "TSQ_ERR_INVALID_ARG", 2: "TSQ_ERR_UNSUPPORTED", 3: "TSQ_ERR_BUFFER_TOO_SMALL",
          4: "TSQ_ERR_CUDA", 5: "TSQ_ERR_CORRUPT_BLOB", 6: "TSQ_ERR_OUTLIER_OVERFLOW", 7: "TSQ_ERR_TIMEOUT"}

VARIANT_MAGNITUDES, VARIANT_SIGNED_VALUES = 0, 1

EXPORTS = ["tsq_plan", "tsq_plan_variant", "tsq_plan_sizes", "tsq_workspace_init", "tsq_workspace_set_wait_limit", "tsq_encode", "tsq_encode_noalloc", "tsq_decode",
           "tsq_blob_info",
           "tsq_workspace_status", "tsq_encode_host", "tsq_decode_host", "tsq_kernel_launch_count",
           "tsq_plan_destroy", "tsq_status_string",
           "tsq_cache_slots", "tsq_cache_store", "tsq_cache_load", "tsq_cache_workspace", "tsq_cache_workspace_init", "tsq_cache_workspace_status", "tsq_cache_attention",
           "tsq_model_kv_bits", "tsq_model_io_bits", "tsq_model_outage", "tsq_model_latency", "tsq_model_best_rate"]

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtsq.so")
_lib: Optional[C.CDLL] = None
_calls = None                     # the extension module, once lib() has run


class TsqError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__("%s failed: %s (%d)" % (where, STATUS.get(status, "?"), status))
        self.status = status


class _Sizes(C.Structure):
    _fields_ = [("blob_bytes", C.c_size_t), ("workspace_bytes", C.c_size_t)]


class _Info(C.Structure):
    _fields_ = [("status", C.c_uint32), ("tokens", C.c_uint32), ("hidden", C.c_uint32), ("dtype", C.c_uint32),
                ("total_words", C.c_uint64), ("total_outliers", C.c_uint64), ("payload_bytes", C.c_uint64)]


class _CacheStruct(C.Structure):
    _fields_ = [("dtype", C.c_int), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_tokens", C.c_int32), ("pages", C.c_int64),
                ("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


def lib() -> C.CDLL:
    """Load libtsq.so and the extension module. Raises if they have not been built: there is no fallback path."""
    global _lib, _calls
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError("tsq CUDA library missing at %s; run `python -m paper_2511_04002_b200.build` "
                           "(needs nvcc). No CPU fallback exists." % _LIB_PATH)
    try:
        from . import _tsq_torch as calls
    except ImportError as e:
        raise RuntimeError("the binding's extension module is missing; run `python -m paper_2511_04002_b200.build`") from e
    L = C.CDLL(_LIB_PATH)
    vp, i64, sz = C.c_void_p, C.c_int64, C.c_size_t
    L.tsq_plan.argtypes = [C.POINTER(vp), C.c_int, C.c_int, C.c_int32, i64, C.c_float, C.POINTER(C.c_int32),
                           C.c_int32, C.c_float, i64]
    L.tsq_plan_variant.argtypes = L.tsq_plan.argtypes + [C.c_int32]
    L.tsq_plan_sizes.argtypes = [vp, i64, C.POINTER(_Sizes)]
    L.tsq_workspace_init.argtypes = [vp, vp, sz, vp]
    L.tsq_workspace_set_wait_limit.argtypes = [vp, C.c_uint32, vp]
    L.tsq_encode.argtypes = [vp, vp, i64, vp, sz, vp, sz, vp]
    L.tsq_encode_noalloc.argtypes = [vp, vp, i64, vp, sz, vp]
    L.tsq_encode_noalloc.restype = C.c_int
    L.tsq_decode.argtypes = [vp, vp, sz, i64, vp, vp, sz, vp]
    L.tsq_blob_info.argtypes = [vp, C.POINTER(_Info), vp]
    L.tsq_workspace_status.argtypes = [vp, C.POINTER(C.c_uint32), C.POINTER(C.c_uint32), vp]
    L.tsq_encode_host.argtypes = [vp, vp, i64, vp, sz, C.POINTER(C.c_uint64), vp, vp, vp, sz, vp]
    L.tsq_decode_host.argtypes = [vp, vp, sz, i64, vp, vp, vp, vp, sz, vp]
    for name in ("tsq_plan", "tsq_plan_variant", "tsq_plan_sizes", "tsq_workspace_init", "tsq_workspace_set_wait_limit", "tsq_encode", "tsq_decode", "tsq_blob_info",
                 "tsq_workspace_status", "tsq_encode_host", "tsq_decode_host"):
        getattr(L, name).restype = C.c_int
    d, i32 = C.c_double, C.c_int32
    cache, ip = C.POINTER(_CacheStruct), C.c_void_p
    L.tsq_cache_slots.argtypes = [i32, ip, ip, i32, ip, i32, ip, ip, ip, i32, ip, i64, ip, vp]
    L.tsq_cache_store.argtypes = [cache, vp, i64, vp, i64, i64, ip, vp]
    L.tsq_cache_load.argtypes = [cache, ip, i64, vp, i64, vp, i64, vp]
    L.tsq_cache_workspace.argtypes = [cache, i64, i32, i32, i32, C.POINTER(sz)]
    L.tsq_cache_workspace_init.argtypes = [vp, sz, vp]
    L.tsq_cache_workspace_status.argtypes = [vp, C.POINTER(C.c_uint32), vp]
    L.tsq_cache_attention.argtypes = [cache, vp, i64, i32, i64, ip, ip, i32, i32, ip, i32, C.c_float, vp, i64, vp, sz, vp]
    for name in ("tsq_cache_slots", "tsq_cache_store", "tsq_cache_load", "tsq_cache_workspace", "tsq_cache_workspace_init", "tsq_cache_workspace_status",
                 "tsq_cache_attention"):
        getattr(L, name).restype = C.c_int
    L.tsq_model_kv_bits.argtypes = [i64, i32, i32, i32, i64, d, d]
    L.tsq_model_io_bits.argtypes = [i64, i32, i32, i32, i64, d, d, i32]
    L.tsq_model_outage.argtypes = [d, d, d]
    L.tsq_model_latency.argtypes = [d, d, d, d, d]
    L.tsq_model_best_rate.argtypes = [d, d, d, d]
    for name in ("tsq_model_kv_bits", "tsq_model_io_bits", "tsq_model_outage", "tsq_model_latency", "tsq_model_best_rate"):
        getattr(L, name).restype = d
    L.tsq_kernel_launch_count.argtypes = []
    L.tsq_kernel_launch_count.restype = C.c_uint64
    L.tsq_plan_destroy.argtypes = [vp]
    L.tsq_plan_destroy.restype = None
    L.tsq_status_string.argtypes = [C.c_int]
    L.tsq_status_string.restype = C.c_char_p
    _calls = calls
    _lib = L
    return L


def _check(status: int, where: str) -> None:
    if status != 0:
        raise TsqError(status, where)


def _stream(stream) -> int:
    if stream is None:
        return _calls.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float16:
        return F16
    if dt == torch.bfloat16:
        return BF16
    raise TypeError("tsq handles float16 and bfloat16, got %s" % dt)


@dataclass
class BlobInfo:
    status: int
    tokens: int
    hidden: int
    dtype: int
    total_words: int
    total_outliers: int
    payload_bytes: int


class Plan:
    """tsq_plan_t wrapper. Methods are the C calls of the same name with pointers filled in."""

    def __init__(self, dtype: torch.dtype, hidden: int, max_tokens: int, tau: float, bits: Sequence[int],
                 delta: float = 0.2, max_outliers: int = 0, device: int = 0, variant: int = VARIANT_MAGNITUDES):
        self._h = C.c_void_p()
        arr = (C.c_int32 * len(bits))(*bits)
        if variant == VARIANT_MAGNITUDES:
            st = lib().tsq_plan(C.byref(self._h), device, dtype_code(dtype), hidden, max_tokens, tau, arr, len(bits),
                                delta, max_outliers)
        else:
            st = lib().tsq_plan_variant(C.byref(self._h), device, dtype_code(dtype), hidden, max_tokens, tau, arr,
                                        len(bits), delta, max_outliers, variant)
        _check(st, "tsq_plan")
        self._addr, self._dtype_code = self._h.value, dtype_code(dtype)
        self.variant = variant
        self.dtype, self.hidden, self.max_tokens, self.device = dtype, hidden, max_tokens, device
        self.tau, self.bits, self.delta, self.max_outliers = tau, tuple(bits), delta, max_outliers

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and _lib is not None:
            _lib.tsq_plan_destroy(h)

    def sizes(self, tokens: int) -> Tuple[int, int]:
        s = _Sizes()
        _check(lib().tsq_plan_sizes(self._h, tokens, C.byref(s)), "tsq_plan_sizes")
        return int(s.blob_bytes), int(s.workspace_bytes)

    def alloc(self, tokens: Optional[int] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Allocate (blob, workspace) with torch on the plan's device and initialise the workspace."""
        tokens = self.max_tokens if tokens is None else tokens
        blob_bytes, ws_bytes = self.sizes(tokens)
        dev = torch.device("cuda", self.device)
        blob = torch.empty(blob_bytes, dtype=torch.uint8, device=dev)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        self.workspace_init(ws)
        return blob, ws

    def workspace_init(self, ws: torch.Tensor, stream=None) -> None:
        _check(lib().tsq_workspace_init(self._h, ws.data_ptr(), ws.numel(), _stream(stream)), "tsq_workspace_init")

    def workspace_set_wait_limit(self, ws: torch.Tensor, polls: int, stream=None) -> None:
        _check(lib().tsq_workspace_set_wait_limit(ws.data_ptr(), polls, _stream(stream)), "tsq_workspace_set_wait_limit")

    def encode(self, x: torch.Tensor, blob: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
        st = _calls.encode(self._addr, self._dtype_code, self.hidden, x, blob, ws, stream)
        if st != 0:
            raise TsqError(st, "tsq_encode")

    def encode_noalloc(self, x: torch.Tensor, blob: torch.Tensor, stream=None) -> None:
        """tsq_encode_noalloc: encode with the library's built-in scratch array instead of a workspace."""
        assert x.is_cuda and x.is_contiguous() and x.dtype == self.dtype and x.dim() == 2 and x.shape[1] == self.hidden
        _check(lib().tsq_encode_noalloc(self._h, x.data_ptr(), x.shape[0], blob.data_ptr(), blob.numel(),
                                        _stream(stream)), "tsq_encode_noalloc")

    def decode(self, blob: torch.Tensor, tokens: int, y: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
        st = _calls.decode(self._addr, self._dtype_code, self.hidden, blob, tokens, y, ws, stream)
        if st != 0:
            raise TsqError(st, "tsq_decode")

    def blob_info(self, blob: torch.Tensor, stream=None) -> BlobInfo:
        i = _Info()
        _check(lib().tsq_blob_info(blob.data_ptr(), C.byref(i), _stream(stream)), "tsq_blob_info")
        return BlobInfo(i.status, i.tokens, i.hidden, i.dtype, i.total_words, i.total_outliers, i.payload_bytes)

    def workspace_status(self, ws: torch.Tensor, stream=None) -> Tuple[int, int]:
        e, d = C.c_uint32(0), C.c_uint32(0)
        _check(lib().tsq_workspace_status(ws.data_ptr(), C.byref(e), C.byref(d), _stream(stream)),
               "tsq_workspace_status")
        return int(e.value), int(d.value)

    def encode_host(self, x_host: torch.Tensor, blob_host: torch.Tensor, x_dev: torch.Tensor, blob_dev: torch.Tensor,
                    ws: torch.Tensor, stream=None) -> int:
        """Host tensor in, host blob out (copies inside). Returns the payload size in bytes."""
        assert not x_host.is_cuda and x_host.is_contiguous() and x_host.dtype == self.dtype
        payload = C.c_uint64(0)
        st = lib().tsq_encode_host(self._h, x_host.data_ptr(), x_host.shape[0], blob_host.data_ptr(),
                                   blob_host.numel(), C.byref(payload), x_dev.data_ptr(), blob_dev.data_ptr(),
                                   ws.data_ptr(), ws.numel(), _stream(stream))
        _check(st, "tsq_encode_host")
        return int(payload.value)

    def decode_host(self, blob_host: torch.Tensor, tokens: int, y_host: torch.Tensor, blob_dev: torch.Tensor,
                    y_dev: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
        assert not y_host.is_cuda and y_host.is_contiguous() and y_host.dtype == self.dtype
        st = lib().tsq_decode_host(self._h, blob_host.data_ptr(), blob_host.numel(), tokens, y_host.data_ptr(),
                                   blob_dev.data_ptr(), y_dev.data_ptr(), ws.data_ptr(), ws.numel(),
                                   _stream(stream))
        _check(st, "tsq_decode_host")


class Cache:
    """The paged 8-bit key/value cache (tsq_cache_t) over four tensors of the caller's: codes int8 [pages, kv_heads, page_tokens, head_dim] and scales
    float32 [pages, kv_heads], for keys and for values.  Methods are the C calls tsq_cache_* with pointers filled in; they run on the tensors' device,
    on `stream` or that device's current one, and raise TsqError where the call refuses its arguments."""

    def __init__(self, dtype: torch.dtype, k_codes: torch.Tensor, v_codes: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        lib()
        for name, t in (("k_codes", k_codes), ("v_codes", v_codes)):
            assert t.is_cuda and t.is_contiguous() and t.dtype == torch.int8 and t.dim() == 4 and t.shape == k_codes.shape and t.device == k_codes.device, \
                "%s must be a contiguous int8 CUDA tensor [pages, kv_heads, page_tokens, head_dim]" % name
        pages, kv_heads, page_tokens, head_dim = k_codes.shape
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            assert t.is_cuda and t.is_contiguous() and t.dtype == torch.float32 and tuple(t.shape) == (pages, kv_heads) and t.device == k_codes.device, \
                "%s must be a contiguous float32 CUDA tensor [pages, kv_heads] on the codes' device" % name
        self.dtype, self.pages, self.kv_heads, self.page_tokens, self.head_dim = dtype, pages, kv_heads, page_tokens, head_dim
        self.k_codes, self.v_codes, self.k_scale, self.v_scale = k_codes, v_codes, k_scale, v_scale
        self.device = k_codes.device.index
        self._c = _CacheStruct(dtype_code(dtype), kv_heads, head_dim, page_tokens, pages, k_codes.data_ptr(), v_codes.data_ptr(),
                               k_scale.data_ptr(), v_scale.data_ptr())
        self._addr = C.addressof(self._c)
        self._scale = head_dim ** -0.5 if head_dim else 1.0

    @classmethod
    def alloc(cls, dtype: torch.dtype, kv_heads: int, head_dim: int, pages: int, page_tokens: int = 64, device: int = 0) -> "Cache":
        """A cache over tensors of its own, every code and scale 0."""
        dev = torch.device("cuda", device)
        codes = [torch.zeros((pages, kv_heads, page_tokens, head_dim), dtype=torch.int8, device=dev) for _ in range(2)]
        scales = [torch.zeros((pages, kv_heads), dtype=torch.float32, device=dev) for _ in range(2)]
        return cls(dtype, *codes, *scales)

    def store(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, stream=None) -> None:
        st = _calls.cache_store(self._addr, self.device, k, v, slots, stream)
        if st != 0:
            raise TsqError(st, "tsq_cache_store")

    def load(self, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        st = _calls.cache_load(self._addr, self.device, slots, k, v, stream)
        if st != 0:
            raise TsqError(st, "tsq_cache_load")

    def workspace_bytes(self, tokens: int, q_heads: int, requests: int, max_query: int) -> int:
        out = C.c_size_t(0)
        with torch.cuda.device(self.device):
            _check(lib().tsq_cache_workspace(C.byref(self._c), tokens, q_heads, requests, max_query, C.byref(out)), "tsq_cache_workspace")
        return int(out.value)

    def workspace(self, tokens: int, q_heads: int, requests: int, max_query: int) -> torch.Tensor:
        """Allocate a workspace for attention calls of up to these sizes with torch and initialise it on the current stream."""
        ws = torch.empty(self.workspace_bytes(tokens, q_heads, requests, max_query), dtype=torch.uint8, device=torch.device("cuda", self.device))
        self.workspace_init(ws)
        return ws

    def _check_workspace(self, ws: torch.Tensor) -> None:
        assert ws.is_cuda and ws.device.index == self.device and ws.dtype == torch.uint8 and ws.is_contiguous(), \
            "ws must be a contiguous uint8 CUDA tensor on the cache's device"

    def workspace_init(self, ws: torch.Tensor, stream=None) -> None:
        self._check_workspace(ws)
        with torch.cuda.device(self.device):
            _check(lib().tsq_cache_workspace_init(ws.data_ptr(), ws.numel(), _stream(stream)), "tsq_cache_workspace_init")

    def workspace_status(self, ws: torch.Tensor, stream=None) -> int:
        self._check_workspace(ws)
        assert ws.numel() >= 16, "ws is no workspace"
        out = C.c_uint32(0)
        with torch.cuda.device(self.device):
            _check(lib().tsq_cache_workspace_status(ws.data_ptr(), C.byref(out), _stream(stream)), "tsq_cache_workspace_status")
        return int(out.value)

    def attention(self, q: torch.Tensor, query_start: torch.Tensor, lengths: torch.Tensor, block_table: torch.Tensor, out: torch.Tensor,
                  ws: torch.Tensor, max_query: int, scale: Optional[float] = None, stream=None) -> None:
        """scale: 1 / sqrt(head_dim) unless given."""
        st = _calls.cache_attention(self._addr, self.device, q, query_start, lengths, block_table, out, ws, max_query,
                                    self._scale if scale is None else scale, stream)
        if st != 0:
            raise TsqError(st, "tsq_cache_attention")


def cache_slots(page_tokens: int, held: torch.Tensor, added: torch.Tensor, free_pages: torch.Tensor, query_start: torch.Tensor,
                lengths: torch.Tensor, block_table: torch.Tensor, slots: torch.Tensor, taken: torch.Tensor, stream=None) -> None:
    """tsq_cache_slots on int32 tensors of one device."""
    lib()
    st = _calls.cache_slots(page_tokens, held, added, free_pages, query_start, lengths, block_table, slots, taken, stream)
    if st != 0:
        raise TsqError(st, "tsq_cache_slots")


def model_kv_bits(w, layer, n_layers, split_layer, hd, qa_front, qa_back) -> float:
    return float(lib().tsq_model_kv_bits(w, layer, n_layers, split_layer, hd, qa_front, qa_back))


def model_io_bits(w, layer, n_layers, split_layer, hd, qa_front, qa_back, send_kv) -> float:
    return float(lib().tsq_model_io_bits(w, layer, n_layers, split_layer, hd, qa_front, qa_back, 1 if send_kv else 0))


def model_outage(rate, bandwidth, snr) -> float:
    return float(lib().tsq_model_outage(rate, bandwidth, snr))


def model_latency(bits, rate, bandwidth, snr, epsilon) -> float:
    return float(lib().tsq_model_latency(bits, rate, bandwidth, snr, epsilon))


def model_best_rate(rate_lo, rate_hi, bandwidth, snr) -> float:
    return float(lib().tsq_model_best_rate(rate_lo, rate_hi, bandwidth, snr))


def kernel_launch_count() -> int:
    return int(lib().tsq_kernel_launch_count())


def status_string(status: int) -> str:
    return lib().tsq_status_string(status).decode()
