"""Thin ctypes binding of the C-ABI library (`include/dd.h`, instrumentation in `include/dd_bench.h`):
argument marshalling only.

Every step of the path runs in the library's CUDA kernels. torch is used for device and
pinned memory and for streams; tensors are passed as raw pointers. There is no CPU
fallback: importing this module raises if `libdd.so` has not been built
(`python -m paper_2607_26475_b200.build`).
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdd.so")

DD_OK = 0
DD_ERR_INVALID_ARG = -1
DD_ERR_NOT_PINNED = -2
DD_ERR_CUDA = -3
DD_ERR_TIMEOUT = -4
DD_ERR_INDEX_RANGE = -5
DD_ERR_STATE = -6
DD_ERR_WAIT_EXPIRED = -7
DD_GATHER_LOADS = 0
DD_GATHER_BULK = 1
DD_GATHER_STAGED = 2
DD_GATHER_STATS_FIELDS = 7
DD_TRACE_FIELDS = 8
DD_ATTN_AUTO = 0
DD_ATTN_SPLIT = 1
DD_ATTN_STREAM = 2
DD_ATTN_TC = 3
DD_SELECT_AUTO = 0
DD_SELECT_TWO_KERNELS = 1
DD_BF16 = 0
DD_FP16 = 1
DD_CACHE_BF16 = 0
DD_CACHE_FP16 = 1
DD_CACHE_E4M3 = 2
DD_CACHE_INT4 = 4
DD_ROPE_HALF = 0
DD_ROPE_INTERLEAVED = 1
DD_ROPE_NONE = 0
DD_ROPE_LINEAR = 1
DD_ROPE_NTK = 2
DD_ROPE_BY_PARTS = 3

EXPORTS = [
    "dd_create", "dd_destroy", "dd_slot_bytes", "dd_ring_bytes", "dd_scratch_bytes", "dd_slot_ptr",
    "dd_strerror", "dd_last_error_message", "dd_device_error", "dd_sync", "dd_build_landmarks",
    "dd_select_topk", "dd_gather_kv_from_host", "dd_sparse_decode_attn", "dd_bind", "dd_prime",
    "dd_decode_layer_step", "dd_get_indices", "dd_static_scratch_capacity", "dd_sparse_decode_attn_static",
    "dd_select_topk_chunked", "dd_sparse_decode_attn_causal", "dd_decode_layer_step_causal", "dd_diff_indices",
    "dd_fetch_missing_from_host", "dd_get_merged_indices", "dd_miss_stats", "dd_probe_attn_loads", "dd_probe_select_loads",
    "dd_trace_begin", "dd_trace_end", "dd_trace_read", "dd_decode_step_host", "dd_last_device_error",
    "dd_gather_stats", "dd_set_bulk_wait", "dd_test_pick_cluster", "dd_test_stage_plan", "dd_test_attn_split",
    "dd_cache_landmark_bytes", "dd_cache_landmarks", "dd_cache_select_workspace", "dd_cache_select",
    "dd_cache_sparse_attn_workspace", "dd_cache_sparse_attn",
    "dd_cache_page_bytes", "dd_rope_turns", "dd_rope_apply", "dd_cache_append", "dd_cache_read",
    "dd_cache_decode_attn_workspace", "dd_cache_decode_attn",
]


class DDConfig(C.Structure):
    """Mirror of `dd_config`."""
    _fields_ = [
        ("n_layers", C.c_int), ("batch", C.c_int), ("n_q_heads", C.c_int), ("n_kv_heads", C.c_int),
        ("head_dim", C.c_int), ("page_tokens", C.c_int), ("max_pages", C.c_int), ("k_pages", C.c_int),
        ("forced_recent_pages", C.c_int), ("n_q_tokens", C.c_int), ("ring_depth", C.c_int),
        ("gather_mode", C.c_int), ("gather_ctas", C.c_int), ("select_mode", C.c_int), ("attn_splits", C.c_int),
        ("compute_stream", C.c_void_p), ("copy_stream", C.c_void_p),
        ("ring_mem", C.c_void_p), ("ring_bytes", C.c_size_t),
        ("landmark_chunk_tokens", C.c_int), ("miss_correction", C.c_int), ("urgent_stream", C.c_void_p),
        ("select_stream", C.c_void_p), ("stage_min_run_pages", C.c_int), ("stage_block_pages", C.c_int), ("attn_mode", C.c_int),
        ("store_format", C.c_int),
    ]


class DDRows(C.Structure):
    """Mirror of `dd_rows`."""
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int), ("n_heads", C.c_int), ("token_stride", C.c_longlong),
                ("head_stride", C.c_longlong)]


class DDRope(C.Structure):
    """Mirror of `dd_rope`."""
    _fields_ = [("turns", C.c_void_p), ("rot_dim", C.c_int), ("layout", C.c_int), ("amplitude", C.c_float)]


class DDCache(C.Structure):
    """Mirror of `dd_cache`."""
    _fields_ = [("data", C.c_void_p), ("format", C.c_int), ("n_kv_heads", C.c_int), ("head_dim", C.c_int),
                ("page_tokens", C.c_int), ("n_blocks", C.c_int), ("block_stride", C.c_longlong), ("head_stride", C.c_longlong),
                ("block_table", C.c_void_p), ("batch", C.c_int), ("max_pages", C.c_int), ("table_stride", C.c_longlong),
                ("status", C.c_void_p)]


class DDError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"dd error {code}: {message}")
        self.code = code


PICK_FITS = C.CFUNCTYPE(C.c_int, C.c_int, C.c_size_t, C.c_void_p)


def _load() -> C.CDLL:
    from . import build as _build
    try:
        _build.build()          # compiles with nvcc when the library is missing or older than its sources
    except Exception as e:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing and could not be built ({e}); build it with "
                              "`python -m paper_2607_26475_b200.build` (there is no CPU fallback)") from e
    lib = C.CDLL(LIB_PATH)
    vp, ip = C.c_void_p, C.c_int
    lib.dd_create.argtypes = [C.POINTER(DDConfig), C.POINTER(vp)]
    lib.dd_destroy.argtypes = [vp]
    for name in ("dd_slot_bytes", "dd_ring_bytes", "dd_scratch_bytes"):
        getattr(lib, name).argtypes = [C.POINTER(DDConfig)]
        getattr(lib, name).restype = C.c_size_t
    lib.dd_slot_ptr.argtypes = [vp, ip, C.POINTER(vp)]
    lib.dd_strerror.argtypes = [ip]
    lib.dd_strerror.restype = C.c_char_p
    lib.dd_last_error_message.argtypes = [vp]
    lib.dd_last_error_message.restype = C.c_char_p
    lib.dd_device_error.argtypes = [vp, C.c_double, C.POINTER(ip), C.POINTER(ip)]
    lib.dd_sync.argtypes = [vp, C.c_double]
    lib.dd_build_landmarks.argtypes = [vp, vp, vp, vp, vp]
    lib.dd_select_topk.argtypes = [vp, vp, ip, vp, vp, vp, vp, vp]
    lib.dd_gather_kv_from_host.argtypes = [vp, vp, vp, vp, ip, vp]
    lib.dd_sparse_decode_attn.argtypes = [vp, vp, ip, vp, vp, vp, vp, vp]
    lib.dd_bind.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), vp, vp]
    lib.dd_prime.argtypes = [vp, vp]
    lib.dd_decode_layer_step.argtypes = [vp, ip, ip, vp, vp]
    lib.dd_get_indices.argtypes = [vp, ip, ip, C.POINTER(vp)]
    lib.dd_select_topk_chunked.argtypes = [vp, vp, ip, vp, vp, vp, vp, vp, vp]
    lib.dd_sparse_decode_attn_causal.argtypes = [vp, vp, ip, vp, vp, vp, vp, vp, vp, vp]
    lib.dd_decode_layer_step_causal.argtypes = [vp, ip, ip, vp, vp, vp, vp]
    lib.dd_diff_indices.argtypes = [vp, vp, vp, ip, vp, vp]
    lib.dd_fetch_missing_from_host.argtypes = [vp, vp, ip, vp]
    lib.dd_get_merged_indices.argtypes = [vp, ip, C.POINTER(vp)]
    lib.dd_miss_stats.argtypes = [vp, C.POINTER(C.c_ulonglong), C.POINTER(C.c_ulonglong), ip]
    lib.dd_decode_step_host.argtypes = [vp, ip, vp, vp]
    lib.dd_trace_begin.argtypes = [vp, ip]
    lib.dd_trace_end.argtypes = [vp, C.POINTER(ip)]
    lib.dd_trace_read.argtypes = [vp, ip, ip, vp]
    lib.dd_probe_attn_loads.argtypes = [vp, ip, vp]
    lib.dd_probe_select_loads.argtypes = [vp, vp, vp, vp]
    lib.dd_last_device_error.argtypes = [vp, C.POINTER(ip), C.POINTER(ip)]
    lib.dd_gather_stats.argtypes = [vp, C.POINTER(C.c_ulonglong), ip]
    lib.dd_set_bulk_wait.argtypes = [vp, C.c_double, ip]
    lib.dd_test_pick_cluster.argtypes = [ip, ip, ip, ip, ip, ip, PICK_FITS, vp, C.POINTER(ip), C.POINTER(C.c_size_t), C.POINTER(ip), C.POINTER(ip)]
    lib.dd_test_stage_plan.argtypes = [vp, vp, ip, ip, ip, ip, ip, ip, C.c_longlong, vp, C.c_longlong, vp, vp, vp, vp, vp, vp]
    lib.dd_test_attn_split.argtypes = [ip, ip, ip, ip, ip, C.POINTER(ip), C.POINTER(ip), C.POINTER(ip)]
    lib.dd_static_scratch_capacity.argtypes = []
    lib.dd_static_scratch_capacity.restype = C.c_size_t
    lib.dd_sparse_decode_attn_static.argtypes = [ip] * 8 + [vp] * 7
    rows, rope, cache = C.POINTER(DDRows), C.POINTER(DDRope), C.POINTER(DDCache)
    lib.dd_cache_page_bytes.argtypes = [ip, ip, ip]
    lib.dd_cache_page_bytes.restype = C.c_size_t
    lib.dd_rope_turns.argtypes = [ip, C.c_double, ip, C.c_double, C.c_double, C.c_double, C.c_double, C.POINTER(C.c_double)]
    lib.dd_rope_apply.argtypes = [rope, ip, ip, vp, rows, rows, rows, rows, ip, vp]
    lib.dd_cache_append.argtypes = [cache, ip, vp, vp, rows, rows, rope, rows, rows, vp]
    lib.dd_cache_read.argtypes = [cache, vp, ip, vp, ip, vp]
    lib.dd_cache_decode_attn_workspace.argtypes = [ip, ip, ip, ip]
    lib.dd_cache_decode_attn_workspace.restype = C.c_size_t
    lib.dd_cache_decode_attn.argtypes = [cache, ip, rows, vp, rows, vp, ip, C.c_float, vp, C.c_size_t, vp]
    for name, n in (("dd_cache_landmark_bytes", 1), ("dd_cache_select_workspace", 3), ("dd_cache_sparse_attn_workspace", 5)):
        getattr(lib, name).argtypes = [ip] * n
        getattr(lib, name).restype = C.c_size_t
    lib.dd_cache_landmarks.argtypes = [cache, vp, ip, vp, vp]
    lib.dd_cache_select.argtypes = [cache, ip, vp, vp, rows, vp, ip, ip, ip, vp, vp, C.c_size_t, vp]
    lib.dd_cache_sparse_attn.argtypes = [cache, ip, vp, vp, rows, vp, ip, rows, vp, C.c_float, vp, C.c_size_t, vp]
    return lib


lib = _load()


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


class _DevMem:
    """Raw device memory as a CUDA-array-interface object, so that torch can view it."""

    def __init__(self, ptr: int, shape, typestr: str):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr, "data": (ptr, False),
                                         "version": 2, "strides": None}


def _view(ptr: int, shape, kind: str) -> torch.Tensor:
    """Zero-copy torch view of library-owned device memory (kind: 'i4' or 'bf16')."""
    if kind == "bf16":
        return torch.as_tensor(_DevMem(ptr, shape, "<i2"), device="cuda").view(torch.bfloat16)
    return torch.as_tensor(_DevMem(ptr, shape, "<" + kind), device="cuda")


# The current stream as a number, without building a Stream object (3 us less per call); torch offers it to generated code.
_raw_stream, _raw_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(s) -> int:
    if s is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _torch_stream(s, device):
    """The stream of `device` behind a raw handle, 0 being the default one (torch makes a new stream of an external 0)."""
    return torch.cuda.ExternalStream(s, device=device) if s else torch.cuda.default_stream(device)


def sparse_decode_attn_static(q, slot, idx, ctx_len, out, out_lse=None, *, n_splits=1, page_tokens=16, stream=None):
    """Attention over a gathered slot without a context and without any allocation: for callers that are
    not allowed to allocate device memory. The library's built-in scratch array (8 MiB per GPU) is shared
    by every call on the device, so calls must not overlap on the GPU; the first call on a device should
    come before any stream capture. q [B, Tq, Hq, d], slot [B, Hkv, 2, k*T, d], idx [B, Hkv, k]."""
    B, Tq, Hq, d = q.shape
    Hkv, k = idx.shape[1], idx.shape[2]
    rc = lib.dd_sparse_decode_attn_static(B, Hq, Hkv, d, page_tokens, k, Tq, n_splits, _ptr(q), _ptr(slot), _ptr(idx),
                                          _ptr(ctx_len), _ptr(out), _ptr(out_lse), _stream(stream))
    if rc != DD_OK:
        raise DDError(rc, lib.dd_last_error_message(None).decode())


_ROW_TYPES = {torch.bfloat16: DD_BF16, torch.float16: DD_FP16}
_PACK_ROWS = struct.Struct("<Qiiqq").pack          # a `dd_rows`, byte for byte
assert C.sizeof(DDRows) == 32


def _invalid(message: str) -> DDError:
    return DDError(DD_ERR_INVALID_ARG, message)


def _handle(name: str, *argtypes):
    """The entry point again, with structures passed by address (ints, packed bytes or None): cheaper to call."""
    f = lib[name]
    f.argtypes, f.restype = argtypes, C.c_int
    return f


_P, _I = C.c_void_p, C.c_int
_rope_apply = _handle("dd_rope_apply", _P, _I, _I, _P, _P, _P, _P, _P, _I, _P)
_cache_append = _handle("dd_cache_append", _P, _I, _P, _P, _P, _P, _P, _P, _P, _P)
_cache_read = _handle("dd_cache_read", _P, _P, _I, _P, _I, _P)
_cache_decode_attn = _handle("dd_cache_decode_attn", _P, _I, _P, _P, _P, _P, _I, C.c_float, _P, C.c_size_t, _P)
_cache_landmarks = _handle("dd_cache_landmarks", _P, _P, _I, _P, _P)
_cache_select = _handle("dd_cache_select", _P, _I, _P, _P, _P, _P, _I, _I, _I, _P, _P, C.c_size_t, _P)
_cache_sparse_attn = _handle("dd_cache_sparse_attn", _P, _I, _P, _P, _P, _P, _I, _P, _P, C.c_float, _P, C.c_size_t, _P)


def _rows(t, name: str, head_dim: int, tokens: int):
    """`dd_rows` of a tensor [tokens, heads, head_dim] whose rows are dense (slices of a larger tensor are fine)."""
    kind, shape = _ROW_TYPES.get(t.dtype), t.shape
    if kind is None:
        raise _invalid(f"{name} must be bfloat16 or float16, not {t.dtype}")
    if len(shape) != 3 or shape[2] != head_dim or shape[0] != tokens:
        raise _invalid(f"{name} must be [{tokens}, heads, {head_dim}], not {tuple(shape)}")
    token, head, one = t.stride()
    if one != 1:
        raise _invalid(f"the elements of a row of {name} must be adjacent")
    h = shape[1]
    # a stride that is never stepped over may be anything: hand on one that passes
    return _PACK_ROWS(t.data_ptr(), kind, h, token if tokens > 1 else head_dim * h, head if h > 1 else head_dim)


def _rows4(t, name: str, head_dim: int):
    """`dd_rows` of [batch, tokens, heads, head_dim] as batch * tokens rows with one stride."""
    kind = _ROW_TYPES.get(t.dtype)
    if kind is None:
        raise _invalid(f"{name} must be bfloat16 or float16, not {t.dtype}")
    b, n, h, d = t.shape
    request, token, head, one = t.stride()
    if d != head_dim or one != 1:
        raise _invalid(f"{name} must be [batch, tokens, heads, {head_dim}] with dense rows, not {tuple(t.shape)}")
    if n == 1:
        token = request
    elif b > 1 and request != n * token:
        raise _invalid(f"the tokens of {name} must lie at one stride: [batch, tokens] has to fold into one dimension")
    return _PACK_ROWS(t.data_ptr(), kind, h, token if b * n > 1 else head_dim * h, head if h > 1 else head_dim)


def _ints(t, name: str, shape):
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        raise _invalid(f"{name} must be a dense int32 tensor of shape {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _raise_last(rc: int):
    raise DDError(rc, lib.dd_last_error_message(None).decode())


class Rope:
    """Rotary positions of one model: the turns per position of every pair (64 bits, on the device), the pair layout and the
    amplitude. See `dd_rope_turns` for the scalings."""

    def __init__(self, *, head_dim=128, rot_dim=None, base=10000.0, layout=DD_ROPE_HALF, scaling=DD_ROPE_NONE, factor=1.0,
                 original_len=0.0, low_turns=1.0, high_turns=32.0, amplitude=1.0, device="cuda"):
        self.head_dim, self.rot_dim = head_dim, head_dim if rot_dim is None else rot_dim
        n = max(1, self.rot_dim // 2)
        host = (C.c_double * n)()
        rc = lib.dd_rope_turns(self.rot_dim, base, scaling, factor, original_len, low_turns, high_turns, host)
        if rc != DD_OK:
            _raise_last(rc)
        self.turns_host = torch.tensor(list(host), dtype=torch.float64)
        self.turns = self.turns_host.to(device)
        self.c = DDRope(self.turns.data_ptr(), self.rot_dim, layout, amplitude)
        self._addr = C.addressof(self.c)

    def apply(self, positions, q, k, q_out=None, k_out=None, *, backward=False, stream=None):
        """Turns q [N, Hq, d] and k [N, Hkv, d] (either may be None) by their positions [N] into q_out and k_out; without
        an output, in place. backward: the transpose, i.e. the gradient with respect to the inputs."""
        n, d = positions.shape[0], self.head_dim
        rq = None if q is None else _rows(q, "q", d, n)
        rk = None if k is None else _rows(k, "k", d, n)
        rc = _rope_apply(self._addr, d, n, _ints(positions, "positions", (n,)), rq, rk,
                         rq if q_out is None else _rows(q_out, "q_out", d, n), rk if k_out is None else _rows(k_out, "k_out", d, n),
                         1 if backward else 0, _stream(stream))
        if rc != DD_OK:
            _raise_last(rc)


class PagedCache:
    """A pool of KV pages and the block tables of the requests that live in it (`dd_cache`). Owns nothing but an error word.

    data         [n_blocks, Hkv, ...]: each (block, head) one dense page of dd_cache_page_bytes() bytes; on the device, or
                 page-locked host memory (append and read only)
    block_table  [batch, max_pages] int32 on the device
    """

    def __init__(self, data, block_table, *, cache_format=DD_CACHE_BF16, head_dim=128, page_tokens=16, n_blocks=None,
                 block_stride=None, head_stride=None, n_kv_heads=None):
        page = lib.dd_cache_page_bytes(cache_format, page_tokens, head_dim)
        if page == 0:
            raise _invalid(f"format {cache_format} with {page_tokens} tokens of {head_dim} elements a page is not supported")
        size = data.element_size()
        if data.numel() == 0 or n_blocks == 0 or n_kv_heads == 0:
            raise _invalid("data is empty")
        if n_blocks is not None and (block_stride is None or head_stride is None or n_kv_heads is None):
            raise _invalid("n_blocks, block_stride, head_stride and n_kv_heads go together")
        if n_blocks is None:
            if data.dim() < 3 or data[0, 0].numel() * size != page or not data[0, 0].is_contiguous():
                raise _invalid(f"data must be [n_blocks, n_kv_heads, ...] with dense pages of {page} bytes, not {tuple(data.shape)}")
            n_blocks, n_kv_heads = data.shape[0], data.shape[1]
            block_stride = data.stride(0) * size if n_blocks > 1 else page * n_kv_heads
            head_stride = data.stride(1) * size if n_kv_heads > 1 else page
        extent = (n_blocks - 1) * block_stride + (n_kv_heads - 1) * head_stride + page
        if extent > data.untyped_storage().nbytes() - data.storage_offset() * size:
            raise _invalid(f"the pages reach over {extent} bytes, behind the end of data")
        if block_table.dtype != torch.int32 or block_table.dim() != 2 or (block_table.shape[1] > 1 and block_table.stride(1) != 1):
            raise _invalid("block_table must be int32 [batch, max_pages] with dense rows")
        batch, max_pages = block_table.shape
        if batch < 1 or max_pages < 1:
            raise _invalid("block_table is empty")
        self.data, self.block_table = data, block_table
        self.head_dim, self.page_tokens, self.cache_format = head_dim, page_tokens, cache_format
        self.status = torch.zeros(2, dtype=torch.int32, device=block_table.device)
        self.c = DDCache(data.data_ptr(), cache_format, n_kv_heads, head_dim, page_tokens, n_blocks, block_stride, head_stride,
                         block_table.data_ptr(), batch, max_pages, block_table.stride(0) if batch > 1 else max_pages,
                         self.status.data_ptr())
        self._addr = C.addressof(self.c)
        self._batch, self._heads, self._device = batch, n_kv_heads, block_table.device
        self._workspace_bytes = {}
        self._max_pages, self._landmark_shape = max_pages, (n_blocks, n_kv_heads, head_dim + 16)
        # the error word is zeroed on the stream the cache is made on: until that has run, calls on other streams wait for it
        self._made_on = self._made = None
        if self.status.is_cuda and not torch.cuda.is_current_stream_capturing():
            made_on = torch.cuda.current_stream(self._device)
            self._made_on, self._made = made_on.cuda_stream, made_on.record_event()

    def _stream(self, s) -> int:
        s, made = _stream(s), self._made
        if made is not None and s != self._made_on and not torch.cuda.is_current_stream_capturing():
            if made.query():
                self._made = None
            else:
                _torch_stream(s, self._device).wait_event(made)
        return s

    @classmethod
    def of_store(cls, kv_layer, *, cache_format=DD_CACHE_BF16, head_dim=128, page_tokens=16, device="cuda"):
        """A layer of the method's store, [B, Hkv, P, ...] dense, seen as a cache: page p of request b is its page p."""
        if kv_layer.dim() < 4 or not kv_layer.is_contiguous():
            raise _invalid("kv_layer must be a dense [batch, n_kv_heads, max_pages, ...] tensor")
        if kv_layer.numel() == 0:
            raise _invalid("kv_layer is empty")
        B, H, P = kv_layer.shape[:3]
        page = lib.dd_cache_page_bytes(cache_format, page_tokens, head_dim)
        if kv_layer[0, 0, 0].numel() * kv_layer.element_size() != page:
            raise _invalid(f"the pages of kv_layer must hold {page} bytes")
        table = (torch.arange(B, dtype=torch.int32).view(-1, 1) * (H * P) + torch.arange(P, dtype=torch.int32)).to(device)
        return cls(kv_layer, table, cache_format=cache_format, head_dim=head_dim, page_tokens=page_tokens,
                   n_blocks=(B - 1) * H * P + P, block_stride=page, head_stride=P * page, n_kv_heads=H)

    def append(self, k, v, positions, requests=None, *, rope=None, q=None, q_out=None, stream=None):
        """Writes k and v [N, Hkv, d] of N new tokens to position positions[n] of request requests[n] (None: N / batch tokens
        of each request in turn); with `rope`, k is turned on the way and q [N, Hq, d] into q_out (None: in place)."""
        n, d = positions.shape[0], self.head_dim
        if rope is not None and rope.head_dim != d:
            raise _invalid("rope and cache differ in head_dim")
        rq = None if q is None else _rows(q, "q", d, n)
        rc = _cache_append(self._addr, n, _ints(positions, "positions", (n,)),
                           None if requests is None else _ints(requests, "requests", (n,)),
                           _rows(k, "k", d, n), _rows(v, "v", d, n), None if rope is None else rope._addr, rq,
                           rq if q_out is None else _rows(q_out, "q_out", d, n), self._stream(stream))
        if rc != DD_OK:
            _raise_last(rc)

    def read(self, idx, out, stream=None):
        """Pages idx [batch, Hkv, k] (numbers within each request) in attention layout into out
        [batch, Hkv, 2, k * page_tokens, d], dense bfloat16 or float16."""
        kind, b, h = _ROW_TYPES.get(out.dtype), self._batch, self._heads
        if idx.dim() != 3:
            raise _invalid(f"idx must be [{b}, {h}, k], not {tuple(idx.shape)}")
        k = idx.shape[2]
        if kind is None or not out.is_contiguous() or out.shape != (b, h, 2, k * self.page_tokens, self.head_dim):
            raise _invalid(f"out must be a dense 16-bit tensor {(b, h, 2, k * self.page_tokens, self.head_dim)}")
        rc = _cache_read(self._addr, _ints(idx, "idx", (b, h, k)), k, out.data_ptr(), kind, self._stream(stream))
        if rc != DD_OK:
            _raise_last(rc)

    def decode_attn(self, q, ctx_len, out, out_lse=None, *, window=0, scale=0.0, workspace=None, stream=None):
        """Attention of the last Tq tokens of every request over its cached tokens. q, out [batch, Tq, Hq, d]; ctx_len
        [batch] int32; out_lse [batch, Tq, Hq] float32. Without a workspace the call takes one from torch's allocator on
        the stream it runs on (safe for several streams and for graph capture)."""
        b, shape = self._batch, q.shape
        if len(shape) != 4 or shape[0] != b or out.shape != shape:
            raise _invalid(f"q and out must be [{b}, tokens, heads, {self.head_dim}], not {tuple(shape)} and {tuple(out.shape)}")
        if not 0 <= window < 1 << 31:
            raise _invalid(f"window must be in [0, 2^31), not {window}")
        Tq, Hq = shape[1], shape[2]
        rq, ro = _rows4(q, "q", self.head_dim), _rows4(out, "out", self.head_dim)
        if out_lse is not None and (out_lse.dtype is not torch.float32 or out_lse.shape != (b, Tq, Hq) or not out_lse.is_contiguous()):
            raise _invalid(f"out_lse must be a dense float32 tensor {(b, Tq, Hq)}")
        if workspace is None:
            need = self._bytes((Hq, Tq), lambda: lib.dd_cache_decode_attn_workspace(Hq, self._heads, self.head_dim, Tq))
            workspace = self._take(need, stream)
        else:
            need = self._given(workspace)
        rc = _cache_decode_attn(self._addr, Tq, rq, _ints(ctx_len, "ctx_len", (b,)), ro,
                                None if out_lse is None else out_lse.data_ptr(), window, scale, workspace.data_ptr(), need,
                                self._stream(stream))
        if rc != DD_OK:
            _raise_last(rc)

    def _take(self, need: int, stream) -> torch.Tensor:
        """A workspace from torch's allocator on the stream of the call."""
        if stream is None:
            return torch.empty(need, dtype=torch.uint8, device=self._device)
        with torch.cuda.stream(_torch_stream(stream, self._device) if isinstance(stream, int) else stream):
            return torch.empty(need, dtype=torch.uint8, device=self._device)

    def _bytes(self, shape, ask) -> int:
        """Workspace bytes of a call of this shape, asked for once (and again when very many shapes have come by)."""
        need = self._workspace_bytes.get(shape)
        if need is None:
            if len(self._workspace_bytes) >= 1024:
                self._workspace_bytes.clear()
            need = self._workspace_bytes[shape] = max(16, ask())
        return need

    @staticmethod
    def _given(workspace) -> int:
        if not workspace.is_contiguous():
            raise _invalid("workspace must be dense")
        return workspace.numel() * workspace.element_size()

    def new_landmarks(self) -> torch.Tensor:
        """Zeroed landmarks for every (block, KV head) of the pool: uint8 [n_blocks, Hkv, dd_cache_landmark_bytes()]."""
        return torch.zeros(self.c.n_blocks, self._heads, lib.dd_cache_landmark_bytes(self.head_dim), dtype=torch.uint8, device=self._device)

    def _check_landmarks(self, landmarks) -> int:
        shape = self._landmark_shape
        if landmarks.dtype is not torch.uint8 or landmarks.shape != shape or not landmarks.is_contiguous():
            raise _invalid(f"landmarks must be a dense uint8 tensor {shape}, not {landmarks.dtype} {tuple(landmarks.shape)}")
        return landmarks.data_ptr()

    def update_landmarks(self, landmarks, ctx_len, *, n_last=0, stream=None):
        """Landmarks of the pages that hold any of the last n_last tokens of every request (0: of all its pages); ctx_len [batch]
        int32, the appended tokens counted in."""
        if not 0 <= n_last < 1 << 31:
            raise _invalid(f"n_last must be in [0, 2^31), not {n_last}")
        rc = _cache_landmarks(self._addr, _ints(ctx_len, "ctx_len", (self._batch,)), n_last, self._check_landmarks(landmarks), self._stream(stream))
        if rc != DD_OK:
            _raise_last(rc)

    def _listed(self, positions, idx, requests):
        """(tokens, pages a token, address of positions, of requests, of idx) of a call on listed pages."""
        n = positions.shape[0] if positions.dim() == 1 else -1
        if idx.dim() != 3 or idx.shape[2] < 1:
            raise _invalid(f"idx must be [tokens, {self._heads}, k], not {tuple(idx.shape)}")
        return (n, idx.shape[2], _ints(positions, "positions", (n,)), None if requests is None else _ints(requests, "requests", (n,)),
                _ints(idx, "idx", (n, self._heads, idx.shape[2])))

    def select(self, q, landmarks, positions, idx, requests=None, *, first_pages=0, recent_pages=1, workspace=None, stream=None):
        """The pages of every query token and KV head into idx [N, Hkv, k] int32 (ascending, -1 behind them): the first first_pages,
        the last recent_pages, and those with the highest scores (of the summed query heads and the landmarks, both as 8-bit whole
        numbers). q [N, Hq, d]; positions, requests [N] int32 as for append."""
        n, k, p, r, i = self._listed(positions, idx, requests)
        if not (0 <= first_pages <= k and 1 <= recent_pages <= k):
            raise _invalid(f"first_pages ({first_pages}) and recent_pages ({recent_pages}, at least 1) must fit the {k} pages of idx")
        rq = _rows(q, "q", self.head_dim, n)
        if workspace is None:
            need = self._bytes((n,), lambda: lib.dd_cache_select_workspace(n, self._heads, self._max_pages))
            workspace = self._take(need, stream)
        else:
            need = self._given(workspace)
        rc = _cache_select(self._addr, n, p, r, rq, self._check_landmarks(landmarks), k, first_pages, recent_pages, i,
                           workspace.data_ptr(), need, self._stream(stream))
        if rc != DD_OK:
            _raise_last(rc)

    def sparse_attn(self, q, idx, positions, out, out_lse=None, requests=None, *, scale=0.0, workspace=None, stream=None):
        """Attention of every query token over the pages idx [N, Hkv, k] listed for it, up to its own position. Only the entries in front are
        looked at, as many as there are pages up to the token's own, holes (-1) and repeats among them: pages come first, -1 behind
        them, as select gives them. q, out [N, Hq, d];
        positions, requests [N] int32 as for append; out_lse [N, Hq] float32. Without a workspace the call takes one from torch's
        allocator on the stream it runs on."""
        n, k, p, r, i = self._listed(positions, idx, requests)
        if q.shape != out.shape:
            raise _invalid(f"q and out must have one shape, not {tuple(q.shape)} and {tuple(out.shape)}")
        rq, ro = _rows(q, "q", self.head_dim, n), _rows(out, "out", self.head_dim, n)
        heads = q.shape[1]
        if out_lse is not None and (out_lse.dtype is not torch.float32 or out_lse.shape != (n, heads) or not out_lse.is_contiguous()):
            raise _invalid(f"out_lse must be a dense float32 tensor {(n, heads)}")
        if workspace is None:
            need = self._bytes((n, heads, k), lambda: lib.dd_cache_sparse_attn_workspace(n, heads, self._heads, self.head_dim, k))
            workspace = self._take(need, stream)
        else:
            need = self._given(workspace)
        rc = _cache_sparse_attn(self._addr, n, p, r, rq, i, k, ro, None if out_lse is None else out_lse.data_ptr(), scale,
                                workspace.data_ptr(), need, self._stream(stream))
        if rc != DD_OK:
            _raise_last(rc)

    def workspace(self, n_q_heads: int, n_q_tokens: int = 1) -> torch.Tensor:
        """A workspace for decode_attn calls of this shape."""
        return torch.empty(max(16, lib.dd_cache_decode_attn_workspace(n_q_heads, self.c.n_kv_heads, self.head_dim, n_q_tokens)),
                           dtype=torch.uint8, device=self.block_table.device)

    def device_error(self):
        """(code, detail) of the first index that a kernel found out of range, whatever stream its call went to; waits for all
        work of the device and clears it."""
        if self.status.is_cuda:
            torch.cuda.synchronize(self._device)
        code, detail = self.status.tolist()
        if code:
            self.status.zero_()
            if self.status.is_cuda:
                torch.cuda.current_stream(self._device).synchronize()      # before a call on another stream reports again
        return code, detail


class Context:
    """Owns one `dd_ctx`. Method names follow the C entry points (without the `dd_` prefix)."""

    def __init__(self, *, n_layers, batch, max_pages, k_pages, n_q_heads=32, n_kv_heads=8, head_dim=128,
                 page_tokens=16, forced_recent_pages=0, n_q_tokens=2, ring_depth=2, gather_mode=DD_GATHER_LOADS,
                 gather_ctas=0, select_mode=DD_SELECT_AUTO, attn_splits=0, compute_stream=None, copy_stream=None, ring=None,
                 miss_correction=False, urgent_stream=None, landmark_chunk_tokens=0, select_stream=None,
                 stage_min_run_pages=0, stage_block_pages=0, attn_mode=DD_ATTN_AUTO, store_format=DD_CACHE_BF16):
        if not torch.cuda.is_available():
            raise RuntimeError("the sparse decode path needs a CUDA device; there is no CPU fallback")
        self.compute_stream = compute_stream if compute_stream is not None else torch.cuda.current_stream()
        self.copy_stream = copy_stream if copy_stream is not None else torch.cuda.Stream()
        self._ring = ring
        self.urgent_stream = urgent_stream
        if miss_correction and urgent_stream is None:
            self.urgent_stream = torch.cuda.Stream(priority=-1)
        self.cfg = DDConfig(n_layers, batch, n_q_heads, n_kv_heads, head_dim, page_tokens, max_pages, k_pages,
                            forced_recent_pages, n_q_tokens, ring_depth, gather_mode, gather_ctas, select_mode, attn_splits,
                            self.compute_stream.cuda_stream, self.copy_stream.cuda_stream,
                            _ptr(ring), ring.numel() * ring.element_size() if ring is not None else 0,
                            landmark_chunk_tokens, 1 if miss_correction else 0,
                            self.urgent_stream.cuda_stream if self.urgent_stream is not None else None,
                            select_stream.cuda_stream if select_stream is not None else None,
                            stage_min_run_pages, stage_block_pages, attn_mode, store_format)
        self.select_stream = select_stream
        self._h = C.c_void_p()
        self._keep = []
        rc = lib.dd_create(C.byref(self.cfg), C.byref(self._h))
        if rc != DD_OK:
            raise DDError(rc, lib.dd_last_error_message(None).decode())

    # -- plumbing
    def _check(self, rc: int):
        if rc != DD_OK:
            raise DDError(rc, lib.dd_last_error_message(self._h).decode())

    def close(self):
        if self._h:
            rc = lib.dd_destroy(self._h)
            self._h = C.c_void_p()
            if rc != DD_OK:
                raise DDError(rc, "dd_destroy failed")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def slot_bytes(self) -> int:
        return lib.dd_slot_bytes(C.byref(self.cfg))

    def ring_bytes(self) -> int:
        return lib.dd_ring_bytes(C.byref(self.cfg))

    def scratch_bytes(self) -> int:
        return lib.dd_scratch_bytes(C.byref(self.cfg))

    def slot_ptr(self, slot: int) -> int:
        p = C.c_void_p()
        self._check(lib.dd_slot_ptr(self._h, slot, C.byref(p)))
        return p.value

    def slot_tensor(self, slot: int) -> torch.Tensor:
        """A copy of ring slot `slot` as [B, Hkv, 2, k*T, d] bf16 (synchronises; for tests)."""
        c = self.cfg
        shape = (c.batch, c.n_kv_heads, 2, c.k_pages * c.page_tokens, c.head_dim)
        torch.cuda.synchronize()
        return _view(self.slot_ptr(slot), shape, "bf16").clone()

    def sync(self, timeout_s: float = 60.0):
        self._check(lib.dd_sync(self._h, timeout_s))

    def device_error(self, timeout_s: float = 60.0):
        code, detail = C.c_int(), C.c_int()
        self._check(lib.dd_device_error(self._h, timeout_s, C.byref(code), C.byref(detail)))
        return code.value, detail.value

    def last_device_error(self):
        """(code, detail) of the first device-side error since the last device_error(), without synchronising."""
        code, detail = C.c_int(), C.c_int()
        self._check(lib.dd_last_device_error(self._h, C.byref(code), C.byref(detail)))
        return code.value, detail.value

    def gather_stats(self, reset=False) -> dict:
        """Host-side counters of the staged gather (see dd_gather_stats)."""
        a = (C.c_ulonglong * DD_GATHER_STATS_FIELDS)()
        self._check(lib.dd_gather_stats(self._h, a, 1 if reset else 0))
        names = ("gathers", "copies", "copied_bytes", "pages_staged", "pages_zero_copy", "host_wait_us", "host_issue_us")
        return dict(zip(names, [int(x) for x in a]))

    def set_bulk_wait(self, wait_seconds: float, inflate_first_stage: bool = False):
        self._check(lib.dd_set_bulk_wait(self._h, wait_seconds, 1 if inflate_first_stage else 0))

    # -- entry points
    def build_landmarks(self, kv_layer, ctx_len, landmarks, stream=None):
        self._check(lib.dd_build_landmarks(self._h, _ptr(kv_layer), _ptr(ctx_len), _ptr(landmarks), _stream(stream)))

    def select_topk(self, q, q_token, landmarks, n_pages, out_idx, out_scores=None, stream=None):
        self._check(lib.dd_select_topk(self._h, _ptr(q), q_token, _ptr(landmarks), _ptr(n_pages), _ptr(out_idx),
                                       _ptr(out_scores), _stream(stream)))

    def select_topk_chunked(self, q, q_token, landmarks, n_pages, ctx_len, out_idx, out_scores=None, stream=None):
        self._check(lib.dd_select_topk_chunked(self._h, _ptr(q), q_token, _ptr(landmarks), _ptr(n_pages), _ptr(ctx_len),
                                               _ptr(out_idx), _ptr(out_scores), _stream(stream)))

    def gather_kv_from_host(self, host_kv_layer, idx, n_pages, slot, stream=None):
        self._check(lib.dd_gather_kv_from_host(self._h, _ptr(host_kv_layer), _ptr(idx), _ptr(n_pages), slot,
                                               _stream(stream)))

    def sparse_decode_attn(self, q, slot, idx, ctx_len, out, out_lse=None, stream=None):
        self._check(lib.dd_sparse_decode_attn(self._h, _ptr(q), slot, _ptr(idx), _ptr(ctx_len), _ptr(out),
                                              _ptr(out_lse), _stream(stream)))

    def sparse_decode_attn_causal(self, q, slot, idx, ctx_len, k_new, v_new, out, out_lse=None, stream=None):
        self._check(lib.dd_sparse_decode_attn_causal(self._h, _ptr(q), slot, _ptr(idx), _ptr(ctx_len), _ptr(k_new),
                                                     _ptr(v_new), _ptr(out), _ptr(out_lse), _stream(stream)))

    def decode_layer_step_causal(self, step, layer, q, k_new, v_new, out):
        self._check(lib.dd_decode_layer_step_causal(self._h, step, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out)))

    def bind(self, landmarks_per_layer, host_kv_per_layer, n_pages, ctx_len):
        L = self.cfg.n_layers
        assert len(landmarks_per_layer) == L and len(host_kv_per_layer) == L
        self._keep = [landmarks_per_layer, host_kv_per_layer, n_pages, ctx_len]    # keep the tensors alive
        lm = (C.c_void_p * L)(*[_ptr(t) for t in landmarks_per_layer])
        kv = (C.c_void_p * L)(*[_ptr(t) for t in host_kv_per_layer])
        self._check(lib.dd_bind(self._h, lm, kv, _ptr(n_pages), _ptr(ctx_len)))

    def prime(self, q_init):
        self._check(lib.dd_prime(self._h, _ptr(q_init)))

    def decode_layer_step(self, step, layer, q, out):
        self._check(lib.dd_decode_layer_step(self._h, step, layer, _ptr(q), _ptr(out)))

    def diff_indices(self, pred_idx, true_idx, slot, merged_idx, stream=None):
        self._check(lib.dd_diff_indices(self._h, _ptr(pred_idx), _ptr(true_idx), slot, _ptr(merged_idx), _stream(stream)))

    def fetch_missing_from_host(self, host_kv_layer, slot, stream=None):
        self._check(lib.dd_fetch_missing_from_host(self._h, _ptr(host_kv_layer), slot, _stream(stream)))

    def get_merged_indices(self, slot) -> torch.Tensor:
        """A copy of the repaired page list [B, Hkv, k] int32 of ring slot `slot` (synchronises)."""
        p = C.c_void_p()
        self._check(lib.dd_get_merged_indices(self._h, slot, C.byref(p)))
        c = self.cfg
        torch.cuda.synchronize()
        return _view(p.value, (c.batch, c.n_kv_heads, c.k_pages), "i4").clone()

    def miss_stats(self, reset=False):
        """(missing pages, selected pages) accumulated by the corrected layer steps (synchronises)."""
        a, b = C.c_ulonglong(), C.c_ulonglong()
        self._check(lib.dd_miss_stats(self._h, C.byref(a), C.byref(b), 1 if reset else 0))
        return a.value, b.value

    def trace_begin(self, max_layer_steps: int):
        self._check(lib.dd_trace_begin(self._h, max_layer_steps))

    def trace_end(self):
        """Stops the trace and returns it as a [n, DD_TRACE_FIELDS] float32 numpy array of microseconds (see
        dd_trace_begin in dd_bench.h)."""
        import numpy as np
        n = C.c_int()
        self._check(lib.dd_trace_end(self._h, C.byref(n)))
        out = np.zeros((n.value, DD_TRACE_FIELDS), dtype=np.float32)
        if n.value:
            self._check(lib.dd_trace_read(self._h, 0, n.value, out.ctypes.data_as(C.c_void_p)))
        return out

    def probe_attn_loads(self, slot, stream=None):
        self._check(lib.dd_probe_attn_loads(self._h, slot, _stream(stream)))

    def probe_select_loads(self, landmarks, n_pages, stream=None):
        self._check(lib.dd_probe_select_loads(self._h, _ptr(landmarks), _ptr(n_pages), _stream(stream)))

    def decode_step_host(self, step, q_host, out_host):
        """One whole step from pinned host tensors [L, B, Tq, Hq, d] (asynchronous on the compute stream)."""
        self._check(lib.dd_decode_step_host(self._h, step, _ptr(q_host), _ptr(out_host)))

    def get_indices(self, step_parity, layer) -> torch.Tensor:
        """A copy of the index set [B, Hkv, k] int32 used at (step parity, layer) (synchronises)."""
        p = C.c_void_p()
        self._check(lib.dd_get_indices(self._h, step_parity, layer, C.byref(p)))
        c = self.cfg
        torch.cuda.synchronize()
        return _view(p.value, (c.batch, c.n_kv_heads, c.k_pages), "i4").clone()
