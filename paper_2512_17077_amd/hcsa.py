"""Thin ctypes binding over libdllm_hcsa.so (include/dllm_hcsa.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  Tensors are torch tensors on the GPU, used for device memory and the
current stream; nothing here computes.  If the library has not been built,
loading raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdllm_hcsa.so")
LIB_PATH_CHECKED = os.path.join(_HERE, "libdllm_hcsa_checked.so")   # built with the device-side precondition checks

DLLM_OK = 0
DLLM_ERR_INVALID_ARG = -1
DLLM_ERR_UNSUPPORTED = -2
DLLM_ERR_WORKSPACE = -3
DLLM_ERR_DEVICE = -4
DLLM_F32, DLLM_BF16 = 0, 1
DLLM_SEQ_SPARSE, DLLM_SEQ_DENSE = 0, 1
DLLM_SELECT_FORM_AUTO, DLLM_SELECT_FORM_TWO_LAUNCHES, DLLM_SELECT_FORM_ONE_LAUNCH = 0, 1, 2

EXPORTS = [
    "dllm_hcsa_select_workspace", "dllm_hcsa_select", "dllm_hcsa_select_ex", "dllm_hcsa_select_static",
    "dllm_hcsa_set_select_form", "dllm_hcsa_select_form_of",
    "dllm_hcsa_attend_workspace", "dllm_hcsa_attend", "dllm_hcsa_attend_form_of",
    "dllm_dense_refresh_attend_workspace", "dllm_dense_refresh_attend",
    "dllm_hcsa_pack", "dllm_hcsa_precondition_errors",
    "dllm_hcsa_cache_scale_slots", "dllm_hcsa_cache_write", "dllm_hcsa_cache_read",
    "dllm_hcsa_select_cached_workspace", "dllm_hcsa_select_cached",
    "dllm_hcsa_attend_cached_workspace", "dllm_hcsa_attend_cached", "dllm_hcsa_attend_cached_form_of",
    "dllm_last_error", "dllm_hcsa_version",
]
DLLM_CHECK_CU_Q, DLLM_CHECK_CU_KV, DLLM_CHECK_CU_K, DLLM_CHECK_K_OVER_L, DLLM_CHECK_FORCED, DLLM_CHECK_IDX = 1, 2, 4, 8, 16, 32


class DllmBatch(ctypes.Structure):
    """Mirror of `dllm_batch`."""
    _fields_ = [
        ("dtype", ctypes.c_int),
        ("batch", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("q", ctypes.c_void_p),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("q_stride_tok", ctypes.c_int64),
        ("q_stride_head", ctypes.c_int64),
        ("kv_stride_tok", ctypes.c_int64),
        ("kv_stride_head", ctypes.c_int64),
        ("cu_q", ctypes.c_void_p),
        ("cu_kv", ctypes.c_void_p),
        ("total_q", ctypes.c_int32),
        ("total_kv", ctypes.c_int32),
        ("max_q", ctypes.c_int32),
        ("max_kv", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
    ]


class DllmCache(ctypes.Structure):
    """Mirror of `dllm_cache`."""
    _fields_ = [
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("stride_tok", ctypes.c_int64),
        ("stride_head", ctypes.c_int64),
        ("scale_stride_head", ctypes.c_int64),
        ("scale_block", ctypes.c_int32),
    ]


class DllmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"dllm status {status}: {message}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """Open the built library (once).  A missing build is an error."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2512_17077_amd.build` "
                "(there is no CPU or PyTorch fallback for this library)")
        L = ctypes.CDLL(LIB_PATH)
        P, vp, i32, sz = ctypes.POINTER(DllmBatch), ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        L.dllm_hcsa_select_workspace.restype = sz
        L.dllm_hcsa_select_workspace.argtypes = [P, i32]
        L.dllm_hcsa_select.restype = ctypes.c_int
        L.dllm_hcsa_select.argtypes = [P, vp, i32, i32, i32, vp, vp, sz, vp]
        L.dllm_hcsa_select_ex.restype = ctypes.c_int
        L.dllm_hcsa_select_ex.argtypes = [P, vp, i32, i32, i32, i32, i32, vp, vp, sz, vp]
        L.dllm_hcsa_set_select_form.restype = i32
        L.dllm_hcsa_set_select_form.argtypes = [i32]
        L.dllm_hcsa_select_form_of.restype = i32
        L.dllm_hcsa_select_form_of.argtypes = [P, i32, i32]
        L.dllm_hcsa_select_static.restype = ctypes.c_int
        L.dllm_hcsa_select_static.argtypes = [P, vp, i32, i32, i32, i32, i32, vp, vp]
        L.dllm_hcsa_attend_workspace.restype = sz
        L.dllm_hcsa_attend_workspace.argtypes = [P, i32]
        L.dllm_hcsa_attend.restype = ctypes.c_int
        L.dllm_hcsa_attend.argtypes = [P, vp, vp, i32, i32, vp, vp, vp, sz, vp]
        L.dllm_hcsa_attend_form_of.restype = ctypes.c_int
        L.dllm_hcsa_attend_form_of.argtypes = [P, i32, i32, i32, ctypes.POINTER(i32)]
        L.dllm_dense_refresh_attend_workspace.restype = sz
        L.dllm_dense_refresh_attend_workspace.argtypes = [P]
        L.dllm_dense_refresh_attend.restype = ctypes.c_int
        L.dllm_dense_refresh_attend.argtypes = [P, vp, vp, sz, vp]
        L.dllm_hcsa_pack.restype = ctypes.c_int
        L.dllm_hcsa_pack.argtypes = [P, vp, vp, i32, i32, vp, vp, vp]
        L.dllm_hcsa_precondition_errors.restype = ctypes.c_int
        L.dllm_hcsa_precondition_errors.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32)]
        C, i64 = ctypes.POINTER(DllmCache), ctypes.c_int64
        L.dllm_hcsa_cache_scale_slots.restype = i64
        L.dllm_hcsa_cache_scale_slots.argtypes = [i32, i32, i32]
        L.dllm_hcsa_cache_write.restype = ctypes.c_int
        L.dllm_hcsa_cache_write.argtypes = [P, C, vp, i32, i32, vp, vp]
        L.dllm_hcsa_cache_read.restype = ctypes.c_int
        L.dllm_hcsa_cache_read.argtypes = [P, C, vp, i32, i32, vp, vp, vp, vp]
        L.dllm_hcsa_select_cached_workspace.restype = sz
        L.dllm_hcsa_select_cached_workspace.argtypes = [P, C, i32]
        L.dllm_hcsa_select_cached.restype = ctypes.c_int
        L.dllm_hcsa_select_cached.argtypes = [P, C, vp, i32, i32, i32, i32, i32, vp, vp, sz, vp]
        L.dllm_hcsa_attend_cached_workspace.restype = sz
        L.dllm_hcsa_attend_cached_workspace.argtypes = [P, C, i32]
        L.dllm_hcsa_attend_cached_form_of.restype = i32
        L.dllm_hcsa_attend_cached_form_of.argtypes = [P, C, i32, i32, i32]
        L.dllm_hcsa_attend_cached.restype = ctypes.c_int
        L.dllm_hcsa_attend_cached.argtypes = [P, C, vp, vp, i32, i32, vp, vp, sz, vp]
        L.dllm_last_error.restype = ctypes.c_char_p
        L.dllm_last_error.argtypes = []
        L.dllm_hcsa_version.restype = i32
        L.dllm_hcsa_version.argtypes = []
        _lib = L
    return _lib


def use_checked_library(on: bool = True):
    """Switch this binding to the library built with the device-side precondition checks (or back).  The
    checked library must have been built (paper_2512_17077_amd.build does both)."""
    global _lib, LIB_PATH
    _lib = None
    LIB_PATH = LIB_PATH_CHECKED if on else os.path.join(_HERE, "libdllm_hcsa.so")


def dllm_hcsa_precondition_errors(stream=None) -> int:
    """Fetch and clear the error word of the checked library (raises DLLM_ERR_UNSUPPORTED in the release one)."""
    out = ctypes.c_uint32(0)
    _raise(lib().dllm_hcsa_precondition_errors(_stream(stream), ctypes.byref(out)))
    return int(out.value)


def last_error() -> str:
    return lib().dllm_last_error().decode()


def _raise(status: int):
    if status != DLLM_OK:
        raise DllmError(status, last_error())


# Addresses and streams go through ctypes as plain integers (the prototypes say c_void_p), and the current stream
# is asked for by device number: torch.cuda.current_stream() builds a Stream object, 2.5 of the 10 us a call of
# two launches took on the host; small calls are bound by exactly that time.
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def make_batch(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_kv: torch.Tensor,
               max_q: int, max_kv: int, softmax_scale: float) -> DllmBatch:
    """Describe packed q [total_q,Hq,D], k/v [total_kv,Hkv,D] (last dim contiguous) to the library."""
    assert q.dim() == 3 and k.dim() == 3 and v.dim() == 3
    assert q.stride(2) == 1 and k.stride(2) == 1 and v.stride(2) == 1
    assert k.shape == v.shape and k.stride() == v.stride() and q.dtype == k.dtype == v.dtype
    assert cu_q.dtype == torch.int32 and cu_kv.dtype == torch.int32
    dt = {torch.float32: DLLM_F32, torch.bfloat16: DLLM_BF16}[q.dtype]
    b = DllmBatch()
    b.dtype = dt
    b.batch = cu_q.numel() - 1
    b.n_q_heads, b.n_kv_heads, b.head_dim = q.shape[1], k.shape[1], q.shape[2]
    b.q, b.k, b.v = q.data_ptr(), k.data_ptr(), v.data_ptr()
    b.q_stride_tok, b.q_stride_head = q.stride(0), q.stride(1)
    b.kv_stride_tok, b.kv_stride_head = k.stride(0), k.stride(1)
    b.cu_q, b.cu_kv = cu_q.data_ptr(), cu_kv.data_ptr()
    b.total_q, b.total_kv = q.shape[0], k.shape[0]
    b.max_q, b.max_kv = int(max_q), int(max_kv)
    b.softmax_scale = float(softmax_scale)
    return b


def _workspace(nbytes: int, device, stream=None) -> Optional[torch.Tensor]:
    """A workspace of the call's own.  It is allocated on the stream that works in it: memory of another stream's pool may
    still be read or written by what is queued there, for which this stream would not wait."""
    if nbytes == 0:
        return None
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)   # torch allocations are >= 256-byte aligned
    if not isinstance(stream, torch.cuda.Stream):   # (anything with a raw stream will do; 0 is the default one)
        raw = stream.cuda_stream
        stream = torch.cuda.ExternalStream(raw, device) if raw else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def dllm_hcsa_select_workspace(batch: DllmBatch, max_k: int) -> int:
    return int(lib().dllm_hcsa_select_workspace(ctypes.byref(batch), int(max_k)))


def dllm_hcsa_select(batch: DllmBatch, cu_k: torch.Tensor, total_k: int, max_k: int, idx_out: torch.Tensor,
                     pool_w: int = 1, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Per-head top-k selection; fills idx_out [Hq, total_k] (int32, device)."""
    if workspace is None:
        workspace = _workspace(dllm_hcsa_select_workspace(batch, max_k), idx_out.device, stream)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _raise(lib().dllm_hcsa_select(ctypes.byref(batch), _ptr(cu_k), int(total_k), int(max_k), int(pool_w),
                                  _ptr(idx_out), _ptr(workspace), nbytes, _stream(stream)))
    return idx_out


def dllm_hcsa_select_ex(batch: DllmBatch, cu_k: torch.Tensor, total_k: int, max_k: int, idx_out: torch.Tensor,
                        pool_w: int = 1, forced_tail: int = 0, head_sum: bool = False,
                        workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Selection with the block's own positions always kept and / or one list shared by all heads."""
    if workspace is None:
        workspace = _workspace(dllm_hcsa_select_workspace(batch, max_k), idx_out.device, stream)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _raise(lib().dllm_hcsa_select_ex(ctypes.byref(batch), _ptr(cu_k), int(total_k), int(max_k), int(pool_w),
                                     int(forced_tail), int(bool(head_sum)), _ptr(idx_out), _ptr(workspace), nbytes,
                                     _stream(stream)))
    return idx_out


DLLM_SELECT_STATIC_BYTES = 32 << 20


def dllm_hcsa_select_form_of(batch: DllmBatch, pool_w: int = 1, head_sum: bool = False) -> int:
    """Which of its two forms a selection call on this batch takes under the current setting (DLLM_SELECT_FORM_*)."""
    form = int(lib().dllm_hcsa_select_form_of(ctypes.byref(batch), int(pool_w), int(bool(head_sum))))
    if form < 0:
        raise ValueError(last_error())
    return form


def dllm_hcsa_set_select_form(form: int) -> int:
    """Process-wide choice between the two forms of selection (DLLM_SELECT_FORM_*); returns the previous one."""
    prev = int(lib().dllm_hcsa_set_select_form(int(form)))
    if prev < 0:
        raise ValueError(f"select form {form} is none of DLLM_SELECT_FORM_AUTO/TWO_LAUNCHES/ONE_LAUNCH")
    return prev


def dllm_hcsa_select_static(batch: DllmBatch, cu_k: torch.Tensor, total_k: int, max_k: int, idx_out: torch.Tensor,
                            pool_w: int = 1, forced_tail: int = 0, head_sum: bool = False, stream=None) -> torch.Tensor:
    """dllm_hcsa_select_ex on the library's built-in scratch buffer: no workspace, nothing allocated."""
    _raise(lib().dllm_hcsa_select_static(ctypes.byref(batch), _ptr(cu_k), int(total_k), int(max_k), int(pool_w),
                                         int(forced_tail), int(bool(head_sum)), _ptr(idx_out), _stream(stream)))
    return idx_out


def dllm_hcsa_attend_workspace(batch: DllmBatch, max_k: int) -> int:
    return int(lib().dllm_hcsa_attend_workspace(ctypes.byref(batch), int(max_k)))


def dllm_hcsa_attend_form_of(batch: DllmBatch, max_k: int = 0, total_k: int = 0, all_dense: bool = False):
    """(chunks per kept list, workgroups per list over head_dim, wave groups over a dense sequence's keys) of a call."""
    form = (ctypes.c_int32 * 3)()
    _raise(lib().dllm_hcsa_attend_form_of(ctypes.byref(batch), int(max_k), int(total_k), int(bool(all_dense)), form))
    return tuple(form)


def dllm_hcsa_attend(batch: DllmBatch, idx: Optional[torch.Tensor], cu_k: Optional[torch.Tensor], total_k: int,
                     max_k: int, seq_mode: Optional[torch.Tensor], o: torch.Tensor,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention over kept rows (and over all rows for sequences flagged dense); fills o."""
    if workspace is None:
        workspace = _workspace(dllm_hcsa_attend_workspace(batch, max_k), o.device, stream)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _raise(lib().dllm_hcsa_attend(ctypes.byref(batch), _ptr(idx), _ptr(cu_k), int(total_k), int(max_k),
                                  _ptr(seq_mode), _ptr(o), _ptr(workspace), nbytes, _stream(stream)))
    return o


def dllm_dense_refresh_attend_workspace(batch: DllmBatch) -> int:
    return int(lib().dllm_dense_refresh_attend_workspace(ctypes.byref(batch)))


def dllm_dense_refresh_attend(batch: DllmBatch, o: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                              stream=None) -> torch.Tensor:
    """Dense bidirectional attention of every sequence; fills o."""
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _raise(lib().dllm_dense_refresh_attend(ctypes.byref(batch), _ptr(o), _ptr(workspace), nbytes, _stream(stream)))
    return o


def dllm_hcsa_pack(batch: DllmBatch, idx: torch.Tensor, cu_k: torch.Tensor, total_k: int, max_k: int,
                   k_packed: torch.Tensor, v_packed: torch.Tensor, stream=None):
    """Copy every head's kept rows into k_packed / v_packed [Hq, total_k, D]."""
    _raise(lib().dllm_hcsa_pack(ctypes.byref(batch), _ptr(idx), _ptr(cu_k), int(total_k), int(max_k),
                                _ptr(k_packed), _ptr(v_packed), _stream(stream)))
    return k_packed, v_packed


def make_packed_batch(q: torch.Tensor, k_packed: torch.Tensor, v_packed: torch.Tensor, cu_q: torch.Tensor,
                      cu_k: torch.Tensor, max_q: int, max_k: int, softmax_scale: float) -> DllmBatch:
    """Describe packed buffers [Hq, total_k, D] as the K/V operand of an attend call: one KV head per
    query head, rows of a head contiguous, sequence b owning list positions cu_k[b] .. cu_k[b+1]-1."""
    assert k_packed.dim() == 3 and k_packed.is_contiguous() and v_packed.is_contiguous()
    return make_batch(q, k_packed.transpose(0, 1), v_packed.transpose(0, 1), cu_q, cu_k, max_q, max_k, softmax_scale)


# ---------------------------------------------------------------- the 8-bit cache
# (Checks cost the host 0.05 us an attribute and 0.04 a Python call, where the smallest calls take 5 us in all.)
_I32 = torch.int32


def _fits(t: torch.Tensor, dtype: torch.dtype, shape, place: int) -> bool:
    """What the kernels take a tensor for: its type, this shape without gaps, on the device numbered `place`."""
    return t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == place


def _check_lists(batch: DllmBatch, place: int, cu_k: torch.Tensor, idx: Optional[torch.Tensor], total_k: int):
    assert cu_k.dtype is _I32 and cu_k.shape == batch.cu_shape and cu_k.is_contiguous() and cu_k.get_device() == place, \
        "cu_k: contiguous int32 [batch + 1], on the cache's device"
    assert idx is None or (idx.dtype is _I32 and idx.shape == (batch.n_q_heads, total_k) and idx.is_contiguous() and
                           idx.get_device() == place), "lists: contiguous int32 [Hq, total_k], on the cache's device"


def cache_scale_slots(total_kv: int, batch: int, scale_block: int) -> int:
    """Entries of one head's row of scales in a cache of `batch` sequences with total_kv tokens together."""
    n = int(lib().dllm_hcsa_cache_scale_slots(int(total_kv), int(batch), int(scale_block)))
    if n < 0:
        raise ValueError(f"no cache has total_kv={total_kv}, batch={batch}, scale_block={scale_block} (16, 32 or 64)")
    return n


def make_cache(k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, scale_block: int) -> DllmCache:
    """Describe codes k/v [total_kv, Hkv, D] (float8_e4m3fn or uint8, last dim contiguous) and their scale bytes [Hkv, slots]
    (uint8, last dim contiguous) to the library.  Zero the memory of a new cache."""
    assert k.dim() == 3 and k.shape == v.shape and k.stride() == v.stride() and k.stride(2) == 1
    assert k.dtype == v.dtype and k.dtype in (torch.uint8, torch.float8_e4m3fn)
    assert k_scale.dtype == v_scale.dtype == torch.uint8 and k_scale.dim() == 2 and k_scale.shape[0] == k.shape[1]
    assert k_scale.shape == v_scale.shape and k_scale.stride() == v_scale.stride() and k_scale.stride(1) == 1
    assert k.device == v.device == k_scale.device == v_scale.device
    assert scale_block in (16, 32, 64)
    c = DllmCache()
    c.k, c.v, c.k_scale, c.v_scale = k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr()
    c.stride_tok, c.stride_head = k.stride(0), k.stride(1)
    # a single head's row is as long as its scales say, whatever stride a tensor of one row has
    c.scale_stride_head = k_scale.stride(0) if k_scale.shape[0] > 1 else k_scale.shape[1]
    c.scale_block = int(scale_block)
    # (not part of the C structure: the tensors stay alive with their descriptor, and what the checks of a call compare)
    c.tensors = (k, v, k_scale, v_scale)
    c.of = (int(k.shape[0]), int(k.shape[1]), int(k.shape[2]), k.device.index)
    c.place = k.get_device()
    c.most_sequences = int(k_scale.shape[1]) - int(k.shape[0]) // c.scale_block
    return c


def make_cached_batch(q: torch.Tensor, cu_q: torch.Tensor, cu_kv: torch.Tensor, total_kv: int, n_kv_heads: int, max_q: int,
                      max_kv: int, softmax_scale: float) -> DllmBatch:
    """Describe packed queries q [total_q,Hq,D] and the sequences of a cache (select_cached, attend_cached)."""
    assert q.dim() == 3 and q.stride(2) == 1
    b = DllmBatch()
    b.dtype = {torch.float32: DLLM_F32, torch.bfloat16: DLLM_BF16}[q.dtype]
    b.batch = cu_q.numel() - 1
    for cu in (cu_q, cu_kv):
        assert _fits(cu, torch.int32, (b.batch + 1,), q.get_device()), "cu_q and cu_kv: contiguous int32 [batch + 1], on q's device"
    b.n_q_heads, b.n_kv_heads, b.head_dim = q.shape[1], int(n_kv_heads), q.shape[2]
    b.q = q.data_ptr()
    b.q_stride_tok, b.q_stride_head = q.stride(0), q.stride(1)
    b.cu_q, b.cu_kv = cu_q.data_ptr(), cu_kv.data_ptr()
    b.total_q, b.total_kv = q.shape[0], int(total_kv)
    b.max_q, b.max_kv = int(max_q), int(max_kv)
    b.softmax_scale = float(softmax_scale)
    b.tensors = (q, cu_q, cu_kv)   # (as in make_cache)
    b.of, b.sequences = (b.total_kv, b.n_kv_heads, b.head_dim, q.device.index), b.batch
    b.q_shape, b.q_dtype, b.cu_shape = q.shape, q.dtype, cu_q.shape
    return b


def make_rows_batch(k: torch.Tensor, v: torch.Tensor, cu_kv: torch.Tensor, total_kv: int, max_kv: int) -> DllmBatch:
    """Describe rows k/v [total_rows,Hkv,D] (bf16 or fp32) and the sequences of the cache that they go to or come from."""
    assert k.dim() == 3 and k.stride(2) == 1 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype
    b = DllmBatch()
    b.dtype = {torch.float32: DLLM_F32, torch.bfloat16: DLLM_BF16}[k.dtype]
    b.batch = cu_kv.numel() - 1
    assert _fits(cu_kv, torch.int32, (b.batch + 1,), k.get_device()), "cu_kv: contiguous int32 [batch + 1], on the rows' device"
    assert v.get_device() == k.get_device(), "k and v are on different devices"
    b.n_q_heads = b.n_kv_heads = k.shape[1]
    b.head_dim = k.shape[2]
    b.k, b.v = k.data_ptr(), v.data_ptr()
    b.kv_stride_tok, b.kv_stride_head = k.stride(0), k.stride(1)
    b.cu_kv = cu_kv.data_ptr()
    b.total_kv, b.max_kv = int(total_kv), int(max_kv)
    b.tensors = (k, v, cu_kv)   # (as in make_cache)
    b.of, b.sequences = (b.total_kv, b.n_kv_heads, b.head_dim, k.device.index), b.batch
    b.rows, b.place = int(k.shape[0]), k.get_device()
    return b


def _cached_stream(batch: DllmBatch, cache: DllmCache, stream) -> int:
    """Checks that the two descriptors belong together and lie on the current device (where the call launches); the stream."""
    assert batch.of == cache.of, "the cache has another shape or device than the batch says"
    assert batch.sequences <= cache.most_sequences, "too few scales (cache_scale_slots)"
    device = torch.cuda.current_device()
    if device != cache.of[3]:
        raise ValueError(f"the tensors are on device {cache.of[3]}, the current device is {device}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    if stream.device_index != device:
        raise ValueError(f"the stream is on device {stream.device_index}, the current device is {device}")
    return stream.cuda_stream


def _rows_moved(batch: DllmBatch, cu_rows, total_rows: Optional[int], max_rows: Optional[int], at):
    """(total_rows, max_rows) of a write or read, checked."""
    if cu_rows is None:
        assert at is None and batch.rows >= batch.of[0], "without cu_rows all rows are moved"
        return batch.of[0], 0
    assert total_rows is not None and max_rows is not None, "cu_rows lies on the device: total_rows and max_rows say what is in it"
    place = batch.place
    assert _fits(cu_rows, torch.int32, (batch.sequences + 1,), place), "cu_rows: contiguous int32 [batch + 1], on the rows' device"
    assert at is None or _fits(at, torch.int32, (batch.sequences,), place), "at: contiguous int32 [batch], on the rows' device"
    assert batch.rows >= total_rows, "fewer rows than total_rows"
    return total_rows, max_rows


def dllm_hcsa_cache_write(batch: DllmBatch, cache: DllmCache, cu_rows: Optional[torch.Tensor] = None,
                          total_rows: Optional[int] = None, max_rows: Optional[int] = None, at: Optional[torch.Tensor] = None,
                          stream=None) -> DllmCache:
    """Quantise the rows of `batch` (make_rows_batch) into the cache: cu_rows[b] .. cu_rows[b+1]-1 to positions at[b] .. of
    sequence b (at None: its last ones), or every sequence whole (cu_rows None)."""
    total_rows, max_rows = _rows_moved(batch, cu_rows, total_rows, max_rows, at)
    stream = _cached_stream(batch, cache, stream)
    status = (_lib or lib()).dllm_hcsa_cache_write(batch, cache, _ptr(cu_rows), total_rows, max_rows, _ptr(at), stream)
    if status:
        _raise(status)
    return cache


def dllm_hcsa_cache_read(batch: DllmBatch, cache: DllmCache, k_out: torch.Tensor, v_out: torch.Tensor,
                         cu_rows: Optional[torch.Tensor] = None, total_rows: Optional[int] = None,
                         max_rows: Optional[int] = None, at: Optional[torch.Tensor] = None, stream=None):
    """Read rows of the cache back into k_out / v_out, the tensors that `batch` describes (make_rows_batch)."""
    assert (batch.k or 0) == k_out.data_ptr() and (batch.v or 0) == v_out.data_ptr(), "batch describes other tensors"
    total_rows, max_rows = _rows_moved(batch, cu_rows, total_rows, max_rows, at)
    stream = _cached_stream(batch, cache, stream)
    _raise(lib().dllm_hcsa_cache_read(batch, cache, _ptr(cu_rows), total_rows, max_rows, _ptr(at), batch.k, batch.v, stream))
    return k_out, v_out


def dllm_hcsa_select_cached_workspace(batch: DllmBatch, cache: DllmCache, max_k: int) -> int:
    return int(lib().dllm_hcsa_select_cached_workspace(ctypes.byref(batch), ctypes.byref(cache), int(max_k)))


def dllm_hcsa_select_cached(batch: DllmBatch, cache: DllmCache, cu_k: torch.Tensor, total_k: int, max_k: int,
                            idx_out: torch.Tensor, pool_w: int = 1, forced_tail: int = 0, head_sum: bool = False,
                            workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Selection over the cached K (batch: make_cached_batch); fills idx_out [Hq, total_k] (int32, device)."""
    raw, place = _cached_stream(batch, cache, stream), cache.place
    _check_lists(batch, place, cu_k, idx_out, total_k)
    if workspace is None:
        workspace = _workspace(dllm_hcsa_select_cached_workspace(batch, cache, max_k), idx_out.device, stream)
    space, nbytes = None, 0
    if workspace is not None:
        assert workspace.is_contiguous() and workspace.get_device() == place, "the workspace is not contiguous or on another device"
        space, nbytes = workspace.data_ptr(), workspace.nbytes
    status = (_lib or lib()).dllm_hcsa_select_cached(batch, cache, cu_k.data_ptr(), total_k, max_k, pool_w, forced_tail,
                                                     1 if head_sum else 0, idx_out.data_ptr(), space, nbytes, raw)
    if status:
        _raise(status)
    return idx_out


def dllm_hcsa_attend_cached_workspace(batch: DllmBatch, cache: DllmCache, max_k: int) -> int:
    return int(lib().dllm_hcsa_attend_cached_workspace(ctypes.byref(batch), ctypes.byref(cache), int(max_k)))


def dllm_hcsa_attend_cached_form_of(batch: DllmBatch, cache: DllmCache, lists: bool, max_k: int, total_k: int) -> int:
    """Rows per piece in which a call cuts its lists, 0 if every list is taken whole."""
    piece = int(lib().dllm_hcsa_attend_cached_form_of(ctypes.byref(batch), ctypes.byref(cache), int(bool(lists)), int(max_k),
                                                      int(total_k)))
    if piece < 0:
        raise ValueError(last_error())
    return piece


def dllm_hcsa_attend_cached(batch: DllmBatch, cache: DllmCache, idx: Optional[torch.Tensor], cu_k: torch.Tensor, total_k: int,
                            max_k: int, o: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention over the cache: every head over its own list, or (idx None) all heads over the first rows of each sequence."""
    raw, place = _cached_stream(batch, cache, stream), cache.place
    _check_lists(batch, place, cu_k, idx, total_k)
    assert o.dtype is batch.q_dtype and o.shape == batch.q_shape and o.is_contiguous() and o.get_device() == place, \
        "o: contiguous, of q's type and shape, on the cache's device"
    if workspace is None:
        workspace = _workspace(dllm_hcsa_attend_cached_workspace(batch, cache, max_k), o.device, stream)
    space, nbytes = None, 0
    if workspace is not None:
        assert workspace.is_contiguous() and workspace.get_device() == place, "the workspace is not contiguous or on another device"
        space, nbytes = workspace.data_ptr(), workspace.nbytes
    status = (_lib or lib()).dllm_hcsa_attend_cached(batch, cache, None if idx is None else idx.data_ptr(), cu_k.data_ptr(), total_k,
                                                     max_k, o.data_ptr(), space, nbytes, raw)
    if status:
        _raise(status)
    return o
