"""ctypes binding of libtq.so: argument marshalling only, same names as include/tq.h.

Host arrays are numpy arrays; device memory is torch CUDA tensors (PyTorch is used for
device memory and streams only).  There is no CPU fallback: if libtq.so cannot be loaded (or
built with nvcc) importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import functools
from dataclasses import dataclass

import numpy as np
import torch

from . import build as _build

TQ_OK = 0
TQ_ERR_INVALID_ARG = -1
TQ_ERR_CORRUPT_STREAM = -2
TQ_ERR_BUFFER_TOO_SMALL = -3
TQ_ERR_UNSUPPORTED_SHAPE = -4
TQ_ERR_CUDA = -5
TQ_ERR_TIMEOUT = -6
TQ_ERR_NOMEM = -7
TQ_LAYOUT_STREAM = 0
TQ_LAYOUT_PLANES = 1
TQ_LAYOUT_TILES = 2
TQ_TILES_TABLE_WORDS = 33024
TQ_TILES_MAX_COLS = 65536
TQ_STATUS_BAD_CODE = 1
TQ_STATUS_BAD_ROW = 2
TQ_STATUS_WAIT_EXPIRED = 4
TQ_STATUS_BAD_PAGE = 8
TQ_STATUS_BAD_POSITION = 16
TQ_TYPE_BF16 = 0
TQ_TYPE_F32 = 1
TQ_NORM_MAX_COLS = 16384
TQ_ROPE_MAX_AXES = 3
TQ_SAMPLE_MAX_VOCAB = 262144
TQ_MAX_CACHES = 128
TQ_TREE_MAX_PATH = 256

EXPORTS = [
    "tq_strerror", "tq_last_cuda_error", "tq_set_num_threads", "tq_quantize_tensor", "tq_quantize_tensor_bits", "tq_quantize_rows",
    "tq_quantize_rows_device", "tq_build_dictionary", "tq_build_dictionary_device_size", "tq_build_dictionary_device", "tq_dict_from_entries", "tq_dict_entries",
    "tq_encode", "tq_dict_free", "tq_dict_upload_size", "tq_dict_upload", "tq_ddict_free",
    "tq_upload_size", "tq_upload", "tq_upload_device_size", "tq_upload_device", "tq_upload_device_rows", "tq_tiles_image_host", "tq_dmat_get_info", "tq_decompress", "tq_fused_gemv",
    "tq_fused_gemv_host", "tq_fused_gemv_host_static", "tq_fused_gemm", "tq_gemm_workspace_size",
    "tq_fused_gemm_ws", "tq_decode_bf16", "tq_gemm_bf16_ws", "tq_decode_bf16_stack", "tq_gemm_plan_size", "tq_gemm_plan_create", "tq_gemm_plan_run",
    "tq_gemm_plan_status", "tq_gemm_plan_free", "tq_stack_size", "tq_stack_plan_host", "tq_stack_create",
    "tq_fused_gemv_stack", "tq_fused_gemv_stack_host", "tq_stack_launches", "tq_test_withhold_table_chunk", "tq_decompress_stack", "tq_stack_free", "tq_device_status", "tq_dmat_free",
    "tq_rmsnorm", "tq_rmsnorm_q8", "tq_rope_append", "tq_attn_workspace_size", "tq_attn_workspace_init", "tq_paged_attention",
    "tq_cross_attention", "tq_attn_status", "tq_test_withhold_cross_entry",
    "tq_qk_norm_rope_append", "tq_tree_attention", "tq_sample", "tq_tree_accept",
]


class TqError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str | None = None):
        self.status = status
        if detail is None:
            detail = _lib.tq_last_cuda_error().decode() if status == TQ_ERR_CUDA else ""
        super().__init__(f"{where}: {_lib.tq_strerror(status).decode()} ({status}) {detail}")


class _Info(C.Structure):
    _fields_ = [("rows", C.c_uint32), ("cols", C.c_uint32), ("K", C.c_uint32),
                ("layout", C.c_int32), ("levels_signed", C.c_int32),
                ("n_hits", C.c_uint64), ("n_miss", C.c_uint64), ("stream_bytes", C.c_uint64),
                ("payload_bytes", C.c_uint64), ("device_bytes", C.c_uint64), ("n_raw_words", C.c_uint64)]


class _KvCache(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("n_pages", C.c_uint32), ("page_size", C.c_uint32),
                ("n_kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("slot_stride", C.c_int64), ("d_status", C.c_void_p)]


class _EncoderKv(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("n_seqs", C.c_uint32), ("n_states", C.c_uint32),
                ("n_kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("batch_stride", C.c_int64), ("state_stride", C.c_int64),
                ("head_stride", C.c_int64)]


def _load() -> C.CDLL:
    path = _build.build_library()  # raises if the library is missing and cannot be built
    lib = C.CDLL(str(path))
    vp, u8p, u16p, u32p, u64p = C.c_void_p, C.POINTER(C.c_uint8), C.POINTER(C.c_uint16), C.POINTER(C.c_uint32), C.POINTER(C.c_uint64)
    f32p = C.POINTER(C.c_float)
    sig = {
        "tq_strerror": (C.c_char_p, [C.c_int]),
        "tq_last_cuda_error": (C.c_char_p, []),
        "tq_set_num_threads": (C.c_int, [C.c_int]),
        "tq_quantize_tensor": (C.c_int, [f32p, C.c_uint64, u8p, f32p, f32p]),
        "tq_quantize_tensor_bits": (C.c_int, [f32p, C.c_uint64, C.c_int, u8p, f32p, f32p]),
        "tq_quantize_rows": (C.c_int, [f32p, C.c_uint32, C.c_uint32, C.POINTER(C.c_int8), f32p]),
        "tq_quantize_rows_device": (C.c_int, [vp, C.c_uint32, C.c_uint32, vp, vp, vp]),
        "tq_build_dictionary": (C.c_int, [C.POINTER(u8p), u64p, C.c_int, C.c_uint32, C.POINTER(vp)]),
        "tq_build_dictionary_device_size": (C.c_int, [u64p, C.c_int, u64p]),
        "tq_build_dictionary_device": (C.c_int, [C.POINTER(vp), u64p, C.c_int, C.c_uint32, vp, C.c_uint64, vp, C.POINTER(vp)]),
        "tq_dict_from_entries": (C.c_int, [u8p, C.c_uint32, C.POINTER(vp)]),
        "tq_dict_entries": (C.c_int, [vp, u32p, C.POINTER(u8p), C.POINTER(u64p)]),
        "tq_encode": (C.c_int, [vp, u8p, C.c_uint64, u16p, C.c_uint64, u64p, u64p, u64p]),
        "tq_dict_free": (None, [vp]),
        "tq_dict_upload_size": (C.c_int, [vp, u64p]),
        "tq_dict_upload": (C.c_int, [vp, vp, C.c_uint64, vp, C.POINTER(vp)]),
        "tq_ddict_free": (None, [vp]),
        "tq_upload_size": (C.c_int, [u16p, C.c_uint64, C.c_uint32, C.c_uint32, C.c_int, u64p]),
        "tq_upload": (C.c_int, [vp, u16p, C.c_uint64, C.c_uint32, C.c_uint32, f32p, f32p, C.c_int,
                                C.c_int, vp, C.c_uint64, vp, C.POINTER(vp)]),
        "tq_upload_device_size": (C.c_int, [C.c_uint32, C.c_uint32, u64p]),
        "tq_upload_device": (C.c_int, [vp, vp, C.c_uint32, C.c_uint32, vp, vp, C.c_int, vp, C.c_uint64, vp, C.POINTER(vp)]),
        "tq_upload_device_rows": (C.c_int, [vp, vp, C.c_uint32, C.c_uint32, C.c_uint32, C.c_uint32, vp, vp, C.c_int, vp, C.c_uint64, vp,
                                            C.POINTER(vp)]),
        "tq_tiles_image_host": (C.c_int, [vp, u16p, C.c_uint64, C.c_uint32, C.c_uint32, f32p, f32p, u8p,
                                          C.c_uint64, u64p, u64p, u32p]),
        "tq_dmat_get_info": (C.c_int, [vp, C.POINTER(_Info)]),
        "tq_decompress": (C.c_int, [vp, vp, vp]),
        "tq_fused_gemv": (C.c_int, [vp, vp, C.c_int, vp, vp]),
        "tq_fused_gemv_host": (C.c_int, [vp, vp, C.c_int, vp, vp, vp, vp]),
        "tq_fused_gemv_host_static": (C.c_int, [vp, vp, C.c_int, vp, vp]),
        "tq_fused_gemm": (C.c_int, [vp, vp, C.c_int, vp, vp]),
        "tq_gemm_workspace_size": (C.c_int, [vp, u64p]),
        "tq_fused_gemm_ws": (C.c_int, [vp, vp, C.c_int, vp, vp, C.c_uint64, vp]),
        "tq_decode_bf16": (C.c_int, [vp, vp, C.c_uint64, vp]),
        "tq_gemm_bf16_ws": (C.c_int, [vp, vp, C.c_int, vp, vp, vp]),
        "tq_decode_bf16_stack": (C.c_int, [vp, vp, vp]),
        "tq_gemm_plan_size": (C.c_int, [C.c_int, u64p]),
        "tq_gemm_plan_create": (C.c_int, [C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.c_int, C.c_int, vp,
                                          C.c_uint64, vp, C.POINTER(vp)]),
        "tq_gemm_plan_run": (C.c_int, [vp, vp]),
        "tq_gemm_plan_status": (C.c_int, [vp, vp, u32p]),
        "tq_gemm_plan_free": (None, [vp]),
        "tq_stack_size": (C.c_int, [C.POINTER(vp), C.c_int, C.c_int, u64p]),
        "tq_stack_plan_host": (C.c_int, [C.c_int, u32p, u32p, C.POINTER(u32p), C.c_uint32, u32p, C.c_uint32, u32p, u32p]),
        "tq_stack_create": (C.c_int, [C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.c_int, C.c_int, vp, C.c_uint64, vp,
                                      C.POINTER(vp)]),
        "tq_fused_gemv_stack": (C.c_int, [vp, vp]),
        "tq_fused_gemv_stack_host": (C.c_int, [vp, vp, vp, C.c_uint64, vp, vp, C.c_uint64, vp]),
        "tq_stack_launches": (C.c_int, [vp]),
        "tq_test_withhold_table_chunk": (None, [C.c_int]),
        "tq_test_withhold_cross_entry": (None, [C.c_int]),
        "tq_decompress_stack": (C.c_int, [vp, vp, vp]),
        "tq_stack_free": (None, [vp]),
        "tq_device_status": (C.c_int, [vp, vp, u32p]),
        "tq_dmat_free": (None, [vp]),
        "tq_rmsnorm": (C.c_int, [vp, C.c_int, C.c_int64, vp, C.c_int, C.c_int64, vp, C.c_float, C.c_uint32, C.c_uint32, vp, vp, vp]),
        "tq_rmsnorm_q8": (C.c_int, [vp, C.c_int, C.c_int64, vp, C.c_int, C.c_int64, vp, C.c_float, C.c_uint32, C.c_uint32, vp, vp,
                                    vp, vp]),
        "tq_rope_append": (C.c_int, [vp, vp, vp, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_uint32, C.c_uint32, vp, C.c_uint32,
                                     C.c_uint32, vp, u32p, C.c_uint32, C.c_int, vp, C.POINTER(_KvCache), vp, vp]),
        "tq_attn_workspace_size": (C.c_int, [u64p]),
        "tq_attn_workspace_init": (C.c_int, [vp, C.c_uint64, vp]),
        "tq_paged_attention": (C.c_int, [C.POINTER(_KvCache), vp, C.c_int64, C.c_uint32, C.c_uint32, vp, C.c_uint32, vp, C.c_float,
                                         vp, vp, vp, C.c_uint64, vp]),
        "tq_cross_attention": (C.c_int, [C.POINTER(_EncoderKv), vp, C.c_int64, C.c_int64, C.c_uint32, C.c_uint32, vp, vp, C.c_uint32,
                                         C.c_float, vp, vp, vp, C.c_uint64, vp]),
        "tq_attn_status": (C.c_int, [vp, vp, u32p]),
        "tq_qk_norm_rope_append": (C.c_int, [vp, vp, vp, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_uint32, C.c_uint32, vp, vp, C.c_float, vp,
                                             C.c_uint32, C.c_uint32, vp, u32p, C.c_uint32, C.c_int, vp, C.POINTER(_KvCache), vp, vp]),
        "tq_tree_attention": (C.c_int, [C.POINTER(_KvCache), vp, C.c_int64, C.c_uint32, C.c_uint32, C.c_uint32, vp, vp, C.c_uint32, vp, vp,
                                        C.c_uint32, C.c_float, vp, vp, vp, C.c_uint64, vp]),
        "tq_sample": (C.c_int, [vp, C.c_int, C.c_int64, C.c_uint32, C.c_uint32, vp, vp, vp, vp, vp, vp, vp, vp]),
        "tq_tree_accept": (C.c_int, [C.POINTER(_KvCache), C.c_uint32, vp, C.c_uint32, C.c_uint32, C.c_uint32, vp, vp, vp, vp, vp, C.c_uint32,
                                     vp, vp, vp, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


_lib = _load()


def _check(status: int, where: str) -> None:
    if status != TQ_OK:
        raise TqError(status, where)


def _np_ptr(a: np.ndarray, ctype):
    return a.ctypes.data_as(C.POINTER(ctype))


def _stream_ptr(stream=None) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def tq_set_num_threads(n: int) -> int:
    return _lib.tq_set_num_threads(n)


# ------------------------------------------------------------------------------ host
def tq_quantize_tensor(x: np.ndarray):
    x = np.ascontiguousarray(x, dtype=np.float32)
    q = np.empty(x.shape, dtype=np.uint8)
    s, z = C.c_float(), C.c_float()
    _check(_lib.tq_quantize_tensor(_np_ptr(x, C.c_float), x.size, _np_ptr(q, C.c_uint8), C.byref(s), C.byref(z)),
           "tq_quantize_tensor")
    return q, np.float32(s.value), np.float32(z.value)


def tq_quantize_tensor_bits(x: np.ndarray, bits: int):
    x = np.ascontiguousarray(x, dtype=np.float32)
    q = np.empty(x.shape, dtype=np.uint8)
    s, z = C.c_float(), C.c_float()
    _check(_lib.tq_quantize_tensor_bits(_np_ptr(x, C.c_float), x.size, int(bits), _np_ptr(q, C.c_uint8), C.byref(s),
                                        C.byref(z)), "tq_quantize_tensor_bits")
    return q, np.float32(s.value), np.float32(z.value)


def tq_quantize_rows(w: np.ndarray):
    w = np.ascontiguousarray(w, dtype=np.float32)
    rows, cols = w.shape
    q = np.empty((rows, cols), dtype=np.int8)
    s = np.empty(rows, dtype=np.float32)
    _check(_lib.tq_quantize_rows(_np_ptr(w, C.c_float), rows, cols, _np_ptr(q, C.c_int8), _np_ptr(s, C.c_float)),
           "tq_quantize_rows")
    return q, s


def tq_quantize_rows_device(w: torch.Tensor, stream=None):
    assert w.is_cuda and w.dtype == torch.float32 and w.is_contiguous() and w.dim() == 2
    rows, cols = w.shape
    q = torch.empty((rows, cols), dtype=torch.int8, device=w.device)
    s = torch.empty(rows, dtype=torch.float32, device=w.device)
    _check(_lib.tq_quantize_rows_device(w.data_ptr(), rows, cols, q.data_ptr(), s.data_ptr(), _stream_ptr(stream)),
           "tq_quantize_rows_device")
    return q, s


class Dict:
    """Owner of a host tq_dict handle."""

    def __init__(self, handle: int):
        self._h = C.c_void_p(handle)

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.tq_dict_free(self._h)
            self._h = None

    def _borrow(self):
        K, e, c = C.c_uint32(), C.POINTER(C.c_uint8)(), C.POINTER(C.c_uint64)()
        _check(_lib.tq_dict_entries(self._h, C.byref(K), C.byref(e), C.byref(c)), "tq_dict_entries")
        return K.value, e, c

    @property
    def K(self) -> int:
        return self._borrow()[0]

    @property
    def entries(self) -> np.ndarray:
        K, e, _ = self._borrow()
        return np.ctypeslib.as_array(e, shape=(K, 4)).copy() if K else np.zeros((0, 4), np.uint8)

    @property
    def counts(self) -> np.ndarray:
        K, _, c = self._borrow()
        return np.ctypeslib.as_array(c, shape=(K,)).copy() if K else np.zeros((0,), np.uint64)


def tq_build_dictionary(mats, top_k: int = 2 ** 16 - 1) -> Dict:
    arrs = [np.ascontiguousarray(m).view(np.uint8).reshape(-1) for m in mats]
    n = len(arrs)
    ptrs = (C.POINTER(C.c_uint8) * max(n, 1))(*[_np_ptr(a, C.c_uint8) for a in arrs])
    lens = (C.c_uint64 * max(n, 1))(*[a.size for a in arrs])
    out = C.c_void_p()
    _check(_lib.tq_build_dictionary(ptrs, lens, n, top_k, C.byref(out)), "tq_build_dictionary")
    return Dict(out.value)


def tq_build_dictionary_device(mats, top_k: int = 2 ** 16 - 1, stream=None) -> Dict:
    """mats: CUDA 1-byte tensors (levels).  Counts the windows on the GPU; same table as tq_build_dictionary."""
    n = len(mats)
    assert n >= 1
    for m in mats:
        assert m.is_cuda and m.is_contiguous() and m.element_size() == 1
    lens = (C.c_uint64 * n)(*[m.numel() for m in mats])
    need = C.c_uint64()
    _check(_lib.tq_build_dictionary_device_size(lens, n, C.byref(need)), "tq_build_dictionary_device_size")
    ws = torch.empty(need.value, dtype=torch.uint8, device=mats[0].device)
    ptrs = (C.c_void_p * n)(*[m.data_ptr() for m in mats])
    out = C.c_void_p()
    with torch.cuda.device(ws.device):
        _check(_lib.tq_build_dictionary_device(ptrs, lens, n, top_k, ws.data_ptr(), ws.numel(), _stream_ptr(stream),
                                               C.byref(out)), "tq_build_dictionary_device")
    return Dict(out.value)


def tq_dict_from_entries(entries: np.ndarray) -> Dict:
    e = np.ascontiguousarray(entries, dtype=np.uint8).reshape(-1, 4)
    out = C.c_void_p()
    _check(_lib.tq_dict_from_entries(_np_ptr(e, C.c_uint8), e.shape[0], C.byref(out)), "tq_dict_from_entries")
    return Dict(out.value)


def tq_encode(d: Dict, codes: np.ndarray):
    """-> (stream uint16, n_hits, n_miss)"""
    w = np.ascontiguousarray(codes).view(np.uint8).reshape(-1)
    n, h, m = C.c_uint64(), C.c_uint64(), C.c_uint64()
    _check(_lib.tq_encode(d._h, _np_ptr(w, C.c_uint8), w.size, None, 0, C.byref(n), C.byref(h), C.byref(m)), "tq_encode")
    out = np.empty(n.value, dtype=np.uint16)
    _check(_lib.tq_encode(d._h, _np_ptr(w, C.c_uint8), w.size, _np_ptr(out, C.c_uint16), out.size,
                          C.byref(n), C.byref(h), C.byref(m)), "tq_encode")
    return out, h.value, m.value


# ------------------------------------------------------------------------------ device
class DeviceDict:
    """A table resident on the GPU: owns the torch buffer and the tq_ddict handle."""

    def __init__(self, handle: int, buf: torch.Tensor, K: int):
        self._h = C.c_void_p(handle)
        self.buf = buf
        self.K = K

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.tq_ddict_free(self._h)
            self._h = None


def tq_dict_upload(d: Dict, device="cuda", stream=None) -> DeviceDict:
    need = C.c_uint64()
    _check(_lib.tq_dict_upload_size(d._h, C.byref(need)), "tq_dict_upload_size")
    buf = torch.empty(need.value, dtype=torch.uint8, device=device)
    out = C.c_void_p()
    with torch.cuda.device(buf.device):
        _check(_lib.tq_dict_upload(d._h, buf.data_ptr(), buf.numel(), _stream_ptr(stream), C.byref(out)), "tq_dict_upload")
    return DeviceDict(out.value, buf, d.K)


@dataclass
class MatInfo:
    rows: int
    cols: int
    K: int
    layout: int
    levels_signed: int
    n_hits: int
    n_miss: int
    stream_bytes: int
    payload_bytes: int
    device_bytes: int
    n_raw_words: int


class DeviceMatrix:
    """One compressed matrix resident on the GPU: owns the torch buffer and the tq_dmat handle."""

    def __init__(self, handle: int, buf: torch.Tensor, ddict: DeviceDict):
        self._h = C.c_void_p(handle)
        self.buf = buf
        self.ddict = ddict  # keeps the table alive
        i = _Info()
        _check(_lib.tq_dmat_get_info(self._h, C.byref(i)), "tq_dmat_get_info")
        self.info = MatInfo(*(getattr(i, f[0]) for f in _Info._fields_))

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.tq_dmat_free(self._h)
            self._h = None


def tq_upload_size(stream: np.ndarray, rows: int, cols: int, layout: int = TQ_LAYOUT_STREAM) -> int:
    s = np.ascontiguousarray(stream, dtype=np.uint16)
    need = C.c_uint64()
    _check(_lib.tq_upload_size(_np_ptr(s, C.c_uint16), s.size, rows, cols, layout, C.byref(need)), "tq_upload_size")
    return need.value


def tq_upload(ddict: DeviceDict, stream: np.ndarray, rows: int, cols: int, row_scale: np.ndarray,
              row_zero=None, levels_signed: bool = True, layout: int = TQ_LAYOUT_STREAM,
              cuda_stream=None) -> DeviceMatrix:
    s = np.ascontiguousarray(stream, dtype=np.uint16)
    sc = np.ascontiguousarray(row_scale, dtype=np.float32)
    assert sc.size == rows
    zp = None
    if row_zero is not None:
        zr = np.ascontiguousarray(row_zero, dtype=np.float32)
        assert zr.size == rows
        zp = _np_ptr(zr, C.c_float)
    need = C.c_uint64()
    _check(_lib.tq_upload_size(_np_ptr(s, C.c_uint16), s.size, rows, cols, layout, C.byref(need)), "tq_upload_size")
    buf = torch.empty(need.value, dtype=torch.uint8, device=ddict.buf.device)
    out = C.c_void_p()
    with torch.cuda.device(buf.device):
        _check(_lib.tq_upload(ddict._h, _np_ptr(s, C.c_uint16), s.size, rows, cols, _np_ptr(sc, C.c_float), zp,
                              int(levels_signed), layout, buf.data_ptr(), buf.numel(), _stream_ptr(cuda_stream),
                              C.byref(out)), "tq_upload")
    return DeviceMatrix(out.value, buf, ddict)


def tq_upload_device(ddict: DeviceDict, levels: torch.Tensor, row_scale: torch.Tensor, row_zero: torch.Tensor | None = None,
                     levels_signed: bool = True, cuda_stream=None) -> DeviceMatrix:
    """levels: CUDA int8/uint8 [rows][cols]; row_scale / row_zero: CUDA fp32 [rows].  Builds the TILES
    image on the GPU, in a buffer sized for the worst case (info.device_bytes tells what is in use)."""
    assert levels.is_cuda and levels.is_contiguous() and levels.element_size() == 1 and levels.dim() == 2
    assert row_scale.is_cuda and row_scale.dtype == torch.float32 and row_scale.is_contiguous()
    rows, cols = levels.shape
    assert row_scale.numel() == rows
    if row_zero is not None:
        assert row_zero.is_cuda and row_zero.dtype == torch.float32 and row_zero.is_contiguous() and row_zero.numel() == rows
    need = C.c_uint64()
    _check(_lib.tq_upload_device_size(rows, cols, C.byref(need)), "tq_upload_device_size")
    buf = torch.empty(need.value, dtype=torch.uint8, device=levels.device)
    out = C.c_void_p()
    with torch.cuda.device(buf.device):
        _check(_lib.tq_upload_device(ddict._h, levels.data_ptr(), rows, cols, row_scale.data_ptr(),
                                     row_zero.data_ptr() if row_zero is not None else None, int(levels_signed),
                                     buf.data_ptr(), buf.numel(), _stream_ptr(cuda_stream), C.byref(out)), "tq_upload_device")
    return DeviceMatrix(out.value, buf, ddict)


def tq_upload_device_rows(ddict: DeviceDict, levels: torch.Tensor, row_begin: int, row_end: int, row_scale: torch.Tensor,
                          row_zero: torch.Tensor | None = None, levels_signed: bool = True, cuda_stream=None) -> DeviceMatrix:
    """Rows row_begin .. row_end-1 of `levels` (CUDA int8/uint8 [rows][cols]) as a compressed matrix of their
    own; row_scale / row_zero are the full [rows] arrays."""
    assert levels.is_cuda and levels.is_contiguous() and levels.element_size() == 1 and levels.dim() == 2
    rows, cols = levels.shape
    assert row_scale.is_cuda and row_scale.dtype == torch.float32 and row_scale.is_contiguous() and row_scale.numel() == rows
    if row_zero is not None:
        assert row_zero.is_cuda and row_zero.dtype == torch.float32 and row_zero.is_contiguous() and row_zero.numel() == rows
    need = C.c_uint64()
    _check(_lib.tq_upload_device_size(max(row_end - row_begin, 1), cols, C.byref(need)), "tq_upload_device_size")
    buf = torch.empty(need.value, dtype=torch.uint8, device=levels.device)
    out = C.c_void_p()
    with torch.cuda.device(buf.device):
        _check(_lib.tq_upload_device_rows(ddict._h, levels.data_ptr(), rows, cols, row_begin, row_end, row_scale.data_ptr(),
                                          row_zero.data_ptr() if row_zero is not None else None, int(levels_signed),
                                          buf.data_ptr(), buf.numel(), _stream_ptr(cuda_stream), C.byref(out)), "tq_upload_device_rows")
    return DeviceMatrix(out.value, buf, ddict)


def tq_tiles_image_host(d: Dict, stream: np.ndarray, rows: int, cols: int, row_scale: np.ndarray, row_zero=None):
    """-> (image uint8, dict of byte offsets, tiles per row block, row blocks)"""
    s = np.ascontiguousarray(stream, dtype=np.uint16)
    sc = np.ascontiguousarray(row_scale, dtype=np.float32)
    zp = None
    if row_zero is not None:
        zr = np.ascontiguousarray(row_zero, dtype=np.float32)
        zp = _np_ptr(zr, C.c_float)
    need = C.c_uint64()
    _check(_lib.tq_tiles_image_host(d._h, _np_ptr(s, C.c_uint16), s.size, rows, cols, None, None, None, 0,
                                    C.byref(need), None, None), "tq_tiles_image_host")
    out = np.zeros(need.value, dtype=np.uint8)
    offs = (C.c_uint64 * 5)()
    dims = (C.c_uint32 * 2)()
    _check(_lib.tq_tiles_image_host(d._h, _np_ptr(s, C.c_uint16), s.size, rows, cols, _np_ptr(sc, C.c_float), zp,
                                    _np_ptr(out, C.c_uint8), out.size, C.byref(need), offs, dims), "tq_tiles_image_host")
    names = ("scale", "zero", "tile_raw", "tokens", "raw")
    return out, dict(zip(names, (int(o) for o in offs))), int(dims[0]), int(dims[1])


def tq_decompress(m: DeviceMatrix, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    if out is None:
        out = torch.empty((m.info.rows, m.info.cols), dtype=torch.uint8, device=m.buf.device)
    assert out.is_cuda and out.is_contiguous() and out.numel() == m.info.rows * m.info.cols and out.element_size() == 1
    _check(_lib.tq_decompress(m._h, out.data_ptr(), _stream_ptr(stream)), "tq_decompress")
    return out


def tq_fused_gemv(m: DeviceMatrix, x: torch.Tensor, y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.is_contiguous()
    x2 = x.view(-1, m.info.cols)
    B = x2.shape[0]
    if y is None:
        y = torch.empty((B, m.info.rows), dtype=torch.float32, device=x.device)
    assert y.is_cuda and y.dtype == torch.float32 and y.is_contiguous() and y.numel() == B * m.info.rows
    _check(_lib.tq_fused_gemv(m._h, x2.data_ptr(), B, y.data_ptr(), _stream_ptr(stream)), "tq_fused_gemv")
    return y


def tq_fused_gemv_host(m: DeviceMatrix, h_x: torch.Tensor, h_y: torch.Tensor, d_x_stage: torch.Tensor,
                       d_y_stage: torch.Tensor, stream=None) -> None:
    """h_x: CPU (pinned) bf16 [B][cols]; h_y: CPU (pinned) fp32 [B][rows]; stages: CUDA tensors."""
    assert (not h_x.is_cuda) and h_x.dtype == torch.bfloat16 and h_x.is_contiguous()
    assert (not h_y.is_cuda) and h_y.dtype == torch.float32 and h_y.is_contiguous()
    B = h_x.numel() // m.info.cols
    assert d_x_stage.is_cuda and d_x_stage.numel() * d_x_stage.element_size() >= B * m.info.cols * 2
    assert d_y_stage.is_cuda and d_y_stage.numel() * d_y_stage.element_size() >= B * m.info.rows * 4
    _check(_lib.tq_fused_gemv_host(m._h, h_x.data_ptr(), B, h_y.data_ptr(), d_x_stage.data_ptr(),
                                   d_y_stage.data_ptr(), _stream_ptr(stream)), "tq_fused_gemv_host")


def tq_fused_gemv_host_static(m: DeviceMatrix, h_x: torch.Tensor, h_y: torch.Tensor, stream=None) -> None:
    """tq_fused_gemv_host without caller staging: the library's built-in 1.5 MiB staging array is
    used, nothing is allocated (B * cols and B * rows are limited to 262144 each)."""
    assert (not h_x.is_cuda) and h_x.dtype == torch.bfloat16 and h_x.is_contiguous()
    assert (not h_y.is_cuda) and h_y.dtype == torch.float32 and h_y.is_contiguous()
    B = h_x.numel() // m.info.cols
    assert h_y.numel() == B * m.info.rows
    with torch.cuda.device(m.buf.device):
        rc = _lib.tq_fused_gemv_host_static(m._h, h_x.data_ptr(), B, h_y.data_ptr(), _stream_ptr(stream))
    if rc == TQ_ERR_UNSUPPORTED_SHAPE:  # the library left the limits in its error text
        raise TqError(rc, "tq_fused_gemv_host_static", _lib.tq_last_cuda_error().decode())
    _check(rc, "tq_fused_gemv_host_static")


def tq_fused_gemm(m: DeviceMatrix, X: torch.Tensor, Y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.is_contiguous()
    X2 = X.view(-1, m.info.cols)
    M = X2.shape[0]
    if Y is None:
        Y = torch.empty((M, m.info.rows), dtype=torch.float32, device=X.device)
    assert Y.is_cuda and Y.dtype == torch.float32 and Y.is_contiguous() and Y.numel() == M * m.info.rows
    _check(_lib.tq_fused_gemm(m._h, X2.data_ptr(), M, Y.data_ptr(), _stream_ptr(stream)), "tq_fused_gemm")
    return Y


def tq_gemm_workspace_size(m: DeviceMatrix) -> int:
    need = C.c_uint64()
    _check(_lib.tq_gemm_workspace_size(m._h, C.byref(need)), "tq_gemm_workspace_size")
    return need.value


def tq_fused_gemm_ws(m: DeviceMatrix, X: torch.Tensor, workspace: torch.Tensor, Y: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    """Two-phase prefill product for the TILES layout; workspace: CUDA tensor of >= tq_gemm_workspace_size(m) bytes."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.is_contiguous() and workspace.is_cuda
    X2 = X.view(-1, m.info.cols)
    M = X2.shape[0]
    if Y is None:
        Y = torch.empty((M, m.info.rows), dtype=torch.float32, device=X.device)
    assert Y.is_cuda and Y.dtype == torch.float32 and Y.is_contiguous() and Y.numel() == M * m.info.rows
    _check(_lib.tq_fused_gemm_ws(m._h, X2.data_ptr(), M, Y.data_ptr(), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream_ptr(stream)), "tq_fused_gemm_ws")
    return Y


def tq_decode_bf16(m: DeviceMatrix, workspace: torch.Tensor, stream=None) -> None:
    assert workspace.is_cuda
    _check(_lib.tq_decode_bf16(m._h, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                               _stream_ptr(stream)), "tq_decode_bf16")


def tq_gemm_bf16_ws(m: DeviceMatrix, X: torch.Tensor, workspace: torch.Tensor, Y: torch.Tensor | None = None,
                    stream=None) -> torch.Tensor:
    """Phase 2 alone: workspace was filled for m by tq_decode_bf16 or tq_decode_bf16_stack."""
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.is_contiguous() and workspace.is_cuda
    assert workspace.numel() * workspace.element_size() >= tq_gemm_workspace_size(m)
    X2 = X.view(-1, m.info.cols)
    M = X2.shape[0]
    if Y is None:
        Y = torch.empty((M, m.info.rows), dtype=torch.float32, device=X.device)
    assert Y.is_cuda and Y.dtype == torch.float32 and Y.is_contiguous() and Y.numel() == M * m.info.rows
    _check(_lib.tq_gemm_bf16_ws(m._h, X2.data_ptr(), M, Y.data_ptr(), workspace.data_ptr(), _stream_ptr(stream)),
           "tq_gemm_bf16_ws")
    return Y


def tq_stack_plan_host(steps, row_blocks, rb_raw, n_ctas: int):
    """-> (segments [(matrix, first row block, end row block)], cta_seg): the work split of a stack, computed on the host."""
    n = len(steps)
    st = np.ascontiguousarray(steps, dtype=np.uint32)
    rbk = np.ascontiguousarray(row_blocks, dtype=np.uint32)
    raws = [np.ascontiguousarray(r, dtype=np.uint32) for r in rb_raw]
    ptrs = (C.POINTER(C.c_uint32) * n)(*[_np_ptr(r, C.c_uint32) for r in raws])
    cap = n + n_ctas
    segs = np.zeros(3 * cap, dtype=np.uint32)
    cta = np.zeros(n_ctas + 1, dtype=np.uint32)
    ns = C.c_uint32()
    _check(_lib.tq_stack_plan_host(n, _np_ptr(st, C.c_uint32), _np_ptr(rbk, C.c_uint32), ptrs, n_ctas,
                                   _np_ptr(segs, C.c_uint32), cap, C.byref(ns), _np_ptr(cta, C.c_uint32)), "tq_stack_plan_host")
    return [tuple(int(v) for v in segs[3 * i: 3 * i + 3]) for i in range(ns.value)], cta.tolist()


class Stack:
    """Several TILES matrices bound to their operands for one persistent launch.  Keeps the
    matrices, the operand tensors and its own device buffer alive."""

    def __init__(self, handle: int, buf: torch.Tensor, mats, xs, ys, B: int):
        self._h = C.c_void_p(handle)
        self.buf, self.mats, self.xs, self.ys, self.B = buf, list(mats), list(xs), list(ys), B

    @property
    def launches(self) -> int:
        return _lib.tq_stack_launches(self._h)

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.tq_stack_free(self._h)
            self._h = None


def tq_test_withhold_table_chunk(on: bool) -> None:
    """Test hook: see tq.h."""
    _lib.tq_test_withhold_table_chunk(int(bool(on)))


def tq_stack_create(mats, xs=None, ys=None, stream=None) -> Stack:
    """mats: DeviceMatrix list (TILES layout, one table); xs[i]: CUDA bf16 [B][cols_i]; ys[i]: CUDA fp32 [B][rows_i].
    Without xs / ys the stack serves tq_decompress_stack only."""
    n = len(mats)
    assert n >= 1 and (xs is None) == (ys is None)
    hm = (C.c_void_p * n)(*[m._h for m in mats])
    B, hx, hy = 0, None, None
    if xs is not None:
        assert len(xs) == n and len(ys) == n
        B = xs[0].numel() // mats[0].info.cols
    need = C.c_uint64()
    _check(_lib.tq_stack_size(hm, n, B, C.byref(need)), "tq_stack_size")
    buf = torch.empty(need.value, dtype=torch.uint8, device=mats[0].buf.device)
    if xs is not None:
        for m, x, y in zip(mats, xs, ys):
            assert x.is_cuda and x.dtype == torch.bfloat16 and x.is_contiguous() and x.numel() == B * m.info.cols
            assert y.is_cuda and y.dtype == torch.float32 and y.is_contiguous() and y.numel() == B * m.info.rows
        hx = (C.c_void_p * n)(*[x.data_ptr() for x in xs])
        hy = (C.c_void_p * n)(*[y.data_ptr() for y in ys])
    out = C.c_void_p()
    with torch.cuda.device(buf.device):
        _check(_lib.tq_stack_create(hm, hx, hy, n, B, buf.data_ptr(), buf.numel(), _stream_ptr(stream), C.byref(out)),
               "tq_stack_create")
    return Stack(out.value, buf, mats, xs or [], ys or [], B)


def tq_decompress_stack(s: Stack, outs, stream=None) -> None:
    """outs[i]: CUDA 1-byte tensor with rows_i * cols_i elements."""
    assert len(outs) == len(s.mats)
    for m, o in zip(s.mats, outs):
        assert o.is_cuda and o.is_contiguous() and o.element_size() == 1 and o.numel() == m.info.rows * m.info.cols
    ptrs = torch.tensor([o.data_ptr() for o in outs], dtype=torch.int64).to(s.buf.device)
    _check(_lib.tq_decompress_stack(s._h, ptrs.data_ptr(), _stream_ptr(stream)), "tq_decompress_stack")
    s._out_ptrs = ptrs  # keep the pointer array alive until the stream has used it


def tq_decode_bf16_stack(s: Stack, workspaces, stream=None) -> None:
    """workspaces[i]: CUDA tensor of >= tq_gemm_workspace_size(mats[i]) bytes, 256-byte aligned."""
    assert len(workspaces) == len(s.mats)
    for m, w in zip(s.mats, workspaces):
        assert w.is_cuda and w.numel() * w.element_size() >= tq_gemm_workspace_size(m) and w.data_ptr() % 256 == 0
    ptrs = torch.tensor([w.data_ptr() for w in workspaces], dtype=torch.int64).to(s.buf.device)
    _check(_lib.tq_decode_bf16_stack(s._h, ptrs.data_ptr(), _stream_ptr(stream)), "tq_decode_bf16_stack")
    s._ws_ptrs = ptrs  # keep the pointer array alive until the stream has used it


class GemmPlan:
    """Several workspace GEMMs of one token count bound for one persistent launch.  Keeps the
    matrices, operands, workspaces and its own device buffer alive."""

    def __init__(self, handle: int, buf: torch.Tensor, mats, Xs, Ys, workspaces, M: int):
        self._h = C.c_void_p(handle)
        self.buf, self.mats, self.Xs, self.Ys, self.workspaces, self.M = buf, list(mats), list(Xs), list(Ys), list(workspaces), M

    def __del__(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.tq_gemm_plan_free(self._h)
            self._h = None


def tq_gemm_plan_create(mats, Xs, workspaces, Ys=None, stream=None) -> GemmPlan:
    """Xs[i]: CUDA bf16 [M][cols_i]; workspaces[i]: filled (now or later, before the run) by tq_decode_bf16(_stack);
    Ys[i]: CUDA fp32 [M][rows_i] (made here when None)."""
    n = len(mats)
    assert n >= 1 and len(Xs) == n and len(workspaces) == n
    M = Xs[0].view(-1, mats[0].info.cols).shape[0]
    dev = Xs[0].device
    if Ys is None:
        Ys = [torch.empty((M, m.info.rows), dtype=torch.float32, device=dev) for m in mats]
    for m, X, Y, w in zip(mats, Xs, Ys, workspaces):
        assert X.is_cuda and X.dtype == torch.bfloat16 and X.is_contiguous() and X.numel() == M * m.info.cols
        assert Y.is_cuda and Y.dtype == torch.float32 and Y.is_contiguous() and Y.numel() == M * m.info.rows
        assert w.is_cuda and w.numel() * w.element_size() >= tq_gemm_workspace_size(m)
    need = C.c_uint64()
    _check(_lib.tq_gemm_plan_size(n, C.byref(need)), "tq_gemm_plan_size")
    buf = torch.empty(need.value + 256, dtype=torch.uint8, device=dev)
    off = (-buf.data_ptr()) % 256
    arr = lambda ts: (C.c_void_p * n)(*[t.data_ptr() for t in ts])  # noqa: E731
    out = C.c_void_p()
    with torch.cuda.device(dev):
        _check(_lib.tq_gemm_plan_create((C.c_void_p * n)(*[m._h for m in mats]), arr(Xs), arr(Ys), arr(workspaces), n, M,
                                        buf.data_ptr() + off, need.value, _stream_ptr(stream), C.byref(out)),
               "tq_gemm_plan_create")
    return GemmPlan(out.value, buf, mats, Xs, Ys, workspaces, M)


def tq_gemm_plan_run(p: GemmPlan, stream=None) -> None:
    _check(_lib.tq_gemm_plan_run(p._h, _stream_ptr(stream)), "tq_gemm_plan_run")


def tq_gemm_plan_status(p: GemmPlan, stream=None) -> int:
    st = C.c_uint32()
    _check(_lib.tq_gemm_plan_status(p._h, _stream_ptr(stream), C.byref(st)), "tq_gemm_plan_status")
    return st.value


def tq_fused_gemv_stack(s: Stack, stream=None) -> None:
    _check(_lib.tq_fused_gemv_stack(s._h, _stream_ptr(stream)), "tq_fused_gemv_stack")


def tq_fused_gemv_stack_host(s: Stack, h_x: torch.Tensor, d_x_arena: torch.Tensor, h_y: torch.Tensor,
                             d_y_arena: torch.Tensor, stream=None) -> None:
    """h_x / h_y: CPU (pinned) images of the x / y arenas the stack's operands live in."""
    assert (not h_x.is_cuda) and (not h_y.is_cuda) and d_x_arena.is_cuda and d_y_arena.is_cuda
    xb = d_x_arena.numel() * d_x_arena.element_size()
    yb = d_y_arena.numel() * d_y_arena.element_size()
    assert h_x.numel() * h_x.element_size() == xb and h_y.numel() * h_y.element_size() == yb
    _check(_lib.tq_fused_gemv_stack_host(s._h, h_x.data_ptr(), d_x_arena.data_ptr(), xb, h_y.data_ptr(),
                                         d_y_arena.data_ptr(), yb, _stream_ptr(stream)), "tq_fused_gemv_stack_host")


def tq_device_status(m: DeviceMatrix, stream=None) -> int:
    st = C.c_uint32()
    _check(_lib.tq_device_status(m._h, _stream_ptr(stream), C.byref(st)), "tq_device_status")
    return st.value


# ------------------------------------------------------------------------------ between the linear layers
_TYPES = {torch.bfloat16: TQ_TYPE_BF16, torch.float32: TQ_TYPE_F32}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # a torch without CUDA still has the host's half of this module
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _load_fast():
    """The native form of the calls below for their usual case (csrc/tq_fast.cpp), or None (it cannot be built or loaded here, or
    torch is without the DLPack exchange interface).  It answers None for whatever it does not take, and the checks here speak."""
    import importlib.util
    import warnings

    path = _build.build_fast()
    if path is None:
        return None
    spec = importlib.util.spec_from_file_location("_tqfast", str(path))
    try:
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError as e:
        warnings.warn(f"the native form of the small calls was not loaded, they go through Python: {e}", RuntimeWarning)
        return None
    names = ("tq_rmsnorm", "tq_rmsnorm_q8", "tq_rope_append", "tq_paged_attention", "tq_cross_attention", "tq_qk_norm_rope_append",
             "tq_tree_attention", "tq_sample", "tq_tree_accept")
    return module if module.setup(torch, *(C.cast(getattr(_lib, n), C.c_void_p).value for n in names)) else None


_fast = _load_fast()


# A decode step makes dozens of these calls of a few microseconds each: the usual case goes through _fast, and the checks
# here use the cheap tensor attributes (get_device() is -1 for a CPU tensor) and build no objects.
def _elsewhere(device: int, stream):
    """None if the call is for the current device and its current stream; else a context in which it is, so that the call's results
    come from that stream's memory."""
    assert device >= 0, "a CUDA tensor is wanted"
    if stream is None:
        return None if _current_device() == device else torch.cuda.device(device)
    assert stream.device.index == device
    return torch.cuda.stream(stream)


def _strides(x: torch.Tensor):
    """Strides, with 0 for dimensions of size 1, whose stride means nothing."""
    return tuple(st if n > 1 else 0 for n, st in zip(x.shape, x.stride()))


def _norm_args(h, weight, delta, h_out, device):
    rows, cols = shape = h.shape
    stride = h.stride()
    assert device >= 0 and h.dtype in _TYPES and (stride[1] == 1 or cols == 1)
    assert weight.get_device() == device and weight.dtype == torch.float32 and weight.is_contiguous() and weight.numel() == cols
    dp, dt, ds = None, 0, 0
    if delta is not None:
        dst = delta.stride()
        assert delta.get_device() == device and delta.shape == shape and (dst[1] == 1 or cols == 1)
        dp, dt, ds = delta.data_ptr(), _TYPES[delta.dtype], dst[0]
        if h_out is None:
            h_out = h
    if h_out is not None and h_out is not h:
        assert h_out.get_device() == device and h_out.dtype == h.dtype and h_out.shape == shape
        assert h_out.stride() == stride or _strides(h_out) == _strides(h)
    return rows, cols, (h.data_ptr(), _TYPES[h.dtype], stride[0], dp, dt, ds, weight.data_ptr()), None if h_out is None else h_out.data_ptr()


def tq_rmsnorm(h: torch.Tensor, weight: torch.Tensor, delta: torch.Tensor | None = None, eps: float = 1e-5,
               out: torch.Tensor | None = None, h_out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """h: CUDA bf16 / fp32 [rows][cols] (rows may be strided); delta: bf16 / fp32 of the same shape; weight: fp32 [cols].
    With a delta the sum h + delta goes to h_out (a tensor like h), or to h itself when h_out is None.  -> bf16 [rows][cols]."""
    if stream is None and _fast is not None:
        r = _fast.rmsnorm(h, weight, delta, eps, out, h_out)
        if r is not None:
            return r
    device = h.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_rmsnorm(h, weight, delta, eps, out, h_out)
    rows, cols, args, ho = _norm_args(h, weight, delta, h_out, device)
    if out is None:
        out = torch.empty((rows, cols), dtype=torch.bfloat16, device=h.device)
    else:
        assert out.get_device() == device and out.dtype == torch.bfloat16 and out.is_contiguous() and out.numel() == rows * cols
    _check(_lib.tq_rmsnorm(*args, eps, rows, cols, ho, out.data_ptr(), _raw_stream(device)), "tq_rmsnorm")
    return out


def tq_rmsnorm_q8(h: torch.Tensor, weight: torch.Tensor, delta: torch.Tensor | None = None, eps: float = 1e-5,
                  q: torch.Tensor | None = None, scale: torch.Tensor | None = None, h_out: torch.Tensor | None = None, stream=None):
    """tq_rmsnorm with the result in 8 bits: -> (int8 [rows][cols], fp32 [rows] scales)."""
    if stream is None and q is None and scale is None and _fast is not None:
        r = _fast.rmsnorm_q8(h, weight, delta, eps, h_out)
        if r is not None:
            return r
    device = h.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_rmsnorm_q8(h, weight, delta, eps, q, scale, h_out)
    rows, cols, args, ho = _norm_args(h, weight, delta, h_out, device)
    if q is None:
        q = torch.empty((rows, cols), dtype=torch.int8, device=h.device)
    if scale is None:
        scale = torch.empty(rows, dtype=torch.float32, device=h.device)
    assert q.get_device() == device and q.dtype == torch.int8 and q.is_contiguous() and q.numel() == rows * cols
    assert scale.get_device() == device and scale.dtype == torch.float32 and scale.is_contiguous() and scale.numel() == rows
    _check(_lib.tq_rmsnorm_q8(*args, eps, rows, cols, ho, q.data_ptr(), scale.data_ptr(), _raw_stream(device)), "tq_rmsnorm_q8")
    return q, scale


class KvCache:
    """A pool of pages of keys and values: keeps the tensors and a status word alive."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        assert k.is_cuda and k.dtype == torch.bfloat16 and k.dim() == 4 and k.stride(3) == 1
        assert v.device == k.device and v.dtype == k.dtype and v.shape == k.shape and _strides(v) == _strides(k)
        self.k, self.v = k, v
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        self.device = k.get_device()
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._c = _KvCache(k.data_ptr(), v.data_ptr(), self.n_pages, self.page_size, self.n_kv_heads, self.head_dim,
                           *_strides(k)[:3], self.status.data_ptr())
        self._ref = C.byref(self._c)
        self._addr = C.addressof(self._c)
        self.scale = self.head_dim ** -0.5  # of the scores, unless a call says otherwise


def tq_kv_cache(k: torch.Tensor, v: torch.Tensor) -> KvCache:
    """k, v: CUDA bf16 [pages][kv heads][page size][head dim] with any strides (a pool laid out as [pages][page size][kv heads][head
    dim] is passed as pool.transpose(1, 2))."""
    return KvCache(k, v)


def tq_kv_cache_status(cache: KvCache) -> int:
    """Reads and clears the cache's status word (TQ_STATUS_BAD_PAGE, TQ_STATUS_BAD_POSITION); synchronises the current stream."""
    st = int(cache.status.item())
    cache.status.zero_()
    return st


def _heads(x: torch.Tensor, tokens: int, n: int, dim: int, device: int, dtype) -> int:
    """Token stride of x, [tokens][n * dim] or [tokens][n][dim]."""
    shape, stride = x.shape, x.stride()
    assert x.get_device() == device and x.dtype == dtype and shape[0] == tokens and stride[-1] == 1
    if len(shape) == 2:
        assert shape[1] == n * dim
    else:
        assert shape[1:] == (n, dim) and (n == 1 or stride[1] == dim)
    return stride[0] if tokens > 1 else 0  # of one token it means nothing


@functools.lru_cache(maxsize=64)
def _sections(sections):
    return (C.c_uint32 * len(sections))(*sections)


def _rope_args(q, k, v, table, positions, slots, cache, sections, out, device):
    """Checks what the calls with rotary positions share; -> tokens, heads, the arguments of q, k, v, those of table and positions, slots,
    the result and its address."""
    D, K, shape, dtype = cache.head_dim, cache.n_kv_heads, q.shape, q.dtype
    T, H = shape[0], (shape[1] if len(shape) == 3 else shape[1] // D)
    assert cache.device == device and dtype in _TYPES
    qs, ks, vs = _heads(q, T, H, D, device, dtype), _heads(k, T, K, D, device, dtype), _heads(v, T, K, D, device, dtype)
    n_positions, rot = table.shape
    assert table.get_device() == device and table.dtype == torch.float32 and table.is_contiguous()
    axes = 1 if positions.dim() == 1 else positions.shape[0]
    assert positions.get_device() == device and positions.dtype == torch.int32 and positions.is_contiguous() and positions.numel() == axes * T
    assert slots.get_device() == device and slots.dtype == torch.int32 and slots.is_contiguous() and slots.numel() == T
    sec = (rot // 2,) if sections is None else tuple(sections)
    assert len(sec) == axes
    if out is None:
        out = torch.empty((T, H, D), dtype=torch.bfloat16, device=q.device)
    else:
        assert out.get_device() == device and out.dtype == torch.bfloat16 and out.is_contiguous() and out.numel() == T * H * D
    return (T, H, (q.data_ptr(), k.data_ptr(), v.data_ptr(), _TYPES[dtype], qs, ks, vs),
            (table.data_ptr(), n_positions, rot, positions.data_ptr(), _sections(sec), axes), slots.data_ptr(), out, out.data_ptr())


def tq_rope_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, positions: torch.Tensor,
                   slots: torch.Tensor, cache: KvCache, sections=None, interleaved: bool = False, out: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
    """q, k, v: CUDA bf16 or fp32 [tokens][heads * head dim] or [tokens][heads][head dim] (tokens may be strided); table: fp32
    [positions][rot dim], cosines then sines; positions: int32 [axes][tokens] or [tokens]; slots: int32 [tokens], -1 for none;
    sections: pairs of each axis (one axis: all).  -> rotated q, bf16 [tokens][q heads][head dim]; k and v are in the cache."""
    if stream is None and _fast is not None:
        r = _fast.rope_append(q, k, v, table, positions, slots, cache._addr, cache.device, sections, interleaved, out)
        if r is not None:
            return r
    device = q.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_rope_append(q, k, v, table, positions, slots, cache, sections, interleaved, out)
    T, H, x, where, at, out, o = _rope_args(q, k, v, table, positions, slots, cache, sections, out, device)
    _check(_lib.tq_rope_append(*x, T, H, *where, interleaved, at, cache._ref, o, _raw_stream(device)), "tq_rope_append")
    return out


class AttnWorkspace:
    """Workspace of tq_paged_attention, tq_cross_attention and tq_tree_attention: one for each stream that makes such calls."""

    def __init__(self, buf: torch.Tensor):
        self.buf = buf
        self.device, self.ptr, self.bytes = buf.get_device(), buf.data_ptr(), buf.numel()


def tq_attn_workspace(device="cuda", stream=None) -> AttnWorkspace:
    with torch.cuda.device(device) if stream is None else torch.cuda.stream(stream):
        need = C.c_uint64()
        _check(_lib.tq_attn_workspace_size(C.byref(need)), "tq_attn_workspace_size")
        buf = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        _check(_lib.tq_attn_workspace_init(buf.data_ptr(), buf.numel(), _stream_ptr()), "tq_attn_workspace_init")
    return AttnWorkspace(buf)


def tq_test_withhold_cross_entry(on: bool) -> None:
    """Test hook: see tq.h."""
    _lib.tq_test_withhold_cross_entry(int(bool(on)))


def tq_attn_status(workspace: AttnWorkspace, stream=None) -> int:
    st = C.c_uint32()
    with torch.cuda.device(workspace.device) if stream is None else torch.cuda.stream(stream):
        _check(_lib.tq_attn_status(workspace.ptr, _stream_ptr(), C.byref(st)), "tq_attn_status")
    return st.value


def _attn_out(q, out, lse, device):
    shape = q.shape
    if out is None:
        out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
    else:
        assert out.get_device() == device and out.dtype == torch.bfloat16 and out.is_contiguous() and out.shape == shape
    if lse is None:
        return out, None
    assert lse.get_device() == device and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == shape[:-1]
    return out, lse.data_ptr()


def tq_paged_attention(q: torch.Tensor, cache: KvCache, page_table: torch.Tensor, lens: torch.Tensor, workspace: AttnWorkspace,
                       scale: float | None = None, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                       stream=None) -> torch.Tensor:
    """q: CUDA bf16 [sequences][q heads][head dim] (sequences may be strided); page_table: int32 [sequences][max pages]; lens: int32
    [sequences]; scale: 1 / sqrt(head dim) when None; lse: fp32 [sequences][q heads], filled when given.  -> bf16 like q."""
    if stream is None and _fast is not None:
        r = _fast.paged_attention(q, cache._addr, cache.device, page_table, lens, workspace.ptr, workspace.bytes, workspace.device,
                                  cache.scale if scale is None else scale, out, lse)
        if r is not None:
            return r
    device = q.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_paged_attention(q, cache, page_table, lens, workspace, scale, out, lse)
    (B, H, D), stride = q.shape, q.stride()
    assert cache.device == device and workspace.device == device and q.dtype == torch.bfloat16
    assert D == cache.head_dim and stride[2] == 1 and (H == 1 or stride[1] == D)
    rows, max_pages = page_table.shape
    assert page_table.get_device() == device and page_table.dtype == torch.int32 and page_table.is_contiguous() and rows == B
    assert lens.get_device() == device and lens.dtype == torch.int32 and lens.is_contiguous() and lens.numel() == B
    out, lse = _attn_out(q, out, lse, device)
    _check(_lib.tq_paged_attention(cache._ref, q.data_ptr(), stride[0] if B > 1 else 0, B, H, page_table.data_ptr(), max_pages, lens.data_ptr(),
                                   cache.scale if scale is None else scale, out.data_ptr(), lse, workspace.ptr, workspace.bytes,
                                   _raw_stream(device)), "tq_paged_attention")
    return out


def tq_cross_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, workspace: AttnWorkspace, kv_len: torch.Tensor | None = None,
                       mask: torch.Tensor | None = None, block_len: int = 1, scale: float | None = None,
                       out: torch.Tensor | None = None, lse: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """q: CUDA bf16 [sequences][tokens][q heads][head dim]; k, v: bf16 [sequences][states][kv heads][head dim], any strides (an
    expanded batch has the same states for every sequence); kv_len: int32 [sequences]; mask: uint8 / bool
    [sequences][tokens][ceil(states / block_len)], nonzero where a token sees the block; lse: fp32 [sequences][tokens][q heads],
    filled when given.  -> bf16 [sequences][tokens][q heads][head dim]."""
    if stream is None and _fast is not None:
        r = _fast.cross_attention(q, k, v, workspace.ptr, workspace.bytes, workspace.device, kv_len, mask, block_len,
                                  q.shape[-1] ** -0.5 if scale is None else scale, out, lse)
        if r is not None:
            return r
    device = q.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_cross_attention(q, k, v, workspace, kv_len, mask, block_len, scale, out, lse)
    (B, T, H, D), stride = q.shape, q.stride()
    assert workspace.device == device and q.dtype == torch.bfloat16 and stride[3] == 1 and (H == 1 or stride[2] == D)
    n, S, K, dim = k.shape
    ks = _strides(k)
    assert k.get_device() == device and k.dtype == torch.bfloat16 and n == B and dim == D and ks[3] == 1
    assert v.get_device() == device and v.dtype == torch.bfloat16 and v.shape == k.shape and _strides(v) == ks
    n_valid = seen = None  # names of their own: an argument that nobody else holds would be freed, and its memory be the result's
    if kv_len is not None:
        assert kv_len.get_device() == device and kv_len.dtype == torch.int32 and kv_len.is_contiguous() and kv_len.numel() == B
        n_valid = kv_len.data_ptr()
    if mask is not None:
        assert mask.get_device() == device and mask.dtype in (torch.uint8, torch.bool) and mask.is_contiguous()
        assert block_len >= 1 and mask.shape == (B, T, -(-S // block_len))
        seen = mask.data_ptr()
    out, lse = _attn_out(q, out, lse, device)
    _check(_lib.tq_cross_attention(_EncoderKv(k.data_ptr(), v.data_ptr(), B, S, K, D, ks[0], ks[1], ks[2]), q.data_ptr(),
                                   stride[0] if B > 1 else 0, stride[1] if T > 1 else 0, T, H, n_valid, seen, block_len,
                                   D ** -0.5 if scale is None else scale, out.data_ptr(), lse, workspace.ptr, workspace.bytes,
                                   _raw_stream(device)), "tq_cross_attention")
    return out


# ------------------------------------------------------------------------------ a decode step with drafted tokens
def _like(x: torch.Tensor, device: int, dtype, *shape) -> int:
    """Address of a contiguous tensor of this type and shape on the call's device.  (The caller keeps the tensor in a name of its own: an
    argument that nobody else holds would be freed, and its memory be the next result's.)"""
    assert x.get_device() == device and x.dtype == dtype and x.is_contiguous() and x.shape == shape, f"{dtype} {shape} on device {device} is wanted"
    return x.data_ptr()


def _count(x: torch.Tensor, device: int, dtype, n: int) -> int:
    """Likewise, of a contiguous tensor of n elements, whatever its shape."""
    assert x.get_device() == device and x.dtype == dtype and x.is_contiguous() and x.numel() == n, f"{n} elements of {dtype} on device {device} are wanted"
    return x.data_ptr()


def tq_qk_norm_rope_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_weight: torch.Tensor, k_weight: torch.Tensor,
                           table: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor, cache: KvCache, eps: float = 1e-5,
                           sections=None, interleaved: bool = False, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """tq_rope_append with every head of q and k normalised first; q_weight, k_weight: fp32 [head dim]."""
    if stream is None and _fast is not None:
        r = _fast.qk_norm_rope_append(q, k, v, table, positions, slots, cache._addr, cache.device, sections, interleaved, out, q_weight, k_weight, eps)
        if r is not None:
            return r
    device = q.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_qk_norm_rope_append(q, k, v, q_weight, k_weight, table, positions, slots, cache, eps, sections, interleaved, out)
    D = cache.head_dim
    weights = _like(q_weight, device, torch.float32, D), _like(k_weight, device, torch.float32, D)
    T, H, x, where, at, out, o = _rope_args(q, k, v, table, positions, slots, cache, sections, out, device)
    _check(_lib.tq_qk_norm_rope_append(*x, T, H, *weights, eps, *where, interleaved, at, cache._ref, o, _raw_stream(device)),
           "tq_qk_norm_rope_append")
    return out


def tq_tree_attention(q: torch.Tensor, cache: KvCache, page_table: torch.Tensor, first: torch.Tensor, lens: torch.Tensor,
                      workspace: AttnWorkspace, mask: torch.Tensor | None = None, scale: float | None = None,
                      out: torch.Tensor | None = None, lse: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """q: CUDA bf16 [tokens][q heads][head dim] (tokens may be strided); first: int32 [sequences + 1], rows of each sequence; page_table:
    int32 [sequences][max pages]; lens: int32 [sequences], new tokens included; mask: int32 [tokens][words], bit j of a row's words set
    where it sees the sequence's new token j (None: a chain); lse: fp32 [tokens][q heads], filled when given.  -> bf16 like q; rows of no
    sequence are not written."""
    if stream is None and _fast is not None:
        r = _fast.tree_attention(q, cache._addr, cache.device, page_table, first, lens, workspace.ptr, workspace.bytes, workspace.device, mask,
                                 cache.scale if scale is None else scale, out, lse)
        if r is not None:
            return r
    device = q.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_tree_attention(q, cache, page_table, first, lens, workspace, mask, scale, out, lse)
    (T, H, D), stride = q.shape, q.stride()
    assert cache.device == device and workspace.device == device and q.dtype == torch.bfloat16
    assert D == cache.head_dim and stride[2] == 1 and (H == 1 or stride[1] == D)
    B, max_pages = page_table.shape
    table, f, n = _like(page_table, device, torch.int32, B, max_pages), _like(first, device, torch.int32, B + 1), _like(lens, device, torch.int32, B)
    words = 0 if mask is None else mask.shape[1]
    m = None if mask is None else _like(mask, device, torch.int32, T, words)
    out, e = _attn_out(q, out, lse, device)
    _check(_lib.tq_tree_attention(cache._ref, q.data_ptr(), stride[0] if T > 1 else 0, T, B, H, f, table, max_pages, n, m, words,
                                  cache.scale if scale is None else scale, out.data_ptr(), e, workspace.ptr, workspace.bytes,
                                  _raw_stream(device)), "tq_tree_attention")
    return out


def tq_sample(logits: torch.Tensor, uniform: torch.Tensor, temperature: torch.Tensor | None = None, top_k: torch.Tensor | None = None,
              top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None, out: torch.Tensor | None = None,
              logprob: torch.Tensor | bool | None = None, stream=None):
    """logits: CUDA bf16 or fp32 [rows][vocab] (rows may be strided); uniform: fp32 [rows] in [0, 1); temperature, top_p, min_p: fp32
    [rows] or of another shape with as many elements; top_k: int32, likewise.  -> int32 [rows] tokens; with logprob (True, or the fp32 [rows] tensor to fill) also their logarithms."""
    if stream is None and out is None and (logprob is None or isinstance(logprob, bool)) and _fast is not None:
        r = _fast.sample(logits, uniform, temperature, top_k, top_p, min_p, logprob is True)
        if r is not None:
            return r
    device = logits.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_sample(logits, uniform, temperature, top_k, top_p, min_p, out, logprob)
    (R, V), stride = logits.shape, logits.stride()
    assert logits.dtype in _TYPES and (stride[1] == 1 or V == 1)
    u = _like(uniform, device, torch.float32, R)
    t, k, p, m = (None if x is None else _count(x, device, dt, R) for x, dt in
                  ((temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32)))
    if out is None:
        out = torch.empty(R, dtype=torch.int32, device=logits.device)
    if logprob is True:
        logprob = torch.empty(R, dtype=torch.float32, device=logits.device)
    lp = None if logprob is None or logprob is False else _like(logprob, device, torch.float32, R)
    _check(_lib.tq_sample(logits.data_ptr(), _TYPES[logits.dtype], stride[0] if R > 1 else 0, R, V, u, t, k, p, m, _like(out, device, torch.int32, R),
                          lp, _raw_stream(device)), "tq_sample")
    return out if lp is None else (out, logprob)


class KvCaches:
    """The caches of a model's layers, alike in shape and strides, that share a page table; keeps them alive."""

    def __init__(self, caches):
        self.caches = list(caches)
        assert len(self.caches) <= TQ_MAX_CACHES and len({c.device for c in self.caches}) <= 1
        self._c = (_KvCache * max(1, len(self.caches)))(*[c._c for c in self.caches])
        self._addr = C.addressof(self._c)
        self.device = self.caches[0].device if self.caches else None

    def __len__(self):
        return len(self.caches)


def tq_kv_caches(caches) -> KvCaches:
    """caches: KvCache objects, one for each layer."""
    return KvCaches(caches)


def tq_tree_accept(caches: KvCaches | None, page_table: torch.Tensor | None, first: torch.Tensor, lens: torch.Tensor, tokens: torch.Tensor,
                   parents: torch.Tensor, sampled: torch.Tensor, max_path: int, stream=None):
    """first: CUDA int32 [sequences + 1]; lens: int32 [sequences], new tokens included; tokens (drafted), parents (counted from the
    sequence's first row), sampled: int32 [rows]; page_table: int32 [sequences][max pages].  -> (samples along the path, int32
    [sequences][max_path]; the path's rows, likewise, both -1 past its end; its length, int32 [sequences]; new lens): the path's keys
    and values lie behind the certain ones in every cache."""
    if stream is None and _fast is not None:
        n = 0 if caches is None else len(caches)
        r = _fast.tree_accept(caches._addr if n else 0, n, caches.device if n else 0, page_table, first, lens, tokens, parents, sampled, max_path)
        if r is not None:
            return r
    device = first.get_device()
    ctx = _elsewhere(device, stream)
    if ctx is not None:
        with ctx:
            return tq_tree_accept(caches, page_table, first, lens, tokens, parents, sampled, max_path)
    n = 0 if caches is None else len(caches)
    assert not n or caches.device == device
    B, T = first.numel() - 1, tokens.numel()
    assert max_path >= 1
    f, length = _like(first, device, torch.int32, B + 1), _like(lens, device, torch.int32, B)
    rows = [_like(tokens, device, torch.int32, T), *(_count(x, device, torch.int32, T) for x in (parents, sampled))]
    max_pages = page_table.shape[1] if n else 0
    table = _like(page_table, device, torch.int32, B, max_pages) if n else None
    both = torch.empty((2, B, max_path), dtype=torch.int32, device=first.device)
    ends = torch.empty((2, B), dtype=torch.int32, device=first.device)
    (out_tokens, path), (count, lens_out) = both.unbind(), ends.unbind()
    _check(_lib.tq_tree_accept(caches._c if n else None, n, table, max_pages, B, T, f, length, *rows, max_path, out_tokens.data_ptr(),
                               path.data_ptr(), count.data_ptr(), lens_out.data_ptr(), _raw_stream(device)), "tq_tree_accept")
    return out_tokens, path, count, lens_out
