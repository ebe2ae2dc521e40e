"""EntQuant inference-time decoding on MI355X: thin ctypes binding of libeq.

Every function here has the name of the C entry point it wraps (include/eq.h,
include/eq_encode.h) and only marshals arguments: torch supplies device memory
and streams, all decoding runs in libeq's gfx950 kernels.  There is no CPU
fallback: if libeq.so is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

from ._build import LIB as _LIB_PATH
from ._build import build as _build_lib

EQ_OK, EQ_EINVAL, EQ_EFORMAT, EQ_EHIP, EQ_ECORRUPT, EQ_ESCRATCH = 0, -1, -2, -3, -4, -5
NOALLOC_SCRATCH_BYTES = 32 << 20
FMT_E4M3, FMT_INT8 = 1, 2  # base formats of the codes (container field base_format)

_lib = None
_vp = ctypes.c_void_p


class EqError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn}: {eq_strerror(code)} ({code})")
        self.code = code


class eq_layer(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint32), ("cols", ctypes.c_uint32),
                ("chunk_syms", ctypes.c_uint32), ("n_chunks", ctypes.c_uint32),
                ("lanes", ctypes.c_uint32), ("prob_bits", ctypes.c_uint32),
                ("n_syms", ctypes.c_uint32), ("base_format", ctypes.c_uint32),
                ("total_words", ctypes.c_uint64), ("padded_words", ctypes.c_uint64),
                ("scale", _vp), ("sym", _vp), ("freq", _vp), ("chunk_off", _vp),
                ("chunk_state", _vp), ("words", _vp), ("lut", _vp), ("status", _vp),
                ("version", ctypes.c_uint32), ("tile_cols", ctypes.c_uint32),
                ("n_quads", ctypes.c_uint32), ("n_pairs", ctypes.c_uint32),
                ("n_singles", ctypes.c_uint32), ("row_order", _vp)]


class eq_kv_cache(ctypes.Structure):
    _fields_ = [("pages", _vp), ("n_pages", ctypes.c_uint32), ("page_tokens", ctypes.c_uint32),
                ("kv_heads", ctypes.c_uint32), ("head_dim", ctypes.c_uint32)]


class eq_kv_batch(ctypes.Structure):
    _fields_ = [("seq_start", _vp), ("kv_len", _vp), ("page_table", _vp),
                ("n_seqs", ctypes.c_uint32), ("max_pages", ctypes.c_uint32),
                ("n_tokens", ctypes.c_uint32), ("max_new", ctypes.c_uint32),
                ("max_len", ctypes.c_uint32)]


class eq_rope(ctypes.Structure):
    _fields_ = [("cos", _vp), ("sin", _vp), ("rows", ctypes.c_uint32), ("dims", ctypes.c_uint32),
                ("pairs", ctypes.c_uint32)]


class eqe_params(ctypes.Structure):
    _fields_ = [("prob_bits", ctypes.c_uint32), ("chunk_syms", ctypes.c_uint32),
                ("lanes", ctypes.c_uint32), ("threads", ctypes.c_uint32),
                ("seed", ctypes.c_uint64), ("target_bits", ctypes.c_float),
                ("base_format", ctypes.c_uint32)]


class eqe_params2(ctypes.Structure):
    _fields_ = [("res_bits", ctypes.c_uint32), ("tile_rows", ctypes.c_uint32),
                ("tile_cols", ctypes.c_uint32), ("threads", ctypes.c_uint32),
                ("seed", ctypes.c_uint64), ("target_bits", ctypes.c_float),
                ("base_format", ctypes.c_uint32), ("row_order", ctypes.c_uint32)]


class eqe_rd_params(ctypes.Structure):
    _fields_ = [("lambda_", ctypes.c_double), ("lr", ctypes.c_double),
                ("iters", ctypes.c_uint32), ("history", ctypes.c_uint32),
                ("threads", ctypes.c_uint32), ("base_format", ctypes.c_uint32)]


# name -> (restype, argtypes): every symbol the public headers declare
SIGNATURES = {
    "eq_lut_bytes": (ctypes.c_size_t, []),
    "eq_layer_init": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp, ctypes.c_uint64, _vp, _vp,
                                     _vp]),
    "eq_layer_prepare": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp]),
    "eq_decode_codes": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp, _vp]),
    "eq_decode_bf16": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp, _vp]),
    "eq_gemv_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(eq_layer), ctypes.c_uint32]),
    "eq_decode_gemv": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp, ctypes.c_uint32, _vp, _vp,
                                      _vp, ctypes.c_size_t, _vp]),
    "eq_decode_gemv_noalloc": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp, ctypes.c_uint32, _vp,
                                              _vp, _vp]),
    "eq_decode_bf16_multi": (ctypes.c_int, [_vp, _vp, ctypes.c_uint32, _vp]),
    "eq_decode_codes_multi": (ctypes.c_int, [_vp, _vp, ctypes.c_uint32, _vp]),
    "eq_gemv_multi_workspace_bytes": (ctypes.c_size_t, [_vp, ctypes.c_uint32, ctypes.c_uint32]),
    "eq_decode_gemv_multi": (ctypes.c_int, [_vp, ctypes.c_uint32, _vp, ctypes.c_uint32, _vp, _vp,
                                            _vp, ctypes.c_size_t, _vp]),
    "eq_gemm_codes_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(eq_layer), ctypes.c_uint32]),
    "eq_gemm_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(eq_layer), ctypes.c_uint32]),
    "eq_gemm_codes": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp, _vp, ctypes.c_uint32, _vp, _vp,
                                     _vp, ctypes.c_size_t, _vp]),
    "eq_decode_gemm": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp, ctypes.c_uint32, _vp, _vp,
                                      _vp, ctypes.c_size_t, _vp]),
    "eq_qk_norm_rope": (ctypes.c_int, [_vp, ctypes.c_uint64, ctypes.c_uint32, _vp, _vp,
                                       _vp, ctypes.c_uint64, ctypes.c_uint32, _vp, _vp,
                                       ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32,
                                       ctypes.c_float, _vp, _vp, _vp]),
    "eq_kv_page_bytes": (ctypes.c_size_t, [ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32]),
    "eq_kv_append": (ctypes.c_int, [_vp, _vp, _vp, ctypes.c_uint64, ctypes.c_uint32, _vp,
                                    ctypes.c_uint64, ctypes.c_uint32, _vp, _vp, _vp]),
    "eq_kv_read": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp]),
    "eq_attn_kv4_workspace_bytes": (ctypes.c_size_t, [_vp, _vp, ctypes.c_uint32]),
    "eq_attn_kv4": (ctypes.c_int, [_vp, _vp, _vp, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_float,
                                   ctypes.c_uint32, _vp, _vp, ctypes.c_size_t, _vp]),
    "eq_tree_mask": (ctypes.c_int, [_vp, _vp, ctypes.c_uint32, _vp, _vp, _vp]),
    "eq_attn_kv4_tree_workspace_bytes": (ctypes.c_size_t, [_vp, _vp, ctypes.c_uint32]),
    "eq_attn_kv4_tree": (ctypes.c_int, [_vp, _vp, _vp, ctypes.c_uint64, ctypes.c_uint32,
                                        ctypes.c_float, ctypes.c_uint32, _vp, _vp, _vp, _vp,
                                        ctypes.c_size_t, _vp]),
    "eq_tree_verify_workspace_bytes": (ctypes.c_size_t, [_vp, ctypes.c_uint32, ctypes.c_int]),
    "eq_tree_verify": (ctypes.c_int, [_vp, _vp, _vp, _vp, ctypes.c_uint64, ctypes.c_uint32, _vp,
                                      ctypes.c_uint64, ctypes.c_uint32, ctypes.c_uint32, _vp, _vp,
                                      ctypes.c_uint32, ctypes.c_uint32, _vp, _vp, _vp, _vp,
                                      ctypes.c_size_t, _vp]),
    "eq_kv_keep": (ctypes.c_int, [_vp, ctypes.c_uint32, _vp, _vp, _vp, _vp, _vp]),
    "eq_get_status": (ctypes.c_int, [ctypes.POINTER(eq_layer), _vp]),
    "eq_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "eqe_alpha_search": (ctypes.c_float, [_vp, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_double,
                                          ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32,
                                          ctypes.POINTER(ctypes.c_double)]),
    "eqe_encode": (ctypes.c_int, [_vp, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_float,
                                  ctypes.POINTER(eqe_params), ctypes.POINTER(ctypes.c_void_p),
                                  ctypes.POINTER(ctypes.c_uint64)]),
    "eqe_encode2": (ctypes.c_int, [_vp, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_float, _vp,
                                   ctypes.POINTER(eqe_params2), ctypes.POINTER(ctypes.c_void_p),
                                   ctypes.POINTER(ctypes.c_uint64)]),
    "eqe_encode_scaled": (ctypes.c_int, [_vp, ctypes.c_uint32, ctypes.c_uint32, _vp,
                                         ctypes.POINTER(eqe_params),
                                         ctypes.POINTER(ctypes.c_void_p),
                                         ctypes.POINTER(ctypes.c_uint64)]),
    "eqe_rd_objective": (ctypes.c_double, [_vp, ctypes.c_uint32, ctypes.c_uint32, ctypes.c_uint32,
                                           ctypes.c_double, _vp, ctypes.c_uint32, _vp, _vp]),
    "eqe_rd_scales": (ctypes.c_int, [_vp, ctypes.c_uint32, ctypes.c_uint32,
                                     ctypes.POINTER(eqe_rd_params), _vp, _vp, _vp]),
    "eqe_rd_lambda_search": (ctypes.c_int, [_vp, ctypes.c_uint32, ctypes.c_uint32,
                                            ctypes.c_double, ctypes.c_uint32,
                                            ctypes.POINTER(eqe_rd_params),
                                            ctypes.POINTER(ctypes.c_double),
                                            ctypes.POINTER(ctypes.c_double)]),
    "eqe_free": (None, [_vp]),
}


def build() -> str:
    """Compile libeq.so (gfx950) in place and reload it."""
    global _lib
    path = _build_lib()
    _lib = None
    return path


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is not built; run __graft_entry__.build() first")
        L = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(fn: str, rc: int) -> None:
    if rc != EQ_OK:
        raise EqError(fn, rc)


def _stream(stream):
    """The stream's handle, or the current device's current stream's (read
    directly where torch has the call: torch.cuda.current_stream() builds a
    Stream object each time)."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


def _dptr(t, dtype=None, numel=None):
    """Device pointer of a contiguous CUDA tensor, with optional checks."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"tensor too small: {t.numel()} < {numel}")
    return t.data_ptr()


# ---------------------------------------------------------------- decode ABI
def eq_strerror(code: int) -> str:
    return lib().eq_strerror(code).decode()


def eq_lut_bytes() -> int:
    return lib().eq_lut_bytes()


def eq_layer_init(host_blob: np.ndarray, dev_blob, dev_lut, dev_status) -> eq_layer:
    host_blob = np.ascontiguousarray(host_blob, dtype=np.uint8)
    L = eq_layer()
    rc = lib().eq_layer_init(ctypes.byref(L), host_blob.ctypes.data, host_blob.size,
                             _dptr(dev_blob, numel=host_blob.size),
                             _dptr(dev_lut, numel=None), _dptr(dev_status))
    _check("eq_layer_init", rc)
    return L


def eq_layer_prepare(L, stream=None) -> None:
    _check("eq_layer_prepare", lib().eq_layer_prepare(ctypes.byref(_raw(L)), _stream(stream)))


def eq_decode_codes(L, codes, stream=None) -> None:
    import torch
    r = _raw(L)
    p = _dptr(codes, torch.uint8, r.rows * r.cols)
    _check("eq_decode_codes", lib().eq_decode_codes(ctypes.byref(r), p, _stream(stream)))


def eq_decode_bf16(L, w, stream=None) -> None:
    import torch
    r = _raw(L)
    if w.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise ValueError("w must hold 16-bit BF16 patterns")
    p = _dptr(w, None, r.rows * r.cols)
    _check("eq_decode_bf16", lib().eq_decode_bf16(ctypes.byref(r), p, _stream(stream)))


def eq_gemv_workspace_bytes(L, B: int) -> int:
    return lib().eq_gemv_workspace_bytes(ctypes.byref(_raw(L)), B)


def eq_decode_gemv(L, x, B: int, bias, y, ws, stream=None) -> None:
    import torch
    r = _raw(L)
    if x.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise ValueError("x must hold 16-bit BF16 patterns")
    px = _dptr(x, None, B * r.cols)
    pb = _dptr(bias, None, r.rows) if bias is not None else None
    py = _dptr(y, torch.float32, B * r.rows)
    pw = _dptr(ws)
    nbytes = ws.numel() * ws.element_size()
    _check("eq_decode_gemv", lib().eq_decode_gemv(ctypes.byref(r), px, B, pb, py, pw, nbytes,
                                                  _stream(stream)))


def eq_decode_gemv_noalloc(L, x, B: int, bias, y, stream=None) -> None:
    """eq_decode_gemv with the library's static per-device scratch as workspace."""
    import torch
    r = _raw(L)
    if x.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise ValueError("x must hold 16-bit BF16 patterns")
    px = _dptr(x, None, B * r.cols)
    pb = _dptr(bias, None, r.rows) if bias is not None else None
    py = _dptr(y, torch.float32, B * r.rows)
    _check("eq_decode_gemv_noalloc",
           lib().eq_decode_gemv_noalloc(ctypes.byref(r), px, B, pb, py, _stream(stream)))


def _layer_array(layers):
    """Host array of eq_layer pointers (the views must outlive the call)."""
    raws = [_raw(L) for L in layers]
    arr = (ctypes.POINTER(eq_layer) * len(raws))(*[ctypes.pointer(r) for r in raws])
    return arr, raws


def _ptr_array(ptrs):
    return (ctypes.c_void_p * len(ptrs))(*ptrs)


def eq_decode_bf16_multi(layers, outs, stream=None) -> None:
    """Block-wise decode of several layers: layer i to outs[i]."""
    import torch
    if len(layers) != len(outs):
        raise ValueError("one output per layer")
    arr, raws = _layer_array(layers)
    for w in outs:
        if w.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
            raise ValueError("outputs must hold 16-bit BF16 patterns")
    ptrs = _ptr_array([_dptr(w, None, r.rows * r.cols) for w, r in zip(outs, raws)])
    _check("eq_decode_bf16_multi",
           lib().eq_decode_bf16_multi(arr, ptrs, len(raws), _stream(stream)))


def eq_decode_codes_multi(layers, outs, stream=None) -> None:
    """Block-wise decode of several layers to one-byte codes: layer i to outs[i]."""
    import torch
    if len(layers) != len(outs):
        raise ValueError("one output per layer")
    arr, raws = _layer_array(layers)
    ptrs = _ptr_array([_dptr(c, torch.uint8, r.rows * r.cols) for c, r in zip(outs, raws)])
    _check("eq_decode_codes_multi",
           lib().eq_decode_codes_multi(arr, ptrs, len(raws), _stream(stream)))


def eq_gemv_multi_workspace_bytes(layers, B: int) -> int:
    arr, raws = _layer_array(layers)
    return lib().eq_gemv_multi_workspace_bytes(arr, len(raws), B)


def eq_decode_gemv_multi(layers, x, B: int, biases, ys, ws, stream=None) -> None:
    """Fused decode-GEMV of several layers sharing the input x: ys[i] for
    layer i; biases is None or a list (entries may be None)."""
    import torch
    if len(layers) != len(ys) or (biases is not None and len(biases) != len(layers)):
        raise ValueError("one output (and bias) per layer")
    arr, raws = _layer_array(layers)
    if x.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise ValueError("x must hold 16-bit BF16 patterns")
    px = _dptr(x, None, B * raws[0].cols)
    py = _ptr_array([_dptr(y, torch.float32, B * r.rows) for y, r in zip(ys, raws)])
    pb = None
    if biases is not None:
        pb = _ptr_array([_dptr(b, None, r.rows) if b is not None else None
                         for b, r in zip(biases, raws)])
    nbytes = ws.numel() * ws.element_size()
    _check("eq_decode_gemv_multi",
           lib().eq_decode_gemv_multi(arr, len(raws), px, B, pb, py, _dptr(ws), nbytes,
                                      _stream(stream)))


def multi_workspace(layers, B: int):
    """A device workspace for eq_decode_gemv_multi over `layers`."""
    import torch
    return torch.empty(eq_gemv_multi_workspace_bytes(layers, B), dtype=torch.uint8,
                       device=layers[0].dev_blob.device)


def eq_gemm_codes_workspace_bytes(L, B: int) -> int:
    return lib().eq_gemm_codes_workspace_bytes(ctypes.byref(_raw(L)), B)


def eq_gemm_workspace_bytes(L, B: int) -> int:
    return lib().eq_gemm_workspace_bytes(ctypes.byref(_raw(L)), B)


def eq_gemm_codes(L, codes, x, B: int, bias, y, ws=None, stream=None) -> None:
    """Prefill GEMM from decoded codes: y[B][M] = x[B][N] W_hat^T + bias; ws:
    eq_gemm_codes_workspace_bytes(L, B) bytes (None when that is 0)."""
    import torch
    r = _raw(L)
    if x.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise ValueError("x must hold 16-bit BF16 patterns")
    pc = _dptr(codes, torch.uint8, r.rows * r.cols)
    px = _dptr(x, None, B * r.cols)
    pb = _dptr(bias, None, r.rows) if bias is not None else None
    py = _dptr(y, torch.float32, B * r.rows)
    pw = _dptr(ws) if ws is not None else None
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    _check("eq_gemm_codes", lib().eq_gemm_codes(ctypes.byref(r), pc, px, B, pb, py, pw, nbytes,
                                                _stream(stream)))


def eq_decode_gemm(L, x, B: int, bias, y, ws, stream=None) -> None:
    """Prefill: decode the codes into ws, then the MFMA GEMM."""
    import torch
    r = _raw(L)
    if x.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
        raise ValueError("x must hold 16-bit BF16 patterns")
    px = _dptr(x, None, B * r.cols)
    pb = _dptr(bias, None, r.rows) if bias is not None else None
    py = _dptr(y, torch.float32, B * r.rows)
    nbytes = ws.numel() * ws.element_size()
    _check("eq_decode_gemm", lib().eq_decode_gemm(ctypes.byref(r), px, B, pb, py, _dptr(ws),
                                                  nbytes, _stream(stream)))


def eq_get_status(L, stream=None) -> int:
    return lib().eq_get_status(ctypes.byref(_raw(L)), _stream(stream))


# ------------------------------------------------- 4-bit key/value cache ABI
class Rope:
    """Rotation by tables cos and sin [rows, dims / 2] (fp32, contiguous):
    channels (c, c + dims/2) turn together, or with pairs (2c, 2c + 1)."""

    def __init__(self, cos, sin, pairs: bool = False):
        import torch
        if cos.dim() != 2 or cos.shape != sin.shape:
            raise ValueError("cos and sin are two [rows, dims / 2] tables")
        if cos.device != sin.device:
            raise ValueError("cos and sin are on two devices")
        self.tables = (cos, sin)
        self.device, self.index = cos.device, cos.get_device()
        self.raw = eq_rope(_dptr(cos, torch.float32), _dptr(sin, torch.float32), cos.shape[0],
                           2 * cos.shape[1], int(bool(pairs)))
        self.ptr = ctypes.addressof(self.raw)


class KvCache:
    """A paged cache of 4-bit keys and values in `pages` (uint8, n_pages x
    eq_kv_page_bytes(), any shape with the pages in order)."""

    def __init__(self, pages, *, page_tokens: int, kv_heads: int, head_dim: int):
        import torch
        nbytes = eq_kv_page_bytes(kv_heads, head_dim, page_tokens)
        if nbytes == 0:
            raise ValueError("unsupported cache: page_tokens a power of two from 32 to 4096, "
                             "kv_heads up to 1024, head_dim 64 or 128")
        ptr = _dptr(pages, torch.uint8)
        if pages.numel() == 0 or pages.numel() % nbytes:
            raise ValueError(f"pages holds {pages.numel()} bytes, not a multiple of {nbytes}")
        self.pages, self.page_bytes = pages, nbytes
        self.device, self.index = pages.device, pages.get_device()
        self.raw = eq_kv_cache(ptr, pages.numel() // nbytes, page_tokens, kv_heads, head_dim)
        self.ptr = ctypes.addressof(self.raw)
        self.kv_heads, self.head_dim = kv_heads, head_dim

    @classmethod
    def empty(cls, n_pages: int, *, page_tokens: int, kv_heads: int, head_dim: int, device="cuda"):
        import torch
        pages = torch.empty(n_pages, eq_kv_page_bytes(kv_heads, head_dim, page_tokens),
                            dtype=torch.uint8, device=device)
        return cls(pages, page_tokens=page_tokens, kv_heads=kv_heads, head_dim=head_dim)


class KvBatch:
    """The tokens of a call (eq_kv_batch): seq_start [n + 1], kv_len [n] and
    page_table [n, max_pages], int32 on the device and read there, so their
    contents may change between calls; n_tokens, max_new and max_len bound
    them."""

    def __init__(self, seq_start, kv_len, page_table, *, n_tokens: int, max_new: int,
                 max_len: int):
        import torch
        n = kv_len.numel()
        if seq_start.numel() != n + 1 or page_table.dim() != 2 or page_table.shape[0] != n:
            raise ValueError("seq_start has n + 1 entries, kv_len n, page_table n rows")
        if not kv_len.device == seq_start.device == page_table.device:
            raise ValueError("the batch's tensors are on several devices")
        if min(n_tokens, max_new, max_len) < 0 or max(n_tokens, max_new, max_len) >> 32:
            raise ValueError("a bound below 0 or beyond 32 bits")
        self.tensors = (seq_start, kv_len, page_table)
        self.device, self.index = kv_len.device, kv_len.get_device()
        self.raw = eq_kv_batch(_dptr(seq_start, torch.int32), _dptr(kv_len, torch.int32),
                               _dptr(page_table, torch.int32), n, page_table.shape[1], n_tokens,
                               max_new, max_len)
        self.ptr = ctypes.addressof(self.raw)
        self.n_tokens, self.n_seqs, self.max_new = n_tokens, n, max_new
        self.mask_words = -(-max_new // 32)  # of a drafted tree's masks


class KvCaches:
    """Caches of one size on one device, such as a model's layers', that
    eq_kv_keep treats alike."""

    def __init__(self, caches):
        self.caches = list(caches)
        if not self.caches:
            raise ValueError("no caches")
        self.index = self.caches[0].index
        if any(c.index != self.index for c in self.caches):
            raise _apart(*self.caches)
        self.array = (_vp * len(self.caches))(*(c.ptr for c in self.caches))
        self.ptr = ctypes.addressof(self.array)


_KINDS = {}  # torch dtype -> EQ_F32 or EQ_BF16, filled by the first call
_BF16 = _I32 = _F32 = _current = _raw_stream = None


def _kinds():
    global _BF16, _I32, _F32, _current, _raw_stream
    import torch
    _BF16, _I32, _F32 = torch.bfloat16, torch.int32, torch.float32
    # the direct calls where torch has them: a device's tensors are there by now
    _current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
        (lambda device: torch.cuda.current_stream(device).cuda_stream)
    _KINDS.update({torch.float32: 0, torch.bfloat16: 1})


def _stream_on(device, stream):
    """_stream(), where the call's tensors are on `device`, which has to be the
    current one."""
    if device != _current():
        raise ValueError(f"the tensors are on device {device}, which is not the current one")
    if stream is None:
        return _raw_stream(device)
    if getattr(stream, "device_index", device) != device:
        raise ValueError(f"the stream is not of device {device}, where the tensors are")
    return stream.cuda_stream


def _apart(*handles):
    return ValueError("the call's tensors are on several devices: "
                      f"{[h.index for h in handles if h is not None]}")


def _head_rows(x, shape, what, device):
    """(pointer, token stride, element type) of x [tokens, heads, head_dim] on
    `device`, whose tokens may be apart and whose heads lie one after another;
    shape: x.shape.  (These checks are most of a small call's host time, hence
    one look at each property.)"""
    if not _KINDS:
        _kinds()
    kind = _KINDS.get(x.dtype)
    tokens, heads, dim = shape
    step, head, one = x.stride()
    if kind is None or device < 0 or x.get_device() != device or one != 1 or \
            (head != dim and heads > 1):
        raise ValueError(f"{what}: expected float32 or bfloat16 [tokens, heads, head_dim] on the "
                         "call's device, the heads of a token contiguous")
    return x.data_ptr(), step if tokens > 1 else heads * dim, kind


def _cache_rows(x, cache, batch, what, device):
    """_head_rows of rows that go into the cache."""
    shape = x.shape
    if len(shape) != 3 or shape[1] != cache.kv_heads or shape[2] != cache.head_dim or \
            shape[0] < batch.n_tokens:
        raise ValueError(f"{what}: expected [{batch.n_tokens} tokens, {cache.kv_heads}, "
                         f"{cache.head_dim}], got {tuple(shape)}")
    return _head_rows(x, shape, what, device)


def _bf16(t, numel, what, device):
    """Pointer of a contiguous BF16 tensor of at least numel elements on `device`, or None."""
    if t is None:
        return None
    if not _KINDS:
        _kinds()
    if t.dtype is not _BF16 or t.get_device() != device or not t.is_contiguous() or \
            t.numel() < numel:
        raise ValueError(f"{what}: expected a contiguous bfloat16 tensor of at least {numel} "
                         "elements on the call's device")
    return t.data_ptr()


def _positions(t, tokens, device):
    if t is None:
        return None
    if t.dtype is not _I32 or t.get_device() != device or not t.is_contiguous() or \
            t.numel() < tokens:
        raise ValueError(f"positions: expected a contiguous int32 tensor of at least {tokens} "
                         "elements on the call's device")
    return t.data_ptr()


def eq_qk_norm_rope(q, k, q_out, k_out, *, q_weight=None, k_weight=None, eps: float = 1e-6,
                    rope=None, positions=None, stream=None) -> None:
    """Norm of each head of q and k [tokens, heads, head_dim] (fp32 or BF16;
    k may be None) and its rotation, to BF16: q_out, k_out contiguous."""
    shape = q.shape
    tokens, heads, dim = shape
    if tokens >> 32:
        raise ValueError("more than 2^32 - 1 tokens")
    dev = q.get_device()
    pq, sq, kind = _head_rows(q, shape, "q", dev)
    pqo = _bf16(q_out, tokens * heads * dim, "q_out", dev)
    pk = pko = None
    sk = hk = 0
    if k is not None:
        shape = k.shape
        n, hk, kd = shape
        pk, sk, kind_k = _head_rows(k, shape, "k", dev)
        if n != tokens or kd != dim or kind_k != kind:
            raise ValueError("q and k differ in tokens, head_dim or type")
        pko = _bf16(k_out, tokens * hk * dim, "k_out", dev)
    pr = None
    if rope is not None:
        if positions is None:
            raise ValueError("a rotation needs positions")
        if rope.index != dev:
            raise ValueError("rope is not on q's device")
        pr = rope.ptr
    rc = lib().eq_qk_norm_rope(pq, sq, heads, _bf16(q_weight, dim, "q_weight", dev), pqo, pk, sk,
                               hk, _bf16(k_weight, dim, "k_weight", dev), pko, kind, tokens, dim,
                               eps, _positions(positions, tokens, dev), pr,
                               _stream_on(dev, stream))
    if rc:
        raise EqError("eq_qk_norm_rope", rc)


def eq_kv_page_bytes(kv_heads: int, head_dim: int, page_tokens: int) -> int:
    if (kv_heads | head_dim | page_tokens) >> 32:  # (ctypes would cut them; below 0 too)
        return 0
    return lib().eq_kv_page_bytes(kv_heads, head_dim, page_tokens)


def eq_kv_append(cache, batch, k, v, *, rope=None, positions=None, stream=None) -> None:
    """Append k and v [n_tokens, kv_heads, head_dim] (fp32 or BF16 each), the
    keys rotated on the way when rope is given: at `positions`, or at the
    tokens' places in their sequences."""
    dev = cache.index
    if batch.index != dev or (rope is not None and rope.index != dev):
        raise _apart(cache, batch, rope)
    pk, sk, kind_k = _cache_rows(k, cache, batch, "k", dev)
    pv, sv, kind_v = _cache_rows(v, cache, batch, "v", dev)
    rc = lib().eq_kv_append(cache.ptr, batch.ptr, pk, sk, kind_k, pv, sv, kind_v,
                            _positions(positions, batch.n_tokens, dev),
                            None if rope is None else rope.ptr,
                            _stream_on(dev, stream))
    if rc:
        raise EqError("eq_kv_append", rc)


def eq_kv_read(cache, batch, k, v, stream=None) -> None:
    """The cache's values of the batch's tokens, as BF16: k and v contiguous
    [n_tokens, kv_heads, head_dim]."""
    n = batch.n_tokens * cache.kv_heads * cache.head_dim
    dev = cache.index
    if batch.index != dev:
        raise _apart(cache, batch)
    rc = lib().eq_kv_read(cache.ptr, batch.ptr, _bf16(k, n, "k", dev), _bf16(v, n, "v", dev),
                          _stream_on(dev, stream))
    if rc:
        raise EqError("eq_kv_read", rc)


def eq_attn_kv4_workspace_bytes(cache, batch, q_heads: int) -> int:
    if q_heads >> 32:
        return 0
    return lib().eq_attn_kv4_workspace_bytes(cache.ptr, batch.ptr, q_heads)


def attn_workspace(cache, batch, q_heads: int):
    """A device workspace for eq_attn_kv4 (None when it needs none)."""
    import torch
    n = eq_attn_kv4_workspace_bytes(cache, batch, q_heads)
    return torch.empty(n, dtype=torch.uint8, device=cache.device) if n else None


def eq_attn_kv4(cache, batch, q, scale: float, out, ws=None, *, window: int = 0,
                stream=None) -> None:
    """Causal attention of q [n_tokens, q_heads, head_dim] (BF16) over the
    cache to out (BF16, contiguous); with window, over the last `window`
    positions only."""
    if window >> 32:  # (below 0 too)
        raise ValueError(f"window {window}: expected 0 (none) to 2^32 - 1")
    shape = q.shape
    n, heads, dim = shape
    dev = cache.index
    if batch.index != dev:
        raise _apart(cache, batch)
    pq, sq, kind = _head_rows(q, shape, "q", dev)
    if kind != 1 or dim != cache.head_dim or n < batch.n_tokens:
        raise ValueError(f"q: expected bfloat16 [{batch.n_tokens} tokens, heads, "
                         f"{cache.head_dim}]")
    po = _bf16(out, batch.n_tokens * heads * dim, "out", dev)
    pw, nbytes = None, 0
    if ws is not None:
        pw, nbytes = _dptr(ws), ws.numel() * ws.element_size()
        if ws.get_device() != dev:
            raise ValueError("ws is not on the call's device")
    rc = lib().eq_attn_kv4(cache.ptr, batch.ptr, pq, sq, heads, scale, window, po, pw, nbytes,
                           _stream_on(dev, stream))
    if rc:
        raise EqError("eq_attn_kv4", rc)


# ---------------------------------------------------------------- drafted trees
def _ints(t, numel, what, device, dtype=None):
    """Pointer of a contiguous int32 (or dtype) tensor of at least numel elements on
    `device`, or None."""
    if t is None:
        return None
    if not _KINDS:
        _kinds()
    if t.dtype is not (dtype or _I32) or t.get_device() != device or not t.is_contiguous() or \
            t.numel() < numel:
        raise ValueError(f"{what}: expected a contiguous {dtype or _I32} tensor of at least {numel} "
                         "elements on the call's device")
    return t.data_ptr()


def _workspace(ws, device):
    if ws is None:
        return None, 0
    if ws.get_device() != device:
        raise ValueError("ws is not on the call's device")
    return _dptr(ws), ws.numel() * ws.element_size()


def _logit_rows(x, batch, vocab, what, device):
    """(pointer, row stride, element type) of logits [n_tokens, vocab]."""
    if not _KINDS:
        _kinds()
    kind = _KINDS.get(x.dtype)
    if kind is None or x.get_device() != device or x.dim() != 2 or x.shape[0] < batch.n_tokens or \
            x.shape[1] != vocab or (x.stride(1) != 1 and vocab > 1):
        raise ValueError(f"{what}: expected float32 or bfloat16 [{batch.n_tokens} rows, {vocab}] on the "
                         "call's device, a row's logits one after another")
    return x.data_ptr(), x.stride(0) if x.shape[0] > 1 else vocab, kind


def tree_buffers(batch):
    """(mask, positions) for eq_tree_mask: int32 [n_tokens, words] and [n_tokens]."""
    import torch
    return (torch.empty(batch.n_tokens, batch.mask_words, dtype=torch.int32, device=batch.device),
            torch.empty(batch.n_tokens, dtype=torch.int32, device=batch.device))


def eq_tree_mask(batch, parents, mask, positions, *, window: int = 0, stream=None) -> None:
    """The masks (int32 [n_tokens, batch.mask_words], a bit for each new token that
    a node sees) and positions (int32 [n_tokens]) of the batch's trees, from each
    node's parent among its sequence's earlier ones (-1: the cached tokens)."""
    if window >> 32:  # (below 0 too)
        raise ValueError(f"window {window}: expected 0 (none) to 2^32 - 1")
    dev, n = batch.index, batch.n_tokens
    rc = lib().eq_tree_mask(batch.ptr, _ints(parents, n, "parents", dev), window,
                            _ints(mask, n * batch.mask_words, "mask", dev),
                            _ints(positions, n, "positions", dev), _stream_on(dev, stream))
    if rc:
        raise EqError("eq_tree_mask", rc)


def eq_attn_kv4_tree_workspace_bytes(cache, batch, q_heads: int) -> int:
    if q_heads >> 32:
        return 0
    return lib().eq_attn_kv4_tree_workspace_bytes(cache.ptr, batch.ptr, q_heads)


def attn_tree_workspace(cache, batch, q_heads: int):
    """A device workspace for eq_attn_kv4_tree (None when it needs none)."""
    import torch
    n = eq_attn_kv4_tree_workspace_bytes(cache, batch, q_heads)
    return torch.empty(n, dtype=torch.uint8, device=cache.device) if n else None


def eq_attn_kv4_tree(cache, batch, q, scale: float, mask, out, ws=None, *, positions=None,
                     window: int = 0, stream=None) -> None:
    """eq_attn_kv4 where each row of q sees, of its sequence's new tokens, those of
    its bits in `mask` (int32 [n_tokens, batch.mask_words]); with window, the cached
    tokens above positions[row] - window."""
    if window >> 32:  # (below 0 too)
        raise ValueError(f"window {window}: expected 0 (none) to 2^32 - 1")
    shape = q.shape
    n, heads, dim = shape
    dev = cache.index
    if batch.index != dev:
        raise _apart(cache, batch)
    pq, sq, kind = _head_rows(q, shape, "q", dev)
    if kind != 1 or dim != cache.head_dim or n < batch.n_tokens:
        raise ValueError(f"q: expected bfloat16 [{batch.n_tokens} tokens, heads, "
                         f"{cache.head_dim}]")
    po = _bf16(out, batch.n_tokens * heads * dim, "out", dev)
    pw, nbytes = _workspace(ws, dev)
    rc = lib().eq_attn_kv4_tree(cache.ptr, batch.ptr, pq, sq, heads, scale, window,
                                _ints(mask, batch.n_tokens * batch.mask_words, "mask", dev),
                                _positions(positions, batch.n_tokens, dev), po, pw, nbytes,
                                _stream_on(dev, stream))
    if rc:
        raise EqError("eq_attn_kv4_tree", rc)


def eq_tree_verify_workspace_bytes(batch, vocab: int, draft: bool) -> int:
    if vocab >> 32:
        return 0
    return lib().eq_tree_verify_workspace_bytes(batch.ptr, vocab, int(bool(draft)))


def verify_workspace(batch, vocab: int, *, draft: bool = True):
    """A device workspace for eq_tree_verify, with a draft's logits or without."""
    import torch
    return torch.empty(eq_tree_verify_workspace_bytes(batch, vocab, draft), dtype=torch.uint8,
                       device=batch.device)


def eq_tree_verify(batch, parents, tokens, target, draft, random, path, kept, next_token, ws, *,
                   temperature=None, replace: bool = False, max_children: int = 256,
                   stream=None) -> None:
    """Verify the batch's drafted tokens against the target's logits [n_tokens, vocab]
    (fp32 or BF16): the kept nodes of each sequence to path (int32 [n_tokens], -1
    behind them), their number to kept and the token behind them to next_token (int32
    [n_seqs]).  draft: the logits that nodes' children were drawn from, without
    replacement unless `replace`, or None where they were not drawn.  random: fp32
    [n_tokens] in [0, 1).  temperature: fp32 [n_seqs], 0 for the largest logit.
    max_children: a bound of a node's children, 1 for chains."""
    if max_children < 1 or max_children >> 32:
        raise ValueError(f"max_children {max_children}: expected 1 to 2^32 - 1")
    dev, n = batch.index, batch.n_tokens
    if target.dim() != 2 or target.shape[1] >> 32:
        raise ValueError("target: expected [rows, vocab]")
    vocab = target.shape[1]
    pt, st, kt = _logit_rows(target, batch, vocab, "target", dev)
    pd = None
    sd = kd = 0
    if draft is not None:
        pd, sd, kd = _logit_rows(draft, batch, vocab, "draft", dev)
    pw, nbytes = _workspace(ws, dev)
    rc = lib().eq_tree_verify(batch.ptr, _ints(parents, n, "parents", dev),
                              _ints(tokens, n, "tokens", dev), pt, st, kt, pd, sd, kd, vocab,
                              _ints(temperature, batch.n_seqs, "temperature", dev, _F32),
                              _ints(random, n, "random", dev, _F32), int(bool(replace)),
                              max_children, _ints(path, n, "path", dev),
                              _ints(kept, batch.n_seqs, "kept", dev),
                              _ints(next_token, batch.n_seqs, "next_token", dev), pw, nbytes,
                              _stream_on(dev, stream))
    if rc:
        raise EqError("eq_tree_verify", rc)


def eq_kv_keep(caches, batch, path, kept, new_len=None, *, stream=None) -> None:
    """Keep a path: in every cache (KvCaches, a list of KvCache, or one) the k-th of a
    sequence's new places takes new token path[seq_start + k], k < kept; new_len
    (int32 [n_seqs], not the batch's kv_len): the lengths without what was not kept."""
    if isinstance(caches, KvCache):
        caches = KvCaches([caches])
    elif not isinstance(caches, KvCaches):
        caches = KvCaches(caches)
    dev = caches.index
    if batch.index != dev:
        raise _apart(caches, batch)
    rc = lib().eq_kv_keep(caches.ptr, len(caches.caches), batch.ptr,
                          _ints(path, batch.n_tokens, "path", dev),
                          _ints(kept, batch.n_seqs, "kept", dev),
                          _ints(new_len, batch.n_seqs, "new_len", dev), _stream_on(dev, stream))
    if rc:
        raise EqError("eq_kv_keep", rc)


# ---------------------------------------------------------------- encoder ABI
def eqe_alpha_search(w: np.ndarray, target_bits: float, sample_rows: int = 0,
                     threads: int = 0, base_format: int = FMT_E4M3):
    w = np.ascontiguousarray(w, dtype=np.uint16)
    h = ctypes.c_double()
    a = lib().eqe_alpha_search(w.ctypes.data, w.shape[0], w.shape[1], target_bits, sample_rows,
                               threads, base_format, ctypes.byref(h))
    if a <= 0:
        raise EqError("eqe_alpha_search", EQ_EINVAL)
    return a, h.value


def eqe_encode(w: np.ndarray, alpha: float, *, prob_bits: int = 12, chunk_syms: int,
               lanes: int, threads: int = 0, seed: int = 0, target_bits: float = 0.0,
               base_format: int = FMT_E4M3, scale_bf16: np.ndarray | None = None) -> np.ndarray:
    """eqe_encode, or eqe_encode_scaled when scale_bf16 (uint16[M]) is given."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    prm = eqe_params(prob_bits, chunk_syms, lanes, threads, seed, target_bits, base_format)
    p = ctypes.c_void_p()
    nb = ctypes.c_uint64()
    if scale_bf16 is None:
        rc = lib().eqe_encode(w.ctypes.data, w.shape[0], w.shape[1], alpha, ctypes.byref(prm),
                              ctypes.byref(p), ctypes.byref(nb))
        _check("eqe_encode", rc)
    else:
        sc = np.ascontiguousarray(scale_bf16, dtype=np.uint16)
        if sc.size != w.shape[0]:
            raise ValueError("one scale per row")
        rc = lib().eqe_encode_scaled(w.ctypes.data, w.shape[0], w.shape[1], sc.ctypes.data,
                                     ctypes.byref(prm), ctypes.byref(p), ctypes.byref(nb))
        _check("eqe_encode_scaled", rc)
    try:
        out = np.empty(nb.value, dtype=np.uint8)
        ctypes.memmove(out.ctypes.data, p.value, nb.value)
    finally:
        lib().eqe_free(p)
    return out


def eqe_encode2(w: np.ndarray, alpha: float, *, tile_rows: int, tile_cols: int,
                res_bits: int = 12, threads: int = 0, seed: int = 0, target_bits: float = 0.0,
                base_format: int = FMT_E4M3, scale_bf16: np.ndarray | None = None,
                row_order: bool = False) -> np.ndarray:
    """A version-2 container (tile-ordered chunks, phrase alphabet); with
    row_order, the tiles are cut over the rows sorted by phrase count."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    prm = eqe_params2(res_bits, tile_rows, tile_cols, threads, seed, target_bits, base_format,
                      int(bool(row_order)))
    sc = None
    if scale_bf16 is not None:
        sc = np.ascontiguousarray(scale_bf16, dtype=np.uint16)
        if sc.size != w.shape[0]:
            raise ValueError("one scale per row")
    p = ctypes.c_void_p()
    nb = ctypes.c_uint64()
    rc = lib().eqe_encode2(w.ctypes.data, w.shape[0], w.shape[1], alpha,
                           None if sc is None else sc.ctypes.data, ctypes.byref(prm),
                           ctypes.byref(p), ctypes.byref(nb))
    _check("eqe_encode2", rc)
    try:
        out = np.empty(nb.value, dtype=np.uint8)
        ctypes.memmove(out.ctypes.data, p.value, nb.value)
    finally:
        lib().eqe_free(p)
    return out


def _rd_params(lam, iters, history, lr, threads, base_format):
    return eqe_rd_params(lam, lr, iters, history, threads, base_format)


def eqe_rd_objective(w: np.ndarray, scale: np.ndarray, lam: float, base_format: int = FMT_E4M3,
                     threads: int = 0):
    """(F, straight-through gradient, distortion term) at the given scales."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    sc = np.ascontiguousarray(scale, dtype=np.float64)
    g = np.empty(w.shape[0], dtype=np.float64)
    d = ctypes.c_double()
    f = lib().eqe_rd_objective(w.ctypes.data, w.shape[0], w.shape[1], base_format, lam,
                               sc.ctypes.data, threads, g.ctypes.data, ctypes.byref(d))
    if np.isnan(f):
        raise EqError("eqe_rd_objective", EQ_EINVAL)
    return f, g, d.value


def eqe_rd_scales(w: np.ndarray, lam: float, *, iters: int = 0, history: int = 0, lr: float = 0.0,
                  threads: int = 0, base_format: int = FMT_E4M3):
    """(scales as float64, scales as BF16 bit patterns, lowest F)."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    M = w.shape[0]
    prm = _rd_params(lam, iters, history, lr, threads, base_format)
    s64 = np.empty(M, dtype=np.float64)
    s16 = np.empty(M, dtype=np.uint16)
    f = ctypes.c_double()
    _check("eqe_rd_scales", lib().eqe_rd_scales(w.ctypes.data, M, w.shape[1], ctypes.byref(prm),
                                                 s64.ctypes.data, s16.ctypes.data, ctypes.byref(f)))
    return s64, s16, f.value


def eqe_rd_lambda_search(w: np.ndarray, target_bits: float, sample_rows: int = 0, *,
                         iters: int = 0, history: int = 0, lr: float = 0.0, threads: int = 0,
                         base_format: int = FMT_E4M3):
    """(lambda, entropy over the rows searched)."""
    w = np.ascontiguousarray(w, dtype=np.uint16)
    prm = _rd_params(0.0, iters, history, lr, threads, base_format)
    lam, h = ctypes.c_double(), ctypes.c_double()
    _check("eqe_rd_lambda_search",
           lib().eqe_rd_lambda_search(w.ctypes.data, w.shape[0], w.shape[1], target_bits,
                                      sample_rows, ctypes.byref(prm), ctypes.byref(lam),
                                      ctypes.byref(h)))
    return lam.value, h.value


# ---------------------------------------------------------------- layer object
class Layer:
    """One compressed layer resident on the device: the container bytes, the
    decode-table scratch and the status word, with its validated eq_layer."""

    def __init__(self, blob: np.ndarray, device="cuda", stream=None):
        import torch
        self.blob = np.ascontiguousarray(blob, dtype=np.uint8)
        self.dev_blob = torch.from_numpy(self.blob).to(device)
        self.lut = torch.empty(eq_lut_bytes(), dtype=torch.uint8, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.raw = eq_layer_init(self.blob, self.dev_blob, self.lut, self.status)
        eq_layer_prepare(self, stream)

    @property
    def rows(self) -> int:
        return self.raw.rows

    @property
    def cols(self) -> int:
        return self.raw.cols

    @property
    def base_format(self) -> int:
        return self.raw.base_format

    def workspace(self, B: int):
        import torch
        return torch.empty(eq_gemv_workspace_bytes(self, B), dtype=torch.uint8,
                           device=self.dev_blob.device)

    def gemm_workspace(self, B: int):
        """Workspace of eq_decode_gemm for B tokens."""
        import torch
        return torch.empty(eq_gemm_workspace_bytes(self, B), dtype=torch.uint8,
                           device=self.dev_blob.device)


def _raw(L) -> eq_layer:
    return L.raw if isinstance(L, Layer) else L


def smoke() -> None:
    """One small decode (codes, BF16), fused GEMV (B = 3) and prefill (24
    tokens) on cuda:0, and the same codes in a version-2 container (codes and
    the batch-1 GEMV), checked against the CPU oracle."""
    import sys

    import torch

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    if root not in sys.path:
        sys.path.insert(0, root)
    import oracle
    import synth
    from synth.configs import small_spec

    spec = small_spec(96, 320, bits=2.5, chunk=1024, lanes=64, seed=77)
    w = synth.weights(spec)
    alpha, _ = eqe_alpha_search(w, spec.target_bits)
    blob = eqe_encode(w, alpha, chunk_syms=spec.chunk_syms, lanes=spec.lanes)
    dev = torch.device("cuda:0")
    L = Layer(blob, dev)
    codes = torch.empty(spec.params, dtype=torch.uint8, device=dev)
    eq_decode_codes(L, codes)
    wb = torch.empty(spec.params, dtype=torch.int16, device=dev)
    eq_decode_bf16(L, wb)
    B = 3
    x = torch.from_numpy(synth.activations(spec, B).view(np.int16)).to(dev)
    y = torch.empty(B, spec.rows, dtype=torch.float32, device=dev)
    ws = L.workspace(B)
    eq_decode_gemv(L, x, B, None, y, ws)
    _check("eq_get_status", eq_get_status(L))

    rc, q_ref = oracle.container_decode(blob)
    assert rc == oracle.OK
    assert np.array_equal(codes.cpu().numpy().reshape(q_ref.shape), q_ref), "codes differ"
    w_ref = oracle.dequant(q_ref, oracle.container_scales(blob))
    assert np.array_equal(wb.cpu().numpy().view(np.uint16).reshape(w_ref.shape), w_ref), \
        "bf16 differs"
    y_ref = oracle.gemv(w_ref, synth.activations(spec, B))
    err = np.abs(y.cpu().numpy() - y_ref).max(axis=1) / np.abs(y_ref).max(axis=1)
    assert (err <= 1e-2).all(), f"gemv error {err}"
    # prefill: decode to codes + matrix-core GEMM over 24 tokens
    T = 24
    xt_bits = np.stack([synth.vector(spec.seed, 40 + t, spec.cols) for t in range(T)])
    xt = torch.from_numpy(xt_bits.view(np.int16)).to(dev)
    yt = torch.empty(T, spec.rows, dtype=torch.float32, device=dev)
    eq_decode_gemm(L, xt, T, None, yt, L.gemm_workspace(T))
    _check("eq_get_status", eq_get_status(L))
    yt_ref = oracle.gemv(w_ref, xt_bits)
    err_t = np.abs(yt.cpu().numpy() - yt_ref).max(axis=1) / np.abs(yt_ref).max(axis=1)
    assert (err_t <= 1e-2).all(), f"prefill error {err_t}"
    # version 2: tiles of 64 x 64, codes and the batch-1 GEMV
    blob2 = eqe_encode2(w, alpha, tile_rows=64, tile_cols=64)
    L2 = Layer(blob2, dev)
    codes2 = torch.empty(spec.params, dtype=torch.uint8, device=dev)
    eq_decode_codes(L2, codes2)
    x1 = x[:1].contiguous()
    y1 = torch.empty(1, spec.rows, dtype=torch.float32, device=dev)
    eq_decode_gemv(L2, x1, 1, None, y1, L2.workspace(1))
    _check("eq_get_status", eq_get_status(L2))
    rc, q2_ref = oracle.container2_decode(blob2)
    assert rc == oracle.OK
    assert np.array_equal(codes2.cpu().numpy().reshape(q2_ref.shape), q2_ref), "v2 codes differ"
    w2_ref = oracle.dequant(q2_ref, oracle.container_scales(blob2))
    y1_ref = oracle.gemv(w2_ref, synth.activations(spec, B)[:1])
    err2 = np.abs(y1.cpu().numpy() - y1_ref).max() / np.abs(y1_ref).max()
    assert err2 <= 1e-2, f"version-2 gemv error {err2}"
    print(f"smoke ok: codes/bf16 bit-exact, gemv max rel err {err.max():.2e}, "
          f"prefill max rel err {err_t.max():.2e}; version 2: codes bit-exact, "
          f"gemv rel err {err2:.2e}")
