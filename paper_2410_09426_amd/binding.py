"""Binding of libflatquant.so: argument marshalling only.

Functions have the names of the C entry points (see include/flatquant.h).  They
accept raw device addresses (ints) or objects with ``data_ptr()`` (torch
tensors); nothing is computed in Python.  There is no fallback for the
kernels: if the library is missing, loading raises.

All entry points have the parameters of their C counterparts, plus ``stream=None, check=True`` where they launch.  Those of a model's
forward pass (``NATIVE``, on the paged key/value cache ``CACHE_CALLS`` and around it ``STEP_CALLS``) are functions of the extension module ``_fqcall`` (csrc/fq_python.cpp), which calls the library that
``lib()`` has loaded.  The module is compiled for one interpreter; under another one, or where it has not been built, the same functions
call through ctypes like the rest (2.6 us of host time for a product's arguments instead of 0.5).
"""
from __future__ import annotations

import ctypes
import importlib
import os
from typing import Optional

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libflatquant.so")

FQ_OK, FQ_INVALID_ARG, FQ_UNSUPPORTED_SHAPE, FQ_MISALIGNED, FQ_LAUNCH_FAILED = range(5)

EXPORTS = (
    "flatquant_transform_quant", "flatquant_kv_transform_quant", "flatquant_kv_transform_quant_bits",
    "flatquant_dequant", "flatquant_dequant_bits", "flatquant_stream_probe", "flatquant_transform_mxfp4", "flatquant_transform_mxfp4_tiled", "fq_mxfp4_tiled_scale_bytes",
    "flatquant_dequant_mxfp4", "flatquant_mxfp4_gemm",
    "flatquant_weight_transform_quant", "fq_inverse_transpose", "flatquant_head_transform", "flatquant_w4a4_gemm",
    "fq_supported", "fq_choose_factors", "fq_default_design_fits", "fq_lds_bytes",
    "fq_status_string", "fq_last_hip_error", "fq_abi_version", "fq_set_tuning",
    "flatquant_cache_write", "flatquant_cache_read", "flatquant_cache_attention", "flatquant_cache_tree_attention", "fq_cache_attention_workspace",
    "flatquant_cache_advance", "flatquant_head_rope", "fq_rope_turns", "flatquant_cache_scored_attention",
)

# parameters of the launching entry points without the stream, and their C types: pointer, int, long (int64_t), float
_ACT = ("P1 P2 clip clip_mode T n1 n2 x_stride out_codes out_scales", "ppppiliilpp")
_GEMM = ("x_codes x_scales w_codes w_scales T m n out out_stride", "ppppliipl")
_NATIVE_PARAMS = {
    "flatquant_transform_quant": ("x " + _ACT[0], _ACT[1]),
    "flatquant_transform_mxfp4": ("x " + _ACT[0], _ACT[1]),
    "flatquant_transform_mxfp4_tiled": ("x " + _ACT[0], _ACT[1]),
    "flatquant_weight_transform_quant": ("w A1 A2 clip clip_mode m n1 n2 w_stride out_codes out_scales", _ACT[1]),
    "flatquant_w4a4_gemm": _GEMM,
    "flatquant_mxfp4_gemm": _GEMM,
    "flatquant_kv_transform_quant": ("kv P Hp clip T H D out_codes out_scales out_zeros", "ppifliippp"),
    "flatquant_kv_transform_quant_bits": ("kv P Hp clip bits T H D out_codes out_scales out_zeros", "ppifiliippp"),
    "flatquant_head_transform": ("x P Hp T H D out", "ppiliip"),
}
NATIVE = tuple(_NATIVE_PARAMS)

# the paged key/value cache: `cache` is a KvCache, `batch` a KvBatch
_CACHE_PARAMS = {
    "flatquant_cache_write": ("cache batch k k_stride v v_stride P_k P_v Hp k_clip v_clip", "ppplplppiff"),
    "flatquant_cache_read": ("cache batch k k_stride v v_stride", "ppplpl"),
    "flatquant_cache_attention": ("cache batch q q_stride Hq scale window sinks out out_stride workspace workspace_bytes", "ppplifiiplpl"),
    "flatquant_cache_tree_attention": ("cache batch q q_stride Hq scale visible out out_stride workspace workspace_bytes", "ppplifpplpl"),
}
CACHE_CALLS = tuple(_CACHE_PARAMS)

# a step around it: `pool` is a PagePool
_STEP_PARAMS = {
    "flatquant_cache_advance": ("batch pool page_tokens pages held keep rows positions slots", "ppilppppp"),
    "flatquant_head_rope": ("q q_stride Hq k k_stride H T positions turns rotary interleaved w_q w_k eps P_q P_k per_head q_out q_out_stride k_out k_out_stride",
                            "pliplilppiippfppiplpl"),
    "flatquant_cache_scored_attention": ("cache batch q q_stride Hq scale cap slopes prefix window sinks visible out out_stride workspace workspace_bytes",
                                         "pppliffppiipplpl"),
}
STEP_CALLS = tuple(_STEP_PARAMS)
_PARAMS = {**_NATIVE_PARAMS, **_CACHE_PARAMS, **_STEP_PARAMS}

_lib = None
_fqcall = None


class FlatQuantError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status}, hip error {last_hip_error()})")


def lib() -> ctypes.CDLL:
    """Load the shared library once.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2410_09426_amd.build` "
                "(there is no CPU fallback for the FlatQuant kernels)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
        for name, (params, types) in _PARAMS.items():
            getattr(L, name).argtypes = [{"p": vp, "i": i32, "l": i64, "f": f32}[t] for t in types] + [vp]
            getattr(L, name).restype = i32
        L.fq_cache_attention_workspace.argtypes = [vp, vp, i32]
        L.fq_cache_attention_workspace.restype = i64
        L.fq_rope_turns.argtypes = [vp, i32, vp]
        L.fq_rope_turns.restype = i32
        L.fq_mxfp4_tiled_scale_bytes.argtypes = [i64, i64]
        L.fq_mxfp4_tiled_scale_bytes.restype = i64
        L.flatquant_dequant_mxfp4.argtypes = [vp, vp, i64, i32, vp, vp]
        L.flatquant_dequant_mxfp4.restype = i32
        L.flatquant_dequant.argtypes = [vp, vp, vp, i64, i32, vp, vp]
        L.flatquant_dequant.restype = i32
        L.flatquant_dequant_bits.argtypes = [vp, vp, vp, i64, i32, i32, vp, vp]
        L.flatquant_dequant_bits.restype = i32
        L.fq_inverse_transpose.argtypes = [vp, i32, vp, ctypes.POINTER(ctypes.c_double)]
        L.fq_inverse_transpose.restype = i32
        L.flatquant_stream_probe.argtypes = [vp, i64, i32, i64, vp, vp]
        L.flatquant_stream_probe.restype = i32
        L.fq_supported.argtypes = [i32, i32]
        L.fq_supported.restype = i32
        L.fq_choose_factors.argtypes = [i64, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.fq_choose_factors.restype = i32
        L.fq_default_design_fits.argtypes = [i32, i32, i64]
        L.fq_default_design_fits.restype = i32
        L.fq_lds_bytes.argtypes = [i32, i32]
        L.fq_lds_bytes.restype = i64
        L.fq_status_string.argtypes = [i32]
        L.fq_status_string.restype = ctypes.c_char_p
        L.fq_last_hip_error.argtypes = []
        L.fq_last_hip_error.restype = i32
        L.fq_set_tuning.argtypes = [ctypes.c_char_p, i32, i32]
        L.fq_set_tuning.restype = i32
        L.fq_abi_version.argtypes = []
        L.fq_abi_version.restype = i32
        _lib = L
        if _fqcall:
            _fqcall.bind({n: ctypes.cast(getattr(L, n), vp).value for n in _PARAMS})
    return _lib


def _ptr(obj) -> Optional[int]:
    if obj is None:
        return None
    if isinstance(obj, int):
        return obj
    return int(obj.data_ptr())


def _stream(stream) -> Optional[int]:
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream or None
    return int(stream.cuda_stream) or None      # torch.cuda.Stream


def _ctypes_call(name: str):
    """A launching entry point through ctypes, written out from its parameters."""
    params, types = _PARAMS[name]
    convert = {"p": "_ptr", "i": "int", "l": "int", "f": "float"}
    values = ", ".join(f"{convert[t]}({p})" for p, t in zip(params.split(), types))
    scope = {}
    exec(f"def {name}({', '.join(params.split())}, stream=None, check=True):\n"
         "    'See include/flatquant.h; returns the status, raises FlatQuantError if check.'\n"
         f"    st = lib().{name}({values}, _stream(stream))\n"
         "    if check and st != FQ_OK:\n"
         f"        raise FlatQuantError(st, {name!r})\n"
         "    return st\n", globals(), scope)
    return scope[name]


try:
    _fqcall = importlib.import_module(__package__ + "._fqcall")
except ModuleNotFoundError:                     # not built, or built for another interpreter
    globals().update((n, _ctypes_call(n)) for n in _PARAMS)
else:
    _fqcall.connect(lib, FlatQuantError)
    globals().update((n, getattr(_fqcall, n)) for n in _PARAMS)


class _HostStruct:
    """A host struct of the C interface whose address the calls take; keeps what its pointers point to."""

    def __init__(self, **values):
        self._kept = tuple(values.values())
        self._struct = self._Fields(**{n: _ptr(values[n]) if t is ctypes.c_void_p else int(values[n]) for n, t in self._Fields._fields_})
        self._address = ctypes.addressof(self._struct)

    def data_ptr(self) -> int:
        return self._address


class KvCache(_HostStruct):
    """fq_kv_cache: the pages of one layer's keys and values (tensors or device addresses)."""

    class _Fields(ctypes.Structure):
        _fields_ = [("k_codes", ctypes.c_void_p), ("k_params", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("v_params", ctypes.c_void_p),
                    ("pages", ctypes.c_int64), ("page_tokens", ctypes.c_int32), ("H", ctypes.c_int32), ("k_bits", ctypes.c_int32),
                    ("v_bits", ctypes.c_int32)]

    def __init__(self, k_codes, k_params, v_codes, v_params, pages: int, page_tokens: int, H: int, k_bits: int, v_bits: int):
        super().__init__(k_codes=k_codes, k_params=k_params, v_codes=v_codes, v_params=v_params, pages=pages, page_tokens=page_tokens, H=H,
                         k_bits=k_bits, v_bits=v_bits)


class KvBatch(_HostStruct):
    """fq_kv_batch: the sequences and rows of a call (tensors or device addresses, and what the host knows of them)."""

    class _Fields(ctypes.Structure):
        _fields_ = [("row_starts", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("page_table", ctypes.c_void_p), ("B", ctypes.c_int64),
                    ("T", ctypes.c_int64), ("table_width", ctypes.c_int64), ("table_stride", ctypes.c_int64), ("max_rows", ctypes.c_int64),
                    ("max_length", ctypes.c_int64)]

    def __init__(self, row_starts, lengths, page_table, B: int, T: int, table_width: int, table_stride: int, max_rows: int, max_length: int):
        super().__init__(row_starts=row_starts, lengths=lengths, page_table=page_table, B=B, T=T, table_width=table_width,
                         table_stride=table_stride, max_rows=max_rows, max_length=max_length)


class PagePool(_HostStruct):
    """fq_page_pool: the ring of free pages (i32 [capacity]), its state (i64 [2]) and what it becomes (i64 [3]; may be the state, of three numbers then)."""

    class _Fields(ctypes.Structure):
        _fields_ = [("ring", ctypes.c_void_p), ("state", ctypes.c_void_p), ("next", ctypes.c_void_p), ("capacity", ctypes.c_int64)]

    def __init__(self, ring, state, next, capacity: int):
        super().__init__(ring=ring, state=state, next=next, capacity=capacity)


def fq_cache_attention_workspace(cache, batch, Hq: int) -> int:
    """Bytes of workspace of the attention calls; raises for arguments that they refuse."""
    n = int(lib().fq_cache_attention_workspace(_ptr(cache), _ptr(batch), int(Hq)))
    if n < 0:
        raise FlatQuantError(FQ_INVALID_ARG, "fq_cache_attention_workspace")
    return n


def status_string(status: int) -> str:
    return lib().fq_status_string(int(status)).decode()


def last_hip_error() -> int:
    return int(lib().fq_last_hip_error())


def fq_mxfp4_tiled_scale_bytes(rows: int, n: int) -> int:
    return int(lib().fq_mxfp4_tiled_scale_bytes(int(rows), int(n)))


def flatquant_dequant_mxfp4(codes, scales, rows: int, n: int, out, stream=None, check: bool = True) -> int:
    st = lib().flatquant_dequant_mxfp4(_ptr(codes), _ptr(scales), int(rows), int(n), _ptr(out), _stream(stream))
    if check and st != FQ_OK:
        raise FlatQuantError(st, "flatquant_dequant_mxfp4")
    return st


def flatquant_dequant_bits(codes, scales, zeros, rows: int, n: int, bits: int, out, stream=None, check: bool = True) -> int:
    st = lib().flatquant_dequant_bits(_ptr(codes), _ptr(scales), _ptr(zeros), int(rows), int(n), int(bits), _ptr(out),
                                      _stream(stream))
    if check and st != FQ_OK:
        raise FlatQuantError(st, "flatquant_dequant_bits")
    return st


def flatquant_dequant(codes, scales, zeros, rows: int, n: int, out, stream=None, check: bool = True) -> int:
    st = lib().flatquant_dequant(_ptr(codes), _ptr(scales), _ptr(zeros), int(rows), int(n), _ptr(out), _stream(stream))
    if check and st != FQ_OK:
        raise FlatQuantError(st, "flatquant_dequant")
    return st


def fq_inverse_transpose(P):
    """Host helper: fp16 [n, n] numpy array -> (fp16 (P^-1)^T, max |P^T out - I|).  Raises on a singular matrix."""
    import numpy as np
    P = np.ascontiguousarray(P, dtype=np.float16)
    n = P.shape[0]
    if P.ndim != 2 or P.shape != (n, n):
        raise ValueError("fq_inverse_transpose expects a square matrix")
    out = np.empty((n, n), dtype=np.float16)
    res = ctypes.c_double(0.0)
    st = lib().fq_inverse_transpose(P.ctypes.data, n, out.ctypes.data, ctypes.byref(res))
    if st != FQ_OK:
        raise FlatQuantError(st, "fq_inverse_transpose")
    return out, res.value


def fq_rope_turns(frequencies):
    """Host helper of flatquant_head_rope: float64 [n] radians a position -> uint64 [n], the angle that a position adds in units of 2^-64 of a turn."""
    import numpy as np
    f = np.ascontiguousarray(frequencies, dtype=np.float64)
    if f.ndim != 1:
        raise ValueError("fq_rope_turns expects a vector")
    turns = np.empty(f.shape, dtype=np.uint64)
    st = lib().fq_rope_turns(f.ctypes.data, len(f), turns.ctypes.data)
    if st != FQ_OK:
        raise FlatQuantError(st, "fq_rope_turns")
    return turns


def flatquant_stream_probe(x, T: int, n: int, x_stride: int, out, stream=None, check: bool = True) -> int:
    st = lib().flatquant_stream_probe(_ptr(x), int(T), int(n), int(x_stride), _ptr(out), _stream(stream))
    if check and st != FQ_OK:
        raise FlatQuantError(st, "flatquant_stream_probe")
    return st


def fq_supported(n1: int, n2: int) -> bool:
    return bool(lib().fq_supported(int(n1), int(n2)))


def fq_choose_factors(n: int):
    a, b = ctypes.c_int(0), ctypes.c_int(0)
    st = lib().fq_choose_factors(int(n), ctypes.byref(a), ctypes.byref(b))
    if st != FQ_OK:
        raise FlatQuantError(st, "fq_choose_factors")
    return a.value, b.value


def fq_default_design_fits(n1: int, n2: int, m_bytes: int) -> bool:
    return bool(lib().fq_default_design_fits(int(n1), int(n2), int(m_bytes)))


def fq_lds_bytes(n1: int, n2: int) -> int:
    return int(lib().fq_lds_bytes(int(n1), int(n2)))


def fq_set_tuning(name: str, value: Optional[int]) -> None:
    """Set a tuning override (value) or remove it (None)."""
    st = lib().fq_set_tuning(name.encode(), 0 if value is None else int(value), 0 if value is None else 1)
    if st != FQ_OK:
        raise FlatQuantError(st, f"fq_set_tuning({name})")


def fq_abi_version() -> int:
    return int(lib().fq_abi_version())
