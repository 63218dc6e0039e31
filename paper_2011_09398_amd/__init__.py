"""MI355X (gfx950) bitpacked binary convolution: Python binding of include/lce.h.

Argument marshalling only: every step of the operator runs in the HIP
kernels of liblce.so.  torch supplies device memory and the current stream.
If the library is not built this module raises; there is no CPU fallback.

    bitpack(x)                        LceQuantize: float [..., C] -> int32 [..., ceil(C/32)]
    bconv2d(x_packed, w_packed, c_in) LceBConv2d with the fused output transform
    quantize_bconv2d(x, w_packed)     LceQuantize + LceBConv2d in one launch (float input)
    pad_correction(w_packed, c_in)    zero-padding correction table of a filter tensor
    fold_thresholds(m, b, k, clamp)   float transform + binarization -> thresholds, flip
    mfma_weights(w_packed, c_in)      filters widened to 4-bit +-1.0 for the matrix-core path
    bconv2d_mfma(x_packed, w_fp4, ..) LceBConv2d on the matrix cores (same result)
    bmaxpool2d(x_packed, channels)    LceBMaxPool2d: AND over each window of packed words
    dequantize(x_packed, channels)    LceDequantize: packed bits -> +-1.0 float32

A transformer's key/value cache in 4 bits:

    KV4Cache(kv_heads, head_dim, ..)  the cache's memory: pages of 64 tokens
    kv4_append(cache, k, v, slots)    quantize keys and values as they are written
    kv4_read(cache, slots)            read tokens back as floats
    kv4_attention(cache, q, table, q_start, lengths)  attention over cached sequences
    kv4_select(cache, q, table, q_start, lengths, n)  the n pages whose key signs fit best
    kv4_workspace(cache, q, table)    memory that the last two keep between calls

The same in 8 bits, and the positions of what goes into either:

    KV8Cache(kv_heads, head_dim, ..)  the cache's memory: pages of 64 tokens
    kv8_append(cache, k, v, table, q_start, lengths)  quantize sequences' last tokens
    kv8_read(cache, slots)            read tokens back as floats
    kv8_attention(cache, q, table, q_start, lengths)  attention over cached sequences, with
                                      capped scores, a bias by distance, a prefix
    kv8_workspace(cache, q, table)    memory that attention keeps between calls
    Rotary(head_dim, ..)              frequencies of rotary positions
    rotary(plan, positions, q, k)     queries and keys turned to their positions
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
from typing import Optional, Sequence, Tuple, Union

from . import build as _build

LCE_OK, LCE_EINVAL, LCE_EUNSUPPORTED, LCE_EALIGN, LCE_EHIP = 0, 1, 2, 3, 4
STATUS_NAMES = {0: "LCE_OK", 1: "LCE_EINVAL", 2: "LCE_EUNSUPPORTED", 3: "LCE_EALIGN",
                4: "LCE_EHIP"}
PADDING = {"valid": 0, "same": 1}
PAD_VALUE = {"one": 0, "zero": 1}
OUT_TYPE = {"float": 0, "bitpacked": 1, "int32": 2}
INT32_MIN = -(2 ** 31)
INT32_MAX = 2 ** 31 - 1

# Every symbol include/lce.h declares.
EXPORTS = ("lce_packed_words", "lce_bconv2d_out_shape", "lce_bitpack", "lce_bconv2d",
           "lce_bconv2d_pad_correction_size", "lce_bconv2d_pad_correction",
           "lce_fold_thresholds", "lce_bmaxpool2d_out_shape", "lce_bmaxpool2d",
           "lce_dequantize", "lce_bconv2d_mfma_weights_size", "lce_bconv2d_mfma_weights",
           "lce_bconv2d_mfma", "lce_quantize_bconv2d", "lce_quantize_bconv2d_mfma",
           "lce_kv4_cache_size", "lce_kv4_append", "lce_kv4_read", "lce_kv4_workspace_size",
           "lce_kv4_attention_workspace_size", "lce_kv4_select_workspace_size",
           "lce_kv4_attention", "lce_kv4_select",
           "lce_kv8_cache_size", "lce_kv8_append", "lce_kv8_read", "lce_kv8_workspace_size",
           "lce_kv8_attention", "lce_rotary_frequencies", "lce_rotary_turns", "lce_rotary",
           "lce_set_tuning", "lce_get_tuning",
           "lce_last_error", "lce_last_schedule")

# lce_tuning_key values, by the names tuning() takes.
TUNING_KEYS = {"xor_nb": 0, "xor_ks": 1, "mfma_schedule": 2, "mfma_fs_ks": 3, "mfma_fs_s": 4,
               "mfma_fs_wpc": 5, "mfma_fs_pad": 6, "mfma_packed": 7, "mfma_tile_m": 8,
               "mfma_tile_n": 9, "mfma_fs_window": 10, "xor_stream": 11, "kv4_chunk": 12,
               "kv4_rows": 13, "kv8_chunk": 14, "kv8_rows": 15}
MFMA_SCHEDULES = {"auto": 0, "fs": 1, "ksplit": 2, "pixel": 3, "stream": 4}


class Desc(ctypes.Structure):
    """lce_bconv2d_desc: fourteen int32 fields, in header order."""
    _fields_ = [(name, ctypes.c_int32) for name in (
        "n", "h", "w", "c_in", "c_out", "kh", "kw", "stride_h", "stride_w",
        "padding", "pad_value", "clamp_min", "clamp_max", "out_type")]


class PoolDesc(ctypes.Structure):
    """lce_bmaxpool2d_desc: nine int32 fields, in header order."""
    _fields_ = [(name, ctypes.c_int32) for name in (
        "n", "h", "w", "channels", "kh", "kw", "stride_h", "stride_w", "padding")]


class KV4CacheDesc(ctypes.Structure):
    """lce_kv4_cache_desc: three int32 fields, in header order."""
    _fields_ = [(name, ctypes.c_int32) for name in ("pages", "kv_heads", "head_dim")]


class KV4QueryDesc(ctypes.Structure):
    """lce_kv4_query_desc: ten int32 fields, a float and two int64, in header order."""
    _fields_ = [(name, ctypes.c_int32) for name in (
        "tokens", "q_heads", "seqs", "table_width", "type", "causal", "window", "list", "max_q",
        "max_len")] + [("scale", ctypes.c_float), ("q_token_stride", ctypes.c_int64),
                       ("q_head_stride", ctypes.c_int64)]


class KV8CacheDesc(ctypes.Structure):
    """lce_kv8_cache_desc: three int32 fields, in header order."""
    _fields_ = KV4CacheDesc._fields_


class KV8QueryDesc(ctypes.Structure):
    """lce_kv8_query_desc: nine int32 fields, two floats and two int64, in header order."""
    _fields_ = [(name, ctypes.c_int32) for name in (
        "tokens", "q_heads", "seqs", "table_width", "type", "causal", "window", "max_q",
        "max_len")] + [("scale", ctypes.c_float), ("softcap", ctypes.c_float),
                       ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64)]


class RotaryDesc(ctypes.Structure):
    """lce_rotary_desc: six int32 fields and a float, in header order."""
    _fields_ = [(name, ctypes.c_int32) for name in (
        "tokens", "head_dim", "rot_dim", "type", "interleaved", "backward")] + [
            ("scale", ctypes.c_float)]


class RotaryRows(ctypes.Structure):
    """lce_rotary_rows: an int32, two pointers and four int64, in header order."""
    _fields_ = [("heads", ctypes.c_int32), ("x", ctypes.c_void_p), ("y", ctypes.c_void_p)] + [
        (name, ctypes.c_int64) for name in ("x_token_stride", "x_head_stride", "y_token_stride",
                                            "y_head_stride")]


class LceError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded liblce.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.LIB):
            raise ImportError(f"{_build.LIB} is not built; run paper_2011_09398_amd.build.build()")
        L = ctypes.CDLL(_build.LIB)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.lce_packed_words.argtypes = [i32]
        L.lce_packed_words.restype = i32
        L.lce_bconv2d_out_shape.argtypes = [ctypes.POINTER(Desc), ctypes.POINTER(i32),
                                            ctypes.POINTER(i32)]
        L.lce_bconv2d_out_shape.restype = ctypes.c_int
        L.lce_bitpack.argtypes = [vp, vp, i64, i32, vp]
        L.lce_bitpack.restype = ctypes.c_int
        L.lce_bconv2d.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.lce_bconv2d.restype = ctypes.c_int
        L.lce_bconv2d_pad_correction_size.argtypes = [ctypes.POINTER(Desc),
                                                       ctypes.POINTER(i64)]
        L.lce_bconv2d_pad_correction_size.restype = ctypes.c_int
        L.lce_bconv2d_pad_correction.argtypes = [ctypes.POINTER(Desc), vp, vp, vp]
        L.lce_bconv2d_pad_correction.restype = ctypes.c_int
        L.lce_fold_thresholds.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp]
        L.lce_fold_thresholds.restype = ctypes.c_int
        L.lce_bmaxpool2d_out_shape.argtypes = [ctypes.POINTER(PoolDesc), ctypes.POINTER(i32),
                                               ctypes.POINTER(i32)]
        L.lce_bmaxpool2d_out_shape.restype = ctypes.c_int
        L.lce_bmaxpool2d.argtypes = [ctypes.POINTER(PoolDesc), vp, vp, vp]
        L.lce_bmaxpool2d.restype = ctypes.c_int
        L.lce_dequantize.argtypes = [vp, vp, i64, i32, vp]
        L.lce_dequantize.restype = ctypes.c_int
        L.lce_bconv2d_mfma_weights_size.argtypes = [ctypes.POINTER(Desc), ctypes.POINTER(i64)]
        L.lce_bconv2d_mfma_weights_size.restype = ctypes.c_int
        L.lce_bconv2d_mfma_weights.argtypes = [ctypes.POINTER(Desc), vp, vp, vp]
        L.lce_bconv2d_mfma_weights.restype = ctypes.c_int
        L.lce_bconv2d_mfma.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, vp, vp, vp]
        L.lce_bconv2d_mfma.restype = ctypes.c_int
        L.lce_quantize_bconv2d.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, vp, vp, vp]
        L.lce_quantize_bconv2d.restype = ctypes.c_int
        L.lce_quantize_bconv2d_mfma.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, vp,
                                                vp, vp]
        L.lce_quantize_bconv2d_mfma.restype = ctypes.c_int
        cd, qd = ctypes.POINTER(KV4CacheDesc), ctypes.POINTER(KV4QueryDesc)
        L.lce_kv4_cache_size.argtypes = [cd, ctypes.POINTER(i64)]
        L.lce_kv4_cache_size.restype = ctypes.c_int
        L.lce_kv4_append.argtypes = [cd, vp, i32, vp, i64, i64, vp, i64, i64, vp, i64, vp]
        L.lce_kv4_append.restype = ctypes.c_int
        L.lce_kv4_read.argtypes = [cd, vp, vp, i64, i32, vp, vp, vp]
        L.lce_kv4_read.restype = ctypes.c_int
        for size in (L.lce_kv4_workspace_size, L.lce_kv4_attention_workspace_size,
                     L.lce_kv4_select_workspace_size):
            size.argtypes = [cd, qd, ctypes.POINTER(i64)]
            size.restype = ctypes.c_int
        L.lce_kv4_attention.argtypes = [cd, vp, qd, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        L.lce_kv4_attention.restype = ctypes.c_int
        L.lce_kv4_select.argtypes = [cd, vp, qd, vp, vp, vp, vp, i32, i32, vp, vp, i64, vp]
        L.lce_kv4_select.restype = ctypes.c_int
        cd, qd = ctypes.POINTER(KV8CacheDesc), ctypes.POINTER(KV8QueryDesc)
        L.lce_kv8_cache_size.argtypes = [cd, ctypes.POINTER(i64)]
        L.lce_kv8_append.argtypes = [cd, vp, i32, vp, i64, i64, vp, i64, i64, i32, i32, i32, vp, vp,
                                     vp, vp]
        L.lce_kv8_read.argtypes = [cd, vp, vp, i64, i32, vp, vp, vp]
        L.lce_kv8_workspace_size.argtypes = [cd, qd, ctypes.POINTER(i64)]
        L.lce_kv8_attention.argtypes = [cd, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
        dp = ctypes.POINTER(ctypes.c_double)
        L.lce_rotary_frequencies.argtypes = [i32, ctypes.c_double, i32, ctypes.c_double,
                                             ctypes.c_double, dp, ctypes.POINTER(ctypes.c_float)]
        L.lce_rotary_turns.argtypes = [dp, i32, ctypes.POINTER(ctypes.c_uint64)]
        L.lce_rotary.argtypes = [vp, vp, vp, vp, vp, vp]
        for name in ("kv8_cache_size", "kv8_append", "kv8_read", "kv8_workspace_size",
                     "kv8_attention", "rotary_frequencies", "rotary_turns", "rotary"):
            getattr(L, "lce_" + name).restype = ctypes.c_int
        L.lce_set_tuning.argtypes = [i32, i32]
        L.lce_set_tuning.restype = ctypes.c_int
        L.lce_get_tuning.argtypes = [i32]
        L.lce_get_tuning.restype = i32
        L.lce_last_error.argtypes = []
        L.lce_last_error.restype = ctypes.c_char_p
        L.lce_last_schedule.argtypes = []
        L.lce_last_schedule.restype = ctypes.c_char_p
        _lib = L
    return _lib


def last_error() -> str:
    return lib().lce_last_error().decode()


def last_schedule() -> str:
    """The schedule of this thread's last convolution or attention (lce_last_schedule)."""
    return lib().lce_last_schedule().decode()


def _check(status: int) -> None:
    if status != LCE_OK:
        raise LceError(status, last_error())


def set_tuning(**overrides) -> None:
    """Schedule overrides (lce_set_tuning), e.g. set_tuning(xor_nb=2,
    mfma_schedule="fs"); 0 restores the automatic choice.  Process-wide."""
    for name, value in overrides.items():
        if name not in TUNING_KEYS:
            raise KeyError(f"unknown tuning key {name!r}")
        if name == "mfma_schedule" and isinstance(value, str):
            value = MFMA_SCHEDULES[value]
        _check(lib().lce_set_tuning(TUNING_KEYS[name], int(value)))


def get_tuning(name: str) -> int:
    return int(lib().lce_get_tuning(TUNING_KEYS[name]))


class tuning:
    """Context manager: the given overrides inside, every key back to
    automatic (0) on exit."""

    def __init__(self, **overrides):
        self.overrides = overrides

    def __enter__(self):
        set_tuning(**self.overrides)
        return self

    def __exit__(self, *exc):
        set_tuning(**{k: 0 for k in TUNING_KEYS})
        return False


def packed_words(channels: int) -> int:
    return int(lib().lce_packed_words(int(channels)))


def make_desc(n, h, w, c_in, c_out, kh, kw, stride=1, padding="same", pad_value="one",
              clamp: Optional[Tuple[int, int]] = None, out_type="float") -> Desc:
    sh, sw = (stride, stride) if isinstance(stride, int) else tuple(stride)
    lo, hi = (INT32_MIN, INT32_MAX) if clamp is None else clamp
    return Desc(n, h, w, c_in, c_out, kh, kw, sh, sw,
                PADDING[padding] if isinstance(padding, str) else padding,
                PAD_VALUE[pad_value] if isinstance(pad_value, str) else pad_value,
                lo, hi, OUT_TYPE[out_type] if isinstance(out_type, str) else out_type)


def out_shape(desc: Desc) -> Tuple[int, int]:
    oh, ow = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().lce_bconv2d_out_shape(ctypes.byref(desc), ctypes.byref(oh), ctypes.byref(ow)))
    return oh.value, ow.value


def _raw_stream():
    """torch's function from a device index to its current stream's handle
    (0.2 us; building a torch.cuda.Stream for its handle takes 2.6 us, as long
    as a short kernel), or one that goes through torch.cuda.current_stream."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw if raw is not None else (lambda i: torch.cuda.current_stream(i).cuda_stream)


_raw = None


def _stream_of(index) -> int:
    """The handle of device `index`'s current stream."""
    global _raw
    if _raw is None:
        _raw = _raw_stream()
    return _raw(index)


def _stream_handle(t) -> int:
    return _stream_of(t.device.index)


def _require(t, dtype, name):
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a device tensor, got {t.device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def bitpack(x, out=None):
    """LceQuantize on a float32 device tensor [..., C] -> int32 [..., ceil(C/32)]."""
    import torch
    _require(x, torch.float32, "x")
    c = x.shape[-1]
    cw = packed_words(c)
    rows = x.numel() // c if c else 0
    if out is None:
        out = torch.empty(tuple(x.shape[:-1]) + (cw,), dtype=torch.int32, device=x.device)
    else:
        _require(out, torch.int32, "out")
        if out.numel() != rows * cw:
            raise ValueError("out has the wrong size")
    _check(lib().lce_bitpack(x.data_ptr(), out.data_ptr(), rows, c, _stream_handle(x)))
    return out


def _filter_desc(w_packed, c_in, padding="same", pad_value="zero", stride=1) -> Desc:
    """A descriptor for filter-only calls (the input dims do not matter)."""
    cout, kh, kw, _ = w_packed.shape
    return make_desc(1, kh, kw, c_in, cout, kh, kw, stride, padding, pad_value, None, "int32")


def pad_correction_size(desc: Desc) -> int:
    n = ctypes.c_int64()
    _check(lib().lce_bconv2d_pad_correction_size(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def pad_correction(w_packed, c_in: int, out=None):
    """Zero-padding correction table of w_packed: int32 [(KH+1)*KW*(KW+1)/2, Cout]."""
    import torch
    _require(w_packed, torch.int32, "w_packed")
    cout, kh, kw, cw = w_packed.shape
    if cw != packed_words(c_in):
        raise ValueError(f"packed channel words {cw} do not match c_in={c_in}")
    desc = _filter_desc(w_packed, c_in)
    size = pad_correction_size(desc)
    if out is None:
        out = torch.empty(((kh + 1) * (kw * (kw + 1) // 2), cout), dtype=torch.int32,
                          device=w_packed.device)
    else:
        _require(out, torch.int32, "out")
        if out.numel() != size:
            raise ValueError(f"out must hold {size} elements")
    _check(lib().lce_bconv2d_pad_correction(ctypes.byref(desc), w_packed.data_ptr(),
                                            out.data_ptr(), _stream_handle(w_packed)))
    return out


def fold_thresholds(multiplier, bias, c_out: int, k: int,
                    clamp: Optional[Tuple[int, int]] = None):
    """Host-side fold of (multiplier, bias) into (thresholds float32 [c_out],
    flip int32 [ceil(c_out/32)]), both numpy arrays.  multiplier/bias: array-likes
    of c_out floats, or None for 1 / 0."""
    import numpy as np
    lo, hi = (INT32_MIN, INT32_MAX) if clamp is None else clamp
    arrs = []
    for a, name in ((multiplier, "multiplier"), (bias, "bias")):
        if a is None:
            arrs.append(None)
        else:
            a = np.ascontiguousarray(a, dtype=np.float32)
            if a.size != c_out:
                raise ValueError(f"{name} must have {c_out} elements")
            arrs.append(a)
    thr = np.empty(c_out, dtype=np.float32)
    flip = np.empty(max(packed_words(c_out), 0), dtype=np.int32)
    ptr = lambda a: None if a is None else a.ctypes.data
    _check(lib().lce_fold_thresholds(ptr(arrs[0]), ptr(arrs[1]), int(c_out), int(k), int(lo),
                                     int(hi), thr.ctypes.data, flip.ctypes.data))
    return thr, flip


def _epilogue_args(cout, kh, kw, multiplier, bias, thresholds, flip, pad_correction=None):
    """Check the optional per-channel tensors of a convolution; their pointers."""
    import torch
    ptrs = []
    for t, name, dtype, numel in ((multiplier, "multiplier", torch.float32, cout),
                                  (bias, "bias", torch.float32, cout),
                                  (thresholds, "thresholds", torch.float32, cout),
                                  (flip, "flip", torch.int32, packed_words(cout)),
                                  (pad_correction, "pad_correction", torch.int32,
                                   (kh + 1) * (kw * (kw + 1) // 2) * cout)):
        if t is None:
            ptrs.append(None)
        else:
            _require(t, dtype, name)
            if t.numel() != numel:
                raise ValueError(f"{name} must have {numel} elements")
            ptrs.append(t.data_ptr())
    return ptrs


def _conv_out(out, out_type, n, oh, ow, cout, device):
    """Check a caller's output tensor, or allocate one."""
    import torch
    oc = packed_words(cout) if out_type == "bitpacked" else cout
    dt = torch.float32 if out_type == "float" else torch.int32
    if out is None:
        return torch.empty((n, oh, ow, oc), dtype=dt, device=device)
    _require(out, dt, "out")
    if out.numel() != n * oh * ow * oc:
        raise ValueError(f"out must hold {n}x{oh}x{ow}x{oc} elements")
    return out


def bconv2d(x_packed, w_packed, c_in: int, *, stride: Union[int, Sequence[int]] = 1,
            padding: str = "same", pad_value: str = "one",
            clamp: Optional[Tuple[int, int]] = None, out_type: str = "float",
            multiplier=None, bias=None, thresholds=None, flip=None, pad_correction=None,
            out=None):
    """LceBConv2d: x_packed int32 [N,H,W,Cw], w_packed int32 [Cout,KH,KW,Cw].

    out_type "float" -> float32 [N,OH,OW,Cout]; "bitpacked" -> int32
    [N,OH,OW,ceil(Cout/32)]; "int32" -> the clamped accumulator [N,OH,OW,Cout].
    flip: int32 [ceil(Cout/32)] direction bits (bitpacked output).
    pad_correction: the table of pad_correction(w_packed, c_in), needed by
    pad_value "zero" when the geometry pads.
    """
    import torch
    _require(x_packed, torch.int32, "x_packed")
    _require(w_packed, torch.int32, "w_packed")
    n, h, w, cw = x_packed.shape
    cout, kh, kw, cw2 = w_packed.shape
    if cw != packed_words(c_in) or cw2 != cw:
        raise ValueError(f"packed channel words {cw}/{cw2} do not match c_in={c_in}")
    desc = make_desc(n, h, w, c_in, cout, kh, kw, stride, padding, pad_value, clamp, out_type)
    oh, ow = out_shape(desc)
    ptrs = _epilogue_args(cout, kh, kw, multiplier, bias, thresholds, flip, pad_correction)
    out = _conv_out(out, out_type, n, oh, ow, cout, x_packed.device)
    _check(lib().lce_bconv2d(ctypes.byref(desc), x_packed.data_ptr(), w_packed.data_ptr(),
                             *ptrs, out.data_ptr(), _stream_handle(x_packed)))
    return out


def quantize_bconv2d(x, w_packed, *, stride: Union[int, Sequence[int]] = 1,
                     padding: str = "same", clamp: Optional[Tuple[int, int]] = None,
                     out_type: str = "float", multiplier=None, bias=None, thresholds=None,
                     flip=None, out=None):
    """LceQuantize + LceBConv2d in one launch: x float32 [N,H,W,C_in] (C_in a
    multiple of 32, 16-byte aligned), w_packed int32 [Cout,KH,KW,C_in/32].

    The result equals bconv2d(bitpack(x), w_packed, C_in, ...) with one
    padding.  Shapes the fused kernel does not cover raise LceError with
    status LCE_EUNSUPPORTED (nothing is launched); run bitpack and bconv2d.
    """
    import torch
    _require(x, torch.float32, "x")
    _require(w_packed, torch.int32, "w_packed")
    n, h, w, c_in = x.shape
    cout, kh, kw, cw = w_packed.shape
    if cw != packed_words(c_in):
        raise ValueError(f"packed channel words {cw} do not match c_in={c_in}")
    desc = make_desc(n, h, w, c_in, cout, kh, kw, stride, padding, "one", clamp, out_type)
    oh, ow = out_shape(desc)
    ptrs = _epilogue_args(cout, kh, kw, multiplier, bias, thresholds, flip)[:4]
    out = _conv_out(out, out_type, n, oh, ow, cout, x.device)
    _check(lib().lce_quantize_bconv2d(ctypes.byref(desc), x.data_ptr(), w_packed.data_ptr(),
                                      *ptrs, out.data_ptr(), _stream_handle(x)))
    return out


def make_pool_desc(n, h, w, channels, kernel=2, stride=None, padding="valid") -> PoolDesc:
    kh, kw = (kernel, kernel) if isinstance(kernel, int) else tuple(kernel)
    if stride is None:
        stride = (kh, kw)
    sh, sw = (stride, stride) if isinstance(stride, int) else tuple(stride)
    return PoolDesc(n, h, w, channels, kh, kw, sh, sw,
                    PADDING[padding] if isinstance(padding, str) else padding)


def pool_out_shape(desc: PoolDesc) -> Tuple[int, int]:
    oh, ow = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().lce_bmaxpool2d_out_shape(ctypes.byref(desc), ctypes.byref(oh),
                                          ctypes.byref(ow)))
    return oh.value, ow.value


def bmaxpool2d(x_packed, channels: int, kernel=2, stride=None, padding: str = "valid",
               out=None):
    """LceBMaxPool2d on int32 [N,H,W,ceil(C/32)] -> int32 [N,OH,OW,ceil(C/32)]
    (stride defaults to the window size, as in TensorFlow)."""
    import torch
    _require(x_packed, torch.int32, "x_packed")
    n, h, w, cw = x_packed.shape
    if cw != packed_words(channels):
        raise ValueError(f"packed words {cw} do not match channels={channels}")
    desc = make_pool_desc(n, h, w, channels, kernel, stride, padding)
    oh, ow = pool_out_shape(desc)
    if out is None:
        out = torch.empty((n, oh, ow, cw), dtype=torch.int32, device=x_packed.device)
    else:
        _require(out, torch.int32, "out")
        if out.numel() != n * oh * ow * cw:
            raise ValueError(f"out must hold {n}x{oh}x{ow}x{cw} words")
    _check(lib().lce_bmaxpool2d(ctypes.byref(desc), x_packed.data_ptr(), out.data_ptr(),
                                _stream_handle(x_packed)))
    return out


def dequantize(x_packed, channels: int, out=None):
    """LceDequantize: int32 [..., ceil(C/32)] -> float32 [..., C] of +-1.0."""
    import torch
    _require(x_packed, torch.int32, "x_packed")
    cw = x_packed.shape[-1]
    if cw != packed_words(channels):
        raise ValueError(f"packed words {cw} do not match channels={channels}")
    rows = x_packed.numel() // cw if cw else 0
    if out is None:
        out = torch.empty(tuple(x_packed.shape[:-1]) + (channels,), dtype=torch.float32,
                          device=x_packed.device)
    else:
        _require(out, torch.float32, "out")
        if out.numel() != rows * channels:
            raise ValueError("out has the wrong size")
    _check(lib().lce_dequantize(x_packed.data_ptr(), out.data_ptr(), rows, channels,
                                _stream_handle(x_packed)))
    return out


def mfma_weights_size(desc: Desc) -> int:
    """Bytes of the widened filter buffer lce_bconv2d_mfma reads for `desc`."""
    n = ctypes.c_int64()
    _check(lib().lce_bconv2d_mfma_weights_size(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def mfma_weights(w_packed, c_in: int, out=None):
    """Widened filters for bconv2d_mfma: uint8 device buffer (16-byte aligned)."""
    import torch
    _require(w_packed, torch.int32, "w_packed")
    cout, kh, kw, cw = w_packed.shape
    if cw != packed_words(c_in):
        raise ValueError(f"packed channel words {cw} do not match c_in={c_in}")
    desc = _filter_desc(w_packed, c_in)
    n = ctypes.c_int64()
    _check(lib().lce_bconv2d_mfma_weights_size(ctypes.byref(desc), ctypes.byref(n)))
    if out is None:
        out = torch.empty(n.value, dtype=torch.uint8, device=w_packed.device)
    elif out.numel() * out.element_size() < n.value:
        raise ValueError(f"out must hold {n.value} bytes")
    _check(lib().lce_bconv2d_mfma_weights(ctypes.byref(desc), w_packed.data_ptr(),
                                          out.data_ptr(), _stream_handle(w_packed)))
    return out


def _mfma_conv(fn, x, x_float: bool, w_fp4, c_in: int, c_out: int, kernel, stride, padding,
               pad_value, clamp, out_type, multiplier, bias, thresholds, flip, out):
    """Shared marshalling of the two matrix-core entry points (packed or
    float input); returns the output tensor."""
    import torch
    if x_float:
        _require(x, torch.float32, "x")
        n, h, w, c = x.shape
        if c != c_in:
            raise ValueError(f"x has {c} channels, c_in={c_in}")
    else:
        _require(x, torch.int32, "x_packed")
        n, h, w, cw = x.shape
        if cw != packed_words(c_in):
            raise ValueError(f"packed channel words {cw} do not match c_in={c_in}")
    if not isinstance(w_fp4, torch.Tensor) or w_fp4.device.type != "cuda":
        raise TypeError("w_fp4 must be a device tensor")
    if not w_fp4.is_contiguous():
        raise ValueError("w_fp4 must be contiguous")
    kh, kw = (kernel, kernel) if isinstance(kernel, int) else tuple(kernel)
    desc = make_desc(n, h, w, c_in, c_out, kh, kw, stride, padding, pad_value, clamp, out_type)
    oh, ow = out_shape(desc)
    need = mfma_weights_size(desc)
    if w_fp4.numel() * w_fp4.element_size() < need:
        raise ValueError(f"w_fp4 holds {w_fp4.numel() * w_fp4.element_size()} bytes; these "
                         f"filters widen to {need} (mfma_weights of the same c_in, c_out "
                         f"and kernel)")
    ptrs = []
    for t, name, dtype, numel in ((multiplier, "multiplier", torch.float32, c_out),
                                  (bias, "bias", torch.float32, c_out),
                                  (thresholds, "thresholds", torch.float32, c_out),
                                  (flip, "flip", torch.int32, packed_words(c_out))):
        if t is None:
            ptrs.append(None)
        else:
            _require(t, dtype, name)
            if t.numel() != numel:
                raise ValueError(f"{name} must have {numel} elements")
            ptrs.append(t.data_ptr())
    oc = packed_words(c_out) if out_type == "bitpacked" else c_out
    dt = torch.float32 if out_type == "float" else torch.int32
    if out is None:
        out = torch.empty((n, oh, ow, oc), dtype=dt, device=x.device)
    else:
        _require(out, dt, "out")
        if out.numel() != n * oh * ow * oc:
            raise ValueError(f"out must hold {n}x{oh}x{ow}x{oc} elements")
    _check(fn(ctypes.byref(desc), x.data_ptr(), w_fp4.data_ptr(), *ptrs, out.data_ptr(),
              _stream_handle(x)))
    return out


def bconv2d_mfma(x_packed, w_fp4, c_in: int, c_out: int, kernel, *, stride=1,
                 padding: str = "same", pad_value: str = "one",
                 clamp: Optional[Tuple[int, int]] = None, out_type: str = "float",
                 multiplier=None, bias=None, thresholds=None, flip=None, out=None):
    """LceBConv2d on the matrix cores: x_packed int32 [N,H,W,Cw], w_fp4 from
    mfma_weights(); kernel = (KH, KW) or an int.  Output as bconv2d."""
    return _mfma_conv(lib().lce_bconv2d_mfma, x_packed, False, w_fp4, c_in, c_out, kernel,
                      stride, padding, pad_value, clamp, out_type, multiplier, bias,
                      thresholds, flip, out)


def quantize_bconv2d_mfma(x, w_fp4, c_out: int, kernel, *, stride=1, padding: str = "same",
                          pad_value: str = "one", clamp: Optional[Tuple[int, int]] = None,
                          out_type: str = "float", multiplier=None, bias=None,
                          thresholds=None, flip=None, out=None):
    """LceQuantize + LceBConv2d on the matrix cores in one launch: x float32
    [N,H,W,C_in] (C_in a multiple of 32, 16-byte aligned), w_fp4 from
    mfma_weights().  The result equals bconv2d_mfma(bitpack(x), ...).  Shapes
    that neither the filter-stationary nor the K-split schedule takes raise
    LceError with status LCE_EUNSUPPORTED (nothing is launched); run bitpack and
    bconv2d_mfma."""
    return _mfma_conv(lib().lce_quantize_bconv2d_mfma, x, True, w_fp4, x.shape[-1], c_out,
                      kernel, stride, padding, pad_value, clamp, out_type, multiplier, bias,
                      thresholds, flip, out)


class PreparedBConv2dMfma:
    """A bconv2d_mfma call marshalled once (see PreparedBConv2d)."""

    def __init__(self, x_packed, w_fp4, c_in, c_out, kernel, out, *, stride=1, padding="same",
                 pad_value="one", clamp=None, out_type="float", multiplier=None, bias=None,
                 thresholds=None, flip=None):
        bconv2d_mfma(x_packed, w_fp4, c_in, c_out, kernel, stride=stride, padding=padding,
                     pad_value=pad_value, clamp=clamp, out_type=out_type,
                     multiplier=multiplier, bias=bias, thresholds=thresholds, flip=flip,
                     out=out)
        n, h, w, _ = x_packed.shape
        kh, kw = (kernel, kernel) if isinstance(kernel, int) else tuple(kernel)
        self.desc = make_desc(n, h, w, c_in, c_out, kh, kw, stride, padding, pad_value, clamp,
                              out_type)
        self._desc_ref = ctypes.byref(self.desc)
        ptr = lambda t: None if t is None else t.data_ptr()
        self.args = (x_packed.data_ptr(), w_fp4.data_ptr(), ptr(multiplier), ptr(bias),
                     ptr(thresholds), ptr(flip), out.data_ptr())
        self.keep = (x_packed, w_fp4, multiplier, bias, thresholds, flip, out)
        self._fn = lib().lce_bconv2d_mfma

    def __call__(self, stream=None):
        st = self._fn(self._desc_ref, *self.args, _current_stream() if stream is None else stream)
        if st != LCE_OK:
            raise LceError(st, last_error())


def _current_stream():
    global _raw
    if _raw is None:
        _raw = _raw_stream()
    import torch
    return _raw(torch.cuda.current_device())


class PreparedBConv2d:
    """A bconv2d call with its descriptor and pointers marshalled once.

    Calling it enqueues the convolution on `stream` (default: torch's current
    stream at call time, so it can be captured in a graph) with no Python-side
    validation; the C ABI still validates.  The tensors must outlive it.
    """

    def __init__(self, x_packed, w_packed, c_in, out, *, stride=1, padding="same",
                 pad_value="one", clamp=None, out_type="float", multiplier=None, bias=None,
                 thresholds=None, flip=None, pad_correction=None):
        # one eager call validates shapes/dtypes and fills `out`
        bconv2d(x_packed, w_packed, c_in, stride=stride, padding=padding, pad_value=pad_value,
                clamp=clamp, out_type=out_type, multiplier=multiplier, bias=bias,
                thresholds=thresholds, flip=flip, pad_correction=pad_correction, out=out)
        n, h, w, _ = x_packed.shape
        cout, kh, kw, _ = w_packed.shape
        self.desc = make_desc(n, h, w, c_in, cout, kh, kw, stride, padding, pad_value, clamp,
                              out_type)
        self._desc_ref = ctypes.byref(self.desc)
        ptr = lambda t: None if t is None else t.data_ptr()
        self.args = (x_packed.data_ptr(), w_packed.data_ptr(), ptr(multiplier), ptr(bias),
                     ptr(thresholds), ptr(flip), ptr(pad_correction), out.data_ptr())
        self.keep = (x_packed, w_packed, multiplier, bias, thresholds, flip, pad_correction, out)
        self._fn = lib().lce_bconv2d

    def __call__(self, stream=None):
        st = self._fn(self._desc_ref, *self.args, _current_stream() if stream is None else stream)
        if st != LCE_OK:
            raise LceError(st, last_error())


class PreparedQuantBConv2dMfma:
    """A quantize_bconv2d_mfma call marshalled once (see PreparedBConv2d)."""

    def __init__(self, x, w_fp4, c_out, kernel, out, *, stride=1, padding="same",
                 pad_value="one", clamp=None, out_type="float", multiplier=None, bias=None,
                 thresholds=None, flip=None):
        quantize_bconv2d_mfma(x, w_fp4, c_out, kernel, stride=stride, padding=padding,
                              pad_value=pad_value, clamp=clamp, out_type=out_type,
                              multiplier=multiplier, bias=bias, thresholds=thresholds,
                              flip=flip, out=out)
        n, h, w, c_in = x.shape
        kh, kw = (kernel, kernel) if isinstance(kernel, int) else tuple(kernel)
        self.desc = make_desc(n, h, w, c_in, c_out, kh, kw, stride, padding, pad_value, clamp,
                              out_type)
        self._desc_ref = ctypes.byref(self.desc)
        ptr = lambda t: None if t is None else t.data_ptr()
        self.args = (x.data_ptr(), w_fp4.data_ptr(), ptr(multiplier), ptr(bias),
                     ptr(thresholds), ptr(flip), out.data_ptr())
        self.keep = (x, w_fp4, multiplier, bias, thresholds, flip, out)
        self._fn = lib().lce_quantize_bconv2d_mfma

    def __call__(self, stream=None):
        st = self._fn(self._desc_ref, *self.args, _current_stream() if stream is None else stream)
        if st != LCE_OK:
            raise LceError(st, last_error())


class PreparedQuantBConv2d:
    """A quantize_bconv2d call marshalled once (see PreparedBConv2d)."""

    def __init__(self, x, w_packed, out, *, stride=1, padding="same", clamp=None,
                 out_type="float", multiplier=None, bias=None, thresholds=None, flip=None):
        quantize_bconv2d(x, w_packed, stride=stride, padding=padding, clamp=clamp,
                         out_type=out_type, multiplier=multiplier, bias=bias,
                         thresholds=thresholds, flip=flip, out=out)
        n, h, w, c_in = x.shape
        cout, kh, kw, _ = w_packed.shape
        self.desc = make_desc(n, h, w, c_in, cout, kh, kw, stride, padding, "one", clamp,
                              out_type)
        self._desc_ref = ctypes.byref(self.desc)
        ptr = lambda t: None if t is None else t.data_ptr()
        self.args = (x.data_ptr(), w_packed.data_ptr(), ptr(multiplier), ptr(bias),
                     ptr(thresholds), ptr(flip), out.data_ptr())
        self.keep = (x, w_packed, multiplier, bias, thresholds, flip, out)
        self._fn = lib().lce_quantize_bconv2d

    def __call__(self, stream=None):
        st = self._fn(self._desc_ref, *self.args, _current_stream() if stream is None else stream)
        if st != LCE_OK:
            raise LceError(st, last_error())


KV4_PAGE = 64
KV4_WORKSPACE_ZERO = 131072
FLOAT_TYPE = {"torch.float32": 0, "torch.float16": 1, "torch.bfloat16": 2}
_float_types = {}      # torch dtype -> lce_float_type, filled at first use


def _float_type(dtype, name):
    code = _float_types.get(dtype)
    if code is None:
        code = FLOAT_TYPE.get(str(dtype))
        if code is None:
            raise TypeError(f"{name} must be float32, float16 or bfloat16, got {dtype}")
        _float_types[dtype] = code
    return code


class _PagedCache:
    """What the caches share: a device buffer of pages, and the quick checks of calls."""

    def __init__(self, kv_heads: int, head_dim: int, pages: Optional[int] = None, *, data=None,
                 device="cuda"):
        import torch
        if (pages is None) == (data is None):
            raise ValueError("give either pages or data")
        record = self._record(head_dim)
        if data is not None:
            _require(data, torch.uint8, "data")
            if data.dim() != 3 or data.shape[1] != kv_heads or data.shape[2] != record:
                raise ValueError(f"data must be [pages, {kv_heads}, {record}], got "
                                 f"{list(data.shape)}")
            pages = data.shape[0]
        self.desc = self._Desc(pages, kv_heads, head_dim)
        n = ctypes.c_int64()
        _check(getattr(lib(), self._size)(ctypes.byref(self.desc), ctypes.byref(n)))
        if data is None:
            if torch.device(device).type != "cuda":
                raise ValueError(f"device must be a GPU, got {device}")
            data = torch.empty((pages, kv_heads, record), dtype=torch.uint8, device=device)
        self._data, self.pages, self.kv_heads, self.head_dim = data, pages, kv_heads, head_dim
        self._ref = ctypes.byref(self.desc)
        # what every call compares its tensors with
        self._index = data.get_device()
        self._int32, self._int64 = torch.int32, torch.int64
        self._uint8, self._float32, self._bfloat16 = torch.uint8, torch.float32, torch.bfloat16
        self._types = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
        self._scale = head_dim ** -0.5
        self._empty, self._empty_like, self._device = torch.empty, torch.empty_like, data.device
        self._contiguous = torch.contiguous_format

    @property
    def data(self):
        """The buffer, uint8 [pages, kv_heads, bytes of a record]."""
        return self._data

    def _holds(self, t, dtype) -> bool:
        """Whether t is a contiguous `dtype` tensor on the cache's device: the quick
        check; _require_like says what is wrong."""
        return (t.dtype is dtype and t.get_device() == self._index and t.is_contiguous())


_current_device = None


def _launch(index, fn, *args) -> None:
    """Calls the library with device `index` current: a default stream is its device's by
    that alone."""
    global _current_device
    if _current_device is None:
        import torch
        _current_device = lambda: torch.cuda.current_device()
    if _current_device() == index:
        st = fn(*args)
    else:
        import torch
        with torch.cuda.device(index):
            st = fn(*args)
    if st != LCE_OK:
        raise LceError(st, last_error())


class KV4Cache(_PagedCache):
    """A 4-bit key/value cache: pages of 64 tokens in one device buffer.

    KV4Cache(kv_heads, head_dim, pages=n) allocates uint8 [n, kv_heads,
    76*head_dim] on `device`; data=t takes an existing buffer of that kind.
    Tokens are addressed by slot = page*64 + place; which pages make up a
    sequence is the caller's table.  head_dim is 64, 128 or 256."""

    _Desc, _size = KV4CacheDesc, "lce_kv4_cache_size"

    @staticmethod
    def _record(head_dim):
        return 76 * head_dim


class KV8Cache(_PagedCache):
    """An 8-bit key/value cache: pages of 64 tokens in one device buffer.

    KV8Cache(kv_heads, head_dim, pages=n) allocates uint8 [n, kv_heads,
    128*head_dim + 128] on `device`; data=t takes an existing buffer of that kind.
    Which pages make up a sequence is the caller's table; its token j is in slot
    table[j//64]*64 + j%64.  head_dim is 64, 128 or 256."""

    _Desc, _size = KV8CacheDesc, "lce_kv8_cache_size"

    @staticmethod
    def _record(head_dim):
        return 128 * head_dim + 128


def _require_like(t, dtype, device, name):
    """An index tensor of a call on `device`."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _require_cache(cache, kind=KV4Cache):
    if not isinstance(cache, kind):
        raise TypeError(f"cache must be a {kind.__name__}")


def _require_heads(t, cache, name):
    """A [tokens, heads, head_dim] float tensor with contiguous channels."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != cache.data.device:
        raise ValueError(f"{name} must be on {cache.data.device}, got {t.device}")
    if t.dim() != 3 or t.shape[2] != cache.head_dim:
        raise ValueError(f"{name} must be [tokens, heads, {cache.head_dim}], got {list(t.shape)}")
    if t.stride(2) != 1 and t.numel():
        raise ValueError(f"{name}'s channels must be contiguous")


def _append_refused(cache, k, v, slots):
    """Raises for what kv4_append does not take."""
    import torch
    _require_cache(cache)
    _require_heads(k, cache, "k")
    _require_heads(v, cache, "v")
    if k.shape != v.shape or k.shape[1] != cache.kv_heads:
        raise ValueError(f"k and v must be [tokens, {cache.kv_heads}, {cache.head_dim}], got "
                         f"{list(k.shape)} and {list(v.shape)}")
    if k.dtype != v.dtype:
        raise TypeError(f"k and v must have one dtype, got {k.dtype} and {v.dtype}")
    _float_type(k.dtype, "k")
    _require_like(slots, torch.int64, cache.data.device, "slots")
    if slots.shape != k.shape[:1]:
        raise ValueError(f"slots must have {k.shape[0]} elements")


def kv4_append(cache: KV4Cache, k, v, slots) -> None:
    """Quantize k and v [tokens, kv_heads, head_dim] (float32, float16 or bfloat16; any
    token and head strides that are multiples of 16 bytes) into the cache's `slots`
    (int64 [tokens]; a slot outside the cache drops its token)."""
    try:
        n, heads, dim = k.shape
        ks, vs = k.stride(), v.stride()
        dtype = k.dtype
        code = cache._types.get(dtype, -1)
        fine = (code >= 0 and heads == cache.kv_heads and dim == cache.head_dim
                and v.shape == k.shape and v.dtype is dtype
                and ks[2] == vs[2] == 1 and k.get_device() == v.get_device() == cache._index
                and cache._holds(slots, cache._int64) and slots.shape == (n,))
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        _append_refused(cache, k, v, slots)
    st = lib().lce_kv4_append(cache._ref, cache._data.data_ptr(), code, k.data_ptr(), ks[0], ks[1],
                              v.data_ptr(), vs[0], vs[1], slots.data_ptr(), n, _stream_handle(k))
    if st != LCE_OK:
        raise LceError(st, last_error())


def kv4_read(cache: KV4Cache, slots, *, dtype=None, out=None):
    """The values that the cache holds for `slots` (int64 [tokens]): a pair k, v
    [tokens, kv_heads, head_dim] of `dtype` (default bfloat16), or into the pair
    `out`.  Slots outside the cache read as zeros."""
    import torch
    _require_cache(cache)
    if not isinstance(slots, torch.Tensor) or not cache._holds(slots, torch.int64):
        _require_like(slots, torch.int64, cache.data.device, "slots")
    if slots.dim() != 1:
        raise ValueError("slots must have one dimension")
    n = slots.shape[0]
    if out is None:
        if dtype is None:
            dtype = torch.bfloat16
        code = _float_type(dtype, "dtype")
        k = torch.empty((n, cache.kv_heads, cache.head_dim), dtype=dtype, device=cache._device)
        v = torch.empty_like(k)
    else:
        k, v = out
        shape = (n, cache.kv_heads, cache.head_dim)
        for t, name in ((k, "out[0]"), (v, "out[1]")):
            _require_like(t, k.dtype if dtype is None else dtype, slots.device, name)
            if t.shape != shape:
                raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
        code = _float_type(k.dtype, "out")
    st = lib().lce_kv4_read(cache._ref, cache._data.data_ptr(), slots.data_ptr(), n, code, k.data_ptr(),
                            v.data_ptr(), _stream_handle(slots))
    if st != LCE_OK:
        raise LceError(st, last_error())
    return k, v


def _int32_refused(**sizes):
    """Raises for a size that an int32 of the C ABI would hold as another one."""
    for name, value in sizes.items():
        if not INT32_MIN <= value <= INT32_MAX:
            raise ValueError(f"{name} must be an int32, got {value}")


def _query_refused(cache, q, table, q_start, lengths):
    """Raises for what attention and selection do not take."""
    import torch
    _require_cache(cache)
    _require_heads(q, cache, "q")
    device = cache.data.device
    _require_like(table, torch.int32, device, "table")
    if table.dim() != 2:
        raise ValueError("table must be [sequences, pages]")
    for t, name, n in ((q_start, "q_start", table.shape[0] + 1),
                       (lengths, "lengths", table.shape[0])):
        _require_like(t, torch.int32, device, name)
        if t.shape != (n,):
            raise ValueError(f"{name} must have {n} elements, got {list(t.shape)}")
    if q.dtype == torch.float32:
        raise TypeError("q must be float16 or bfloat16, got torch.float32")
    _float_type(q.dtype, "q")


def _kv4_query(cache, q, table, q_start, lengths, causal, window, count, max_q, max_len, scale):
    """Checks the arguments that attention and selection share; their descriptor."""
    try:
        tokens, heads, dim = q.shape
        seqs, width = table.shape
        strides = q.stride()
        code = cache._types.get(q.dtype, 0)
        i32 = cache._int32
        fine = (code > 0 and dim == cache.head_dim and strides[2] == 1
                and table.dtype is q_start.dtype is lengths.dtype is i32
                and q.get_device() == table.get_device() == q_start.get_device()
                == lengths.get_device() == cache._index
                and table.is_contiguous() and q_start.is_contiguous() and lengths.is_contiguous()
                and q_start.shape == (seqs + 1,) and lengths.shape == (seqs,))
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        _query_refused(cache, q, table, q_start, lengths)
    max_q, max_len = max_q or 0, max_len or 0
    if (tokens | heads | seqs | width | window | count | max_q | max_len) >> 31:
        _int32_refused(tokens=tokens, heads=heads, sequences=seqs, table=width, window=window,
                       count=count, max_q=max_q, max_len=max_len)
    return KV4QueryDesc(tokens, heads, seqs, width, code, 1 if causal else 0, window, count,
                        max_q, max_len, scale, strides[0], strides[1])


def kv4_workspace(cache: KV4Cache, q, table, *, only: Optional[str] = None):
    """Workspace (uint8, zeroed) for kv4_attention and kv4_select calls with q's and
    table's shapes, or with fewer tokens; only="attention" or "select": for calls of that
    kind.  At most 69 MB for attention; for selection 2 bytes for each token, cache head
    and page of the table.  Calls that may overlap need one each."""
    import torch
    _require_cache(cache)
    _require_heads(q, cache, "q")
    _require_like(table, torch.int32, cache.data.device, "table")
    if table.dim() != 2:
        raise ValueError("table must be [sequences, pages]")
    if only not in (None, "attention", "select"):
        raise ValueError(f"only must be 'attention', 'select' or None, got {only!r}")
    _int32_refused(tokens=q.shape[0], heads=q.shape[1], sequences=table.shape[0],
                   table=table.shape[1])
    d = KV4QueryDesc(q.shape[0], q.shape[1], table.shape[0], table.shape[1])
    n = ctypes.c_int64()
    size = getattr(lib(), f"lce_kv4_{only}_workspace_size" if only else "lce_kv4_workspace_size")
    _check(size(cache._ref, ctypes.byref(d), ctypes.byref(n)))
    ws = torch.empty(n.value, dtype=torch.uint8, device=cache.data.device)
    ws[:KV4_WORKSPACE_ZERO].zero_()
    return ws


def _workspace(workspace, cache, q, table, only):
    import torch
    if workspace is None:
        return kv4_workspace(cache, q, table, only=only)
    _require_like(workspace, torch.uint8, cache.data.device, "workspace")
    return workspace


def kv4_attention(cache: KV4Cache, q, table, q_start, lengths, *, scale: Optional[float] = None,
                  causal: bool = True, window: int = 0, pages=None, max_q: Optional[int] = None,
                  max_len: Optional[int] = None, out=None, return_lse: bool = False,
                  workspace=None):
    """Attention of new tokens over cached sequences (lce_kv4_attention).

    q [tokens, q_heads, head_dim], float16 or bfloat16: the tokens of sequence b are rows
    q_start[b]:q_start[b+1] and stand at its end; table int32 [seqs, pages], lengths int32
    [seqs] (cached tokens, the new ones included).  window > 0 hides tokens further back;
    pages int32 [tokens, kv_heads, n] restricts every token and cache head to the pages
    listed (negative: none).  max_q and max_len, the most new tokens and the longest
    length, help to split the work.  Returns out, or (out, lse float32 [tokens, q_heads]).
    """
    count = 0 if pages is None else _list_length(cache, q, pages)
    d = _kv4_query(cache, q, table, q_start, lengths, causal, window, count, max_q, max_len,
                   cache._scale if scale is None else scale)
    if out is None:
        out = cache._empty_like(q) if q.is_contiguous() else q.new_empty(q.shape)
    else:
        _require_like(out, q.dtype, q.device, "out")
        if out.shape != q.shape:
            raise ValueError(f"out must be {list(q.shape)}, got {list(out.shape)}")
    lse = (cache._empty(q.shape[:2], dtype=cache._float32, device=cache._device) if return_lse
           else None)
    if workspace is None or not cache._holds(workspace, cache._uint8):
        workspace = _workspace(workspace, cache, q, table, "attention")
    st = lib().lce_kv4_attention(
        cache._ref, cache._data.data_ptr(), ctypes.byref(d), q.data_ptr(), table.data_ptr(),
        q_start.data_ptr(), lengths.data_ptr(), None if pages is None else pages.data_ptr(),
        out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(),
        workspace.numel(), _stream_handle(q))
    if st != LCE_OK:
        raise LceError(st, last_error())
    return (out, lse) if return_lse else out


def _list_length(cache, q, pages):
    import torch
    _require_cache(cache)
    _require_heads(q, cache, "q")
    _require_like(pages, torch.int32, cache.data.device, "pages")
    if pages.dim() != 3 or pages.shape[:2] != (q.shape[0], cache.kv_heads) or not pages.shape[2]:
        raise ValueError(f"pages must be [{q.shape[0]}, {cache.kv_heads}, n], got "
                         f"{list(pages.shape)}")
    return pages.shape[2]


def kv4_select(cache: KV4Cache, q, table, q_start, lengths, count: int, *, keep_first: int = 1,
               keep_last: int = 1, causal: bool = True, window: int = 0,
               max_len: Optional[int] = None, out=None, workspace=None):
    """The `count` pages of each token and cache head whose key signs agree best with the
    query signs (lce_kv4_select): int32 [tokens, kv_heads, count], ascending, then -1.
    The first keep_first and the last keep_last pages are always among them."""
    if (keep_first | keep_last) >> 31:
        _int32_refused(keep_first=keep_first, keep_last=keep_last)
    d = _kv4_query(cache, q, table, q_start, lengths, causal, window, count, None, max_len, 1.0)
    shape = (q.shape[0], cache.kv_heads, count)
    if out is None:
        out = table.new_empty(shape)
    else:
        _require_like(out, table.dtype, q.device, "out")
        if out.shape != shape:
            raise ValueError(f"out must be {list(shape)}, got {list(out.shape)}")
    if workspace is None or not cache._holds(workspace, cache._uint8):
        workspace = _workspace(workspace, cache, q, table, "select")
    st = lib().lce_kv4_select(
        cache._ref, cache._data.data_ptr(), ctypes.byref(d), q.data_ptr(), table.data_ptr(),
        q_start.data_ptr(), lengths.data_ptr(), keep_first, keep_last, out.data_ptr(),
        workspace.data_ptr(), workspace.numel(), _stream_handle(q))
    if st != LCE_OK:
        raise LceError(st, last_error())
    return out


KV8_PAGE = 64
KV8_BLOCK = 16
KV8_WORKSPACE_ZERO = 131072
# lce_kv8_query_desc, lce_rotary_desc and lce_rotary_rows as bytes: packing them takes a
# third of the time that filling the ctypes structures does.
_pack_kv8_query = struct.Struct("@9i2f2q").pack
_pack_rotary = struct.Struct("@6if").pack
_pack_rotary_rows = struct.Struct("@i2P4q").pack


def _require_sequences(cache, table, q_start, lengths):
    """The index tensors of a call over sequences."""
    import torch
    device = cache.data.device
    _require_like(table, torch.int32, device, "table")
    if table.dim() != 2:
        raise ValueError("table must be [sequences, pages]")
    for t, name, n in ((q_start, "q_start", table.shape[0] + 1),
                       (lengths, "lengths", table.shape[0])):
        _require_like(t, torch.int32, device, name)
        if t.shape != (n,):
            raise ValueError(f"{name} must have {n} elements, got {list(t.shape)}")


def _kv8_append_refused(cache, k, v, table, q_start, lengths):
    """Raises for what kv8_append does not take."""
    _require_cache(cache, KV8Cache)
    _require_heads(k, cache, "k")
    _require_heads(v, cache, "v")
    if k.shape != v.shape or k.shape[1] != cache.kv_heads:
        raise ValueError(f"k and v must be [tokens, {cache.kv_heads}, {cache.head_dim}], got "
                         f"{list(k.shape)} and {list(v.shape)}")
    if k.dtype != v.dtype:
        raise TypeError(f"k and v must have one dtype, got {k.dtype} and {v.dtype}")
    _float_type(k.dtype, "k")
    _require_sequences(cache, table, q_start, lengths)


def kv8_append(cache: KV8Cache, k, v, table, q_start, lengths) -> None:
    """Quantize the last tokens of sequences into the cache (lce_kv8_append).

    k and v [tokens, kv_heads, head_dim], float32, float16 or bfloat16, any token and head
    strides that are multiples of 16 bytes: those of sequence b are rows
    q_start[b]:q_start[b+1] and become its last tokens; table int32 [seqs, pages], lengths
    int32 [seqs] (the new tokens included).  No two sequences may append to one block of
    16 tokens."""
    try:
        n, heads, dim = k.shape
        seqs, width = table.shape
        ks, vs = k.stride(), v.stride()
        dtype = k.dtype
        code = cache._types.get(dtype, -1)
        fine = (type(cache) is KV8Cache and code >= 0 and heads == cache.kv_heads
                and dim == cache.head_dim and v.shape == k.shape and v.dtype is dtype
                and ks[2] == vs[2] == 1 and k.get_device() == v.get_device() == cache._index
                and cache._holds(table, cache._int32) and cache._holds(q_start, cache._int32)
                and cache._holds(lengths, cache._int32) and q_start.shape == (seqs + 1,)
                and lengths.shape == (seqs,))
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        _kv8_append_refused(cache, k, v, table, q_start, lengths)
        n, code, (seqs, width), ks, vs = (k.shape[0], _float_type(k.dtype, "k"), table.shape,
                                          k.stride(), v.stride())
    if (n | seqs | width) >> 31:
        _int32_refused(tokens=n, sequences=seqs, table=width)
    _launch(cache._index, lib().lce_kv8_append, cache._ref, cache._data.data_ptr(), code,
            k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], n, seqs, width,
            table.data_ptr(), q_start.data_ptr(), lengths.data_ptr(), _stream_of(cache._index))


def kv8_read(cache: KV8Cache, slots, *, dtype=None, out=None):
    """The values that the cache holds for `slots` (int64 [tokens]): a pair k, v
    [tokens, kv_heads, head_dim] of `dtype` (default bfloat16), or into the pair
    `out`.  Slots outside the cache read as zeros."""
    try:
        n, = slots.shape
        fine = type(cache) is KV8Cache and cache._holds(slots, cache._int64)
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        _require_cache(cache, KV8Cache)
        _require_like(slots, cache._int64, cache.data.device, "slots")
        if slots.dim() != 1:
            raise ValueError("slots must have one dimension")
        n, = slots.shape
    shape = (n, cache.kv_heads, cache.head_dim)
    if out is None:
        if dtype is None:
            dtype = cache._bfloat16
        code = cache._types.get(dtype)
        if code is None:
            code = _float_type(dtype, "dtype")
        k = cache._data.new_empty(shape, dtype=dtype)
        v = cache._empty_like(k)
    else:
        k, v = out
        if dtype is None:
            dtype = getattr(k, "dtype", cache._bfloat16)
        for t, name in ((k, "out[0]"), (v, "out[1]")):
            _require_like(t, dtype, slots.device, name)
            if t.shape != shape:
                raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
        if k.numel() and k.data_ptr() == v.data_ptr():
            raise ValueError("out must be two tensors")
        code = _float_type(dtype, "out")
    _launch(cache._index, lib().lce_kv8_read, cache._ref, cache._data.data_ptr(),
            slots.data_ptr(), n, code, k.data_ptr(), v.data_ptr(), _stream_of(cache._index))
    return k, v


def kv8_workspace(cache: KV8Cache, q, table):
    """Workspace (uint8, zeroed) for kv8_attention calls with q's and table's shapes, or
    with fewer tokens: at most 69 MB.  Calls that may overlap need one each."""
    import torch
    _require_cache(cache, KV8Cache)
    _require_heads(q, cache, "q")
    _require_like(table, torch.int32, cache.data.device, "table")
    if table.dim() != 2:
        raise ValueError("table must be [sequences, pages]")
    _int32_refused(tokens=q.shape[0], heads=q.shape[1], sequences=table.shape[0],
                   table=table.shape[1])
    d = KV8QueryDesc(q.shape[0], q.shape[1], table.shape[0], table.shape[1])
    n = ctypes.c_int64()
    _check(lib().lce_kv8_workspace_size(cache._ref, ctypes.byref(d), ctypes.byref(n)))
    ws = torch.empty(n.value, dtype=torch.uint8, device=cache.data.device)
    ws[:KV8_WORKSPACE_ZERO].zero_()
    return ws


def _kv8_attention_refused(cache, q, table, q_start, lengths, slopes, prefix):
    """Raises for what kv8_attention does not take."""
    import torch
    _require_cache(cache, KV8Cache)
    _require_heads(q, cache, "q")
    _require_sequences(cache, table, q_start, lengths)
    if q.dtype == torch.float32:
        raise TypeError("q must be float16 or bfloat16, got torch.float32")
    _float_type(q.dtype, "q")
    for t, name, dtype, n in ((slopes, "slopes", torch.float32, q.shape[1]),
                              (prefix, "prefix", torch.int32, table.shape[0])):
        if t is not None:
            _require_like(t, dtype, cache.data.device, name)
            if t.shape != (n,):
                raise ValueError(f"{name} must have {n} elements, got {list(t.shape)}")


def kv8_attention(cache: KV8Cache, q, table, q_start, lengths, *, scale: Optional[float] = None,
                  causal: bool = True, window: int = 0, softcap: float = 0.0, slopes=None,
                  prefix=None, max_q: Optional[int] = None, max_len: Optional[int] = None,
                  out=None, return_lse: bool = False, workspace=None):
    """Attention of new tokens over cached sequences (lce_kv8_attention).

    q [tokens, q_heads, head_dim], float16 or bfloat16: the tokens of sequence b are rows
    q_start[b]:q_start[b+1] and stand at its end; table int32 [seqs, pages], lengths int32
    [seqs] (cached tokens, the new ones included).  window > 0 hides tokens further back;
    softcap > 0 caps scores at softcap*tanh(score/softcap); slopes float32 [q_heads] takes
    slope times the distance off them; prefix int32 [seqs] is the number of a sequence's
    first tokens that all its rows see (causal).  max_q and max_len, the most new tokens
    and the longest length, help to split the work.  Returns out, or (out, lse float32
    [tokens, q_heads]); autograd does not follow them."""
    try:
        tokens, heads, dim = q.shape
        seqs, width = table.shape
        strides = q.stride()
        code = cache._types.get(q.dtype, 0)
        i32 = cache._int32
        fine = (type(cache) is KV8Cache and code > 0 and dim == cache.head_dim and strides[2] == 1
                and table.dtype is q_start.dtype is lengths.dtype is i32
                and q.get_device() == table.get_device() == q_start.get_device()
                == lengths.get_device() == cache._index
                and table.is_contiguous() and q_start.is_contiguous() and lengths.is_contiguous()
                and q_start.shape == (seqs + 1,) and lengths.shape == (seqs,)
                and (slopes is None or cache._holds(slopes, cache._float32)
                     and slopes.shape == (heads,))
                and (prefix is None or cache._holds(prefix, i32) and prefix.shape == (seqs,)))
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        _kv8_attention_refused(cache, q, table, q_start, lengths, slopes, prefix)
        (tokens, heads, _), (seqs, width), strides = q.shape, table.shape, q.stride()
        code = _float_type(q.dtype, "q")
    max_q, max_len = max_q or 0, max_len or 0
    if (tokens | heads | seqs | width | window | max_q | max_len) >> 31:
        _int32_refused(tokens=tokens, heads=heads, sequences=seqs, table=width, window=window,
                       max_q=max_q, max_len=max_len)
    try:
        d = _pack_kv8_query(tokens, heads, seqs, width, code, 1 if causal else 0, window, max_q,
                            max_len, cache._scale if scale is None else scale, softcap, strides[0],
                            strides[1])
    except OverflowError:
        raise ValueError(f"scale {scale} or softcap {softcap} is past float32's range") from None
    except struct.error as e:
        raise TypeError(f"scale {scale!r}, softcap {softcap!r}, window {window!r}, max_q "
                        f"{max_q!r} and max_len {max_len!r} must be numbers ({e})") from None
    if out is None:
        out = cache._empty_like(q, memory_format=cache._contiguous)
    else:
        _require_like(out, q.dtype, q.device, "out")
        if out.shape != q.shape:
            raise ValueError(f"out must be {list(q.shape)}, got {list(out.shape)}")
    lse = q.new_empty((tokens, heads), dtype=cache._float32) if return_lse else None
    if workspace is None:
        workspace = kv8_workspace(cache, q, table)
    elif not cache._holds(workspace, cache._uint8):
        _require_like(workspace, cache._uint8, cache.data.device, "workspace")
    _launch(cache._index, lib().lce_kv8_attention, cache._ref, cache._data.data_ptr(), d,
            q.data_ptr(), table.data_ptr(), q_start.data_ptr(),
            lengths.data_ptr(), None if slopes is None else slopes.data_ptr(),
            None if prefix is None else prefix.data_ptr(), out.data_ptr(),
            None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.numel(),
            _stream_of(cache._index))
    return (out, lse) if return_lse else out


ROTARY_SCALING = {None: 0, "linear": 1, "ntk": 2, "yarn": 3}


class Rotary:
    """Frequencies of rotary positions, for rotary().

    The first rot_dim channels (default: all) of heads of head_dim are turned, in pairs
    (i, i + rot_dim/2) or, interleaved, (2i, 2i + 1), pair i by base**(-2i/rot_dim) radians a
    position.  scaling, for contexts `factor` times as long as trained: "linear", "ntk" or
    "yarn" (trained on `original` positions); see lce_rotary_frequencies.  freqs (float64
    [rot_dim/2], host) gives frequencies instead, and scale what results are multiplied
    by."""

    def __init__(self, head_dim: int, *, rot_dim: Optional[int] = None, base: float = 10000.0,
                 interleaved: bool = False, scaling: Optional[str] = None, factor: float = 1.0,
                 original: int = 4096, freqs=None, scale: Optional[float] = None, device="cuda"):
        import torch
        rot_dim = head_dim if rot_dim is None else rot_dim
        _int32_refused(head_dim=head_dim, rot_dim=rot_dim)
        if not 2 <= head_dim <= 65536:
            raise ValueError(f"head_dim must be in [2, 65536], got {head_dim}")
        if rot_dim < 2 or rot_dim % 2 or rot_dim > head_dim:
            raise ValueError(f"rot_dim must be an even number in [2, {head_dim}], got {rot_dim}")
        if scaling not in ROTARY_SCALING:
            raise ValueError(f"scaling must be one of {list(ROTARY_SCALING)}, got {scaling!r}")
        n = rot_dim // 2
        values, factor_out = (ctypes.c_double * n)(), ctypes.c_float(1.0)
        if freqs is None:
            _check(lib().lce_rotary_frequencies(rot_dim, base, ROTARY_SCALING[scaling], factor,
                                                original, values, ctypes.byref(factor_out)))
        else:
            if scaling is not None:
                raise ValueError("give either freqs or scaling")
            freqs = torch.as_tensor(freqs, dtype=torch.float64, device="cpu")
            if freqs.shape != (n,):
                raise ValueError(f"freqs must have {n} elements, got {list(freqs.shape)}")
            values[:] = freqs.tolist()
        turns = (ctypes.c_uint64 * n)()
        _check(lib().lce_rotary_turns(values, n, turns))
        self.head_dim, self.rot_dim, self.interleaved = head_dim, rot_dim, bool(interleaved)
        self.scale = factor_out.value if scale is None else ctypes.c_float(scale).value
        if not math.isfinite(self.scale):
            raise ValueError(f"scale {scale} is not a finite float32")
        self.freqs = torch.tensor(list(values), dtype=torch.float64)
        if torch.device(device).type != "cuda":
            raise ValueError(f"device must be a GPU, got {device}")
        # (as int64: the same bits)
        self._turns = torch.tensor([t - (1 << 64) if t >> 63 else t for t in turns],
                                   dtype=torch.int64).to(device)
        self._index, self._turns_ptr = self._turns.get_device(), self._turns.data_ptr()
        self._interleaved = int(self.interleaved)
        # what every call compares its tensors with
        self._int64, self._empty_like = torch.int64, torch.empty_like
        self._is_grad_enabled = torch.is_grad_enabled
        self._types = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _rotary_refused(plan, positions, q, k):
    """Raises for what rotary does not take."""
    import torch
    if not isinstance(plan, Rotary):
        raise TypeError("plan must be a Rotary")
    device = plan._turns.device
    for t, name in ((q, "q"), (k, "k")):
        if t is None and name == "k":
            continue
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")
        if t.device != device:
            raise ValueError(f"{name} must be on {device}, got {t.device}")
        _float_type(t.dtype, name)
        if t.dtype != q.dtype:
            raise TypeError(f"q and k must have one dtype, got {q.dtype} and {t.dtype}")
        if t.dim() != 3 or t.shape[0] != q.shape[0] or t.shape[2] != plan.head_dim:
            raise ValueError(f"{name} must be [{q.shape[0]}, heads, {plan.head_dim}], got "
                             f"{list(t.shape)}")
        if t.stride(2) != 1 and t.numel():
            raise ValueError(f"{name}'s channels must be contiguous")
    _require_like(positions, torch.int64, device, "positions")
    if positions.shape != q.shape[:1]:
        raise ValueError(f"positions must have {q.shape[0]} elements, got {list(positions.shape)}")


def _rotary_out(t, out, name):
    """Checks a tensor that rotary writes t's result to."""
    import torch
    if not isinstance(out, torch.Tensor):
        raise TypeError(f"out of {name} must be a torch.Tensor")
    if (out.shape, out.dtype, out.device) != (t.shape, t.dtype, t.device):
        raise ValueError(f"out of {name} must be like it: {list(t.shape)} {t.dtype} on {t.device}, "
                         f"got {list(out.shape)} {out.dtype} on {out.device}")
    if out.stride(2) != 1 and out.numel():
        raise ValueError(f"out of {name}: channels must be contiguous")
    return out


_recorded_rotary = None


def _rotary_recorded(plan, positions, q, k, backward, out):
    """rotary() of tensors that autograd follows: the gradients of a turn are the turn back."""
    global _recorded_rotary
    import torch
    if out is not None:
        raise ValueError("out does not go with tensors that require a gradient: leave it away, or "
                         "call under torch.no_grad()")
    # (a captured backward pass beside an eager one of the same leaves can end the process)
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("rotary of tensors that require a gradient is not captured: call it "
                           "under torch.no_grad(), and with backward=True for gradients")
    if _recorded_rotary is None:
        class Recorded(torch.autograd.Function):
            @staticmethod
            def forward(ctx, plan, backward, positions, q, k):
                ctx.plan, ctx.turned_back = plan, backward
                ctx.save_for_backward(positions)
                ctx.set_materialize_grads(False)
                return rotary(plan, positions, q, k, backward=backward)

            @staticmethod
            def backward(ctx, *grads):
                positions, = ctx.saved_tensors
                # (sums' gradients are views of one number)
                there = [i for i, g in enumerate(grads) if g is not None and ctx.needs_input_grad[3 + i]]
                xs = [grads[i] if grads[i].stride(2) == 1 else grads[i].contiguous() for i in there]
                out = [None, None]
                if xs:
                    ys = rotary(ctx.plan, positions, *xs, backward=not ctx.turned_back)
                    for i, y in zip(there, ys if len(xs) == 2 else (ys,)):
                        out[i] = y
                return (None, None, None, *out)

        _recorded_rotary = Recorded
    return _recorded_rotary.apply(plan, bool(backward), positions, q, k)


def rotary(plan: Rotary, positions, q, k=None, *, backward: bool = False, out=None):
    """q [tokens, q_heads, head_dim], and k [tokens, kv_heads, head_dim] unless it is None,
    turned to `positions` (int64 [tokens]) in one launch (lce_rotary): float32, float16 or
    bfloat16, any token and head strides.  backward: q and k are gradients of what was
    turned, and get turned back (and scaled) to those of what went in.  Returns new
    tensors, or writes `out` (q's, or a pair), which may be q and k themselves.  Autograd
    follows q and k where they require a gradient and there is no `out` (which is then
    refused, as is a call that is being captured into a graph)."""
    try:
        n, heads, dim = q.shape
        x = q.stride()
        code = plan._types.get(q.dtype, -1)
        fine = (type(plan) is Rotary and code >= 0 and dim == plan.head_dim and x[2] == 1
                and q.get_device() == positions.get_device() == plan._index
                and positions.dtype is plan._int64 and positions.shape == (n,)
                and positions.is_contiguous())
        if k is not None:
            shape, y = k.shape, k.stride()
            fine = (fine and len(shape) == 3 and shape[0] == n and shape[2] == dim and y[2] == 1
                    and k.dtype is q.dtype and k.get_device() == plan._index)
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        _rotary_refused(plan, positions, q, k)
        n, heads, dim, x, code = *q.shape, q.stride(), _float_type(q.dtype, "q")
        if k is not None:
            shape, y = k.shape, k.stride()
    if (n | heads) >> 31 or k is not None and shape[1] >> 31:
        _int32_refused(tokens=n, heads=heads if k is None else max(heads, shape[1]))
    if (q.requires_grad or k is not None and k.requires_grad) and plan._is_grad_enabled():
        return _rotary_recorded(plan, positions, q, k, backward, out)
    if out is None:
        first = plan._empty_like(q)
        second = None if k is None else plan._empty_like(k)
    elif k is None:
        first = _rotary_out(q, out, "q")
    else:
        if len(out) != 2:
            raise ValueError("out must be a pair of tensors")
        first, second = _rotary_out(q, out[0], "q"), _rotary_out(k, out[1], "k")
    to = first.stride()
    if to[2] != 1 and out is None:          # like a q whose channels are not next to each other
        first = q.new_empty(q.shape)
        to = first.stride()
    qr = _pack_rotary_rows(heads, q.data_ptr(), first.data_ptr(), x[0], x[1], to[0], to[1])
    kr = None
    if k is not None:
        to = second.stride()
        if to[2] != 1 and out is None:
            second = k.new_empty(k.shape)
            to = second.stride()
        kr = _pack_rotary_rows(shape[1], k.data_ptr(), second.data_ptr(), y[0], y[1], to[0], to[1])
    _launch(plan._index, lib().lce_rotary,
            _pack_rotary(n, dim, plan.rot_dim, code, plan._interleaved, 1 if backward else 0,
                         plan.scale),
            plan._turns_ptr, positions.data_ptr(), qr, kr, _stream_of(plan._index))
    return first if k is None else (first, second)


class PreparedBitpack:
    """A bitpack call marshalled once (see PreparedBConv2d)."""

    def __init__(self, x, out):
        bitpack(x, out=out)
        c = x.shape[-1]
        self.args = (x.data_ptr(), out.data_ptr(), x.numel() // c, c)
        self.keep = (x, out)
        self._fn = lib().lce_bitpack

    def __call__(self, stream=None):
        st = self._fn(*self.args, _current_stream() if stream is None else stream)
        if st != LCE_OK:
            raise LceError(st, last_error())
