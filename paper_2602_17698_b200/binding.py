"""Thin ctypes binding of the C-ABI library (`include/scalebits.h`), same names.

Argument marshalling only: tensors are torch CUDA tensors (device memory and streams are
torch's job), every step runs in the library's kernels.  There is no CPU path: loading
fails loudly when `libscalebits.so` has not been built.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# SCALEBITS_LIB selects another build of the same library (the bounds-checked one, for tests)
LIB_PATH = os.environ.get("SCALEBITS_LIB") or os.path.join(_PKG, "libscalebits.so")

SB_OK, SB_ERR_INVALID, SB_ERR_SHAPE, SB_ERR_BUDGET, SB_ERR_SCRATCH, SB_ERR_CUDA, \
    SB_ERR_NOCONVERGE, SB_ERR_NONFINITE, SB_ERR_TIMEOUT = range(9)
SB_ALLOC_SCALEBITS, SB_ALLOC_GREEDY = 0, 1
SB_ACC_ROW, SB_ACC_COL = 1, 2
SB_FP4_MX, SB_FP4_NV = 0, 1
SB_KV_INT8, SB_KV_E4M3 = 0, 1
SB_KV8_BLOCK = 16
FP4_FORMATS = {"mx": SB_FP4_MX, "nv": SB_FP4_NV}
# a module's attribute is looked up at every use, which the calls of a decode step notice
_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8

EXPORTS = ["sb_create", "sb_destroy", "sb_sync", "sb_last_error", "sb_kernel_launches", "sb_debug_lookback",
           "sb_checked_build",
           "sb_calib_moments", "sb_reorder_channels", "sb_fold_segment_scores",
           "sb_expand_segment_perm", "sb_sum_scores", "sb_permute_matrix", "sb_block_scores", "sb_allocate_bits", "sb_allocate_bits_async",
           "sb_pack_blocks",
           "sb_calib_moments_noalloc", "sb_first_order_scores", "sb_exchange_step",
           "sb_reorder_channels_first_order", "sb_calib_gram",
           "sb_block_scores_full", "sb_dequant_gemm",
           "sb_fp4_code_bytes", "sb_fp4_scale_bytes", "sb_fp4_quantize", "sb_fp4_dequantize", "sb_fp4_gemm",
           "sb_kv8_append", "sb_kv8_read", "sb_kv8_attention",
           "sb_kv4_append", "sb_kv4_read", "sb_kv4_attention", "sb_rotary", "sb_lora_add"]


class SbError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"scalebits status {status}: {msg}")
        self.status = status


class AllocReport(C.Structure):
    _fields_ = [("cap_bits", C.c_int64), ("used_bits", C.c_int64),
                ("iterations", C.c_int32), ("accepted", C.c_int32),
                ("rejected", C.c_int32), ("expansions", C.c_int32),
                ("proxy_loss_init", C.c_double), ("proxy_loss_final", C.c_double),
                ("level_hist", C.c_int64 * 8)]

    def as_dict(self):
        return {"cap_bits": self.cap_bits, "used_bits": self.used_bits,
                "iterations": self.iterations, "accepted": self.accepted,
                "rejected": self.rejected, "expansions": self.expansions,
                "proxy_loss_init": self.proxy_loss_init,
                "proxy_loss_final": self.proxy_loss_final,
                "level_hist": list(self.level_hist)}


class StepReport(C.Structure):
    _fields_ = [("cap_bits", C.c_int64), ("used_in", C.c_int64), ("used_out", C.c_int64),
                ("expansion", C.c_int32), ("moved", C.c_int32),
                ("n_up", C.c_int64), ("n_down", C.c_int64),
                ("sum_up", C.c_double), ("sum_down", C.c_double)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class Kv8CacheStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("table", C.c_void_p), ("table_stride", C.c_int64), ("pages", C.c_int64),
                ("requests", C.c_int32), ("heads", C.c_int32), ("page_tokens", C.c_int32), ("dim", C.c_int32),
                ("type", C.c_int32), ("table_pages", C.c_int32)]


class Kv4CacheStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("k_head", C.c_void_p), ("v_head", C.c_void_p), ("table", C.c_void_p), ("table_stride", C.c_int64), ("pages", C.c_int64),
                ("requests", C.c_int32), ("heads", C.c_int32), ("page_tokens", C.c_int32), ("dim", C.c_int32),
                ("table_pages", C.c_int32), ("reserved", C.c_int32)]


class RotaryTableStruct(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("rotated", C.c_int32), ("interleaved", C.c_int32), ("inverse", C.c_int32), ("factor", C.c_float)]


class RotaryPartStruct(C.Structure):
    _fields_ = [("x", C.c_void_p), ("x_token_stride", C.c_int64), ("x_head_stride", C.c_int64),
                ("y", C.c_void_p), ("y_token_stride", C.c_int64), ("y_head_stride", C.c_int64), ("heads", C.c_int32), ("reserved", C.c_int32)]


class LoraAdaptersStruct(C.Structure):
    _fields_ = [("a", C.c_void_p), ("b", C.c_void_p), ("scale", C.c_void_p), ("in_", C.c_int64), ("out", C.c_int64),
                ("adapters", C.c_int32), ("rank", C.c_int32)]


_lib = None


def lib() -> C.CDLL:
    """Loads libscalebits.so (built in-tree by `python -m paper_2602_17698_b200.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2602_17698_b200.build` "
                "(nvcc, sm_100a). There is no CPU fallback.")
        L = C.CDLL(LIB_PATH)
        vp, i64, i32, f32, f64 = C.c_void_p, C.c_int64, C.c_int, C.c_float, C.c_double
        L.sb_create.argtypes = [C.POINTER(vp), i32, vp]
        L.sb_destroy.argtypes = [vp]
        L.sb_sync.argtypes = [vp]
        L.sb_debug_lookback.argtypes = [vp, i64, i64]
        L.sb_checked_build.argtypes = []
        L.sb_last_error.argtypes = [vp]
        L.sb_last_error.restype = C.c_char_p
        L.sb_kernel_launches.argtypes = [vp]
        L.sb_kernel_launches.restype = i64
        L.sb_calib_moments.argtypes = [vp, vp, i64, i64, i64, vp, i32, f32]
        L.sb_reorder_channels.argtypes = [vp, vp, i64, i64, i64, vp, vp, i32, i32, vp, vp, i32,
                                          i64, i64, vp, vp]
        L.sb_fold_segment_scores.argtypes = [vp, vp, vp, i64, i32, i64]
        L.sb_expand_segment_perm.argtypes = [vp, vp, vp, i64, i32, i64]
        L.sb_sum_scores.argtypes = [vp, vp, C.POINTER(C.c_void_p), i32, i64, i32]
        L.sb_permute_matrix.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp]
        L.sb_block_scores.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp, vp, i32, i32, i32,
                                      C.POINTER(C.c_int), i32, vp, vp, vp]
        L.sb_allocate_bits.argtypes = [vp, vp, i64, vp, i64, C.POINTER(C.c_int), i32, f64, i32,
                                       f64, f64, vp, C.POINTER(AllocReport)]
        L.sb_allocate_bits_async.argtypes = [vp, vp, i64, vp, i64, C.POINTER(C.c_int), i32, f64, i32,
                                             f64, f64, vp, vp]
        L.sb_pack_blocks.argtypes = [vp, vp, i64, i64, i64, vp, vp, i32, i32, i32,
                                     C.POINTER(C.c_int), i32, vp, vp, i64, vp, vp]
        L.sb_first_order_scores.argtypes = [vp, vp, vp, i64, i64, i64, i64, vp, vp, i32, i32, i32,
                                            C.POINTER(C.c_int), i32, vp, vp, vp, vp]
        L.sb_exchange_step.argtypes = [vp, vp, vp, vp, i64, vp, i64, C.POINTER(C.c_int), i32, f64, i64,
                                       vp, C.POINTER(StepReport)]
        L.sb_calib_moments_noalloc.argtypes = [vp, vp, i64, i64, i64, vp, i32, f32]
        L.sb_calib_gram.argtypes = [vp, vp, i64, i64, i64, vp, i32, f32]
        L.sb_block_scores_full.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp, vp, i32, i32, i32,
                                           C.POINTER(C.c_int), i32, vp, vp, vp]
        L.sb_dequant_gemm.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, i64, i64, i32, i32, i32,
                                      C.POINTER(C.c_int), i32, vp, i64]
        L.sb_reorder_channels_first_order.argtypes = [vp, vp, vp, i64, i64, i64, i64, i32, i32, vp, vp, i32,
                                                      i64, i64, vp, vp]
        L.sb_fp4_code_bytes.argtypes = [i64, i64]
        L.sb_fp4_scale_bytes.argtypes = [i64, i64, i32]
        L.sb_fp4_quantize.argtypes = [vp, vp, i64, i64, i64, i32, vp, vp, vp]
        L.sb_fp4_dequantize.argtypes = [vp, vp, vp, i64, i64, i32, vp, vp, i64]
        L.sb_fp4_gemm.argtypes = [vp, vp, vp, vp, i64, vp, vp, vp, i64, i64, i32, vp, i32, i64]
        cp = C.POINTER(Kv8CacheStruct)
        L.sb_kv8_append.argtypes = [vp, cp, vp, i64, i64, vp, i64, i64, i64, vp, vp, i64]
        L.sb_kv8_read.argtypes = [vp, cp, i64, vp, vp, i64, vp, vp]
        L.sb_kv8_attention.argtypes = [vp, cp, vp, i64, i64, i32, i64, vp, vp, i64, i64, f32, i64, vp, i64, i64, vp]
        c4 = C.POINTER(Kv4CacheStruct)
        L.sb_kv4_append.argtypes = [vp, c4, vp, i64, i64, vp, i64, i64, i64, vp, vp, i64]
        L.sb_kv4_read.argtypes = [vp, c4, i64, vp, vp, i64, vp, vp]
        L.sb_kv4_attention.argtypes = [vp, c4, vp, i64, i64, i32, i64, vp, vp, i64, i64, f32, i64, vp, i64, i64, vp]
        L.sb_rotary.argtypes = [vp, C.POINTER(RotaryTableStruct), vp, i32, i32, i32, i64, vp, vp, vp, i32, i64]
        L.sb_lora_add.argtypes = [vp, C.POINTER(LoraAdaptersStruct), vp, i64, vp, i64, vp, i64, i32, i64, vp, vp, i32, i64]
        L.sb_fp4_code_bytes.restype = L.sb_fp4_scale_bytes.restype = i64
        for name in EXPORTS:
            if name not in ("sb_last_error", "sb_kernel_launches", "sb_fp4_code_bytes", "sb_fp4_scale_bytes"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _ptr(t: Optional[torch.Tensor], dtype=None, cuda=True):
    if t is None:
        return None
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    if cuda and not t.is_cuda:
        raise ValueError("expected a CUDA tensor (the library has no CPU path)")
    return C.c_void_p(t.data_ptr())


def _dev(t: Optional[torch.Tensor]):
    """Address of a CUDA tensor (None: NULL); the calls of a decode step are as long as this binding."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor (the library has no CPU path)")
    return t.data_ptr()


def _bits(bits: Sequence[int]):
    return (C.c_int * len(bits))(*[int(b) for b in bits]), len(bits)


def _mat(W: torch.Tensor):
    if W.dim() != 2 or W.dtype != _BF16 or W.stride(1) != 1:
        raise ValueError("expected a row-major 2-D bf16 tensor")
    return W.shape[0], W.shape[1], W.stride(0)


def fp4_code_bytes(rows: int, cols: int) -> int:
    """Bytes of the codes of a 4-bit matrix (rows padded to 32 columns)."""
    return int(lib().sb_fp4_code_bytes(rows, cols))


def fp4_scale_bytes(rows: int, cols: int, fmt: str) -> int:
    """Bytes of its scales (tiles of 128 rows x 4 blocks)."""
    return int(lib().sb_fp4_scale_bytes(rows, cols, FP4_FORMATS[fmt]))


class Fp4Matrix:
    """A matrix in a microscaled 4-bit format ("mx" or "nv"): codes uint8 [rows][padded cols / 2],
    scales uint8 (tiles), and for "nv" the fp32 scale of the whole matrix, a tensor of one element
    on the device (None: 1)."""
    __slots__ = ("codes", "scales", "rows", "cols", "fmt", "tensor_scale")

    def __init__(self, codes, scales, rows: int, cols: int, fmt: str = "nv", tensor_scale=None):
        if fmt not in FP4_FORMATS:
            raise ValueError(f"unknown 4-bit format {fmt!r}")
        pitch = (cols + 31) // 32 * 16
        tiles = (rows + 127) // 128 * ((pitch * 2 // (32 if fmt == "mx" else 16) + 3) // 4)
        if codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or not codes.is_contiguous() or not scales.is_contiguous():
            raise TypeError("codes and scales are contiguous uint8 tensors")
        if codes.numel() != rows * pitch or scales.numel() != tiles * 512:
            raise ValueError("codes or scales have another size than the format's")
        if tensor_scale is not None and (tensor_scale.dtype is not torch.float32 or tensor_scale.numel() != 1):
            raise TypeError("tensor_scale is one fp32 element")
        self.codes, self.scales, self.rows, self.cols, self.fmt, self.tensor_scale = codes, scales, rows, cols, fmt, tensor_scale

    @classmethod
    def empty(cls, rows: int, cols: int, fmt: str = "nv", tensor_scale=None, device="cuda"):
        return cls(torch.empty((rows, (cols + 31) // 32 * 16), dtype=torch.uint8, device=device),
                   torch.empty(fp4_scale_bytes(rows, cols, fmt), dtype=torch.uint8, device=device), rows, cols, fmt, tensor_scale)


_E4M3_BYTES = (torch.uint8, torch.float8_e4m3fn)
_KV8_TYPES = {torch.int8: SB_KV_INT8, torch.float8_e4m3fn: SB_KV_E4M3}


class Kv8Cache:
    """A paged key/value cache in 8 bits: k, v int8 or float8_e4m3fn [pages][heads][page tokens][dim],
    k_scale, v_scale bf16 [pages][heads][page tokens / 16], table int32 [requests][pages of a request]: rows may
    be part of longer ones (table[:, :n]), or for reading the same one (expand)."""
    __slots__ = ("k", "v", "k_scale", "v_scale", "table", "struct")

    def __init__(self, k, v, k_scale, v_scale, table):
        shape = k.shape
        pages, heads, page_tokens, dim = shape
        kind = _KV8_TYPES.get(k.dtype)
        if kind is None or v.dtype is not k.dtype:
            raise TypeError("keys and values are int8 or float8_e4m3fn")
        if k_scale.dtype is not _BF16 or v_scale.dtype is not _BF16 or table.dtype is not _I32:
            raise TypeError("scales are bf16 and page numbers int32")
        n = k_scale.numel()
        if v.shape != shape or n * SB_KV8_BLOCK != pages * heads * page_tokens or v_scale.numel() != n:
            raise ValueError("keys, values and scales do not fit one another")
        requests, per = table.shape
        stride, one = table.stride()
        if per < 1:
            raise ValueError("a request needs room for a page in the table")
        if not (k.is_contiguous() and v.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()) or one != 1:
            raise ValueError("the cache's tensors are contiguous")
        self.k, self.v, self.k_scale, self.v_scale, self.table = k, v, k_scale, v_scale, table
        self.struct = Kv8CacheStruct(_dev(k), _dev(v), _dev(k_scale), _dev(v_scale), _dev(table), stride if requests > 1 else per,
                                     pages, requests, heads, page_tokens, dim, kind, per)

    @classmethod
    def empty(cls, pages: int, heads: int, page_tokens: int, dim: int, table, dtype=torch.int8):
        kv = torch.zeros((2, pages, heads, page_tokens, dim), dtype=torch.uint8, device=table.device).view(dtype)
        sc = torch.zeros((2, pages, heads, page_tokens // SB_KV8_BLOCK), dtype=torch.bfloat16, device=table.device)
        return cls(kv[0], kv[1], sc[0], sc[1], table)


class Kv4Cache:
    """A paged key/value cache in 4 bits: k, v uint8 [pages][heads][page tokens][padded dim / 2] (e2m1, two to a byte, rows padded with zeros to 32
    elements), k_scale, v_scale uint8 or float8_e4m3fn [pages][heads][page tokens][scales of a row, padded to 4], k_head, v_head fp32 [heads] (None: 1),
    table int32 [requests][pages of a request] as in Kv8Cache."""
    __slots__ = ("k", "v", "k_scale", "v_scale", "table", "dim", "k_head", "v_head", "struct")

    def __init__(self, k, v, k_scale, v_scale, table, dim: int, k_head=None, v_head=None):
        pages, heads, page_tokens, row = shape = k.shape
        if k.dtype is not _U8 or v.dtype is not _U8 or k_scale.dtype not in _E4M3_BYTES or v_scale.dtype not in _E4M3_BYTES or table.dtype is not _I32:
            raise TypeError("codes are uint8, scales uint8 or float8_e4m3fn, page numbers int32")
        scales = k_scale.shape
        if v.shape != shape or row != (dim + 31) // 32 * 16 or scales != (pages, heads, page_tokens, (dim + 63) // 64 * 4) or v_scale.shape != scales:
            raise ValueError("codes and scales do not fit one another and dim")
        requests, per = table.shape
        stride, one = table.stride()
        if per < 1:
            raise ValueError("a request needs room for a page in the table")
        if not (k.is_contiguous() and v.is_contiguous() and k_scale.is_contiguous() and v_scale.is_contiguous()) or one != 1:
            raise ValueError("the cache's tensors are contiguous")
        if k_head is not None and (k_head.dtype is not _F32 or k_head.shape != (heads,) or not k_head.is_contiguous()) \
                or v_head is not None and (v_head.dtype is not _F32 or v_head.shape != (heads,) or not v_head.is_contiguous()):
            raise ValueError("k_head, v_head: contiguous fp32 [heads]")
        self.k, self.v, self.k_scale, self.v_scale, self.table, self.dim, self.k_head, self.v_head = k, v, k_scale, v_scale, table, dim, k_head, v_head
        self.struct = Kv4CacheStruct(_dev(k), _dev(v), _dev(k_scale), _dev(v_scale), _dev(k_head), _dev(v_head), _dev(table),
                                     stride if requests > 1 else per, pages, requests, heads, page_tokens, dim, per, 0)

    @classmethod
    def empty(cls, pages: int, heads: int, page_tokens: int, dim: int, table, k_head=None, v_head=None):
        kv = torch.zeros((2, pages, heads, page_tokens, (dim + 31) // 32 * 16), dtype=torch.uint8, device=table.device)
        sc = torch.zeros((2, pages, heads, page_tokens, (dim + 63) // 64 * 4), dtype=torch.uint8, device=table.device)
        return cls(kv[0], kv[1], sc[0], sc[1], table, dim, k_head, v_head)


class RotaryTable:
    """Frequencies of rotary positions: fp32 [rotated / 2] on the device, radians per position (`rotary_frequencies` makes them), how a head's
    elements pair up, and the factor on cos and sin."""
    __slots__ = ("freq", "rotated", "interleaved", "factor", "_structs")

    def __init__(self, freq: torch.Tensor, interleaved: bool = False, factor: float = 1.0):
        if freq.dtype is not _F32 or freq.dim() != 1 or not freq.is_contiguous() or freq.numel() < 1:
            raise ValueError("freq: contiguous fp32 [rotated / 2]")
        self.freq, self.rotated, self.interleaved, self.factor = freq, 2 * freq.numel(), bool(interleaved), float(factor)
        self._structs = [None, None]                                 # forward and inverse, made when they are used

    def struct(self, inverse: bool = False) -> RotaryTableStruct:
        s = self._structs[bool(inverse)]
        if s is None:
            s = self._structs[bool(inverse)] = RotaryTableStruct(_dev(self.freq), self.rotated, self.interleaved, bool(inverse), self.factor)
        return s


# sb_rotary_part as bytes: a third of the time that filling a ctypes structure takes
_ROTARY_PART = struct.Struct("PqqPqqii")


def _rotary_part(x: torch.Tensor, y: torch.Tensor, tokens: int, dim: int, dtype) -> bytes:
    n, heads, d = shape = x.shape
    xt, xh, one = x.stride()
    if y is x:
        yt, yh, two = xt, xh, one
    else:
        yt, yh, two = y.stride()
        if y.shape != shape or y.dtype is not dtype:
            raise ValueError("rotary: out has the shape and type of its input")
    if n != tokens or d != dim or x.dtype is not dtype:
        raise ValueError("rotary: tensors of one type, [tokens][heads][dim] with the same tokens and dim")
    if one != 1 or two != 1:
        raise ValueError("rotary: elements of a head are contiguous")
    px = _dev(x)
    return _ROTARY_PART.pack(px, xt, xh, px if y is x else _dev(y), yt, yh, heads, 0)


class LoraAdapters:
    """Low-rank adapters of one projection: a bf16 [adapters][rank][in], b bf16 [adapters][out][rank], scale fp32 [adapters] (None: 1).  The rank is a
    multiple of 8, up to 128; smaller ones are padded with zeros."""
    __slots__ = ("a", "b", "scale", "adapters", "rank", "inner", "outer", "struct")

    def __init__(self, a: torch.Tensor, b: torch.Tensor, scale: Optional[torch.Tensor] = None):
        if a.dtype is not _BF16 or b.dtype is not _BF16 or not a.is_contiguous() or not b.is_contiguous():
            raise TypeError("a and b are contiguous bf16 tensors")
        n, rank, inner = a.shape
        outer = b.shape[1]
        if b.shape != (n, outer, rank):
            raise ValueError("a: [adapters][rank][in], b: [adapters][out][rank]")
        if scale is not None and (scale.dtype is not _F32 or scale.shape != (n,) or not scale.is_contiguous()):
            raise ValueError("scale: contiguous fp32 [adapters]")
        self.a, self.b, self.scale, self.adapters, self.rank, self.inner, self.outer = a, b, scale, n, rank, inner, outer
        self.struct = LoraAdaptersStruct(_dev(a), _dev(b), _dev(scale), inner, outer, n, rank)


def rotary_frequencies(rotated: int, base: float = 10000.0, scaling: Optional[str] = None, stretch: float = 1.0, trained: int = 8192,
                       low: float = 1.0, high: float = 4.0) -> torch.Tensor:
    """Frequencies base^(-2 i / rotated), fp32 on the host (computed in 64 bits), scaled for contexts `stretch` times as long as the
    `trained` one: None: not; "linear": all divided by stretch; "base": with a base of base stretch^(rotated / (rotated - 2)), under which the slowest pair turns
    stretch times as slowly and the fastest as before; "parts": divided by stretch where a pair turns less than `low` times in the trained
    length, left where it turns more than `high` times, and in between by both in proportion."""
    if rotated < 2 or rotated % 2 or stretch <= 0:
        raise ValueError("rotated is even and at least 2, stretch positive")
    i = torch.arange(rotated // 2, dtype=torch.float64)
    if scaling == "base" and rotated > 2:
        base = base * stretch ** (rotated / (rotated - 2))
    f = base ** (-2 * i / rotated)
    if scaling == "linear":
        f = f / stretch
    elif scaling == "parts":
        if not 0 <= low < high:
            raise ValueError("0 <= low < high")
        keep = ((f * trained / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * (keep + (1 - keep) / stretch)
    elif scaling not in (None, "base"):
        raise ValueError(f"unknown scaling {scaling!r}")
    return f.float()


def _heads(x: torch.Tensor, what: str):
    """(address, token stride, head stride) of a bf16 [tokens][heads][dim] tensor."""
    token, head, one = x.stride()
    if x.dtype is not _BF16 or one != 1 or not x.is_cuda:
        raise ValueError(f"{what}: expected a bf16 [tokens][heads][dim] CUDA tensor with contiguous rows")
    tokens, heads, _ = x.shape
    # the stride of an axis of one element is never used
    return x.data_ptr(), token if tokens > 1 else 0, head if heads > 1 else 0


class Context:
    """One sb_ctx on the current torch device and stream."""

    def __init__(self, device: Optional[int] = None, stream: Optional[torch.cuda.Stream] = None):
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: the scalebits library has no CPU fallback")
        self.device = torch.cuda.current_device() if device is None else int(device)
        self.stream = torch.cuda.current_stream(self.device) if stream is None else stream
        h = C.c_void_p()
        st = lib().sb_create(C.byref(h), self.device, C.c_void_p(self.stream.cuda_stream))
        if st != SB_OK:
            raise SbError(st, "sb_create failed (needs an sm_100 device)")
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().sb_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != SB_OK:
            raise SbError(st, lib().sb_last_error(self._h).decode())

    def _result(self, shape, dtype, device) -> torch.Tensor:
        """Memory for a result of the 4-bit and cache calls: the context's stream writes it, so it comes from what that
        stream has let go, and it is not given away before the stream that is torch's current one now is done with it."""
        here = torch.cuda.current_stream(self.device)
        if here == self.stream:
            return torch.empty(shape, dtype=dtype, device=device)
        with torch.cuda.stream(self.stream):
            out = torch.empty(shape, dtype=dtype, device=device)
        out.record_stream(here)
        return out

    # ---- the C-ABI calls, one method each -------------------------------------------------
    def sync(self):
        self._check(lib().sb_sync(self._h))

    def kernel_launches(self) -> int:
        return int(lib().sb_kernel_launches(self._h))

    def calib_moments(self, X: torch.Tensor, sumsq: Optional[torch.Tensor] = None,
                      accumulate: bool = False, scale: Optional[float] = None) -> torch.Tensor:
        T, K, ldx = _mat(X)
        if sumsq is None:
            sumsq = torch.empty(K, dtype=torch.float32, device=X.device)
            accumulate = False
        if scale is None:
            scale = 1.0 / T
        self._check(lib().sb_calib_moments(self._h, _ptr(X), T, K, ldx, _ptr(sumsq, torch.float32),
                                           int(accumulate), float(scale)))
        return sumsq

    def calib_gram(self, X: torch.Tensor, H: Optional[torch.Tensor] = None, accumulate: bool = False,
                   scale: Optional[float] = None) -> torch.Tensor:
        T, K, ldx = _mat(X)
        if H is None:
            H = torch.empty((K, K), dtype=torch.float32, device=X.device)
            accumulate = False
        if scale is None:
            scale = 1.0 / max(T, 1)
        self._check(lib().sb_calib_gram(self._h, _ptr(X), T, K, ldx, _ptr(H, torch.float32), int(accumulate),
                                        float(scale)))
        return H

    def reorder_channels(self, W: Optional[torch.Tensor], col_moment: Optional[torch.Tensor],
                         ref_bits: int, group: int, row_score=None, col_score=None,
                         accumulate_row: bool = False, accumulate_col: bool = False,
                         row_segment: int = 0, col_segment: int = 0,
                         row_perm=None, col_perm=None, row_weight=None, shape=None):
        if W is not None:
            R, Cc, ldw = _mat(W)
        else:
            R, Cc = shape
            ldw = Cc
        self._check(lib().sb_reorder_channels(
            self._h, _ptr(W), R, Cc, ldw, _ptr(col_moment, torch.float32),
            _ptr(row_weight, torch.float32), int(ref_bits), int(group),
            _ptr(row_score, torch.float32), _ptr(col_score, torch.float32),
            (SB_ACC_ROW if accumulate_row else 0) | (SB_ACC_COL if accumulate_col else 0),
            int(row_segment), int(col_segment), _ptr(row_perm, torch.int32), _ptr(col_perm, torch.int32)))

    def fold_segment_scores(self, dst: torch.Tensor, src: torch.Tensor, reps: int, seg: int):
        assert dst.numel() * reps == src.numel()
        self._check(lib().sb_fold_segment_scores(self._h, _ptr(dst, torch.float32),
                                                 _ptr(src, torch.float32), dst.numel(), reps, seg))

    def sum_scores(self, dst: torch.Tensor, srcs: Sequence[torch.Tensor], accumulate: bool = False):
        """dst = (dst +) srcs[0] + srcs[1] + ... left to right in fp32 (the score vectors of the
        matrices of a coupled channel set, in the order a one-stream accumulation would take)."""
        n = dst.numel()
        assert 1 <= len(srcs) <= 8 and all(t.numel() == n and t.is_contiguous() for t in srcs)
        arr = (C.c_void_p * len(srcs))(*[_ptr(t, torch.float32).value for t in srcs])
        self._check(lib().sb_sum_scores(self._h, _ptr(dst, torch.float32), arr, len(srcs), n, int(accumulate)))
        return dst

    def expand_segment_perm(self, perm: torch.Tensor, reps: int, seg: int, out=None) -> torch.Tensor:
        if out is None:
            out = torch.empty(perm.numel() * reps, dtype=torch.int32, device=perm.device)
        assert out.numel() == perm.numel() * reps and out.dtype == torch.int32
        self._check(lib().sb_expand_segment_perm(self._h, _ptr(out), _ptr(perm, torch.int32),
                                                 perm.numel(), reps, seg))
        return out

    def debug_lookback(self, wait_ns: int = -1, mute_tile: int = -1):
        """Test hook: the time limit of a look-back wait and a tile that publishes nothing."""
        self._check(lib().sb_debug_lookback(self._h, int(wait_ns), int(mute_tile)))

    def permute_matrix(self, W: torch.Tensor, row_perm=None, col_perm=None, out=None) -> torch.Tensor:
        """out[r][j] = W[row_perm[r]][col_perm[j]] (a matrix that is moved along with a channel
        permutation but not scored: embedding, language-model head)."""
        R, Cc, ldw = _mat(W)
        if out is None:
            out = torch.empty((R, Cc), dtype=torch.bfloat16, device=W.device)
        self._check(lib().sb_permute_matrix(self._h, _ptr(W), R, Cc, ldw, _ptr(row_perm, torch.int32),
                                            _ptr(col_perm, torch.int32), _ptr(out)))
        return out

    def block_scores(self, W: torch.Tensor, col_moment: torch.Tensor, bits: Sequence[int],
                     block_rows: int = 128, block_cols: int = 128, group: int = 128,
                     row_perm=None, col_perm=None, row_weight=None, err=None, gain=None,
                     want_gain: bool = True, W_perm_out=None):
        R, Cc, ldw = _mat(W)
        barr, L = _bits(bits)
        nb = (R // block_rows) * (Cc // block_cols)
        if err is None:
            err = torch.empty((nb, L), dtype=torch.float32, device=W.device)
        if gain is None and want_gain and L > 1:
            gain = torch.empty((nb, L - 1), dtype=torch.float32, device=W.device)
        self._check(lib().sb_block_scores(
            self._h, _ptr(W), R, Cc, ldw, _ptr(row_perm, torch.int32), _ptr(col_perm, torch.int32),
            _ptr(col_moment, torch.float32), _ptr(row_weight, torch.float32),
            block_rows, block_cols, group, barr, L, _ptr(err, torch.float32),
            _ptr(gain, torch.float32), _ptr(W_perm_out, torch.bfloat16)))
        return err, gain

    def block_scores_full(self, W: torch.Tensor, H: torch.Tensor, bits: Sequence[int],
                          block_rows: int = 128, block_cols: int = 128, group: int = 128,
                          row_perm=None, col_perm=None, row_weight=None, err=None, gain=None,
                          want_gain: bool = True, W_perm_out=None):
        R, Cc, ldw = _mat(W)
        assert H.shape == (Cc, Cc) and H.is_contiguous()
        barr, L = _bits(bits)
        nb = (R // block_rows) * (Cc // block_cols)
        if err is None:
            err = torch.empty((nb, L), dtype=torch.float32, device=W.device)
        if gain is None and want_gain and L > 1:
            gain = torch.empty((nb, L - 1), dtype=torch.float32, device=W.device)
        self._check(lib().sb_block_scores_full(
            self._h, _ptr(W), R, Cc, ldw, _ptr(row_perm, torch.int32), _ptr(col_perm, torch.int32),
            _ptr(H, torch.float32), _ptr(row_weight, torch.float32), block_rows, block_cols, group, barr, L,
            _ptr(err, torch.float32), _ptr(gain, torch.float32), _ptr(W_perm_out, torch.bfloat16)))
        return err, gain

    def allocate_bits(self, err: torch.Tensor, bits: Sequence[int], budget: float,
                      mode: int = SB_ALLOC_SCALEBITS, gamma0: float = 0.05, gammaT: float = 0.02,
                      uniform_block_elems: int = 128 * 128, block_elems=None, level=None):
        N, L = err.shape
        barr, Lb = _bits(bits)
        assert L == Lb and err.is_contiguous()
        if level is None:
            level = torch.empty(N, dtype=torch.uint8, device=err.device)
        rep = AllocReport()
        st = lib().sb_allocate_bits(self._h, _ptr(err, torch.float32), N, _ptr(block_elems, torch.int64),
                                    int(uniform_block_elems), barr, L, float(budget), int(mode),
                                    float(gamma0), float(gammaT), _ptr(level, torch.uint8), C.byref(rep))
        self._check(st)
        return level, rep.as_dict()

    def allocate_bits_async(self, err: torch.Tensor, bits: Sequence[int], budget: float,
                            mode: int = SB_ALLOC_SCALEBITS, gamma0: float = 0.05, gammaT: float = 0.02,
                            uniform_block_elems: int = 128 * 128, block_elems=None, level=None,
                            report=None):
        """The allocation enqueued only (no host round trip; can be captured in a CUDA graph).
        Returns (level, report): `report` is a uint8 device tensor holding the report struct;
        `read_report(report)` decodes it after a synchronisation."""
        N, L = err.shape
        barr, Lb = _bits(bits)
        assert L == Lb and err.is_contiguous()
        if level is None:
            level = torch.empty(N, dtype=torch.uint8, device=err.device)
        if report is None:
            report = torch.zeros(C.sizeof(AllocReport), dtype=torch.uint8, device=err.device)
        assert report.dtype == torch.uint8 and report.numel() >= C.sizeof(AllocReport) and report.is_contiguous()
        st = lib().sb_allocate_bits_async(self._h, _ptr(err, torch.float32), N, _ptr(block_elems, torch.int64),
                                          int(uniform_block_elems), barr, L, float(budget), int(mode),
                                          float(gamma0), float(gammaT), _ptr(level, torch.uint8),
                                          _ptr(report, torch.uint8))
        self._check(st)
        return level, report

    @staticmethod
    def read_report(report: torch.Tensor) -> dict:
        """Decodes the device report of `allocate_bits_async` (copies it to the host: the
        stream that wrote it must have been synchronised, or be the current one)."""
        raw = bytes(report.cpu().numpy().tobytes()[:C.sizeof(AllocReport)])
        return AllocReport.from_buffer_copy(raw).as_dict()

    def reorder_channels_first_order(self, W: torch.Tensor, G: torch.Tensor, ref_bits: int, group: int,
                                     row_score=None, col_score=None, accumulate_row: bool = False,
                                     accumulate_col: bool = False, row_segment: int = 0, col_segment: int = 0,
                                     row_perm=None, col_perm=None):
        R, Cc, ldw = _mat(W)
        Rg, Cg, ldg = _mat(G)
        assert (R, Cc) == (Rg, Cg)
        acc = (SB_ACC_ROW if accumulate_row else 0) | (SB_ACC_COL if accumulate_col else 0)
        self._check(lib().sb_reorder_channels_first_order(
            self._h, _ptr(W), _ptr(G), R, Cc, ldw, ldg, int(ref_bits), int(group),
            _ptr(row_score, torch.float32), _ptr(col_score, torch.float32), acc, int(row_segment),
            int(col_segment), _ptr(row_perm, torch.int32), _ptr(col_perm, torch.int32)))
        return row_score, col_score

    def first_order_scores(self, W: torch.Tensor, G: torch.Tensor, bits: Sequence[int], level: torch.Tensor,
                           block_rows: int = 128, block_cols: int = 128, group: int = 128,
                           row_perm=None, col_perm=None, s_up=None, s_down=None, s_l1=None,
                           want_l1: bool = True):
        R, Cc, ldw = _mat(W)
        Rg, Cg, ldg = _mat(G)
        assert (R, Cc) == (Rg, Cg)
        barr, L = _bits(bits)
        nb = (R // block_rows) * (Cc // block_cols)
        f32 = dict(dtype=torch.float32, device=W.device)
        if s_up is None:
            s_up = torch.empty(nb, **f32)
        if s_down is None:
            s_down = torch.empty(nb, **f32)
        if s_l1 is None and want_l1:
            s_l1 = torch.empty(nb, **f32)
        self._check(lib().sb_first_order_scores(
            self._h, _ptr(W), _ptr(G), R, Cc, ldw, ldg, _ptr(row_perm, torch.int32),
            _ptr(col_perm, torch.int32), block_rows, block_cols, group, barr, L, _ptr(level, torch.uint8),
            _ptr(s_up, torch.float32), _ptr(s_down, torch.float32), _ptr(s_l1, torch.float32)))
        return s_up, s_down, s_l1

    def exchange_step(self, s_up: torch.Tensor, s_down: torch.Tensor, level: torch.Tensor,
                      bits: Sequence[int], budget: float, k: int, uniform_block_elems: int = 128 * 128,
                      block_elems=None, level_out=None):
        N = level.numel()
        barr, L = _bits(bits)
        if level_out is None:
            level_out = torch.empty_like(level)
        rep = StepReport()
        st = lib().sb_exchange_step(self._h, _ptr(s_up, torch.float32), _ptr(s_down, torch.float32),
                                    _ptr(level, torch.uint8), N, _ptr(block_elems, torch.int64),
                                    int(uniform_block_elems), barr, L, float(budget), int(k),
                                    _ptr(level_out, torch.uint8), C.byref(rep))
        self._check(st)
        return level_out, rep.as_dict()

    def pack_blocks(self, W: torch.Tensor, bits: Sequence[int], level: torch.Tensor,
                    block_rows: int = 128, block_cols: int = 128, group: int = 128,
                    row_perm=None, col_perm=None, packed=None, block_off=None, meta=None):
        R, Cc, ldw = _mat(W)
        barr, L = _bits(bits)
        nb = (R // block_rows) * (Cc // block_cols)
        if packed is None:
            packed = torch.empty(R * Cc * max(bits) // 32, dtype=torch.int32, device=W.device)
        if block_off is None:
            block_off = torch.empty(nb + 1, dtype=torch.int64, device=W.device)
        if meta is None:
            meta = torch.empty((R * Cc // group, 2), dtype=torch.float32, device=W.device)
        self._check(lib().sb_pack_blocks(
            self._h, _ptr(W), R, Cc, ldw, _ptr(row_perm, torch.int32), _ptr(col_perm, torch.int32),
            block_rows, block_cols, group, barr, L, _ptr(level, torch.uint8), _ptr(packed),
            packed.numel(), _ptr(block_off, torch.int64), _ptr(meta, torch.float32)))
        return packed, block_off, meta


    def dequant_gemm(self, X: torch.Tensor, packed: torch.Tensor, block_off: torch.Tensor, meta: torch.Tensor,
                     level: torch.Tensor, R: int, Cc: int, bits: Sequence[int], block_rows: int = 128,
                     block_cols: int = 128, group: int = 128, Y: Optional[torch.Tensor] = None):
        """Y[t][r] = sum_c X[t][c] (lo + scale q)[r][c] on the output of pack_blocks -> fp32 [T][R]."""
        T, Kx, ldx = _mat(X)
        if Kx != Cc:
            raise ValueError("X must have one column per packed column")
        barr, L = _bits(bits)
        if Y is None:
            Y = torch.empty((T, R), dtype=torch.float32, device=X.device)
        self._check(lib().sb_dequant_gemm(
            self._h, _ptr(X), T, ldx, _ptr(packed), _ptr(block_off, torch.int64), _ptr(meta, torch.float32),
            _ptr(level, torch.uint8), R, Cc, block_rows, block_cols, group, barr, L,
            _ptr(Y, torch.float32), Y.stride(0)))
        return Y

    # ---- microscaled 4-bit matrices ---------------------------------------------------------
    def fp4_quantize(self, X: torch.Tensor, out: Fp4Matrix) -> Fp4Matrix:
        """X (bf16 [rows][cols]) into `out`, whose format and tensor scale it takes."""
        R, Cc, ldx = _mat(X)
        if R != out.rows or Cc != out.cols:
            raise ValueError("X and the 4-bit matrix have different sizes")
        self._check(lib().sb_fp4_quantize(self._h, _dev(X), R, Cc, ldx if R > 1 else (Cc + 7) // 8 * 8, FP4_FORMATS[out.fmt],
                                          _dev(out.tensor_scale), _dev(out.codes), _dev(out.scales)))
        return out

    def fp4_dequantize(self, m: Fp4Matrix, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The bf16 values a 4-bit matrix stands for."""
        if out is None:
            out = self._result((m.rows, m.cols), torch.bfloat16, m.codes.device)
        R, Cc, ldy = _mat(out)
        if R != m.rows or Cc != m.cols:
            raise ValueError("out and the 4-bit matrix have different sizes")
        self._check(lib().sb_fp4_dequantize(self._h, _dev(m.codes), _dev(m.scales), R, Cc, FP4_FORMATS[m.fmt], _dev(m.tensor_scale),
                                            _dev(out), ldy if R > 1 else Cc))
        return out

    def fp4_gemm(self, a: Fp4Matrix, b: Fp4Matrix, out: Optional[torch.Tensor] = None, out_dtype=torch.bfloat16) -> torch.Tensor:
        """a [M][K] times the transpose of b [N][K] -> [M][N] in bf16 or fp32 (out's type, or out_dtype)."""
        M, N = a.rows, b.rows
        if a.cols != b.cols or a.fmt != b.fmt:
            raise ValueError("the two matrices need the same format and number of columns")
        if out is None:
            out = self._result((M, N), out_dtype, a.codes.device)
        dtype, shape = out.dtype, out.shape
        ldy, one = out.stride()
        if dtype is not _BF16 and dtype is not _F32 or shape[0] != M or shape[1] != N or one != 1:
            raise ValueError("out: a row-major bf16 or fp32 [M][N] tensor")
        self._check(lib().sb_fp4_gemm(self._h, _dev(a.codes), _dev(a.scales), _dev(a.tensor_scale), M, _dev(b.codes), _dev(b.scales),
                                      _dev(b.tensor_scale), N, a.cols, FP4_FORMATS[a.fmt], _dev(out), int(dtype is _F32),
                                      ldy if M > 1 else N))
        return out

    # ---- key/value cache in 8 bits ----------------------------------------------------------
    @staticmethod
    def _kv8_rows(cache: Kv8Cache, starts: torch.Tensor, lens: torch.Tensor):
        n = cache.struct.requests
        if starts.dtype is not _I32 or lens.dtype is not _I32 or starts.numel() != n + 1 or lens.numel() != n \
                or not starts.is_contiguous() or not lens.is_contiguous():
            raise ValueError("starts: contiguous int32 [requests + 1], lens: contiguous int32 [requests]")
        return _dev(starts), _dev(lens)

    def kv8_append(self, cache: Kv8Cache, K: torch.Tensor, V: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, max_new: int):
        """Writes the new tokens' keys and values (bf16 [tokens][heads][dim]); request b's rows are
        starts[b] .. starts[b + 1], its length with them lens[b]."""
        s, n = self._kv8_rows(cache, starts, lens)
        tokens, heads, dim = shape = K.shape
        if V.shape != shape or heads != cache.struct.heads or dim != cache.struct.dim:
            raise ValueError("K and V: [tokens][heads][dim] of the cache")
        k, kt, kh = _heads(K, "K")
        v, vt, vh = _heads(V, "V")
        self._check(lib().sb_kv8_append(self._h, cache.struct, k, kt, kh, v, vt, vh, tokens, s, n, max_new))

    def kv8_read(self, cache: Kv8Cache, starts: torch.Tensor, lens: torch.Tensor, max_new: int, total: Optional[int] = None, out=None):
        """The values of the last starts[b + 1] - starts[b] tokens of every request, as bf16
        [tokens][heads][dim] keys and values; `out`, or `total` = starts[-1] to allocate them."""
        s, n = self._kv8_rows(cache, starts, lens)
        if out is None:
            shape = (int(starts[-1]) if total is None else total, cache.struct.heads, cache.struct.dim)
            out = tuple(self._result(shape, _BF16, cache.k.device) for _ in range(2))
        K, V = out
        tokens, heads, dim = shape = K.shape
        if V.shape != shape or heads != cache.struct.heads or dim != cache.struct.dim or not K.is_contiguous() or not V.is_contiguous() \
                or K.dtype is not _BF16 or V.dtype is not _BF16:
            raise ValueError("out: two contiguous bf16 [tokens][heads][dim] tensors")
        self._check(lib().sb_kv8_read(self._h, cache.struct, tokens, s, n, max_new, _dev(K), _dev(V)))
        return K, V

    def kv8_attention(self, cache: Kv8Cache, Q: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, max_new: int, max_len: int,
                      scale: Optional[float] = None, window: int = 0, out: Optional[torch.Tensor] = None,
                      lse: Optional[torch.Tensor] = None, want_lse: bool = False):
        """Causal attention of the new tokens (Q bf16 [tokens][query heads][dim]) over the cache, which
        holds them already.  Returns (out, lse); lse is None unless given or asked for."""
        s, n = self._kv8_rows(cache, starts, lens)
        tokens, heads, dim = shape = Q.shape
        if dim != cache.struct.dim:
            raise ValueError("Q: [tokens][query heads][dim of the cache]")
        q, qt, qh = _heads(Q, "Q")
        if out is None:
            out = self._result(shape, _BF16, Q.device)
        elif out.shape != shape:
            raise ValueError("out: the shape of Q")
        o, ot, oh = _heads(out, "out")
        if lse is None and want_lse:
            lse = self._result(shape[:2], _F32, Q.device)
        if lse is not None and (lse.shape != shape[:2] or not lse.is_contiguous() or lse.dtype is not _F32):
            raise ValueError("lse: contiguous fp32 [tokens][query heads]")
        self._check(lib().sb_kv8_attention(self._h, cache.struct, q, qt, qh, heads, tokens, s, n, max_new, max_len,
                                           dim ** -0.5 if scale is None else scale, window, o, ot, oh, _dev(lse)))
        return out, lse

    # ---- key/value cache in 4 bits ----------------------------------------------------------
    def kv4_append(self, cache: Kv4Cache, K: torch.Tensor, V: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, max_new: int):
        """Writes the new tokens' keys and values (bf16 [tokens][heads][dim]); requests as in kv8_append."""
        s, n = self._kv8_rows(cache, starts, lens)
        tokens, heads, dim = shape = K.shape
        if V.shape != shape or heads != cache.struct.heads or dim != cache.dim:
            raise ValueError("K and V: [tokens][heads][dim] of the cache")
        k, kt, kh = _heads(K, "K")
        v, vt, vh = _heads(V, "V")
        self._check(lib().sb_kv4_append(self._h, cache.struct, k, kt, kh, v, vt, vh, tokens, s, n, max_new))

    def kv4_read(self, cache: Kv4Cache, starts: torch.Tensor, lens: torch.Tensor, max_new: int, total: Optional[int] = None, out=None):
        """The values of the last starts[b + 1] - starts[b] tokens of every request, as bf16
        [tokens][heads][dim] keys and values; `out`, or `total` = starts[-1] to allocate them."""
        s, n = self._kv8_rows(cache, starts, lens)
        if out is None:
            shape = (int(starts[-1]) if total is None else total, cache.struct.heads, cache.dim)
            out = tuple(self._result(shape, _BF16, cache.k.device) for _ in range(2))
        K, V = out
        tokens, heads, dim = shape = K.shape
        if V.shape != shape or heads != cache.struct.heads or dim != cache.dim or not K.is_contiguous() or not V.is_contiguous() \
                or K.dtype is not _BF16 or V.dtype is not _BF16:
            raise ValueError("out: two contiguous bf16 [tokens][heads][dim] tensors")
        self._check(lib().sb_kv4_read(self._h, cache.struct, tokens, s, n, max_new, _dev(K), _dev(V)))
        return K, V

    def kv4_attention(self, cache: Kv4Cache, Q: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, max_new: int, max_len: int,
                      scale: Optional[float] = None, window: int = 0, out: Optional[torch.Tensor] = None,
                      lse: Optional[torch.Tensor] = None, want_lse: bool = False):
        """Causal attention of the new tokens (Q bf16 [tokens][query heads][dim]) over the cache, which
        holds them already.  Returns (out, lse); lse is None unless given or asked for."""
        s, n = self._kv8_rows(cache, starts, lens)
        tokens, heads, dim = shape = Q.shape
        if dim != cache.dim:
            raise ValueError("Q: [tokens][query heads][dim of the cache]")
        q, qt, qh = _heads(Q, "Q")
        if out is None:
            out = self._result(shape, _BF16, Q.device)
        elif out.shape != shape:
            raise ValueError("out: the shape of Q")
        o, ot, oh = _heads(out, "out")
        if lse is None and want_lse:
            lse = self._result(shape[:2], _F32, Q.device)
        if lse is not None and (lse.shape != shape[:2] or not lse.is_contiguous() or lse.dtype is not _F32):
            raise ValueError("lse: contiguous fp32 [tokens][query heads]")
        self._check(lib().sb_kv4_attention(self._h, cache.struct, q, qt, qh, heads, tokens, s, n, max_new, max_len,
                                           dim ** -0.5 if scale is None else scale, window, o, ot, oh, _dev(lse)))
        return out, lse

    # ---- rotary positions -------------------------------------------------------------------
    def rotary(self, table: RotaryTable, q: torch.Tensor, k: Optional[torch.Tensor] = None, starts: Optional[torch.Tensor] = None,
               lens: Optional[torch.Tensor] = None, max_new: Optional[int] = None, positions: Optional[torch.Tensor] = None, inverse: bool = False, out=None):
        """Turns q and, if given, k ([tokens][heads][dim], bf16 or fp32) by their positions: those of the requests' new tokens (starts, lens, max_new
        as in the cache calls; max_new None: any number of q's rows), or `positions`, int32 [tokens].  In place, or into `out` (a tensor for each); inverse: the way
        back of gradients.  Returns (q, k) as written."""
        dtype = q.dtype
        if dtype is not _BF16 and dtype is not _F32:
            raise TypeError("rotary: bf16 or fp32 tensors")
        if out is None:
            yq, yk = q, k
        elif isinstance(out, torch.Tensor):
            yq, yk = out, None
        else:
            yq, yk = out[0], out[1] if len(out) > 1 else None
        if (k is None) != (yk is None):
            if k is not None:
                raise ValueError("out: a tensor for q and, where it is given, one for k")
            yk = None
        tokens, _, dim = q.shape
        parts = _rotary_part(q, yq, tokens, dim, dtype)
        if k is not None:
            parts += _rotary_part(k, yk, tokens, dim, dtype)
        if positions is None:
            if starts is None or lens is None:
                raise ValueError("rotary: positions, or starts and lens")
            requests = lens.numel()
            if starts.dtype is not _I32 or lens.dtype is not _I32 or starts.numel() != requests + 1 or not starts.is_contiguous() or not lens.is_contiguous():
                raise ValueError("starts: contiguous int32 [requests + 1], lens: contiguous int32 [requests]")
            at, s, n = None, _dev(starts), _dev(lens)
            if max_new is None:
                max_new = tokens
        else:
            if starts is not None or lens is not None:
                raise ValueError("rotary: positions, or starts and lens")
            if positions.dtype is not _I32 or positions.shape != (tokens,) or not positions.is_contiguous():
                raise ValueError("positions: contiguous int32 [tokens]")
            requests, at, s, n = 0, _dev(positions), None, None
            if max_new is None:
                max_new = 0
        self._check(lib().sb_rotary(self._h, table.struct(inverse), parts, 1 if k is None else 2, dim, dtype is _F32, tokens, at, s, n,
                                    requests, max_new))
        return yq, yk

    # ---- low-rank adapters ------------------------------------------------------------------
    def lora_add(self, adapters: LoraAdapters, X: torch.Tensor, base: torch.Tensor, ids: torch.Tensor, starts: torch.Tensor, max_new: int,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """base (bf16 or fp32 [tokens][out]) plus what the requests' adapters make of X (bf16 [tokens][in]): request b has the rows starts[b] ..
        starts[b + 1] and the adapter ids[b] (-1: none).  In place, or into `out`."""
        tokens, inner, ldx = _mat(X)
        if out is None:
            out = base
        shape, dtype = (tokens, adapters.outer), base.dtype
        if inner != adapters.inner or base.shape != shape or out.shape != shape:
            raise ValueError("X: [tokens][in of the adapters], base and out: [tokens][out]")
        if dtype is not _BF16 and dtype is not _F32 or out.dtype is not dtype:
            raise TypeError("base and out: both bf16 or both fp32")
        ldb, one = base.stride()
        ldy, two = out.stride()
        if one != 1 and shape[1] > 1 or two != 1 and shape[1] > 1:
            raise ValueError("base and out: row-major")
        requests = ids.numel()
        if starts.dtype is not _I32 or ids.dtype is not _I32 or starts.numel() != requests + 1 or not starts.is_contiguous() or not ids.is_contiguous():
            raise ValueError("starts: contiguous int32 [requests + 1], ids: contiguous int32 [requests]")
        self._check(lib().sb_lora_add(self._h, adapters.struct, _dev(X), ldx, _dev(base), ldb, _dev(out), ldy, int(dtype is _F32), tokens,
                                      _dev(starts), _dev(ids), requests, max_new))
        return out


def checked_build() -> bool:
    """True if the loaded library is the bounds-checked build (-DSB_CHECKED)."""
    return bool(lib().sb_checked_build())


def calib_moments_noalloc(X: torch.Tensor, sumsq: Optional[torch.Tensor] = None,
                          accumulate: bool = False, scale: Optional[float] = None,
                          stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """sb_calib_moments_noalloc: second moments without a context and without any device
    allocation inside the library (fixed in-library scratch, K <= 65536).

    For callers that cannot allocate when they need the moments (device memory fully handed
    out at start-up, code under a caching allocator, latency-critical loops).  X's device
    must be current.  Calls share the scratch: do not let two of them overlap on the GPU.
    """
    T, K, ldx = _mat(X)
    if sumsq is None:
        sumsq = torch.empty(K, dtype=torch.float32, device=X.device)
        accumulate = False
    if scale is None:
        scale = 1.0 / max(T, 1)
    s = torch.cuda.current_stream(X.device) if stream is None else stream
    fn = lib().sb_calib_moments_noalloc
    st = fn(C.c_void_p(s.cuda_stream), _ptr(X), T, K, ldx, _ptr(sumsq, torch.float32),
            int(accumulate), float(scale))
    if st != SB_OK:
        raise SbError(st, "sb_calib_moments_noalloc failed (see stderr)")
    return sumsq
