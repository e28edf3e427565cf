"""ctypes binding of libmxq.so: same names as the C ABI, argument marshalling only.

torch is used for device memory and streams: tensors are passed as raw device pointers and
the current CUDA stream's handle.  Code and scale buffers are ``torch.uint8`` tensors.
"""
from __future__ import annotations

import ctypes
import importlib.util
import math
import os
import struct
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmxq.so")

F32, BF16 = 0, 1
FQ_DIRECT, FQ_VIA_ANCHOR = 0, 1

#: format name -> mxq_format enum value (include/mxq.h)
FORMATS = {
    "int8": 0, "int6": 1, "int4": 2, "e4m3": 3, "e3m2": 4, "e2m3": 5, "e2m1": 6,
    "int7": 7, "int5": 8, "int3": 9, "int2": 10, "e3m3": 11, "e2m2": 12,
}


class MxqError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s failed: %s" % (what, status_string(status)))


class _FqItem(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("n", ctypes.c_size_t)]


class _QItem(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("n", ctypes.c_size_t), ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class _DqItem(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("n", ctypes.c_size_t), ("dst", ctypes.c_void_p)]


class _Item(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("n", ctypes.c_size_t),
                ("out_codes", ctypes.c_void_p), ("out_scales", ctypes.c_void_p)]


class _PairItem(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("n", ctypes.c_size_t),
                ("out_codes1", ctypes.c_void_p), ("out_scales1", ctypes.c_void_p),
                ("out_codes2", ctypes.c_void_p), ("out_scales2", ctypes.c_void_p)]


class _TiledItem(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_size_t),
                ("cols", ctypes.c_size_t), ("out_codes", ctypes.c_void_p), ("out_tiled_scales", ctypes.c_void_p)]


class _MoeLayer(ctypes.Structure):
    _fields_ = [("up_codes", ctypes.c_void_p), ("up_scales", ctypes.c_void_p), ("down_codes", ctypes.c_void_p),
                ("down_scales", ctypes.c_void_p), ("hidden", ctypes.c_size_t), ("inner", ctypes.c_size_t),
                ("experts", ctypes.c_int), ("fmt", ctypes.c_int), ("block", ctypes.c_int)]


class _Cache(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("pages", ctypes.c_size_t), ("page", ctypes.c_int), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("fmt", ctypes.c_int), ("block", ctypes.c_int)]


class _Batch(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("starts", ctypes.c_void_p), ("batch", ctypes.c_size_t),
                ("width", ctypes.c_size_t)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_size_t), ("head_stride", ctypes.c_size_t)]


_lib: Optional[ctypes.CDLL] = None
_host = None            # the native module _mxq_host (csrc/host_calls.cpp): the plain case of the per-tensor calls

#: the entry points that _mxq_host calls
_HOST_CALLS = ("mxq_quantize", "mxq_slice_scale", "mxq_slice_scale_multi", "mxq_dequantize", "mxq_tiled_scales_bytes",
               "mxq_quantize_tiled", "mxq_slice_scale_tiled", "mxq_fake_quant", "mxq_fake_quant_bwd", "mxq_codes_bytes",
               "mxq_matmul", "mxq_quantize_matrix", "mxq_matrix_codes_bytes", "mxq_matrix_scales_bytes", "mxq_moe",
               "mxq_moe_workspace_bytes", "mxq_cache_write", "mxq_cache_read", "mxq_cache_attention", "mxq_cache_attention_workspace_bytes")


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load libmxq.so (built in-tree by ``python -m paper_2604_00529_b200.build``)."""
    global _lib, _host
    if _lib is not None:
        return _lib
    from .build import host_module_path
    if not os.path.exists(_LIB_PATH):
        raise ImportError("libmxq.so is not built: run `python -m paper_2604_00529_b200.build` "
                          "(there is no fallback path)")
    if _host is None:
        path = host_module_path()
        if not os.path.exists(path):
            raise ImportError("%s, the binding's module for this torch and Python, is not built: run "
                              "`python -m paper_2604_00529_b200.build`" % os.path.basename(path))
        spec = importlib.util.spec_from_file_location(__package__ + "._mxq_host", path)
        _host = importlib.util.module_from_spec(spec)
    L = ctypes.CDLL(_LIB_PATH)
    vp, sz, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    L.mxq_status_string.argtypes = [i]
    L.mxq_status_string.restype = ctypes.c_char_p
    L.mxq_format_bits.argtypes = [i]
    L.mxq_format_bits.restype = i
    L.mxq_codes_bytes.argtypes = [sz, i]
    L.mxq_codes_bytes.restype = sz
    L.mxq_scales_bytes.argtypes = [sz, i]
    L.mxq_scales_bytes.restype = sz
    L.mxq_block_supported.argtypes = [i]
    L.mxq_block_supported.restype = i
    L.mxq_quantize.argtypes = [vp, i, sz, i, i, vp, vp, vp]
    L.mxq_slice_scale.argtypes = [vp, vp, sz, i, i, i, vp, vp, vp]
    L.mxq_dequantize.argtypes = [vp, vp, sz, i, i, vp, i, vp]
    L.mxq_slice_scale_multi.argtypes = [vp, vp, sz, i, i, i, ctypes.POINTER(i), ctypes.POINTER(vp), ctypes.POINTER(vp), vp]
    L.mxq_slice_scale_multi.restype = i
    L.mxq_fake_quant.argtypes = [vp, i, sz, i, i, i, vp, vp]
    L.mxq_fake_quant_batched.argtypes = [ctypes.POINTER(_FqItem), i, i, i, i, i, vp]
    L.mxq_fake_quant_batched.restype = i
    L.mxq_quantize_batched.argtypes = [ctypes.POINTER(_QItem), i, i, i, i, vp]
    L.mxq_quantize_batched.restype = i
    L.mxq_dequantize_batched.argtypes = [ctypes.POINTER(_DqItem), i, i, i, i, vp]
    L.mxq_dequantize_batched.restype = i
    L.mxq_tiled_scales_bytes.argtypes = [sz, sz]
    L.mxq_tiled_scales_bytes.restype = sz
    L.mxq_tile_scales.argtypes = [vp, sz, sz, vp, vp]
    L.mxq_tile_scales.restype = i
    L.mxq_quantize_tiled.argtypes = [vp, i, sz, sz, i, i, vp, vp, vp]
    L.mxq_quantize_tiled.restype = i
    L.mxq_slice_scale_tiled.argtypes = [vp, vp, sz, sz, i, i, i, vp, vp, vp]
    L.mxq_slice_scale_tiled.restype = i
    L.mxq_slice_scale_tiled_batched.argtypes = [ctypes.POINTER(_TiledItem), i, i, i, i, vp]
    L.mxq_slice_scale_tiled_batched.restype = i
    L.mxq_fake_quant_bwd.argtypes = [vp, i, sz, vp, vp]
    L.mxq_slice_scale_batched.argtypes = [ctypes.POINTER(_Item), i, i, i, i, vp]
    L.mxq_slice_scale_pair_batched.argtypes = [ctypes.POINTER(_PairItem), i, i, i, i, i, vp]
    L.mxq_slice_scale_pair_batched.restype = i
    L.mxq_slice_scale_batched_static.argtypes = [ctypes.POINTER(_Item), i, i, i, i, vp]
    L.mxq_slice_scale_batched_static.restype = i
    L.mxq_matmul.argtypes = [vp, vp, vp, vp, sz, sz, sz, i, i, vp, i, vp]
    L.mxq_matmul.restype = i
    L.mxq_wait_status.argtypes = [i]
    L.mxq_wait_status.restype = i
    L.mxq_matrix_codes_bytes.argtypes = [sz, sz, i]
    L.mxq_matrix_codes_bytes.restype = sz
    L.mxq_matrix_scales_bytes.argtypes = [sz, sz, i]
    L.mxq_matrix_scales_bytes.restype = sz
    L.mxq_quantize_matrix.argtypes = [vp, i, sz, sz, i, i, vp, vp, vp, vp, vp]
    L.mxq_quantize_matrix.restype = i
    L.mxq_moe_workspace_bytes.argtypes = [sz, i, sz, i]
    L.mxq_moe_workspace_bytes.restype = sz
    L.mxq_moe.argtypes = [ctypes.POINTER(_MoeLayer), vp, i, vp, sz, i, i, vp, vp, sz, vp]
    L.mxq_moe.restype = i
    cache, batch, rows = ctypes.POINTER(_Cache), ctypes.POINTER(_Batch), ctypes.POINTER(_Rows)
    L.mxq_cache_write.argtypes = [cache, batch, rows, rows, i, sz, vp]
    L.mxq_cache_write.restype = i
    L.mxq_cache_read.argtypes = [cache, batch, sz, vp, vp, i, vp]
    L.mxq_cache_read.restype = i
    L.mxq_cache_attention_workspace_bytes.argtypes = [cache, batch, i, i, sz]
    L.mxq_cache_attention_workspace_bytes.restype = sz
    L.mxq_cache_attention.argtypes = [cache, batch, rows, i, i, sz, ctypes.c_float, i, sz, vp, vp, vp, sz, vp]
    L.mxq_cache_attention.restype = i
    for name in ("mxq_quantize", "mxq_slice_scale", "mxq_dequantize", "mxq_fake_quant", "mxq_fake_quant_bwd",
                 "mxq_slice_scale_batched"):
        getattr(L, name).restype = i
    _host.bind({name: ctypes.cast(getattr(L, name), vp).value for name in _HOST_CALLS}, FORMATS, torch.nn.Parameter,
               MxqError)
    _lib = L
    return L


def status_string(status: int) -> str:
    return load_library().mxq_status_string(int(status)).decode()


def format_bits(fmt: str) -> int:
    return load_library().mxq_format_bits(FORMATS[fmt])


def codes_bytes(n: int, fmt: str) -> int:
    return load_library().mxq_codes_bytes(n, FORMATS[fmt])


def scales_bytes(n: int, block: int = 32) -> int:
    return load_library().mxq_scales_bytes(n, block)


def _dtype_id(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("mxq tensors are float32 or bfloat16, got %s" % t.dtype)


def _dev(t: torch.Tensor, what: str) -> int:
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor (libmxq has no CPU path)" % what)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    return t.data_ptr()


# torch.cuda.current_stream() builds a Stream object per call (about 3 us, more than the launch itself);
# the raw handle of the current device's current stream comes straight from the C layer when torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise MxqError(rc, what)


def quantize(src: torch.Tensor, fmt: str, block: int = 32, codes: Optional[torch.Tensor] = None,
             scales: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """mxq_quantize: returns (packed codes uint8[n*bits/8], scales uint8[n/block])."""
    L = _lib or load_library()
    out = _host.quantize(src, fmt, block, codes, scales, stream)
    if out is not None:
        return out
    n = src.numel()
    if codes is None:
        codes = torch.empty(codes_bytes(n, fmt), dtype=torch.uint8, device=src.device)
    if scales is None:
        scales = torch.empty(n // block if block > 0 else 0, dtype=torch.uint8, device=src.device)
    _check(L.mxq_quantize(_dev(src, "src"), _dtype_id(src), n, FORMATS[fmt], block, _dev(codes, "codes"),
                          _dev(scales, "scales"), _stream(stream)), "mxq_quantize")
    return codes, scales


def slice_scale(codes: torch.Tensor, scales: torch.Tensor, n: int, src_fmt: str, dst_fmt: str, block: int = 32,
                out_codes: Optional[torch.Tensor] = None, out_scales: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """mxq_slice_scale: anchor codes + scales -> lower-format codes + scales."""
    L = _lib or load_library()
    out = _host.slice_scale(codes, scales, n, src_fmt, dst_fmt, block, out_codes, out_scales, stream)
    if out is not None:
        return out
    if out_codes is None:
        out_codes = torch.empty(codes_bytes(n, dst_fmt), dtype=torch.uint8, device=codes.device)
    if out_scales is None:
        out_scales = torch.empty(n // block if block > 0 else 0, dtype=torch.uint8, device=codes.device)
    _check(L.mxq_slice_scale(_dev(codes, "codes"), _dev(scales, "scales"), n, block, FORMATS[src_fmt],
                             FORMATS[dst_fmt], _dev(out_codes, "out_codes"), _dev(out_scales, "out_scales"),
                             _stream(stream)), "mxq_slice_scale")
    return out_codes, out_scales


def slice_scale_multi(codes: torch.Tensor, scales: torch.Tensor, n: int, src_fmt: str, dst_fmts: Sequence[str],
                      block: int = 32, outs: Optional[Sequence[Tuple[torch.Tensor, torch.Tensor]]] = None, stream=None):
    """mxq_slice_scale_multi: one anchor -> several lower formats; returns [(codes, scales), ...]."""
    L = _lib or load_library()
    made = _host.slice_scale_multi(codes, scales, n, src_fmt, dst_fmts, block, outs, stream)
    if made is not None:
        return made
    k = len(dst_fmts)
    if outs is None:
        outs = [(torch.empty(codes_bytes(n, f), dtype=torch.uint8, device=codes.device),
                 torch.empty(n // block if block > 0 else 0, dtype=torch.uint8, device=codes.device)) for f in dst_fmts]
    fm = (ctypes.c_int * k)(*[FORMATS[f] for f in dst_fmts])
    oc = (ctypes.c_void_p * k)(*[_dev(c, "out_codes") for c, _ in outs])
    os_ = (ctypes.c_void_p * k)(*[_dev(s, "out_scales") for _, s in outs])
    _check(L.mxq_slice_scale_multi(_dev(codes, "codes"), _dev(scales, "scales"), n, block, FORMATS[src_fmt], k, fm, oc,
                                   os_, _stream(stream)), "mxq_slice_scale_multi")
    return list(outs)


def dequantize(codes: torch.Tensor, scales: torch.Tensor, n: int, fmt: str, block: int = 32,
               dtype: torch.dtype = torch.float32, dst: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """mxq_dequantize: V^ = X P as float32 or bfloat16."""
    L = _lib or load_library()
    out = _host.dequantize(codes, scales, n, fmt, block, dtype, dst, stream)
    if out is not None:
        return out
    if dst is None:
        dst = torch.empty(n, dtype=dtype, device=codes.device)
    _check(L.mxq_dequantize(_dev(codes, "codes"), _dev(scales, "scales"), n, FORMATS[fmt], block, _dev(dst, "dst"),
                            _dtype_id(dst), _stream(stream)), "mxq_dequantize")
    return dst


def tiled_scales_bytes(rows: int, kblocks: int) -> int:
    return load_library().mxq_tiled_scales_bytes(rows, kblocks)


def tile_scales(scales: torch.Tensor, rows: int, kblocks: int, tiled: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
    """mxq_tile_scales: row-major [rows, kblocks] scale bytes -> the 128 x 4 tiled order a block-scaled
    tensor-core matmul reads."""
    L = load_library()
    if tiled is None:
        tiled = torch.empty(tiled_scales_bytes(rows, kblocks), dtype=torch.uint8, device=scales.device)
    _check(L.mxq_tile_scales(_dev(scales, "scales"), rows, kblocks, _dev(tiled, "tiled"), _stream(stream)),
           "mxq_tile_scales")
    return tiled


def quantize_tiled(src: torch.Tensor, fmt: str, block: int = 32, codes: Optional[torch.Tensor] = None,
                   tiled_scales: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """mxq_quantize_tiled: a 2-D [rows, cols] tensor -> (packed codes, scale bytes in the 128 x 4 tiled order)."""
    L = _lib or load_library()
    out = _host.quantize_tiled(src, fmt, block, codes, tiled_scales, stream)
    if out is not None:
        return out
    if src.dim() != 2:
        raise ValueError("quantize_tiled takes a [rows, cols] matrix")
    rows, cols = src.shape
    if codes is None:
        codes = torch.empty(codes_bytes(rows * cols, fmt), dtype=torch.uint8, device=src.device)
    if tiled_scales is None:
        tiled_scales = torch.empty(tiled_scales_bytes(rows, cols // 32), dtype=torch.uint8, device=src.device)
    _check(L.mxq_quantize_tiled(_dev(src, "src"), _dtype_id(src), rows, cols, FORMATS[fmt], block, _dev(codes, "codes"),
                                _dev(tiled_scales, "tiled_scales"), _stream(stream)), "mxq_quantize_tiled")
    return codes, tiled_scales


def slice_scale_tiled(codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int, src_fmt: str, dst_fmt: str,
                      block: int = 32, out_codes: Optional[torch.Tensor] = None,
                      out_tiled_scales: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """mxq_slice_scale_tiled: anchor codes + plain scales of a [rows, cols] matrix -> lower-format codes and
    scale bytes in the 128 x 4 tiled order."""
    L = _lib or load_library()
    out = _host.slice_scale_tiled(codes, scales, rows, cols, src_fmt, dst_fmt, block, out_codes, out_tiled_scales, stream)
    if out is not None:
        return out
    if out_codes is None:
        out_codes = torch.empty(codes_bytes(rows * cols, dst_fmt), dtype=torch.uint8, device=codes.device)
    if out_tiled_scales is None:
        out_tiled_scales = torch.empty(tiled_scales_bytes(rows, cols // 32), dtype=torch.uint8, device=codes.device)
    _check(L.mxq_slice_scale_tiled(_dev(codes, "codes"), _dev(scales, "scales"), rows, cols, block, FORMATS[src_fmt],
                                   FORMATS[dst_fmt], _dev(out_codes, "out_codes"),
                                   _dev(out_tiled_scales, "out_tiled_scales"), _stream(stream)), "mxq_slice_scale_tiled")
    return out_codes, out_tiled_scales


def fake_quant(src: torch.Tensor, fmt: str, block: int = 32, mode: int = FQ_DIRECT,
               dst: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """mxq_fake_quant: quantize-dequantize in one pass (dst may be src)."""
    L = _lib or load_library()
    out = _host.fake_quant(src, fmt, block, mode, dst, stream)
    if out is not None:
        return out
    if dst is None:
        dst = torch.empty_like(src)
    _check(L.mxq_fake_quant(_dev(src, "src"), _dtype_id(src), src.numel(), FORMATS[fmt], block, mode,
                            _dev(dst, "dst"), _stream(stream)), "mxq_fake_quant")
    return dst


class FqTable:
    """A marshalled mxq_fq_item array for tensors that persist (e.g. a model's weights): build it once
    with ``make_fq_items`` and pass it to ``fake_quant_batched`` every step."""

    def __init__(self, pairs):
        self.tensors = [(s, d if d is not None else s) for s, d in pairs]
        if not self.tensors:
            raise ValueError("no tensors")
        self.dtype = _dtype_id(self.tensors[0][0])
        self.array = (_FqItem * len(self.tensors))()
        for k, (s, d) in enumerate(self.tensors):
            if _dtype_id(s) != self.dtype or d.dtype != s.dtype or d.numel() != s.numel():
                raise TypeError("all tensors of a batch share one dtype; dst matches src")
            self.array[k] = _FqItem(_dev(s, "src"), _dev(d, "dst"), s.numel())

    def __len__(self):
        return len(self.tensors)


def make_fq_items(pairs) -> FqTable:
    """Marshal (src, dst) tensor pairs (dst None = in place) into an mxq_fq_item array."""
    return FqTable(pairs)


def fake_quant_batched(pairs, fmt: str, block: int = 32, mode: int = FQ_DIRECT, stream=None) -> None:
    """mxq_fake_quant_batched over (src, dst) pairs or an FqTable made from them."""
    L = load_library()
    table = pairs if isinstance(pairs, FqTable) else FqTable(pairs)
    _check(L.mxq_fake_quant_batched(table.array, len(table), table.dtype, FORMATS[fmt], block, mode, _stream(stream)),
           "mxq_fake_quant_batched")


class QTable:
    """A marshalled mxq_q_item array over (src, codes, scales) tensor triples that persist (keeps them alive)."""

    def __init__(self, triples):
        self.tensors = list(triples)
        if not self.tensors:
            raise ValueError("no tensors")
        self.dtype = _dtype_id(self.tensors[0][0])
        self.array = (_QItem * len(self.tensors))()
        for k, (src, codes, scales) in enumerate(self.tensors):
            if _dtype_id(src) != self.dtype:
                raise TypeError("all tensors of a batch share one dtype")
            self.array[k] = _QItem(_dev(src, "src"), src.numel(), _dev(codes, "codes"), _dev(scales, "scales"))

    def __len__(self):
        return len(self.tensors)


def make_q_items(triples) -> QTable:
    """Marshal (src, codes, scales) tensor triples into an mxq_q_item array."""
    return QTable(triples)


def quantize_batched(triples, fmt: str, block: int = 32, stream=None) -> None:
    """mxq_quantize_batched over (src, codes, scales) triples or a QTable made from them."""
    L = load_library()
    table = triples if isinstance(triples, QTable) else QTable(triples)
    _check(L.mxq_quantize_batched(table.array, len(table), table.dtype, FORMATS[fmt], block, _stream(stream)),
           "mxq_quantize_batched")


class DqTable:
    """A marshalled mxq_dq_item array over (codes, scales, n, dst) tuples that persist (keeps them alive)."""

    def __init__(self, items):
        self.tensors = list(items)
        if not self.tensors:
            raise ValueError("no tensors")
        self.dtype = _dtype_id(self.tensors[0][3])
        self.array = (_DqItem * len(self.tensors))()
        for k, (codes, scales, n, dst) in enumerate(self.tensors):
            if _dtype_id(dst) != self.dtype or dst.numel() != n:
                raise TypeError("all outputs of a batch share one dtype and hold n elements")
            self.array[k] = _DqItem(_dev(codes, "codes"), _dev(scales, "scales"), n, _dev(dst, "dst"))

    def __len__(self):
        return len(self.tensors)


def make_dq_items(items) -> DqTable:
    """Marshal (codes, scales, n, dst) tuples into an mxq_dq_item array."""
    return DqTable(items)


def dequantize_batched(items, fmt: str, block: int = 32, stream=None) -> None:
    """mxq_dequantize_batched over (codes, scales, n, dst) tuples or a DqTable made from them."""
    L = load_library()
    table = items if isinstance(items, DqTable) else DqTable(items)
    _check(L.mxq_dequantize_batched(table.array, len(table), FORMATS[fmt], block, table.dtype, _stream(stream)),
           "mxq_dequantize_batched")


def fake_quant_bwd(grad_out: torch.Tensor, grad_in: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """mxq_fake_quant_bwd: straight-through gradient (identity)."""
    L = _lib or load_library()
    out = _host.fake_quant_bwd(grad_out, grad_in, stream)
    if out is not None:
        return out
    if grad_in is None:
        grad_in = torch.empty_like(grad_out)
    _check(L.mxq_fake_quant_bwd(_dev(grad_out, "grad_out"), _dtype_id(grad_out), grad_out.numel(),
                                _dev(grad_in, "grad_in"), _stream(stream)), "mxq_fake_quant_bwd")
    return grad_in


#: the calls that can be prepared, in the order of _mxq_host.run_prepared's kinds
_PREPARED = ("mxq_quantize", "mxq_slice_scale", "mxq_dequantize", "mxq_fake_quant", "mxq_fake_quant_bwd")


class PreparedCall:
    """One C-ABI call with its arguments already marshalled, for buffers that persist (a model's
    weights and their code buffers): ``prepare_*`` checks and converts the arguments once, calling the
    object enqueues the operation on the current stream (or on ``stream``).  It keeps the tensors alive.
    Per call this leaves the stream lookup and the launch."""

    __slots__ = ("fn", "args", "what", "keep", "kind", "packed")

    def __init__(self, fn, args, what, keep):
        self.fn, self.args, self.what, self.keep = fn, args, what, keep
        self.kind = _PREPARED.index(what)
        try:
            self.packed = struct.pack("9q", *args, *(0,) * (9 - len(args)))
        except struct.error:
            self.packed = None          # no 64-bit integers: ctypes converts or refuses them at the call

    def __call__(self, stream=None) -> None:
        if stream is None and self.packed is not None:
            rc = _host.run_prepared(self.kind, self.packed)
        else:
            rc = self.fn(*self.args, _stream(stream))
        if rc != 0:
            raise MxqError(rc, self.what)


def prepare_quantize(src: torch.Tensor, fmt: str, block: int, codes: torch.Tensor, scales: torch.Tensor) -> PreparedCall:
    """mxq_quantize(src -> codes, scales) as a PreparedCall."""
    L = load_library()
    return PreparedCall(L.mxq_quantize, (_dev(src, "src"), _dtype_id(src), src.numel(), FORMATS[fmt], block,
                                         _dev(codes, "codes"), _dev(scales, "scales")), "mxq_quantize",
                        (src, codes, scales))


def prepare_slice_scale(codes: torch.Tensor, scales: torch.Tensor, n: int, src_fmt: str, dst_fmt: str, block: int,
                        out_codes: torch.Tensor, out_scales: torch.Tensor) -> PreparedCall:
    """mxq_slice_scale as a PreparedCall."""
    L = load_library()
    return PreparedCall(L.mxq_slice_scale, (_dev(codes, "codes"), _dev(scales, "scales"), n, block, FORMATS[src_fmt],
                                            FORMATS[dst_fmt], _dev(out_codes, "out_codes"),
                                            _dev(out_scales, "out_scales")), "mxq_slice_scale",
                        (codes, scales, out_codes, out_scales))


def prepare_dequantize(codes: torch.Tensor, scales: torch.Tensor, n: int, fmt: str, block: int,
                       dst: torch.Tensor) -> PreparedCall:
    """mxq_dequantize as a PreparedCall."""
    L = load_library()
    return PreparedCall(L.mxq_dequantize, (_dev(codes, "codes"), _dev(scales, "scales"), n, FORMATS[fmt], block,
                                           _dev(dst, "dst"), _dtype_id(dst)), "mxq_dequantize", (codes, scales, dst))


def prepare_fake_quant(src: torch.Tensor, fmt: str, block: int, mode: int, dst: torch.Tensor) -> PreparedCall:
    """mxq_fake_quant as a PreparedCall."""
    L = load_library()
    return PreparedCall(L.mxq_fake_quant, (_dev(src, "src"), _dtype_id(src), src.numel(), FORMATS[fmt], block, mode,
                                           _dev(dst, "dst")), "mxq_fake_quant", (src, dst))


def prepare_fake_quant_bwd(grad_out: torch.Tensor, grad_in: torch.Tensor) -> PreparedCall:
    """mxq_fake_quant_bwd as a PreparedCall."""
    L = load_library()
    return PreparedCall(L.mxq_fake_quant_bwd, (_dev(grad_out, "grad_out"), _dtype_id(grad_out), grad_out.numel(),
                                               _dev(grad_in, "grad_in")), "mxq_fake_quant_bwd", (grad_out, grad_in))


class _FakeQuantSTE(torch.autograd.Function):
    """Eq. 6 inside autograd: forward is mxq_fake_quant, backward the straight-through estimator."""

    @staticmethod
    def forward(ctx, x, fmt, block, mode, copy_grad):
        ctx.copy_grad = copy_grad
        return fake_quant(x.detach(), fmt, block, mode)

    @staticmethod
    def backward(ctx, grad_out):
        # identity: the incoming gradient itself, or a copy of it made by mxq_fake_quant_bwd
        g = fake_quant_bwd(grad_out.contiguous()) if ctx.copy_grad else grad_out
        return g, None, None, None, None


def fake_quant_ste(x: torch.Tensor, fmt: str, block: int = 32, mode: int = FQ_VIA_ANCHOR,
                   copy_grad: bool = False) -> torch.Tensor:
    """W_t of Eq. 6 as a differentiable function of W: the value is ``fake_quant(x, fmt, block, mode)``,
    the gradient passes straight through (``copy_grad`` hands autograd a fresh copy instead of the
    incoming tensor)."""
    if _lib is None:
        load_library()
    y = _host.fake_quant_ste(x, fmt, block, mode, copy_grad)
    return y if y is not None else _FakeQuantSTE.apply(x, fmt, block, mode, copy_grad)


class ItemTable:
    """A marshalled mxq_ss_item array: build it once with ``make_items`` for buffers that persist and
    pass it to ``slice_scale_batched`` as often as needed (it keeps the tensors alive)."""

    def __init__(self, items):
        self.tensors = list(items)
        self.array = (_Item * len(self.tensors))()
        for k, (c, s, n, oc, os_) in enumerate(self.tensors):
            self.array[k] = _Item(_dev(c, "codes"), _dev(s, "scales"), n, _dev(oc, "out_codes"), _dev(os_, "out_scales"))

    def __len__(self):
        return len(self.tensors)


def make_items(items: Sequence[Tuple[torch.Tensor, torch.Tensor, int, torch.Tensor, torch.Tensor]]) -> ItemTable:
    """Marshal (codes, scales, n, out_codes, out_scales) tuples into an mxq_ss_item array."""
    return ItemTable(items)


def slice_scale_batched(items, src_fmt: str, dst_fmt: str, block: int = 32, stream=None) -> None:
    """mxq_slice_scale_batched over (codes, scales, n, out_codes, out_scales) tuples, or over an
    ItemTable made from them."""
    L = load_library()
    table = items if isinstance(items, ItemTable) else ItemTable(items)
    _check(L.mxq_slice_scale_batched(table.array, len(table), block, FORMATS[src_fmt], FORMATS[dst_fmt],
                                     _stream(stream)), "mxq_slice_scale_batched")


class PairItemTable:
    """A marshalled mxq_ss_pair_item array over (codes, scales, n, out_codes1, out_scales1, out_codes2,
    out_scales2) tuples that persist (keeps the tensors alive)."""

    def __init__(self, items):
        self.tensors = list(items)
        self.array = (_PairItem * len(self.tensors))()
        for k, (c, s, n, c1, s1, c2, s2) in enumerate(self.tensors):
            self.array[k] = _PairItem(_dev(c, "codes"), _dev(s, "scales"), n, _dev(c1, "out_codes1"), _dev(s1, "out_scales1"),
                                      _dev(c2, "out_codes2"), _dev(s2, "out_scales2"))

    def __len__(self):
        return len(self.tensors)


def make_pair_items(items) -> PairItemTable:
    """Marshal (codes, scales, n, out_codes1, out_scales1, out_codes2, out_scales2) tuples into an mxq_ss_pair_item array."""
    return PairItemTable(items)


def slice_scale_pair_batched(items, src_fmt: str, dst_fmt1: str, dst_fmt2: str, block: int = 32, stream=None) -> None:
    """mxq_slice_scale_pair_batched: every anchor of a set of tensors to two lower formats, one read of the anchor."""
    L = load_library()
    table = items if isinstance(items, PairItemTable) else PairItemTable(items)
    _check(L.mxq_slice_scale_pair_batched(table.array, len(table), block, FORMATS[src_fmt], FORMATS[dst_fmt1],
                                          FORMATS[dst_fmt2], _stream(stream)), "mxq_slice_scale_pair_batched")


class TiledItemTable:
    """A marshalled mxq_ss_tiled_item array (keeps the tensors alive), for buffers that persist."""

    def __init__(self, items):
        self.tensors = list(items)
        self.array = (_TiledItem * len(self.tensors))()
        for k, (c, s, rows, cols, oc, ot) in enumerate(self.tensors):
            self.array[k] = _TiledItem(_dev(c, "codes"), _dev(s, "scales"), rows, cols, _dev(oc, "out_codes"),
                                       _dev(ot, "out_tiled_scales"))

    def __len__(self):
        return len(self.tensors)


def make_tiled_items(items) -> TiledItemTable:
    """Marshal (codes, scales, rows, cols, out_codes, out_tiled_scales) tuples into an mxq_ss_tiled_item array."""
    return TiledItemTable(items)


def slice_scale_tiled_batched(items, src_fmt: str, dst_fmt: str, block: int = 32, stream=None) -> None:
    """mxq_slice_scale_tiled_batched over (codes, scales, rows, cols, out_codes, out_tiled_scales) tuples or a
    TiledItemTable made from them."""
    L = load_library()
    table = items if isinstance(items, TiledItemTable) else TiledItemTable(items)
    _check(L.mxq_slice_scale_tiled_batched(table.array, len(table), block, FORMATS[src_fmt], FORMATS[dst_fmt],
                                           _stream(stream)), "mxq_slice_scale_tiled_batched")


#: largest item count mxq_slice_scale_batched_static accepts (MXQ_STATIC_BATCH_MAX in include/mxq.h)
STATIC_BATCH_MAX = 1024


def slice_scale_batched_static(items: Sequence[Tuple[torch.Tensor, torch.Tensor, int, torch.Tensor, torch.Tensor]],
                               src_fmt: str, dst_fmt: str, block: int = 32, stream=None) -> None:
    """mxq_slice_scale_batched_static: slice_scale_batched for callers that may not allocate device
    memory (a process whose own pool owns all of HBM, or a loop that cannot afford the device-wide
    stall of cudaMalloc).  The item table is a fixed array inside libmxq, so at most STATIC_BATCH_MAX
    items fit, and calls that can overlap on the GPU must not share a device.  The marshalling here
    builds one small ctypes array on the host and touches no torch allocator."""
    L = load_library()
    arr = (_Item * len(items))()
    for k, (c, s, n, oc, os_) in enumerate(items):
        arr[k] = _Item(_dev(c, "codes"), _dev(s, "scales"), n, _dev(oc, "out_codes"), _dev(os_, "out_scales"))
    _check(L.mxq_slice_scale_batched_static(arr, len(items), block, FORMATS[src_fmt], FORMATS[dst_fmt],
                                            _stream(stream)), "mxq_slice_scale_batched_static")


# ---- products that read the codes -----------------------------------------------------------------------------


def _operand(t: torch.Tensor, what: str, nbytes: int, device: torch.device) -> int:
    """The pointer of a code or scale buffer of at least `nbytes` bytes on `device`."""
    if t.dtype != torch.uint8:
        raise TypeError("%s must be uint8, got %s" % (what, t.dtype))
    if t.numel() < nbytes:
        raise ValueError("%s holds %d bytes, the operation takes %d" % (what, t.numel(), nbytes))
    return _on(t, what, device)


def _on(t: torch.Tensor, what: str, device: torch.device) -> int:
    p = _dev(t, what)
    if t.device != device:
        raise ValueError("%s is on %s, the other tensors on %s" % (what, t.device, device))
    return p


class _Place:
    """Makes `device` current and the work's stream (None: the device's current one) the allocator's while a call is put together:
    temporary and result buffers then belong to the stream that uses them."""

    __slots__ = ("device", "stream", "inner")

    def __init__(self, device, stream):
        self.device, self.stream, self.inner = device, stream, None

    def __enter__(self):
        if self.stream is not None:
            s = self.stream
            if not hasattr(s, "cuda_stream"):   # a handle; torch has no stream of the handle 1 (cudaStreamLegacy), which is the default one
                s = torch.cuda.ExternalStream(0 if int(s) == 1 else int(s), device=self.device)
            if s.device != self.device:
                raise ValueError("the stream is on %s, the tensors on %s" % (s.device, self.device))
            self.inner = torch.cuda.stream(s)
        elif self.device.index != torch.cuda.current_device():
            self.inner = torch.cuda.device(self.device)
        if self.inner is not None:
            self.inner.__enter__()

    def __exit__(self, *exc):
        if self.inner is not None:
            self.inner.__exit__(*exc)


def matmul(a_codes: torch.Tensor, a_scales: torch.Tensor, b_codes: torch.Tensor, b_scales: torch.Tensor, m: int, n: int, k: int,
           fmt: str = "e4m3", block: int = 32, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
           stream=None) -> torch.Tensor:
    """mxq_matmul: A^ B^T of two quantized operands [m, k] and [n, k] (``quantize``'s codes and scales), as [m, n] of
    ``dtype`` (``out``'s where it is given)."""
    L = _lib or load_library()
    made = _host.matmul(a_codes, a_scales, b_codes, b_scales, m, n, k, fmt, block, dtype, out, stream)
    if made is not None:
        return made
    dev = a_codes.device
    sizes = (m * k, m * k // block, n * k, n * k // block) if block > 0 and min(m, n, k) >= 0 else (0, 0, 0, 0)
    if min(m, n, k) < 0:
        raise ValueError("negative size")
    ptrs = [_operand(t, what, size, dev) for t, what, size in zip((a_codes, a_scales, b_codes, b_scales),
                                                                 ("a_codes", "a_scales", "b_codes", "b_scales"), sizes)]
    with _Place(dev, stream):
        if out is None:
            out = torch.empty(m, n, dtype=dtype, device=dev)
        elif out.numel() != m * n:
            raise ValueError("out holds %d elements, the product %d" % (out.numel(), m * n))
        _check(L.mxq_matmul(*ptrs, m, n, k, FORMATS[fmt], block, _on(out, "out", dev), _dtype_id(out), _stream(None)), "mxq_matmul")
    return out


def quantize_matrix(src: torch.Tensor, fmt: str = "e4m3", block: int = 32, rows: bool = True, cols: bool = True, stream=None):
    """mxq_quantize_matrix: a 2-D tensor -> (codes, scales, codes_t, scales_t), its quantization along the rows and that of its
    transpose, rows padded with zeros to whole blocks; ``rows=False`` / ``cols=False`` leave one of them out (None)."""
    L = _lib or load_library()
    made = _host.quantize_matrix(src, fmt, block, rows, cols, stream)
    if made is not None:
        return made
    if src.dim() != 2:
        raise ValueError("quantize_matrix takes a [rows, cols] matrix")
    r, c = src.shape
    p, dt = _dev(src, "src"), _dtype_id(src)
    with _Place(src.device, stream):
        got = []
        for wanted, x, y in ((rows, r, c), (cols, c, r)):
            if wanted:
                got += [torch.empty(L.mxq_matrix_codes_bytes(x, y, block), dtype=torch.uint8, device=src.device),
                        torch.empty(L.mxq_matrix_scales_bytes(x, y, block), dtype=torch.uint8, device=src.device)]
            else:
                got += [None, None]
        _check(L.mxq_quantize_matrix(p, dt, r, c, FORMATS[fmt], block, *[None if t is None else t.data_ptr() for t in got],
                                     _stream(None)), "mxq_quantize_matrix")
    return tuple(got)


def _up(v: int, block: int) -> int:
    return -(-v // block) * block


def _placed(t: torch.Tensor) -> torch.Tensor:
    """t, contiguous and at an address that the kernels take, a multiple of 32: itself where it is both already."""
    t = t.contiguous()
    return t.clone(memory_format=torch.contiguous_format) if t.data_ptr() % 32 else t


class _Once(torch.autograd.Function):
    """The gradients of a layer that has no second derivative: themselves, and an error where they are differentiated."""

    @staticmethod
    def forward(ctx, *grads):
        return tuple(None if g is None else g.clone() for g in grads)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("linear_ste can be differentiated once only")


class _LinearSTE(torch.autograd.Function):
    """y = Q(x) Q(w)^T; backward dx = Q(dy) Q(w^T)^T and dw = Q(dy^T) Q(x^T)^T, the quantizers passed straight through."""

    @staticmethod
    def forward(ctx, x, w, block):
        m, k, n = x.shape[0], x.shape[1], w.shape[0]
        need_x, need_w = ctx.needs_input_grad[:2]
        xc, xs, xct, xst = quantize_matrix(_placed(x), "e4m3", block, cols=need_w)
        wc, ws, wct, wst = quantize_matrix(_placed(w), "e4m3", block, cols=need_x)
        ctx.save_for_backward(xct, xst, wct, wst)
        ctx.sizes, ctx.block, ctx.dtypes = (m, n, k), block, (x.dtype, w.dtype)
        return matmul(xc, xs, wc, ws, m, n, _up(k, block), "e4m3", block, x.dtype)

    @staticmethod
    def backward(ctx, dy):
        xct, xst, wct, wst = ctx.saved_tensors
        (m, n, k), block = ctx.sizes, ctx.block
        need_x, need_w = ctx.needs_input_grad[:2]
        with torch.no_grad():
            dc, ds, dct, dst = quantize_matrix(_placed(dy), "e4m3", block, rows=need_x, cols=need_w)
            dx = matmul(dc, ds, wct, wst, m, k, _up(n, block), "e4m3", block, ctx.dtypes[0]) if need_x else None
            dw = matmul(dct, dst, xct, xst, n, k, _up(m, block), "e4m3", block, ctx.dtypes[1]) if need_w else None
        if torch.is_grad_enabled():         # (create_graph: dx depends on w, dw on x, even for a constant dy)
            dx, dw = _Once.apply(*[None if g is None else g.requires_grad_() for g in (dx, dw)])
        return dx, dw, None


def linear_ste(x: torch.Tensor, w: torch.Tensor, block: int = 32) -> torch.Tensor:
    """A linear layer whose three products run on MXFP8 E4M3 operands, differentiable: y = Q(x) Q(w)^T for x [..., k] and
    w [n, k] (float32 or bfloat16), with dx = Q(dy) Q(w^T)^T and dw = Q(dy^T) Q(x^T)^T, each operand quantized in blocks
    along the dimension that its product sums over and the quantizers passed straight through.  Any sizes, strides and offsets (what
    is not contiguous at an address that is a multiple of 32 is copied first); y and dx have x's type, dw has w's.  The backward pass
    keeps the transposes' codes (a byte per element), not x and w.  There is no second derivative: gradients taken with create_graph raise
    where they are differentiated.  Under vmap, torch.func's derivatives and forward-mode derivatives it raises; jit.trace
    records it as one call."""
    if _lib is None:
        load_library()
    made = _host.linear_ste(x, w, block)
    if made is not None:
        return made
    if w.dim() != 2 or x.dim() < 1 or x.shape[-1] != w.shape[1]:
        raise ValueError("linear_ste takes x [..., k] and w [n, k], got %s and %s" % (tuple(x.shape), tuple(w.shape)))
    if block not in (32, 64, 128):
        raise MxqError(-3, "linear_ste")
    for t, what in ((x, "x"), (w, "w")):
        _dtype_id(t)
        if not t.is_cuda or t.device != x.device:
            raise ValueError("%s must be a CUDA tensor on x's device (libmxq has no CPU path)" % what)
    y = _LinearSTE.apply(x.reshape(math.prod(x.shape[:-1]), x.shape[-1]), w, block)
    return y.view(*x.shape[:-1], w.shape[0])


#: limits of ``moe`` (MXQ_MOE_*_MAX in include/mxq.h)
MOE_TOKENS_MAX, MOE_EXPERTS_MAX, MOE_TOP_K_MAX = 64, 512, 16


def moe_workspace_bytes(tokens: int, top_k: int, inner: int, dtype: torch.dtype = torch.bfloat16) -> int:
    return load_library().mxq_moe_workspace_bytes(tokens, top_k, inner, F32 if dtype == torch.float32 else BF16)


def moe(x: torch.Tensor, logits: torch.Tensor, up_codes: torch.Tensor, up_scales: torch.Tensor, down_codes: torch.Tensor,
        down_scales: torch.Tensor, inner: int, top_k: int, fmt: str, block: int = 32, renormalize: bool = True,
        out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """mxq_moe: a mixture-of-experts layer for up to MOE_TOKENS_MAX tokens x [tokens, hidden] with the router's float32 logits
    [tokens, experts] over experts held as codes: up matrices [experts, 2 * inner, hidden] (gate rows first) and
    down matrices [experts, hidden, inner], as ``quantize`` writes them.  ``workspace`` (uint8, ``moe_workspace_bytes``) saves
    the allocation of one per call; calls that can overlap on the GPU must not share it.  For serving: the result has no gradient,
    whatever x and the logits require."""
    L = _lib or load_library()
    made = _host.moe(x, logits, up_codes, up_scales, down_codes, down_scales, inner, top_k, fmt, block, renormalize, out, workspace, stream)
    if made is not None:
        return made
    if x.dim() != 2 or logits.dim() != 2 or logits.shape[0] != x.shape[0]:
        raise ValueError("moe takes x [tokens, hidden] and logits [tokens, experts]")
    if logits.dtype != torch.float32:
        raise TypeError("logits are float32, got %s" % logits.dtype)
    (tokens, hidden), experts, dev, dt = x.shape, logits.shape[1], x.device, _dtype_id(x)
    weights = experts * hidden * max(inner, 0)
    per = block if block > 0 else 1
    ptrs = [_operand(t, what, size, dev) for t, what, size in
            ((up_codes, "up_codes", codes_bytes(2 * weights, fmt)), (up_scales, "up_scales", 2 * weights // per),
             (down_codes, "down_codes", codes_bytes(weights, fmt)), (down_scales, "down_scales", weights // per))]
    if inner < 0:
        raise ValueError("negative size")
    layer = _MoeLayer(*ptrs, hidden, inner, experts, FORMATS[fmt], block)
    with _Place(dev, stream):
        if out is None:
            out = torch.empty_like(x)
        elif out.shape != x.shape or out.dtype != x.dtype:
            raise ValueError("out must have x's shape and type")
        if workspace is None:
            workspace = torch.empty(L.mxq_moe_workspace_bytes(tokens, top_k, inner, dt), dtype=torch.uint8, device=dev)
        _check(L.mxq_moe(ctypes.byref(layer), _dev(x, "x"), dt, _on(logits, "logits", dev), tokens, top_k, int(bool(renormalize)),
                         _on(out, "out", dev), _operand(workspace, "workspace", 0, dev), workspace.numel(), _stream(None)), "mxq_moe")
    return out


# ---- a paged cache of keys and values held as codes -----------------------------------------------------------------


def make_cache(pages: int, heads: int, head_dim: int, fmt: str, block: int = 32, page: int = 64, device="cuda"):
    """Buffers of an empty cache: (k_codes, k_scales, v_codes, v_scales), codes [pages, heads, page, head_dim * bits / 8] and
    scales [pages, heads, page, head_dim / block], uint8, zeros (every token of it reads as zeros)."""
    if fmt not in ("e4m3", "e2m1", "int8", "int4"):
        raise MxqError(-2, "make_cache")
    if block not in (32, 64, 128):
        raise MxqError(-3, "make_cache")
    if head_dim not in (64, 128, 256) or head_dim % block or page not in (16, 32, 64, 128, 256) or pages < 0 or not 1 <= heads <= CACHE_HEADS_MAX:
        raise MxqError(-4, "make_cache")
    codes, scales = (pages, heads, page, head_dim * (8 if fmt in ("e4m3", "int8") else 4) // 8), (pages, heads, page, head_dim // block)
    return tuple(torch.zeros(shape, dtype=torch.uint8, device=device) for shape in (codes, scales, codes, scales))


#: limit of a cache's heads (MXQ_CACHE_HEADS_MAX in include/mxq.h)
CACHE_HEADS_MAX = 1024


def _cache(k_codes, k_scales, v_codes, v_scales, fmt: str, block: int) -> _Cache:
    """The marshalled description of a cache's four buffers, whose shapes must agree."""
    f = FORMATS[fmt]
    for t, what in ((k_codes, "k_codes"), (k_scales, "k_scales"), (v_codes, "v_codes"), (v_scales, "v_scales")):
        if t.dtype != torch.uint8:
            raise TypeError("%s must be uint8, got %s" % (what, t.dtype))
        if t.dim() != 4:
            raise ValueError("%s has the shape [pages, heads, page, bytes of a row], got %s" % (what, tuple(t.shape)))
    pages, heads, page, row = k_codes.shape
    bits = load_library().mxq_format_bits(f)
    dim = row * 8 // bits
    srow = (pages, heads, page, dim // block if block > 0 else 0)
    if v_codes.shape != k_codes.shape or k_scales.shape != srow or v_scales.shape != srow:
        raise ValueError("the cache's buffers do not belong together: codes %s and %s, scales %s and %s, block %d" % (
            tuple(k_codes.shape), tuple(v_codes.shape), tuple(k_scales.shape), tuple(v_scales.shape), block))
    dev = k_codes.device
    return _Cache(_on(k_codes, "k_codes", dev), _on(k_scales, "k_scales", dev), _on(v_codes, "v_codes", dev), _on(v_scales, "v_scales", dev),
                  pages, page, heads, dim, f, block)


def _ints(t: torch.Tensor, what: str, shape, device) -> int:
    if t.dtype != torch.int32:
        raise TypeError("%s must be int32, got %s" % (what, t.dtype))
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have the shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))
    return _on(t, what, device)


def _batch(table, lengths, starts, device) -> _Batch:
    if table.dim() != 2:
        raise ValueError("table has the shape [batch, pages of the longest sequence], got %s" % (tuple(table.shape),))
    n, width = table.shape
    return _Batch(_ints(table, "table", (n, width), device), None if lengths is None else _ints(lengths, "lengths", (n,), device),
                  None if starts is None else _ints(starts, "starts", (n + 1,), device), n, width)


def _rows(t: torch.Tensor, what: str, shape, device) -> Tuple[_Rows, torch.Tensor]:
    """A [tokens, heads, head_dim] tensor as the kernels take it: itself, or a contiguous copy where its last dimension is not
    contiguous or its address or strides are no multiples of 32 bytes."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have the shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor (libmxq has no CPU path)" % what)
    if t.device != device:
        raise ValueError("%s is on %s, the other tensors on %s" % (what, t.device, device))
    size = t.element_size()
    if t.stride(2) != 1 or t.stride(0) * size % 32 or t.stride(1) * size % 32 or t.stride(0) < 0 or t.stride(1) < 0 or t.data_ptr() % 32:
        t = t.clone(memory_format=torch.contiguous_format)
    return _Rows(t.data_ptr(), t.stride(0), t.stride(1)), t


def cache_write(k: torch.Tensor, v: torch.Tensor, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor, v_scales: torch.Tensor,
                table: torch.Tensor, lengths: torch.Tensor, fmt: str, block: int = 32, starts: Optional[torch.Tensor] = None,
                stream=None) -> None:
    """mxq_cache_write: quantizes the new tokens' keys and values [tokens, heads, head_dim] into their pages of a cache (``make_cache``'s
    buffers).  ``table`` [batch, width], ``lengths`` [batch] (the new tokens counted) and ``starts`` [batch + 1] are int32 tensors on the
    device; without ``starts`` row b is sequence b's one new token.  Any strides (rows that are no multiples of 32 bytes apart are copied
    first).  Two sequences of a call must not write to the same place."""
    L = _lib or load_library()
    if _host.cache_write(k, v, k_codes, k_scales, v_codes, v_scales, table, lengths, fmt, block, starts, stream):
        return
    dev = k_codes.device
    c, b = _cache(k_codes, k_scales, v_codes, v_scales, fmt, block), _batch(table, lengths, starts, dev)
    with _Place(dev, stream):
        if k.dim() != 3 or k.dtype != v.dtype:
            raise ValueError("cache_write takes k and v [tokens, heads, head_dim] of one type")
        shape = (k.shape[0], c.heads, c.head_dim)
        kr, k = _rows(k, "k", shape, dev)
        vr, v = _rows(v, "v", shape, dev)
        _check(L.mxq_cache_write(ctypes.byref(c), ctypes.byref(b), ctypes.byref(kr), ctypes.byref(vr), _dtype_id(k), shape[0], _stream(None)),
               "mxq_cache_write")


def cache_read(k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor, v_scales: torch.Tensor, table: torch.Tensor,
               starts: torch.Tensor, total: int, fmt: str, block: int = 32, dtype: torch.dtype = torch.bfloat16,
               out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """mxq_cache_read: keys and values, [total, heads, head_dim] each, of the first starts[b + 1] - starts[b] tokens of every sequence, in
    rows starts[b] ...  ``out`` (a pair): rows behind starts[batch] are left as they were."""
    L = _lib or load_library()
    made = _host.cache_read(k_codes, k_scales, v_codes, v_scales, table, starts, total, fmt, block, dtype, out, stream)
    if made is not None:
        return made
    dev = k_codes.device
    if total < 0:
        raise ValueError("negative size")
    c, b = _cache(k_codes, k_scales, v_codes, v_scales, fmt, block), _batch(table, None, starts, dev)
    with _Place(dev, stream):
        shape = (total, c.heads, c.head_dim)
        if out is None:
            out = (torch.empty(shape, dtype=dtype, device=dev), torch.empty(shape, dtype=dtype, device=dev))
        k, v = out
        if tuple(k.shape) != shape or tuple(v.shape) != shape or k.dtype != v.dtype:
            raise ValueError("out holds two tensors of the shape %s and one type" % (shape,))
        _check(L.mxq_cache_read(ctypes.byref(c), ctypes.byref(b), total, _on(k, "out[0]", dev), _on(v, "out[1]", dev), _dtype_id(k), _stream(None)),
               "mxq_cache_read")
    return k, v


def cache_attention_workspace_bytes(tokens: int, q_heads: int, batch: int, width: int, page: int, heads: int, head_dim: int,
                                    dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of ``cache_attention``'s workspace for `tokens` queries of `batch` sequences with tables of `width` pages (0: refused)."""
    c = _Cache(None, None, None, None, 0, page, heads, head_dim, FORMATS["e4m3"], 32)
    b = _Batch(None, None, 1, batch, width)
    return load_library().mxq_cache_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), q_heads, F32 if dtype == torch.float32 else BF16, tokens)


def cache_attention(q: torch.Tensor, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor, v_scales: torch.Tensor,
                    table: torch.Tensor, lengths: torch.Tensor, fmt: str, block: int = 32, starts: Optional[torch.Tensor] = None,
                    scale: Optional[float] = None, causal: bool = True, window: int = 0, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """mxq_cache_attention: softmax(scale q K^T) V of the new tokens' queries q [tokens, q_heads, head_dim] over their sequences' cached
    tokens, K and V as the cache's codes stand for them; q_heads is a multiple of the cache's heads, query head j uses head
    j // (q_heads // heads).  ``table``, ``lengths`` and ``starts`` as in ``cache_write``; scale: 1 / sqrt(head_dim) by default; causal: a
    query sees the tokens up to its own, with ``window`` only the last so many of them; lse: a float32 tensor [tokens, q_heads] for the
    logarithms of the softmax's sums.  ``workspace`` (uint8, ``cache_attention_workspace_bytes``) saves the allocation of one per call; calls that
    can overlap on the GPU must not share it.  A query that sees nothing gives zeros.  For serving: the result has no gradient."""
    L = _lib or load_library()
    made = _host.cache_attention(q, k_codes, k_scales, v_codes, v_scales, table, lengths, fmt, block, starts, scale, causal, window, out, lse, workspace,
                                 stream)
    if made is not None:
        return made
    dev = k_codes.device
    c, b = _cache(k_codes, k_scales, v_codes, v_scales, fmt, block), _batch(table, lengths, starts, dev)
    with _Place(dev, stream):
        if q.dim() != 3 or q.shape[2] != c.head_dim:
            raise ValueError("q has the shape [tokens, q_heads, %d], got %s" % (c.head_dim, tuple(q.shape)))
        if window < 0:
            raise ValueError("negative size")
        tokens, q_heads = q.shape[:2]
        dt = _dtype_id(q)
        qr, q = _rows(q.detach(), "q", q.shape, dev)
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=dev)
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out must have q's shape and type")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2]):
            raise ValueError("lse is float32 of the shape [tokens, q_heads]")
        if workspace is None:
            workspace = torch.empty(L.mxq_cache_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(b), q_heads, dt, tokens), dtype=torch.uint8,
                                    device=dev)
        _check(L.mxq_cache_attention(ctypes.byref(c), ctypes.byref(b), ctypes.byref(qr), q_heads, dt, tokens,
                                     1 / math.sqrt(c.head_dim) if scale is None else scale, int(bool(causal)), window, _on(out, "out", dev),
                                     None if lse is None else _on(lse, "lse", dev), _operand(workspace, "workspace", 0, dev), workspace.numel(),
                                     _stream(None)), "mxq_cache_attention")
    return out
