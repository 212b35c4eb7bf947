"""Python binding of the sparkattn C-ABI library (``libsparkattn.so``).

Argument marshalling only, for the per-layer calls in native code
(``_sparkattn.so``, ``csrc/binding.cpp``), for the others through ctypes: every
step of the path (block selection, FP8 quantisation, block-sparse attention)
runs in the CUDA kernels behind the ``extern "C"`` entry points declared in
``include/sparkattn.h``.  PyTorch is used for device memory and streams.  There
is no CPU fallback: if the shared library is missing or cannot be loaded, every call raises.

Without ``stream`` a per-layer call uses the current stream.  With it, outputs and workspace that the call allocates come from that
stream's memory; an output is read on the current stream once that has waited for the other.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsparkattn.so")
VERSION = 1

OK = 0
E_INVALID_ARG = -1
E_UNSUPPORTED_SHAPE = -2
E_MISALIGNED = -3
E_WORKSPACE_TOO_SMALL = -4
E_CUDA = -5
E_DEVICE_TIMEOUT = -6
E_BAD_INDEX = -7
E_NO_DEVICE = -8
E_OUT_OF_PAGES = -9

BF16 = 0
FP8_E4M3 = 1
FP32 = 2

EXPORTS = (
    "sparkattn_version", "sparkattn_status_string", "sparkattn_workspace_bytes", "sparkattn_select",
    "sparkattn_quant_fp8", "sparkattn_quant_fp8_per_token", "sparkattn_fwd", "sparkattn_read_status", "sparkattn_arena_bytes",
    "sparkattn_attention_host", "sparkattn_select_noalloc", "sparkattn_select_noalloc_max_bytes",
    "sparkattn_select_noalloc_status", "sparkattn_comp_workspace_bytes", "sparkattn_comp_state",
    "sparkattn_comp_apply", "sparkattn_select_window", "sparkattn_fwd_window", "sparkattn_brick_count",
    "sparkattn_brick_layout", "sparkattn_gather_tokens", "sparkattn_select_padded", "sparkattn_fwd_padded",
    "sparkattn_quant_fp8_pooled", "sparkattn_select_pooled", "sparkattn_fwd_gated_workspace_bytes", "sparkattn_fwd_gated",
    "sparkattn_cache_workspace_bytes", "sparkattn_cache_append", "sparkattn_cache_fwd", "sparkattn_cache_fwd_sink",
    "sparkattn_cache_append_norm", "sparkattn_norm_rotate", "sparkattn_pages_workspace_bytes", "sparkattn_pages_fork",
    "sparkattn_pages_reserve", "sparkattn_pages_trim", "sparkattn_pages_compact", "sparkattn_cache_copy_pages", "sparkattn_pages_reserve_len",
)


class Shape(ctypes.Structure):
    """Mirror of ``sparkattn_shape_t``."""
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("version", ctypes.c_uint32),
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("d", ctypes.c_int32),
        ("block", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64),
        ("softmax_scale", ctypes.c_float), ("pad", ctypes.c_uint32),
    ]


_SHAPE_BYTES = ctypes.sizeof(Shape)


class CacheShape(ctypes.Structure):
    """Mirror of ``sparkattn_cache_t``."""
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("version", ctypes.c_uint32),
        ("dtype", ctypes.c_int32), ("pages", ctypes.c_int32), ("H", ctypes.c_int32), ("page", ctypes.c_int32),
        ("d", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("stride_page", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64),
    ]


class Batch(ctypes.Structure):
    """Mirror of ``sparkattn_batch_t``."""
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("version", ctypes.c_uint32),
        ("B", ctypes.c_int32), ("T", ctypes.c_int32), ("max_new", ctypes.c_int32), ("max_pages", ctypes.c_int32),
        ("page_table", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("q_start", ctypes.c_void_p),
    ]


class Rows(ctypes.Structure):
    """Mirror of ``sparkattn_rows_t``."""
    _fields_ = [("data", ctypes.c_void_p), ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class RotaryShape(ctypes.Structure):
    """Mirror of ``sparkattn_rotary_t``."""
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("version", ctypes.c_uint32),
        ("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("rows", ctypes.c_int32), ("axes", ctypes.c_int32),
        ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("axis", ctypes.c_void_p),
    ]


class BookShape(ctypes.Structure):
    """Mirror of ``sparkattn_book_t``."""
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("version", ctypes.c_uint32),
        ("B", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("pages", ctypes.c_int32), ("page", ctypes.c_int32),
        ("page_table", ctypes.c_void_p), ("refs", ctypes.c_void_p),
    ]


class NormShape(ctypes.Structure):
    """Mirror of ``sparkattn_norm_t``."""
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("version", ctypes.c_uint32),
        ("weight_dtype", ctypes.c_int32), ("per_head", ctypes.c_int32), ("eps", ctypes.c_float), ("pad", ctypes.c_uint32),
        ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
    ]


class SparkAttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


# What the native marshalling of the per-layer calls (csrc/binding.cpp) calls, in its order.
_BOUND = ("workspace_bytes", "select", "select_window", "select_padded", "select_pooled", "quant_fp8", "quant_fp8_pooled",
          "quant_fp8_per_token", "fwd", "fwd_window", "fwd_padded", "gather_tokens", "comp_workspace_bytes", "comp_state", "comp_apply",
          "fwd_gated_workspace_bytes", "fwd_gated", "cache_workspace_bytes", "cache_append", "cache_fwd",
          "cache_fwd_sink", "cache_append_norm", "norm_rotate", "pages_workspace_bytes", "pages_fork", "pages_reserve", "pages_trim",
          "pages_compact", "cache_copy_pages", "pages_reserve_len")
_NO_WORKSPACE = 1        # the library does not serve the shape: the workspace query returned 0

_lib = None
_native = None


def lib() -> ctypes.CDLL:
    """Loads the shared library (once).  Raises if it has not been built."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2609_23153_b200.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        sp = ctypes.POINTER(Shape)
        L.sparkattn_version.restype = ctypes.c_int
        L.sparkattn_status_string.restype = ctypes.c_char_p
        L.sparkattn_status_string.argtypes = [ctypes.c_int]
        L.sparkattn_workspace_bytes.restype = sz
        L.sparkattn_workspace_bytes.argtypes = [sp, i32, i32]
        L.sparkattn_select.restype = ctypes.c_int
        L.sparkattn_select.argtypes = [sp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.sparkattn_quant_fp8.restype = ctypes.c_int
        L.sparkattn_quant_fp8.argtypes = [sp, vp, vp, vp, ctypes.c_uint32, vp]
        L.sparkattn_quant_fp8_pooled.restype = ctypes.c_int
        L.sparkattn_quant_fp8_pooled.argtypes = [sp, vp, vp, vp, i32, vp, sz, vp]
        L.sparkattn_select_pooled.restype = ctypes.c_int
        L.sparkattn_select_pooled.argtypes = [sp, i32, vp, vp, vp, sz, vp]
        L.sparkattn_quant_fp8_per_token.restype = ctypes.c_int
        L.sparkattn_quant_fp8_per_token.argtypes = [sp, vp, vp, vp, vp]
        L.sparkattn_fwd.restype = ctypes.c_int
        L.sparkattn_fwd.argtypes = [sp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.sparkattn_read_status.restype = ctypes.c_int
        L.sparkattn_read_status.argtypes = [vp, vp]
        L.sparkattn_brick_count.restype = ctypes.c_int64
        L.sparkattn_brick_count.argtypes = [vp, vp]
        L.sparkattn_brick_layout.restype = ctypes.c_int
        L.sparkattn_brick_layout.argtypes = [vp, vp, i32, vp, vp, vp, vp]
        L.sparkattn_gather_tokens.restype = ctypes.c_int
        L.sparkattn_gather_tokens.argtypes = [sp, vp, sp, vp, vp, vp, sz, vp]
        L.sparkattn_select_padded.restype = ctypes.c_int
        L.sparkattn_select_padded.argtypes = [sp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.sparkattn_fwd_padded.restype = ctypes.c_int
        L.sparkattn_fwd_padded.argtypes = [sp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
        L.sparkattn_arena_bytes.restype = sz
        L.sparkattn_arena_bytes.argtypes = [sp, i32, i32]
        L.sparkattn_attention_host.restype = ctypes.c_int
        L.sparkattn_attention_host.argtypes = [sp, i32, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.sparkattn_select_noalloc.restype = ctypes.c_int
        L.sparkattn_select_noalloc.argtypes = [sp, vp, vp, i32, vp, vp, vp]
        L.sparkattn_select_noalloc_max_bytes.restype = sz
        L.sparkattn_select_noalloc_status.restype = ctypes.c_int
        L.sparkattn_select_noalloc_status.argtypes = [vp]
        L.sparkattn_select_window.restype = ctypes.c_int
        L.sparkattn_select_window.argtypes = [sp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        L.sparkattn_fwd_window.restype = ctypes.c_int
        L.sparkattn_fwd_window.argtypes = [sp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        L.sparkattn_comp_workspace_bytes.restype = sz
        L.sparkattn_comp_workspace_bytes.argtypes = [sp, vp]
        L.sparkattn_comp_state.restype = ctypes.c_int
        L.sparkattn_comp_state.argtypes = [sp, vp, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.sparkattn_comp_apply.restype = ctypes.c_int
        L.sparkattn_comp_apply.argtypes = [sp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp, sz, vp]
        L.sparkattn_fwd_gated_workspace_bytes.restype = sz
        L.sparkattn_fwd_gated_workspace_bytes.argtypes = [sp, i32, vp]
        L.sparkattn_fwd_gated.restype = ctypes.c_int
        L.sparkattn_fwd_gated.argtypes = [sp, vp, vp, vp, vp, vp, i32, vp, i32, vp, vp, vp, vp, vp, ctypes.c_float, vp,
                                          vp, vp, sz, vp]
        cp, bp, rp = ctypes.POINTER(CacheShape), ctypes.POINTER(Batch), ctypes.POINTER(Rows)
        L.sparkattn_cache_workspace_bytes.restype = sz
        L.sparkattn_cache_workspace_bytes.argtypes = [cp, bp, i32]
        L.sparkattn_cache_append.restype = ctypes.c_int
        L.sparkattn_cache_append.argtypes = [cp, bp, ctypes.POINTER(RotaryShape), rp, i32, rp, rp, vp, vp, vp, vp, rp, vp, sz, vp]
        L.sparkattn_cache_fwd.restype = ctypes.c_int
        L.sparkattn_cache_fwd.argtypes = [cp, bp, rp, i32, vp, vp, vp, vp, i32, i32, ctypes.c_float, rp, vp, vp, sz, vp]
        np = ctypes.POINTER(NormShape)
        L.sparkattn_cache_append_norm.restype = ctypes.c_int
        L.sparkattn_cache_append_norm.argtypes = [cp, bp, np, ctypes.POINTER(RotaryShape), rp, i32, rp, rp, vp, vp, vp, vp, rp, vp, sz, vp]
        L.sparkattn_norm_rotate.restype = ctypes.c_int
        L.sparkattn_norm_rotate.argtypes = [sp, vp, sp, vp, sp, vp, sp, vp, np, ctypes.POINTER(RotaryShape), vp, sz, vp]
        kp = ctypes.POINTER(BookShape)
        L.sparkattn_pages_workspace_bytes.restype = sz
        L.sparkattn_pages_workspace_bytes.argtypes = [kp]
        for name, args in (("fork", [vp, vp, i32, vp, vp, vp]), ("reserve", [vp, vp, vp, vp, vp, vp]), ("reserve_len", [vp, vp, vp, vp, vp, vp, vp]), ("trim", [vp, i32, i32, i32, vp, vp]),
                           ("compact", [vp, vp, vp, vp])):
            call = getattr(L, "sparkattn_pages_" + name)
            call.restype = ctypes.c_int
            call.argtypes = [kp, *args, vp, sz, vp]
        L.sparkattn_cache_copy_pages.restype = ctypes.c_int
        L.sparkattn_cache_copy_pages.argtypes = [cp, vp, vp, vp, vp, cp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        L.sparkattn_cache_fwd_sink.restype = ctypes.c_int
        L.sparkattn_cache_fwd_sink.argtypes = [cp, bp, rp, i32, vp, vp, vp, vp, i32, i32, i32, ctypes.c_float, rp, vp, vp, sz, vp]
        from . import _sparkattn
        _sparkattn.bind(*(ctypes.cast(getattr(L, "sparkattn_" + name), vp).value for name in _BOUND))
        _native = _sparkattn
        _lib = L
    return _lib


def _calls():
    if _lib is None:
        lib()
    return _native


def status_string(status: int) -> str:
    return lib().sparkattn_status_string(int(status)).decode()


def _check(rc: int, where: str) -> None:
    if rc != OK:
        if rc == _NO_WORKSPACE:
            raise SparkAttnError(E_UNSUPPORTED_SHAPE, "sparkattn_workspace_bytes")
        raise SparkAttnError(rc, where)


# The current stream's handle alone: building a torch.cuda.Stream object around it takes 3.4 us, a seventh of a small
# call.  The name is not part of torch's public interface: where it is missing the public way is taken.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is None and _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def make_shape(x: torch.Tensor, block: int, softmax_scale: float = 0.0) -> Shape:
    """Shape descriptor for a [B, H, N, d] tensor (d contiguous, arbitrary outer strides)."""
    stride = x.stride()
    if len(stride) != 4 or stride[3] != 1:
        raise ValueError("expected a [B, H, N, d] tensor with a contiguous last dimension")
    B, H, N, d = x.shape
    return Shape(_SHAPE_BYTES, VERSION, B, H, N, d, block, 0, stride[0], stride[1], stride[2], float(softmax_scale), 0)


def _same_layout(ref: torch.Tensor, *others: torch.Tensor) -> None:
    for o in others:
        if o.shape != ref.shape or o.stride() != ref.stride():
            raise ValueError("tensors of one call must share shape and strides")


def workspace_bytes(shape: Shape, which: int, topk_or_kmax: int) -> int:
    return int(lib().sparkattn_workspace_bytes(ctypes.byref(shape), which, topk_or_kmax))


def alloc_workspace(shape: Shape, which: int, topk_or_kmax: int, device) -> torch.Tensor:
    n = workspace_bytes(shape, which, topk_or_kmax)
    if n == 0:
        raise SparkAttnError(E_UNSUPPORTED_SHAPE, "sparkattn_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def read_status(workspace: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> int:
    return int(lib().sparkattn_read_status(_ptr(workspace), _stream_ptr(stream)))


def select(q: torch.Tensor, k: torch.Tensor, block: int, topk: int, *,
           kept_idx: Optional[torch.Tensor] = None, kept_cnt: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
           frame_tokens: int = 0, window: int = 0, block_valid: Optional[torch.Tensor] = None,
           ) -> Tuple[torch.Tensor, torch.Tensor]:
    """``sparkattn_select`` (``sparkattn_select_window`` when ``frame_tokens`` > 0, ``sparkattn_select_padded``
    with ``block_valid``, device int32 [nb]): q, k bf16 [B,H,N,d] on the device -> (kept_idx int32
    [B,H,nb,topk] ascending, kept_cnt int32 [B,H,nb])."""
    if block_valid is not None and frame_tokens > 0:
        raise ValueError("block_valid and a causal window cannot be combined")
    rc, kept_idx, kept_cnt = _calls().select(q, k, block, topk, kept_idx, kept_cnt, workspace,
                                             None if stream is None else stream.cuda_stream, frame_tokens, window, block_valid)
    if rc != OK:
        _check(rc, "sparkattn_select_padded" if block_valid is not None else
               "sparkattn_select_window" if frame_tokens > 0 else "sparkattn_select")
    return kept_idx, kept_cnt


def select_noalloc(q: torch.Tensor, k: torch.Tensor, block: int, topk: int, kept_idx: torch.Tensor,
                   kept_cnt: Optional[torch.Tensor], stream: Optional[torch.cuda.Stream] = None) -> None:
    """``sparkattn_select_noalloc``: same selection as :func:`select`, for callers that
    must not allocate device memory at call time.  The caller passes the output
    buffers; the scratch is a fixed 32 MiB array inside the library, shared by all
    calls on the device (do not overlap calls; make the first call on a device
    before any stream capture)."""
    _same_layout(q, k)
    shape = make_shape(q, block)
    rc = lib().sparkattn_select_noalloc(ctypes.byref(shape), _ptr(q), _ptr(k), topk, _ptr(kept_idx), _ptr(kept_cnt),
                                        _stream_ptr(stream))
    _check(rc, "sparkattn_select_noalloc")


def quant_fp8(x: torch.Tensor, block: int, *, codes: Optional[torch.Tensor] = None,
              scales: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
              ) -> Tuple[torch.Tensor, torch.Tensor]:
    """``sparkattn_quant_fp8``: x bf16 [B,H,N,d] -> (codes uint8, same strides; scales fp32 [B,H,nb])."""
    rc, codes, scales = _calls().quant_fp8(x, block, codes, scales, None if stream is None else stream.cuda_stream)
    _check(rc, "sparkattn_quant_fp8")
    return codes, scales


def quant_fp8_pooled(x: torch.Tensor, block: int, key_side: bool, select_workspace: torch.Tensor, *,
                     codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``sparkattn_quant_fp8_pooled``: :func:`quant_fp8` that also leaves the pooled block means of ``x`` (the query
    tensor, or the key tensor with ``key_side``) in ``select_workspace`` for :func:`select_pooled`."""
    rc, codes, scales = _calls().quant_fp8_pooled(x, block, key_side, select_workspace, codes, scales,
                                                  None if stream is None else stream.cuda_stream)
    _check(rc, "sparkattn_quant_fp8_pooled")
    return codes, scales


def select_pooled(ref: torch.Tensor, block: int, topk: int, workspace: torch.Tensor, *,
                  kept_idx: Optional[torch.Tensor] = None, kept_cnt: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``sparkattn_select_pooled``: scores + top-k on the pooled means two :func:`quant_fp8_pooled` calls left in
    ``workspace``; ``ref`` is any [B,H,N,d] tensor of the problem (for the shape)."""
    rc, kept_idx, kept_cnt = _calls().select_pooled(ref, block, topk, workspace, kept_idx, kept_cnt,
                                                    None if stream is None else stream.cuda_stream)
    _check(rc, "sparkattn_select_pooled")
    return kept_idx, kept_cnt


def quant_fp8_per_token(x: torch.Tensor, *, codes: Optional[torch.Tensor] = None,
                        scales: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                        ) -> Tuple[torch.Tensor, torch.Tensor]:
    """``sparkattn_quant_fp8_per_token``: x bf16 [B,H,N,d] -> (codes uint8, same strides; scales fp32 [B,H,N])."""
    rc, codes, scales = _calls().quant_fp8_per_token(x, codes, scales, None if stream is None else stream.cuda_stream)
    _check(rc, "sparkattn_quant_fp8_per_token")
    return codes, scales


def fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, kept_idx: torch.Tensor,
        kept_cnt: Optional[torch.Tensor], block: int, *,
        scales: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None,
        softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None, return_lse: bool = False,
        workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
        check_status: bool = False, frame_tokens: int = 0, window: int = 0,
        block_valid: Optional[torch.Tensor] = None):
    """``sparkattn_fwd`` (``sparkattn_fwd_window`` when ``frame_tokens`` > 0, ``sparkattn_fwd_padded`` with
    ``block_valid``, device int32 [nb]).  bf16 q,k,v, or uint8
    E4M3 codes with ``scales=(q_scale, k_scale, v_scale)``.  Returns out bf16 [B,H,N,d] (and lse
    fp32 [B,H,N])."""
    if block_valid is not None and frame_tokens > 0:
        raise ValueError("block_valid and a causal window cannot be combined")
    sq, sk, sv = scales if scales is not None else (None, None, None)
    rc, out, lse, workspace = _calls().fwd(q, k, v, kept_idx, kept_cnt, block, BF16 if scales is None else FP8_E4M3, sq, sk, sv,
                                           softmax_scale, out, return_lse, workspace,
                                           None if stream is None else stream.cuda_stream, frame_tokens, window, block_valid)
    _check(rc, "sparkattn_fwd")
    if check_status:
        _check(read_status(workspace, stream), "sparkattn_fwd (device status)")
    return (out, lse) if return_lse else out


def brick_layout(grid, brick, block: int, device="cuda:0", stream: Optional[torch.cuda.Stream] = None):
    """``sparkattn_brick_layout``: (gather int32 [bricks * block] with -1 for padding, block_valid int32 [bricks],
    scatter int32 [N]) for a (T, Hg, Wg) grid cut into (bt, bh, bw) bricks, one block per brick."""
    g = (ctypes.c_int32 * 3)(*[int(v) for v in grid])
    b = (ctypes.c_int32 * 3)(*[int(v) for v in brick])
    bricks = int(lib().sparkattn_brick_count(ctypes.cast(g, ctypes.c_void_p), ctypes.cast(b, ctypes.c_void_p)))
    if bricks == 0:
        raise SparkAttnError(E_INVALID_ARG, "sparkattn_brick_count")
    n = int(grid[0]) * int(grid[1]) * int(grid[2])
    with torch.cuda.stream(stream):      # (None: the current one)
        gather = torch.empty(bricks * block, dtype=torch.int32, device=device)
        valid = torch.empty(bricks, dtype=torch.int32, device=device)
        scatter = torch.empty(n, dtype=torch.int32, device=device)
    if stream is not None:
        for x in (gather, valid, scatter):
            x.record_stream(torch.cuda.current_stream(x.device))
    rc = lib().sparkattn_brick_layout(ctypes.cast(g, ctypes.c_void_p), ctypes.cast(b, ctypes.c_void_p), block, _ptr(gather),
                                      _ptr(valid), _ptr(scatter), _stream_ptr(stream))
    _check(rc, "sparkattn_brick_layout")
    return gather, valid, scatter


def gather_tokens(x: torch.Tensor, index: torch.Tensor, *, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                  check_status: bool = False) -> torch.Tensor:
    """``sparkattn_gather_tokens``: out[b,h,i,:] = x[b,h,index[i],:] (zero row for index -1); x bf16 [B,H,N,d],
    index int32 [N_out] on the device, out bf16 [B,H,N_out,d]."""
    rc, out, workspace = _calls().gather_tokens(x, index, out, workspace, None if stream is None else stream.cuda_stream)
    _check(rc, "sparkattn_gather_tokens")
    if check_status:
        _check(read_status(workspace, stream), "sparkattn_gather_tokens (device status)")
    return out


def arena_bytes(shape: Shape, dtype: int, topk: int) -> int:
    return int(lib().sparkattn_arena_bytes(ctypes.byref(shape), dtype, topk))


def attention_host(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, block: int, topk: int, *,
                   dtype: int = BF16, out: Optional[torch.Tensor] = None,
                   kept_idx: Optional[torch.Tensor] = None, arena: Optional[torch.Tensor] = None,
                   device="cuda:0", stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``sparkattn_attention_host``: q, k, v contiguous bf16 HOST tensors (pinned for
    speed); runs copy-in, select, (quant,) fwd, copy-out and returns the host output."""
    for t in (q, k, v):
        if t.device.type != "cpu" or not t.is_contiguous() or t.dtype != torch.bfloat16:
            raise ValueError("attention_host expects contiguous bf16 CPU tensors")
    shape = make_shape(q, block)
    if out is None:
        out = torch.empty_like(q).pin_memory()
    if arena is None:
        with torch.cuda.stream(stream):      # (None: the current one)
            arena = torch.empty(arena_bytes(shape, dtype, topk), dtype=torch.uint8, device=device)
    rc = lib().sparkattn_attention_host(ctypes.byref(shape), dtype, _ptr(q), _ptr(k), _ptr(v), topk, _ptr(out),
                                        _ptr(kept_idx), _ptr(arena), arena.numel(), _stream_ptr(stream))
    _check(rc, "sparkattn_attention_host")
    return out


def comp_workspace_bytes(shape: Shape, grid) -> int:
    g = (ctypes.c_int32 * 3)(*[int(x) for x in grid])
    return int(lib().sparkattn_comp_workspace_bytes(ctypes.byref(shape), g))


def comp_state(k: torch.Tensor, v: torch.Tensor, pk: torch.Tensor, grid, axis: torch.Tensor, freq: torch.Tensor, *,
               state: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None, check_status: bool = False) -> torch.Tensor:
    """``sparkattn_comp_state``: k, v bf16 [B,H,N,d]; pk bf16 [H,r,d]; grid (T,Hg,Wg); axis/freq the
    rotary tables (rank/2 entries, any device).  Returns the state fp32 [B,H,r,d]."""
    T, Hg, Wg = grid
    rc, state, workspace = _calls().comp_state(k, v, pk, int(T), int(Hg), int(Wg), axis, freq, state, workspace,
                                               None if stream is None else stream.cuda_stream)
    _check(rc, "sparkattn_comp_state")
    if check_status:
        _check(read_status(workspace, stream), "sparkattn_comp_state (device status)")
    return state


def comp_apply(q: torch.Tensor, pq: torch.Tensor, state: torch.Tensor, gate: torch.Tensor, o_sparse: torch.Tensor,
               grid, axis: torch.Tensor, freq: torch.Tensor, *, eps: float = 1e-6,
               out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None, check_status: bool = False) -> torch.Tensor:
    """``sparkattn_comp_apply``: q, o_sparse bf16 [B,H,N,d]; pq bf16 [H,r,d]; state fp32 [B,H,r,d];
    gate fp32 [B,H,N].  Returns the fused output bf16 [B,H,N,d]."""
    T, Hg, Wg = grid
    rc, out, workspace = _calls().comp_apply(q, pq, state, gate, o_sparse, int(T), int(Hg), int(Wg), axis, freq, eps, out, workspace,
                                             None if stream is None else stream.cuda_stream)
    _check(rc, "sparkattn_comp_apply")
    if check_status:
        _check(read_status(workspace, stream), "sparkattn_comp_apply (device status)")
    return out


def fwd_gated_workspace_bytes(shape: Shape, kmax: int, grid) -> int:
    g = (ctypes.c_int32 * 3)(*[int(x) for x in grid])
    return int(lib().sparkattn_fwd_gated_workspace_bytes(ctypes.byref(shape), kmax, g))


def fwd_gated(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, kept_idx: torch.Tensor,
              kept_cnt: Optional[torch.Tensor], pq: torch.Tensor, state: torch.Tensor, gate: torch.Tensor,
              grid, axis: torch.Tensor, freq: torch.Tensor, *, eps: float = 1e-6, softmax_scale: float = 0.0,
              out: Optional[torch.Tensor] = None, return_lse: bool = False, workspace: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None, check_status: bool = False):
    """``sparkattn_fwd_gated``: the bf16 forward over 128-token blocks whose epilogue adds the gated
    compensation term.  Arguments as in ``fwd`` and ``comp_apply``; returns the module output bf16
    [B,H,N,d] (and the lse of the sparse branch, fp32 [B,H,N])."""
    T, Hg, Wg = grid
    rc, out, lse, workspace = _calls().fwd_gated(q, k, v, kept_idx, kept_cnt, pq, state, gate, int(T), int(Hg), int(Wg), axis, freq,
                                                 eps, softmax_scale, out, return_lse, workspace,
                                                 None if stream is None else stream.cuda_stream)
    _check(rc, "sparkattn_fwd_gated")
    if check_status:
        _check(read_status(workspace, stream), "sparkattn_fwd_gated (device status)")
    return (out, lse) if return_lse else out


class KVCache(NamedTuple):
    """Pools of a paged cache: ``k``, ``v`` [pages, H, page, d] of the same strides (d contiguous), bfloat16 or E4M3 codes
    (float8_e4m3fn or uint8); E4M3 pools have ``k_scale``, ``v_scale`` float32 [pages, H]."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


class Rotary(NamedTuple):
    """Rotation of the first ``2 * cos.shape[1]`` channels of queries and keys: tables ``cos``, ``sin`` float32 [rows, rot/2];
    pair m of token t turns by the angle of row ``positions[t, axis[m]]`` (int32 [T] or [T, axes]; None: the token's position in
    its sequence).  Pairs are channels (2m, 2m+1) where ``interleaved``, else (m, m + rot/2)."""
    cos: torch.Tensor
    sin: torch.Tensor
    positions: Optional[torch.Tensor] = None
    axis: Optional[torch.Tensor] = None
    interleaved: bool = False


class Norm(NamedTuple):
    """RMS norm over the channels of each head of queries and keys, in front of their rotation: x / sqrt(mean(x^2) + eps) * weight.  Weights
    ``q``, ``k`` float32 or bfloat16, [d] or [heads, d], both alike; None: ones.  (Not the norm of models that take one mean over all heads'
    channels, such as Wan2.1's: apply that in front, and rotate with ``norm=None``.)"""
    q: Optional[torch.Tensor] = None
    k: Optional[torch.Tensor] = None
    eps: float = 1e-6


_NO_ROTARY = (None, None, None, None, False)
_NO_NORM = (False, None, None, 1.0)


def norm_rotate(q: torch.Tensor, k: Optional[torch.Tensor] = None, *, norm: Optional[Norm] = None, rotary: Optional[Rotary] = None,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None, check_status: bool = False):
    """``sparkattn_norm_rotate``: q, k bf16 [B, H, N, d] (k with heads of its own number) normalised head by head and rotated, in one pass;
    ``rotary.positions`` are int32 [N] or [N, axes] (None: the token's index).  Returns (q, k), or q alone, with the strides of the inputs;
    ``q_out`` may be q, ``k_out`` k."""
    rc, q_out, k_out, workspace = _calls().norm_rotate(q, k, q_out, k_out, *(_NO_ROTARY if rotary is None else rotary),
                                                       *(_NO_NORM if norm is None else (True, *norm)), workspace,
                                                       None if stream is None else stream.cuda_stream)
    if rc != OK:
        _check(rc, "sparkattn_norm_rotate")
    if check_status:
        _check(read_status(workspace, stream), "sparkattn_norm_rotate (device status)")
    return q_out if k is None else (q_out, k_out)


def alloc_cache(pages: int, heads: int, page: int, d: int, fp8: bool = True, device="cuda:0") -> KVCache:
    """A cache of ``pages`` pages of ``page`` tokens (16, 32, 64 or 128) for ``heads`` key heads of ``d`` channels (64 or 128)."""
    k, v = (torch.zeros((pages, heads, page, d), dtype=torch.uint8 if fp8 else torch.bfloat16, device=device) for _ in range(2))
    if not fp8:
        return KVCache(k, v)
    return KVCache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn),
                   *(torch.ones((pages, heads), dtype=torch.float32, device=device) for _ in range(2)))


def cache_append(cache: KVCache, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, kv_len: torch.Tensor, *,
                 q_start: Optional[torch.Tensor] = None, max_new: int = 0, q: Optional[torch.Tensor] = None,
                 norm: Optional[Norm] = None, rotary: Optional[Rotary] = None, q_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None, check_status: bool = False) -> Optional[torch.Tensor]:
    """``sparkattn_cache_append`` (``sparkattn_cache_append_norm`` with ``norm``): stores k, v bf16 [T, H_kv, d] (k normalised and rotated)
    as the newest tokens of the sequences, and returns q bf16 [T, H, d] normalised and rotated (None without q; ``q_out`` may be q).  page_table int32 [B, max_pages]; kv_len int32 [B] with the
    new tokens; rows q_start[b] .. q_start[b+1] - 1 (int32 [B+1]) belong to sequence b, T / B each without it; max_new:
    no sequence has more new tokens (0: T with q_start, which is slow where many sequences share the rows, else T / B)."""
    args = (*cache, page_table, kv_len, q_start, max_new, k, v, q, q_out, *(_NO_ROTARY if rotary is None else rotary))
    last = (workspace, None if stream is None else stream.cuda_stream)
    rc, q_out, workspace = _calls().cache_append(*args, *last) if norm is None else _calls().cache_append_norm(*args, True, *norm, *last)
    if rc != OK:
        _check(rc, "sparkattn_cache_append")
    if check_status:
        _check(read_status(workspace, stream), "sparkattn_cache_append (device status)")
    return q_out


def cache_fwd(q: torch.Tensor, cache: KVCache, page_table: torch.Tensor, kv_len: torch.Tensor, *,
              q_start: Optional[torch.Tensor] = None, max_new: int = 0, frame_tokens: int = 1, window: int = 0, sink: int = 0,
              softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None, return_lse: bool = False,
              workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None, check_status: bool = False):
    """``sparkattn_cache_fwd`` (``sparkattn_cache_fwd_sink`` where ``sink`` > 0): softmax attention of the newest tokens' queries
    q bf16 [T, H, d] over the cache, H a multiple of the cache's heads; causal by frames of ``frame_tokens`` tokens (1: by token,
    0: not), over the last ``window`` frames (0: all) and the sequence's first ``sink`` tokens.
    The batch as in :func:`cache_append`; kernel and split go by ``max_new`` and the width of ``page_table``, so both should be what the
    batch needs.  Returns out bf16 [T, H, d] (and lse float32 [T, H])."""
    args = (*cache, page_table, kv_len, q_start, max_new, q, frame_tokens, window)
    last = (softmax_scale, out, return_lse, workspace, None if stream is None else stream.cuda_stream)
    rc, out, lse, workspace = _calls().cache_fwd(*args, *last) if sink == 0 else _calls().cache_fwd_sink(*args, sink, *last)
    if rc != OK:
        _check(rc, "sparkattn_cache_fwd")
    if check_status:
        _check(read_status(workspace, stream), "sparkattn_cache_fwd (device status)")
    return (out, lse) if return_lse else out


def _book(rc: int, what: str, workspace: torch.Tensor, stream: Optional[torch.cuda.Stream], check_status: bool) -> None:
    if rc != OK:
        _check(rc, what)
    if check_status:
        _check(read_status(workspace, stream), what + " (device status)")


def pages_fork(page_table: torch.Tensor, kv_len: torch.Tensor, refs: torch.Tensor, parent: torch.Tensor, *,
               page_table_out: Optional[torch.Tensor] = None, kv_len_out: Optional[torch.Tensor] = None, refs_out: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None, check_status: bool = False):
    """``sparkattn_pages_fork``: sequence b of the new batch goes on from sequence ``parent[b]`` of the old one (int32; -1: empty); what is nobody's
    parent gives its pages back.  page_table int32 [B, max_pages] (-1: none), kv_len int32 [B], refs int32 [pages] (users of each page).
    Returns (page_table, kv_len, refs); ``refs_out`` may be refs."""
    rc, table, length, refs, workspace = _calls().pages_fork(page_table, kv_len, refs, parent, page_table_out, kv_len_out, refs_out, workspace,
                                                             None if stream is None else stream.cuda_stream)
    _book(rc, "sparkattn_pages_fork", workspace, stream, check_status)
    return table, length, refs


def pages_reserve(page_table: torch.Tensor, kv_len: torch.Tensor, refs: torch.Tensor, kv_new: torch.Tensor, page: int, *,
                  page_table_out: Optional[torch.Tensor] = None, refs_out: Optional[torch.Tensor] = None, src: Optional[torch.Tensor] = None,
                  dst: Optional[torch.Tensor] = None, kv_len_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None, check_status: bool = False):
    """``sparkattn_pages_reserve`` (``sparkattn_pages_reserve_len`` with ``kv_len_out``): pages for the tokens kv_len[b] .. kv_new[b] - 1 of every sequence, pages of ``page`` tokens, in front of
    :func:`cache_append`.  Returns (page_table, refs, src, dst): src, dst int32 [B] go to :func:`cache_copy_pages`, for every layer's cache.  All
    or nothing: with too few free pages the status is E_OUT_OF_PAGES, the book stays as it was, and nothing may be appended.  ``kv_len_out`` int32 [B]
    gets the lengths for the calls of the step, kv_new[b], or -1 where sequence b has not got its pages, by which they leave it alone: for a captured
    step, or any that does not read the status first.  The other outputs may be the inputs."""
    rc, table, refs, src, dst, workspace = _calls().pages_reserve(page_table, kv_len, refs, kv_new, page, page_table_out, refs_out, src, dst, kv_len_out,
                                                                  workspace, None if stream is None else stream.cuda_stream)
    _book(rc, "sparkattn_pages_reserve", workspace, stream, check_status)
    return table, refs, src, dst


def pages_trim(page_table: torch.Tensor, kv_len: torch.Tensor, refs: torch.Tensor, page: int, *, frame_tokens: int = 1, window: int = 0, sink: int = 0,
               page_table_out: Optional[torch.Tensor] = None, refs_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None, check_status: bool = False):
    """``sparkattn_pages_trim``: gives back the pages that no token from position kv_len[b] on reads through :func:`cache_fwd` with the same
    ``frame_tokens``, ``window`` and ``sink``, and those behind kv_len[b].  Returns (page_table, refs); they may be the inputs."""
    rc, table, refs, workspace = _calls().pages_trim(page_table, kv_len, refs, page, frame_tokens, window, sink, page_table_out, refs_out, workspace,
                                                     None if stream is None else stream.cuda_stream)
    _book(rc, "sparkattn_pages_trim", workspace, stream, check_status)
    return table, refs


def pages_compact(page_table: torch.Tensor, refs: torch.Tensor, *, page_table_out: Optional[torch.Tensor] = None, refs_out: Optional[torch.Tensor] = None,
                  src: Optional[torch.Tensor] = None, dst: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None, check_status: bool = False):
    """``sparkattn_pages_compact``: the pages in use become the pool's first.  Returns (page_table, refs, src, dst): src, dst int32 [pages // 2] go
    to :func:`cache_copy_pages`, for every layer's cache, before the new table is used.  The outputs may be the inputs."""
    rc, table, refs, src, dst, workspace = _calls().pages_compact(page_table, refs, page_table_out, refs_out, src, dst, workspace,
                                                                  None if stream is None else stream.cuda_stream)
    _book(rc, "sparkattn_pages_compact", workspace, stream, check_status)
    return table, refs, src, dst


def cache_copy_pages(cache: KVCache, src: torch.Tensor, dst: torch.Tensor, *, to: Optional[KVCache] = None, workspace: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None, check_status: bool = False) -> None:
    """``sparkattn_cache_copy_pages``: page src[i] of the cache to page dst[i] of it, or of the cache ``to`` (int32; pairs of -1 are passed over)."""
    rc, workspace = _calls().cache_copy_pages(*cache, *(cache if to is None else to), src, dst, workspace, None if stream is None else stream.cuda_stream)
    _book(rc, "sparkattn_cache_copy_pages", workspace, stream, check_status)
