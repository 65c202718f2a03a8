"""ctypes binding of libhadacore (``include/hadacore.h``).

Argument marshalling only: every step of the transform runs in the HIP
kernels of ``libhadacore.so``.  The library is loaded from this package
directory; if it is missing, every call raises (there is no fallback).

The raw entry points take device addresses as integers and keep the C names:
``hadamard_transform``, ``hadamard_transform_strided``, ``hadamard_transform_ws``,
``hadamard_transform_ws_noalloc``, ``hadamard_transform_workspace_size``, ``hadamard_transform_fp8``,
``hadamard_transform_int8``, ``hadamard_transform_fp8_blocks``, ``hadacore_padded_tokens``,
``hadacore_quantize_fp8_columns``, ``hadacore_quantize_fp8_tiles``, ``hadacore_matmul_fp8``,
``hadacore_matmul_fp8_grouped``, ``hadacore_weight_gradient_fp8_grouped``, ``hadacore_route``,
``hadacore_route_gradient``, ``hadacore_group_tokens``, ``hadacore_dispatch_rows``,
``hadacore_combine_rows``, ``hadacore_combine_gradient``, ``hadacore_adapters``,
``hadacore_adapter_gradient`` and their ``*_workspace_size``,
``hadacore_stream_copy``, ``hadacore_status_string``, ``hadacore_version``.  ``transform``,
``transform_fp8`` and ``transform_int8`` are convenience wrappers for 2-D torch tensors on a
ROCm device, and so are, for codes with a scale per block of 128, ``transform_fp8_blocks``,
``quantize_fp8_columns``, ``quantize_fp8_tiles``, ``matmul_fp8``, ``grouped_matmul_fp8`` and
``grouped_weight_gradient_fp8``; for tokens and weights of their own ``route_tokens``,
``route_tokens_gradient``, ``group_tokens``, ``dispatch_rows``, ``combine_rows``,
``combine_rows_gradient``, ``adapt_rows`` and ``adapter_gradient``.

Wrappers work on torch's current stream, or on ``stream`` (a torch stream or its handle) as if it were the
current one: outputs that they create, and workspaces, are of its memory.  As with torch's own streams, the
caller has ``stream`` wait for the inputs and keeps them until its work is done, and waits for it
before using the outputs elsewhere.
"""
from __future__ import annotations

import ctypes
import functools
import math
from pathlib import Path
from typing import NamedTuple

LIBRARY = Path(__file__).resolve().parent / "libhadacore.so"

FP16 = 0
BF16 = 1
FP32 = 2  # outputs of the FP8 products; logits, exchange, adapters
BLOCK = 128  # values that share a scale in the block quantizers and the products
SUCCESS = 0
STATUS_NAMES = {
    0: "SUCCESS", 1: "INVALID_VALUE", 2: "INVALID_SIZE", 3: "INVALID_DTYPE",
    4: "INVALID_STRIDE", 5: "MISALIGNED", 6: "OVERLAP", 7: "LAUNCH",
    8: "UNSUPPORTED_DEVICE", 9: "TOO_LARGE", 10: "WORKSPACE", 11: "SCRATCH",
}
NOALLOC_SCRATCH_BYTES = 32 << 20  # HADACORE_NOALLOC_SCRATCH_BYTES
EXPORTS = ("hadamard_transform", "hadamard_transform_strided", "hadamard_transform_ws",
           "hadamard_transform_ws_noalloc", "hadamard_transform_workspace_size", "hadamard_transform_fp8",
           "hadamard_transform_int8", "hadamard_transform_fp8_blocks", "hadacore_padded_tokens",
           "hadacore_quantize_fp8_columns", "hadacore_quantize_fp8_tiles", "hadacore_matmul_fp8",
           "hadacore_matmul_fp8_grouped", "hadacore_weight_gradient_fp8_grouped",
           "hadacore_route_workspace_size", "hadacore_route", "hadacore_route_gradient",
           "hadacore_group_workspace_size", "hadacore_group_tokens", "hadacore_dispatch_rows",
           "hadacore_combine_rows", "hadacore_combine_gradient", "hadacore_adapters_workspace_size",
           "hadacore_adapters", "hadacore_adapter_gradient_workspace_size", "hadacore_adapter_gradient",
           "hadacore_stream_copy", "hadacore_status_string", "hadacore_version")


class HadacoreError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} "
                         f"({hadacore_status_string(status)})")


_lib = None


def _load_torch_runtime() -> None:
    """Import torch, if it is installed, before the library is loaded.

    The device pointers and streams passed to the library come from torch, which
    ships its own copy of the HIP runtime.  libhadacore.so needs libamdhip64.so.7:
    if torch's copy is already loaded, that need is met by it; if the library were
    loaded first, the dynamic loader would map the system ROCm runtime instead and
    torch would then map its own, leaving two runtimes in one process -- the
    library's would see none of torch's memory or streams (and reports no device).
    """
    try:
        import torch  # noqa: F401
    except ImportError:
        pass


def library() -> ctypes.CDLL:
    """The loaded libhadacore.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not LIBRARY.exists():
            raise RuntimeError(f"{LIBRARY} is missing: build it with "
                               "`python -m paper_2412_08832_amd.build`")
        _load_torch_runtime()
        lib = ctypes.CDLL(str(LIBRARY))
        i64, vp, f32, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_int32
        lib.hadamard_transform.argtypes = [vp, vp, i64, i64, i32, f32, vp]
        lib.hadamard_transform.restype = i32
        lib.hadamard_transform_strided.argtypes = [vp, i64, vp, i64, i64, i64, i32, f32, vp]
        lib.hadamard_transform_strided.restype = i32
        lib.hadamard_transform_ws.argtypes = [vp, i64, vp, i64, i64, i64, i32, f32, vp, i64, vp]
        lib.hadamard_transform_ws.restype = i32
        lib.hadamard_transform_ws_noalloc.argtypes = [vp, i64, vp, i64, i64, i64, i32, f32, vp]
        lib.hadamard_transform_ws_noalloc.restype = i32
        lib.hadamard_transform_workspace_size.argtypes = [i64, i64]
        lib.hadamard_transform_workspace_size.restype = i64
        lib.hadamard_transform_fp8.argtypes = [vp, i64, vp, i64, vp, i64, i64, i32, f32, vp]
        lib.hadamard_transform_fp8.restype = i32
        lib.hadamard_transform_int8.argtypes = [vp, i64, vp, i64, vp, i64, i64, i32, f32, vp]
        lib.hadamard_transform_int8.restype = i32
        lib.hadamard_transform_fp8_blocks.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, i32,
                                                      f32, vp]
        lib.hadamard_transform_fp8_blocks.restype = i32
        lib.hadacore_padded_tokens.argtypes = [i64, i64]
        lib.hadacore_padded_tokens.restype = i64
        lib.hadacore_quantize_fp8_columns.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i64, i64,
                                                      i32, vp]
        lib.hadacore_quantize_fp8_columns.restype = i32
        lib.hadacore_quantize_fp8_tiles.argtypes = [vp, i64, i64, vp, i64, i64, vp, i64, i64, vp,
                                                    i64, i64, i64, i64, i64, i32, vp]
        lib.hadacore_quantize_fp8_tiles.restype = i32
        lib.hadacore_matmul_fp8.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, i64, i32,
                                            i64, i64, i64, vp]
        lib.hadacore_matmul_fp8.restype = i32
        lib.hadacore_matmul_fp8_grouped.argtypes = [vp, i64, vp, i64, vp, i64, i64, vp, i64, i64, vp,
                                                    i64, vp, i64, i32, i64, i64, i64, vp]
        lib.hadacore_matmul_fp8_grouped.restype = i32
        lib.hadacore_weight_gradient_fp8_grouped.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp,
                                                             i64, vp, i64, i64, i32, i64, i64, i64,
                                                             vp]
        lib.hadacore_weight_gradient_fp8_grouped.restype = i32
        lib.hadacore_route_workspace_size.argtypes = [i64, i64]
        lib.hadacore_route_workspace_size.restype = i64
        lib.hadacore_route.argtypes = [vp, i64, i32, vp, i64, i64, i64, i32, vp, vp, vp, vp, vp, vp,
                                       i64, vp]
        lib.hadacore_route.restype = i32
        lib.hadacore_route_gradient.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp, i64, i64, i64, i32,
                                                vp, i64, vp]
        lib.hadacore_route_gradient.restype = i32
        lib.hadacore_group_workspace_size.argtypes = [i64, i64]
        lib.hadacore_group_workspace_size.restype = i64
        lib.hadacore_group_tokens.argtypes = [vp, i64, i64, vp, vp, vp, vp, i64, vp]
        lib.hadacore_group_tokens.restype = i32
        lib.hadacore_dispatch_rows.argtypes = [vp, i64, i32, vp, vp, i64, vp, i64, i64, i64, i64, vp]
        lib.hadacore_dispatch_rows.restype = i32
        lib.hadacore_combine_rows.argtypes = [vp, i64, i64, i32, vp, vp, vp, i64, i64, i64, i64, vp]
        lib.hadacore_combine_rows.restype = i32
        lib.hadacore_combine_gradient.argtypes = [vp, i64, vp, i64, i32, vp, vp, i64, vp, vp, i64, vp,
                                                  i64, i64, i64, vp]
        lib.hadacore_combine_gradient.restype = i32
        lib.hadacore_adapters_workspace_size.argtypes = [i64, i64, i64, i64, i64]
        lib.hadacore_adapters_workspace_size.restype = i64
        lib.hadacore_adapters.argtypes = [vp, i64, vp, i64, i64, vp, i64, i64, vp, vp, vp, i64, vp,
                                          i64, vp, i64, i32, i32, vp, i64, i64, i64, i64, i64, vp,
                                          i64, vp]
        lib.hadacore_adapters.restype = i32
        lib.hadacore_adapter_gradient_workspace_size.argtypes = [i64, i64, i64, i64]
        lib.hadacore_adapter_gradient_workspace_size.restype = i64
        lib.hadacore_adapter_gradient.argtypes = [vp, i64, vp, i64, i32, vp, vp, vp, i64, vp, i64, i64,
                                                  i32, i64, i64, i64, vp, i64, vp]
        lib.hadacore_adapter_gradient.restype = i32
        lib.hadacore_stream_copy.argtypes = [vp, vp, i64, vp]
        lib.hadacore_stream_copy.restype = i32
        lib.hadacore_status_string.argtypes = [i32]
        lib.hadacore_status_string.restype = ctypes.c_char_p
        lib.hadacore_version.argtypes = []
        lib.hadacore_version.restype = i32
        _lib = lib
    return _lib


def _check(status: int, where: str) -> None:
    if status != SUCCESS:
        raise HadacoreError(status, where)


def hadamard_transform(in_ptr: int, out_ptr: int, m: int, n: int, dtype: int, scale: float,
                       stream: int = 0, check: bool = True) -> int:
    st = library().hadamard_transform(in_ptr, out_ptr, m, n, dtype, scale, stream)
    if check:
        _check(st, "hadamard_transform")
    return st


def hadamard_transform_strided(in_ptr: int, in_row_stride: int, out_ptr: int,
                               out_row_stride: int, m: int, n: int, dtype: int, scale: float,
                               stream: int = 0, check: bool = True) -> int:
    st = library().hadamard_transform_strided(in_ptr, in_row_stride, out_ptr, out_row_stride,
                                              m, n, dtype, scale, stream)
    if check:
        _check(st, "hadamard_transform_strided")
    return st


def hadamard_transform_ws(in_ptr: int, in_row_stride: int, out_ptr: int, out_row_stride: int,
                          m: int, n: int, dtype: int, scale: float, workspace_ptr: int,
                          workspace_bytes: int, stream: int = 0, check: bool = True) -> int:
    st = library().hadamard_transform_ws(in_ptr, in_row_stride, out_ptr, out_row_stride, m, n,
                                         dtype, scale, workspace_ptr, workspace_bytes, stream)
    if check:
        _check(st, "hadamard_transform_ws")
    return st


def hadamard_transform_ws_noalloc(in_ptr: int, in_row_stride: int, out_ptr: int,
                                  out_row_stride: int, m: int, n: int, dtype: int, scale: float,
                                  stream: int = 0, check: bool = True) -> int:
    st = library().hadamard_transform_ws_noalloc(in_ptr, in_row_stride, out_ptr, out_row_stride,
                                                 m, n, dtype, scale, stream)
    if check:
        _check(st, "hadamard_transform_ws_noalloc")
    return st


def hadamard_transform_workspace_size(m: int, n: int) -> int:
    return int(library().hadamard_transform_workspace_size(m, n))


def hadamard_transform_fp8(in_ptr: int, in_row_stride: int, codes_ptr: int, codes_row_stride: int,
                           scales_ptr: int, m: int, n: int, dtype: int, scale: float,
                           stream: int = 0, check: bool = True) -> int:
    st = library().hadamard_transform_fp8(in_ptr, in_row_stride, codes_ptr, codes_row_stride,
                                          scales_ptr, m, n, dtype, scale, stream)
    if check:
        _check(st, "hadamard_transform_fp8")
    return st


def hadamard_transform_int8(in_ptr: int, in_row_stride: int, codes_ptr: int,
                            codes_row_stride: int, scales_ptr: int, m: int, n: int, dtype: int,
                            scale: float, stream: int = 0, check: bool = True) -> int:
    st = library().hadamard_transform_int8(in_ptr, in_row_stride, codes_ptr, codes_row_stride,
                                           scales_ptr, m, n, dtype, scale, stream)
    if check:
        _check(st, "hadamard_transform_int8")
    return st


def hadamard_transform_fp8_blocks(in_ptr: int, in_row_stride: int, codes_ptr: int,
                                  codes_row_stride: int, scales_ptr: int, scales_row_stride: int,
                                  m: int, k: int, n: int, dtype: int, scale: float,
                                  stream: int = 0, check: bool = True) -> int:
    st = library().hadamard_transform_fp8_blocks(in_ptr, in_row_stride, codes_ptr,
                                                 codes_row_stride, scales_ptr, scales_row_stride,
                                                 m, k, n, dtype, scale, stream)
    if check:
        _check(st, "hadamard_transform_fp8_blocks")
    return st


def hadacore_padded_tokens(tokens: int, groups: int) -> int:
    return int(library().hadacore_padded_tokens(tokens, groups))


def hadacore_quantize_fp8_columns(in_ptr: int, in_row_stride: int, ends_ptr: int, groups: int,
                                  codes_ptr: int, codes_row_stride: int, scales_ptr: int,
                                  scales_row_stride: int, m: int, k: int, dtype: int,
                                  stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_quantize_fp8_columns(in_ptr, in_row_stride, ends_ptr, groups, codes_ptr,
                                                 codes_row_stride, scales_ptr, scales_row_stride,
                                                 m, k, dtype, stream)
    if check:
        _check(st, "hadacore_quantize_fp8_columns")
    return st


def hadacore_quantize_fp8_tiles(in_ptr: int, in_row_stride: int, in_batch_stride: int,
                                codes_ptr: int, codes_row_stride: int, codes_batch_stride: int,
                                codes_t_ptr: int, codes_t_row_stride: int,
                                codes_t_batch_stride: int, scales_ptr: int,
                                scales_row_stride: int, scales_batch_stride: int, batch: int,
                                m: int, k: int, dtype: int, stream: int = 0,
                                check: bool = True) -> int:
    st = library().hadacore_quantize_fp8_tiles(
        in_ptr, in_row_stride, in_batch_stride, codes_ptr, codes_row_stride, codes_batch_stride,
        codes_t_ptr, codes_t_row_stride, codes_t_batch_stride, scales_ptr, scales_row_stride,
        scales_batch_stride, batch, m, k, dtype, stream)
    if check:
        _check(st, "hadacore_quantize_fp8_tiles")
    return st


def hadacore_matmul_fp8(a_ptr: int, a_row_stride: int, a_scales_ptr: int, a_scales_row_stride: int,
                        b_ptr: int, b_row_stride: int, b_scales_ptr: int, b_scales_row_stride: int,
                        b_scale_rows: int, out_ptr: int, out_row_stride: int, out_dtype: int,
                        m: int, n: int, k: int, stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_matmul_fp8(a_ptr, a_row_stride, a_scales_ptr, a_scales_row_stride,
                                       b_ptr, b_row_stride, b_scales_ptr, b_scales_row_stride,
                                       b_scale_rows, out_ptr, out_row_stride, out_dtype, m, n, k,
                                       stream)
    if check:
        _check(st, "hadacore_matmul_fp8")
    return st


def hadacore_matmul_fp8_grouped(a_ptr: int, a_row_stride: int, a_scales_ptr: int,
                                a_scales_row_stride: int, b_ptr: int, b_row_stride: int,
                                b_batch_stride: int, b_scales_ptr: int, b_scales_row_stride: int,
                                b_scales_batch_stride: int, ends_ptr: int, groups: int,
                                out_ptr: int, out_row_stride: int, out_dtype: int, m: int, n: int,
                                k: int, stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_matmul_fp8_grouped(
        a_ptr, a_row_stride, a_scales_ptr, a_scales_row_stride, b_ptr, b_row_stride,
        b_batch_stride, b_scales_ptr, b_scales_row_stride, b_scales_batch_stride, ends_ptr, groups,
        out_ptr, out_row_stride, out_dtype, m, n, k, stream)
    if check:
        _check(st, "hadacore_matmul_fp8_grouped")
    return st


def hadacore_weight_gradient_fp8_grouped(a_ptr: int, a_row_stride: int, a_scales_ptr: int,
                                         a_scales_row_stride: int, b_ptr: int, b_row_stride: int,
                                         b_scales_ptr: int, b_scales_row_stride: int,
                                         ends_ptr: int, groups: int, out_ptr: int,
                                         out_row_stride: int, out_batch_stride: int,
                                         out_dtype: int, places: int, n: int, k: int,
                                         stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_weight_gradient_fp8_grouped(
        a_ptr, a_row_stride, a_scales_ptr, a_scales_row_stride, b_ptr, b_row_stride, b_scales_ptr,
        b_scales_row_stride, ends_ptr, groups, out_ptr, out_row_stride, out_batch_stride,
        out_dtype, places, n, k, stream)
    if check:
        _check(st, "hadacore_weight_gradient_fp8_grouped")
    return st


def hadacore_route_workspace_size(m: int, experts: int) -> int:
    return int(library().hadacore_route_workspace_size(m, experts))


def hadacore_route(logits_ptr: int, logits_row_stride: int, dtype: int, valid_ptr: int, m: int,
                   experts: int, k: int, renormalize: int, experts_ptr: int, weights_ptr: int,
                   counts_ptr: int, loss_ptr: int, slopes_ptr: int, workspace_ptr: int,
                   workspace_bytes: int, stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_route(logits_ptr, logits_row_stride, dtype, valid_ptr, m, experts, k,
                                  renormalize, experts_ptr, weights_ptr, counts_ptr, loss_ptr,
                                  slopes_ptr, workspace_ptr, workspace_bytes, stream)
    if check:
        _check(st, "hadacore_route")
    return st


def hadacore_route_gradient(logits_ptr: int, logits_row_stride: int, dtype: int, chosen_ptr: int,
                            weights_ptr: int, slopes_ptr: int, dweights_ptr: int, dloss_ptr: int,
                            m: int, experts: int, k: int, renormalize: int, out_ptr: int,
                            out_row_stride: int, stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_route_gradient(logits_ptr, logits_row_stride, dtype, chosen_ptr,
                                           weights_ptr, slopes_ptr, dweights_ptr, dloss_ptr, m,
                                           experts, k, renormalize, out_ptr, out_row_stride, stream)
    if check:
        _check(st, "hadacore_route_gradient")
    return st


def hadacore_group_workspace_size(slots: int, groups: int) -> int:
    return int(library().hadacore_group_workspace_size(slots, groups))


def hadacore_group_tokens(ids_ptr: int, slots: int, groups: int, ends_ptr: int, rows_ptr: int,
                          slots_ptr: int, workspace_ptr: int, workspace_bytes: int, stream: int = 0,
                          check: bool = True) -> int:
    st = library().hadacore_group_tokens(ids_ptr, slots, groups, ends_ptr, rows_ptr, slots_ptr,
                                         workspace_ptr, workspace_bytes, stream)
    if check:
        _check(st, "hadacore_group_tokens")
    return st


def hadacore_dispatch_rows(in_ptr: int, in_row_stride: int, value_bytes: int, rows_ptr: int,
                           ends_ptr: int, groups: int, out_ptr: int, out_row_stride: int, m: int,
                           k: int, width: int, stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_dispatch_rows(in_ptr, in_row_stride, value_bytes, rows_ptr, ends_ptr,
                                          groups, out_ptr, out_row_stride, m, k, width, stream)
    if check:
        _check(st, "hadacore_dispatch_rows")
    return st


def hadacore_combine_rows(in_ptr: int, in_row_stride: int, places: int, dtype: int, rows_ptr: int,
                          weights_ptr: int, out_ptr: int, out_row_stride: int, m: int, k: int,
                          width: int, stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_combine_rows(in_ptr, in_row_stride, places, dtype, rows_ptr, weights_ptr,
                                         out_ptr, out_row_stride, m, k, width, stream)
    if check:
        _check(st, "hadacore_combine_rows")
    return st


def hadacore_combine_gradient(dout_ptr: int, dout_row_stride: int, y_ptr: int, y_row_stride: int,
                              dtype: int, rows_ptr: int, ends_ptr: int, groups: int,
                              weights_ptr: int, dy_ptr: int, dy_row_stride: int, dweights_ptr: int,
                              m: int, k: int, width: int, stream: int = 0,
                              check: bool = True) -> int:
    st = library().hadacore_combine_gradient(dout_ptr, dout_row_stride, y_ptr, y_row_stride, dtype,
                                             rows_ptr, ends_ptr, groups, weights_ptr, dy_ptr,
                                             dy_row_stride, dweights_ptr, m, k, width, stream)
    if check:
        _check(st, "hadacore_combine_gradient")
    return st


def hadacore_adapters_workspace_size(m: int, k: int, n: int, rank: int, groups: int) -> int:
    return int(library().hadacore_adapters_workspace_size(m, k, n, rank, groups))


def hadacore_adapters(x_ptr: int, x_row_stride: int, down_ptr: int, down_row_stride: int,
                      down_batch_stride: int, up_ptr: int, up_row_stride: int, up_batch_stride: int,
                      scales_ptr: int, ends_ptr: int, slots_ptr: int, groups: int, y_ptr: int,
                      y_row_stride: int, out_ptr: int, out_row_stride: int, dtype: int,
                      out_dtype: int, hidden_ptr: int, hidden_row_stride: int, m: int, k: int, n: int,
                      rank: int, workspace_ptr: int, workspace_bytes: int, stream: int = 0,
                      check: bool = True) -> int:
    st = library().hadacore_adapters(
        x_ptr, x_row_stride, down_ptr, down_row_stride, down_batch_stride, up_ptr, up_row_stride,
        up_batch_stride, scales_ptr, ends_ptr, slots_ptr, groups, y_ptr, y_row_stride, out_ptr,
        out_row_stride, dtype, out_dtype, hidden_ptr, hidden_row_stride, m, k, n, rank,
        workspace_ptr, workspace_bytes, stream)
    if check:
        _check(st, "hadacore_adapters")
    return st


def hadacore_adapter_gradient_workspace_size(m: int, width: int, rank: int, groups: int) -> int:
    return int(library().hadacore_adapter_gradient_workspace_size(m, width, rank, groups))


def hadacore_adapter_gradient(hidden_ptr: int, hidden_row_stride: int, x_ptr: int, x_row_stride: int,
                              dtype: int, scales_ptr: int, ends_ptr: int, slots_ptr: int, groups: int,
                              out_ptr: int, out_row_stride: int, out_batch_stride: int,
                              out_dtype: int, m: int, width: int, rank: int, workspace_ptr: int,
                              workspace_bytes: int, stream: int = 0, check: bool = True) -> int:
    st = library().hadacore_adapter_gradient(
        hidden_ptr, hidden_row_stride, x_ptr, x_row_stride, dtype, scales_ptr, ends_ptr, slots_ptr,
        groups, out_ptr, out_row_stride, out_batch_stride, out_dtype, m, width, rank, workspace_ptr,
        workspace_bytes, stream)
    if check:
        _check(st, "hadacore_adapter_gradient")
    return st


def hadacore_stream_copy(src_ptr: int, dst_ptr: int, nbytes: int, stream: int = 0,
                         check: bool = True) -> int:
    st = library().hadacore_stream_copy(src_ptr, dst_ptr, nbytes, stream)
    if check:
        _check(st, "hadacore_stream_copy")
    return st


def hadacore_status_string(status: int) -> str:
    return library().hadacore_status_string(status).decode()


def hadacore_version() -> int:
    return int(library().hadacore_version())


# What the tensor wrappers need of torch, looked up on the first call: a call is a
# few microseconds, of which module and attribute lookups, stream objects and
# device contexts were half.
_torch = None
_dtype_codes: dict = {}
_out_codes: dict = {}
_code_types: tuple = ()
_float32 = None
_raw_stream = None
_current_device = None
_one_device = False
# the default scale fp32(1/sqrt(n)) of every supported n
_SCALES = {1 << k: float(ctypes.c_float(1.0 / math.sqrt(1 << k)).value) for k in range(21)}


def _init_torch() -> None:
    global _torch, _raw_stream, _current_device, _one_device, _code_types, _float32
    import torch
    _dtype_codes.update({torch.float16: FP16, torch.bfloat16: BF16})
    _out_codes.update({torch.float16: FP16, torch.bfloat16: BF16, torch.float32: FP32})
    _code_types = (torch.uint8, torch.float8_e4m3fn)
    _float32 = torch.float32
    _current_device = torch.cuda.current_device
    _one_device = torch.cuda.device_count() == 1
    # the current stream's handle without building a Stream object
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
        lambda index: torch.cuda.current_stream(index).cuda_stream)
    _torch = torch


def _dtype_code(t) -> int:
    code = _dtype_codes.get(t.dtype)
    if code is None:
        raise TypeError(f"expected float16 or bfloat16, got {t.dtype}")
    return code


def _default_scale(n: int) -> float:
    scale = _SCALES.get(n)
    return float(ctypes.c_float(1.0 / math.sqrt(n)).value) if scale is None else scale


def _call(name: str, device: int, *args) -> None:
    """The library's entry point ``name`` with ``device`` current, which it nearly
    always is already (and is where there is only one)."""
    entry = getattr(_lib or library(), name)
    if _one_device or _current_device() == device:
        status = entry(*args)
    else:
        with _torch.cuda.device(device):
            status = entry(*args)
    if status != SUCCESS:
        raise HadacoreError(status, name)


class _Entered:
    """A stream given to a wrapper, which is torch's current one now."""
    __slots__ = ("stream", "cuda_stream")

    def __init__(self, stream):
        self.stream, self.cuda_stream = stream, stream.cuda_stream


def _on_stream(stream, x, call):
    """``call`` with ``stream`` (a torch stream or a handle; 0 is the default one), made torch's current one
    for the time: new outputs and workspaces are of its memory, which is handed out in its order.  Of
    torch's current stream they could be in use by work that is still to run there, or be handed out
    again before ``stream`` is done.  Outputs are marked as used on the caller's stream, too."""
    device = x.get_device()
    if device < 0:
        return call(None)  # which refuses such a tensor
    here = _torch.cuda.current_stream(device)
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else stream
    if handle == here.cuda_stream:
        return call(_Entered(here))
    if not isinstance(stream, _torch.cuda.Stream):
        stream = (_torch.cuda.ExternalStream(handle, device=device) if handle
                  else _torch.cuda.default_stream(device))
    elif stream.device_index != device:
        raise ValueError(f"the stream is of device {stream.device_index}, the tensors of {device}")
    with _torch.cuda.stream(stream):
        result = call(_Entered(stream))
    for t in result if isinstance(result, tuple) else (result,):
        if isinstance(t, _torch.Tensor):
            t.record_stream(here)
    return result


def transform(x, out=None, scale: float | None = None, n: int | None = None, stream=None,
              workspace=None):
    """out = scale * x @ H_n over the first ``n`` columns of each row of a 2-D tensor.

    ``x`` and ``out`` are 2-D float16/bfloat16 ROCm tensors with unit column
    stride; ``out=None`` allocates a new tensor, ``out=x`` runs in place.  The
    default scale is fp32(1/sqrt(n)); the default stream is torch's current one.
    n above 2^16 runs through ``hadamard_transform_ws``; ``workspace`` (a
    contiguous ROCm tensor of at least hadamard_transform_workspace_size(m, n)
    bytes) is allocated here when not given.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, x, lambda s: transform(x, out, scale, n, s, workspace))
    if x.dim() != 2 or not x.is_cuda:
        raise ValueError("expected a 2-D tensor on a ROCm device")
    in_stride, column = x.stride()
    if column != 1:
        raise ValueError("rows must be contiguous (column stride 1)")
    code = _dtype_code(x)
    m, columns = x.shape
    n = columns if n is None else int(n)
    if out is None:
        out = _torch.empty((m, n), dtype=x.dtype, device=x.device)
    elif (out is not x) and (out.dtype != x.dtype or out.device != x.device or out.dim() != 2
                             or out.stride(1) != 1):
        raise ValueError("out must be a 2-D tensor of the same dtype/device with column stride 1")
    rows, width = out.shape
    if rows != m or width < n or columns < n:
        raise ValueError("shape mismatch between x, out and n")
    if scale is None:
        scale = _default_scale(n)
    device = x.get_device()
    stream = _raw_stream(device) if stream is None else stream.cuda_stream
    # a single row's stride is never used to address anything; report n
    if m > 1:
        out_stride = out.stride(0)
    else:
        in_stride = out_stride = n
    if n > 1 << 16:
        if workspace is None:
            need = hadamard_transform_workspace_size(m, n)
            workspace = _torch.empty(max(need, 16), dtype=_torch.uint8, device=x.device)
        _call("hadamard_transform_ws", device, x.data_ptr(), in_stride, out.data_ptr(), out_stride,
              m, n, code, scale, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
              stream)
    else:
        _call("hadamard_transform_strided", device, x.data_ptr(), in_stride, out.data_ptr(),
              out_stride, m, n, code, scale, stream)
    return out


def _transform_quantized(x, codes, scales, scale, stream, entry, int8):
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, x, lambda s: _transform_quantized(x, codes, scales, scale, s, entry,
                                                                    int8))
    codes_dtype = _torch.int8 if int8 else _torch.uint8
    if x.dim() != 2 or not x.is_cuda or x.stride(1) != 1:
        raise ValueError("expected a 2-D ROCm tensor with contiguous rows")
    code = _dtype_code(x)
    m, n = x.shape
    if codes is None:
        codes = _torch.empty((m, n), dtype=codes_dtype, device=x.device)
    elif codes.dtype != codes_dtype or codes.dim() != 2 or codes.stride(1) != 1 \
            or tuple(codes.shape) != (m, n):
        raise ValueError(f"codes must be a (m, n) {codes_dtype} tensor with contiguous rows")
    if scales is None:
        scales = _torch.empty((m,), dtype=_torch.float32, device=x.device)
    elif scales.dtype != _torch.float32 or scales.numel() != m or not scales.is_contiguous():
        raise ValueError("scales must be a contiguous float32 tensor of m elements")
    if scale is None:
        scale = _default_scale(n)
    device = x.get_device()
    stream = _raw_stream(device) if stream is None else stream.cuda_stream
    in_stride = x.stride(0) if m > 1 else n
    codes_stride = codes.stride(0) if m > 1 else ((n + 15) // 16) * 16
    _call(entry, device, x.data_ptr(), in_stride, codes.data_ptr(), codes_stride,
          scales.data_ptr(), m, n, code, scale, stream)
    return codes, scales


def transform_fp8(x, codes=None, scales=None, scale: float | None = None, stream=None):
    """Fused transform + per-row e4m3 quantization of a 2-D float16/bfloat16 tensor.

    Returns (codes, scales): codes is a (m, n) torch.uint8 tensor of e4m3 bit
    patterns and scales a (m,) float32 tensor, so that
    x @ H_n * scale ~ codes.view(torch.float8_e4m3fn).float() * scales[:, None].
    """
    return _transform_quantized(x, codes, scales, scale, stream, "hadamard_transform_fp8", False)


def transform_int8(x, codes=None, scales=None, scale: float | None = None, stream=None):
    """Fused transform + symmetric per-row INT8 quantization of a 2-D float16/bfloat16
    tensor.  Returns (codes, scales): a (m, n) torch.int8 tensor and a (m,) float32
    tensor, so that x @ H_n * scale ~ codes.float() * scales[:, None].
    """
    return _transform_quantized(x, codes, scales, scale, stream, "hadamard_transform_int8", True)


# ---- e4m3 codes with a scale for each block of 128, and their products ----------


def _stream_of(stream, device: int):
    return _raw_stream(device) if stream is None else stream.cuda_stream


# The wrappers below allocate with empty_strided, a few tenths of a microsecond faster
# than empty, and read each attribute of a tensor once: their calls are as short as the others'.


def _padded_rows(shape: tuple, device):
    """A uint8 tensor whose rows start on 16-byte boundaries and are readable up to the
    next one (what lies there is ignored): what the quantizers write and the products read.
    Returns it and its row stride."""
    k = shape[-1]
    pitch = (k + 15) & ~15
    if len(shape) == 2:
        padded, steps = (shape[0], pitch), (pitch, 1)
    else:
        padded, steps = (shape[0], shape[1], pitch), (shape[1] * pitch, pitch, 1)
    codes = _torch.empty_strided(padded, steps, dtype=_torch.uint8, device=device)
    return codes if pitch == k else codes.narrow(-1, 0, k), pitch


def _operand(name: str, codes, scales, rows: int, device: int):
    """Checks of an operand's codes (2-D, or 3-D for a batch) and scales, of which there are
    ``rows`` to a matrix: types, devices, unit column strides, shapes, and that every row of
    codes is readable up to the next multiple of 16 bytes.  Returns the row strides of both;
    of a single row, whose stride is never used, one that passes."""
    if codes.dtype not in _code_types:
        raise TypeError(f"{name}: codes must be uint8 or float8_e4m3fn, got {codes.dtype}")
    if scales.dtype is not _float32:
        raise TypeError(f"{name}: scales must be float32, got {scales.dtype}")
    shape = codes.shape
    k = shape[-1]
    blocks = (k + 127) >> 7
    want = (rows, blocks) if len(shape) == 2 else (*shape[:-2], rows, blocks)
    if scales.shape != want:
        raise ValueError(f"{name}: expected scales of shape {want}, got {tuple(scales.shape)}")
    if codes.get_device() != device or scales.get_device() != device:
        raise ValueError(f"{name}: all tensors must be on the same ROCm device")
    steps, scale_steps = codes.stride(), scales.stride()
    if (steps[-1] != 1 and k > 1) or (scale_steps[-1] != 1 and blocks > 1):
        raise ValueError(f"{name}: rows must be contiguous (column stride 1)")
    if k & 15 and codes.numel():
        last = sum((n - 1) * s for n, s in zip(shape[:-1], steps))
        if codes.storage_offset() + last + ((k + 15) & ~15) > codes.untyped_storage().nbytes():
            raise ValueError(f"{name}: the last row of codes must be readable up to a multiple of "
                             "16 bytes (as the quantizers allocate it)")
    return (0 if k == 0 else steps[-2] if shape[-2] > 1 else (k + 15) & ~15,
            scale_steps[-2] if rows > 1 else blocks)


def _row_stride(t, least: int) -> int:
    """The row stride; of a single row, whose stride is never used, one that passes."""
    return t.stride(-2) if t.shape[-2] > 1 else least


def _new_scales(scales, shape: tuple, device):
    if scales is None:
        return _torch.empty_strided(shape, (shape[1], 1), dtype=_float32, device=device)
    if scales.dtype != _torch.float32 or tuple(scales.shape) != shape or scales.device != device \
            or (shape[-1] > 1 and scales.stride(-1) != 1):
        raise ValueError(f"scales must be a {shape} float32 tensor with contiguous rows")
    return scales


def _new_codes(codes, shape: tuple, device):
    """The codes' tensor and row stride (of a single row: its padded length; of empty rows 0)."""
    if codes is None:
        return _padded_rows(shape, device)
    if codes.dtype not in _code_types or tuple(codes.shape) != shape or codes.device != device \
            or (shape[-1] > 1 and codes.stride(-1) != 1):
        raise ValueError(f"codes must be a {shape} uint8 tensor with contiguous rows")
    k = shape[-1]
    return codes, 0 if k == 0 else codes.stride(-2) if shape[-2] > 1 else (k + 15) & ~15


def transform_fp8_blocks(x, n: int | None = None, codes=None, scales=None,
                         scale: float | None = None, stream=None):
    """Rotate each row of a 2-D float16/bfloat16 tensor in blocks of ``n`` and quantize it to
    e4m3 with one scale for every 128 columns.

    ``n`` is a power of two up to 32768 that divides the columns (default: all of them; 1:
    no rotation) and ``scale`` defaults to fp32(1/sqrt(n)).  Returns (codes, scales): (m, k)
    uint8 and (m, ceil(k / 128)) float32, the operand that ``matmul_fp8`` takes:
    (x.view(m, -1, n) @ H_n * scale).view(m, k) ~ codes * scales, a scale per 128 columns.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, x, lambda s: transform_fp8_blocks(x, n, codes, scales, scale, s))
    device = x.get_device()
    if device < 0 or x.dim() != 2:
        raise ValueError("expected a 2-D tensor on a ROCm device")
    m, k = x.shape
    in_stride, column = x.stride()
    if column != 1 and k > 1:
        raise ValueError("rows must be contiguous (column stride 1)")
    code = _dtype_code(x)
    n = max(k, 1) if n is None else int(n)
    blocks = (k + 127) >> 7
    where = x.device
    codes, pitch = _new_codes(codes, (m, k), where)
    scales = _new_scales(scales, (m, blocks), where)
    _call("hadamard_transform_fp8_blocks", device, x.data_ptr(), in_stride if m > 1 else k,
          codes.data_ptr(), pitch, scales.data_ptr(), _row_stride(scales, blocks), m, k, n,
          code, _default_scale(n) if scale is None else scale, _stream_of(stream, device))
    return codes, scales


def _check_ends(ends, device: int) -> None:
    if ends.dtype != _torch.int32 or ends.dim() != 1 or not ends.is_contiguous():
        raise ValueError("ends must be a contiguous 1-D int32 tensor: the end of each group")
    if ends.get_device() != device:
        raise ValueError("ends must be on the same ROCm device")


def quantize_fp8_columns(x, ends=None, codes=None, scales=None, stream=None):
    """Quantize the columns of a 2-D float16/bfloat16 tensor (tokens x features) to
    transposed e4m3 codes with one scale for every 128 tokens: the operands of
    ``grouped_weight_gradient_fp8``.

    ``ends`` (int32, on the device) holds the end of each group of tokens; None is one
    group.  Each group is padded with zeros to a multiple of 128 places.  Returns (codes,
    scales): (k, p) uint8 and (k, p / 128) float32 with p =
    hadacore_padded_tokens(tokens, groups).
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, x, lambda s: quantize_fp8_columns(x, ends, codes, scales, s))
    device = x.get_device()
    if device < 0 or x.dim() != 2:
        raise ValueError("expected a 2-D tensor on a ROCm device")
    m, k = x.shape
    in_stride, column = x.stride()
    if column != 1 and k > 1:
        raise ValueError("rows must be contiguous (column stride 1)")
    code = _dtype_code(x)
    groups, ends_ptr = 1, None
    if ends is not None:
        _check_ends(ends, device)
        groups, ends_ptr = ends.shape[0], ends.data_ptr()
    blocks = (m + 127 * min(groups, m)) >> 7  # hadacore_padded_tokens
    where = x.device
    codes, pitch = _new_codes(codes, (k, blocks << 7), where)
    scales = _new_scales(scales, (k, blocks), where)
    _call("hadacore_quantize_fp8_columns", device, x.data_ptr(), in_stride if m > 1 else k, ends_ptr,
          groups, codes.data_ptr(), pitch, scales.data_ptr(), _row_stride(scales, blocks), m,
          k, code, _stream_of(stream, device))
    return codes, scales


def quantize_fp8_tiles(w, transposed: bool = False, stream=None):
    """Quantize float16/bfloat16 weights (n x k, or experts x n x k) to e4m3 with one scale
    for every tile of 128 x 128.

    Returns (codes, scales), codes of w's shape and scales ceil(n / 128) x ceil(k / 128) for
    each matrix; with ``transposed`` (codes, scales, codes_t), where codes_t holds the same
    codes as k x n matrices, whose scales are ``scales.transpose(-1, -2).contiguous()``.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, w, lambda s: quantize_fp8_tiles(w, transposed, s))
    device = w.get_device()
    lead = w.shape[:-2]
    if device < 0 or len(lead) != w.dim() - 2 or len(lead) > 1:
        raise ValueError("expected a 2-D or 3-D tensor on a ROCm device")
    n, k = w.shape[-2:]
    steps, where = w.stride(), w.device
    if steps[-1] != 1 and k > 1:
        raise ValueError("rows must be contiguous (column stride 1)")
    code = _dtype_code(w)
    rows, blocks = (n + 127) >> 7, (k + 127) >> 7
    batch = lead[0] if lead else 1
    codes, pitch = _padded_rows((batch, n, k) if lead else (n, k), where)
    scales = _torch.empty_strided((batch, rows, blocks) if lead else (rows, blocks),
                                  (rows * blocks, blocks, 1) if lead else (blocks, 1),
                                  dtype=_float32, device=where)
    codes_t, address_t, pitch_t = None, None, 0
    if transposed:
        codes_t, pitch_t = _padded_rows((batch, k, n) if lead else (k, n), where)
        address_t = codes_t.data_ptr()
    # the steps from one matrix to the next are not used for a single one
    _call("hadacore_quantize_fp8_tiles", device, w.data_ptr(), steps[-2] if n > 1 else k,
          steps[0] if lead else 0, codes.data_ptr(), pitch, n * pitch, address_t, pitch_t,
          k * pitch_t, scales.data_ptr(), blocks, rows * blocks, batch, n, k, code,
          _stream_of(stream, device))
    return (codes, scales, codes_t) if transposed else (codes, scales)


def _product_out(out, shape: tuple, dtype, like):
    """The output of a product, its type's code and its row stride."""
    if out is None:
        dtype = dtype or _torch.bfloat16
        code = _out_codes.get(dtype)
        if code is not None:
            n = shape[-1]
            steps = (n, 1) if len(shape) == 2 else (shape[1] * n, n, 1)
            return (_torch.empty_strided(shape, steps, dtype=dtype, device=like.device), code, n)
        raise TypeError(f"expected an output of float16, bfloat16 or float32, got {dtype}")
    if out.shape != shape or out.device != like.device or \
            (shape[-1] > 1 and out.stride(-1) != 1) or (dtype is not None and out.dtype != dtype):
        raise ValueError(f"out must be a {shape} tensor of the output type with contiguous rows")
    code = _out_codes.get(out.dtype)
    if code is None:
        raise TypeError(f"expected an output of float16, bfloat16 or float32, got {out.dtype}")
    return out, code, out.stride(-2) if shape[-2] > 1 else shape[-1]


def matmul_fp8(a, a_scales, b, b_scales, out=None, dtype=None, stream=None):
    """out = A @ B^T for e4m3 codes with a scale for each block of 128.

    ``a`` (m x k) and ``a_scales`` (m x ceil(k / 128)) are as ``transform_fp8_blocks`` gives
    them.  ``b`` (n x k) has a scale per tile of 128 x 128 (``quantize_fp8_tiles``) or one per
    row and 128 columns, told apart by the rows of ``b_scales``.  The product of two scales
    has to be in fp32's range: they are multiplied first.  ``dtype`` is the output's:
    bfloat16 (default), float16 or float32.  Blocks are added in 32 bits and the result is
    rounded once; inside a block a float32 output's sums are fp32, and a 16-bit output's
    are within 2^-9 of the block's largest product (about 17 bits below it are kept), which
    shows where large products cancel.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, a, lambda s: matmul_fp8(a, a_scales, b, b_scales, out, dtype, s))
    device = a.get_device()
    if device < 0 or a.dim() != 2 or b.dim() != 2:
        raise ValueError("expected 2-D tensors on a ROCm device")
    m, k = a.shape
    n, k_b = b.shape
    if k_b != k:
        raise ValueError(f"a has {k} columns and b {k_b}")
    tiles = (n + 127) >> 7
    by_row = n != tiles and b_scales.dim() == 2 and b_scales.shape[0] == n
    a_stride, sa_stride = _operand("a", a, a_scales, m, device)
    b_stride, sb_stride = _operand("b", b, b_scales, n if by_row else tiles, device)
    out, code, out_stride = _product_out(out, (m, n), dtype, a)
    _call("hadacore_matmul_fp8", device, a.data_ptr(), a_stride, a_scales.data_ptr(), sa_stride,
          b.data_ptr(), b_stride, b_scales.data_ptr(), sb_stride, 1 if by_row else 128,
          out.data_ptr(), out_stride, code, m, n, k, _stream_of(stream, device))
    return out


def grouped_matmul_fp8(a, a_scales, b, b_scales, ends, out=None, dtype=None, stream=None):
    """``matmul_fp8`` with a weight of its own for each group of rows (tokens by expert).

    The rows of ``a`` (m x k) are sorted by group and ``ends`` (int32, on the device) holds
    the end of each group, which may be empty; ``b`` is groups x n x k with a scale per tile
    of 128 x 128.  Row i of group g gets a[i] @ b[g]^T; rows after the last end get zeros.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, a, lambda s: grouped_matmul_fp8(a, a_scales, b, b_scales, ends,
                                                                  out, dtype, s))
    device = a.get_device()
    if device < 0 or a.dim() != 2 or b.dim() != 3:
        raise ValueError("expected a 2-D and a 3-D tensor on a ROCm device")
    m, k = a.shape
    groups, n, k_b = b.shape
    if k_b != k:
        raise ValueError(f"a has {k} columns and b {k_b}")
    _check_ends(ends, device)
    if ends.shape[0] != groups:
        raise ValueError(f"{ends.shape[0]} ends for {groups} groups")
    a_stride, sa_stride = _operand("a", a, a_scales, m, device)
    b_stride, sb_stride = _operand("b", b, b_scales, (n + 127) >> 7, device)
    out, code, out_stride = _product_out(out, (m, n), dtype, a)
    _call("hadacore_matmul_fp8_grouped", device, a.data_ptr(), a_stride, a_scales.data_ptr(),
          sa_stride, b.data_ptr(), b_stride, b.stride(0), b_scales.data_ptr(), sb_stride,
          b_scales.stride(0), ends.data_ptr(), groups, out.data_ptr(), out_stride, code, m, n, k,
          _stream_of(stream, device))
    return out


def grouped_weight_gradient_fp8(dy, dy_scales, x, x_scales, ends=None, out=None, dtype=None,
                                stream=None):
    """The weight gradients of ``grouped_matmul_fp8``: for each group, dy^T x over its tokens.

    ``dy`` (n x places) and ``x`` (k x places) are the transposed codes that
    ``quantize_fp8_columns`` gives for the output's gradient and the input, with the same
    ``ends``; a group without tokens gets zeros.  ``ends=None`` is one group of all places.
    Returns groups x n x k, or n x k without ends.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, dy, lambda s: grouped_weight_gradient_fp8(dy, dy_scales, x,
                                                                            x_scales, ends, out,
                                                                            dtype, s))
    device = dy.get_device()
    if device < 0 or dy.dim() != 2 or x.dim() != 2:
        raise ValueError("expected 2-D tensors on a ROCm device")
    n, places = dy.shape
    k, places_x = x.shape
    if places_x != places:
        raise ValueError(f"dy has {places} places and x {places_x}")
    dy_stride, sdy_stride = _operand("dy", dy, dy_scales, n, device)
    x_stride, sx_stride = _operand("x", x, x_scales, k, device)
    if ends is None:
        groups, ends_ptr, shape = 1, None, (n, k)
    else:
        _check_ends(ends, device)
        groups, ends_ptr = ends.shape[0], ends.data_ptr()
        shape = (groups, n, k)
    out, code, out_stride = _product_out(out, shape, dtype, dy)
    _call("hadacore_weight_gradient_fp8_grouped", device, dy.data_ptr(), dy_stride,
          dy_scales.data_ptr(), sdy_stride, x.data_ptr(), x_stride, x_scales.data_ptr(), sx_stride,
          ends_ptr, groups, out.data_ptr(), out_stride, out.stride(0) if groups > 1 else 0, code,
          places, n, k, _stream_of(stream, device))
    return out


# ---- tokens and weights of their own: routing, the exchange by expert, adapters ----------


class Routes(NamedTuple):
    """What ``route_tokens`` gives: the experts of each token (m x k, -1: none), their weights
    (m x k), how many tokens each expert got, the balance loss (a scalar), and its derivative to
    each token's probability of an expert."""
    experts: "torch.Tensor"  # noqa: F821
    weights: "torch.Tensor"  # noqa: F821
    counts: "torch.Tensor"  # noqa: F821
    loss: "torch.Tensor"  # noqa: F821
    slopes: "torch.Tensor"  # noqa: F821
    renormalize: bool


class Groups(NamedTuple):
    """What ``group_tokens`` gives: the ends of the groups, the place of each slot (in the ids'
    shape, -1: none) and the slot of each place."""
    ends: "torch.Tensor"  # noqa: F821
    rows: "torch.Tensor"  # noqa: F821
    slots: "torch.Tensor"  # noqa: F821


_route_workspace = functools.lru_cache(maxsize=1024)(hadacore_route_workspace_size)
_group_workspace = functools.lru_cache(maxsize=1024)(hadacore_group_workspace_size)
_adapters_workspace = functools.lru_cache(maxsize=1024)(hadacore_adapters_workspace_size)
_adapter_gradient_workspace = functools.lru_cache(maxsize=1024)(
    hadacore_adapter_gradient_workspace_size)


def _words(n: int, device, dtype=None):
    return _torch.empty_strided((n,), (1,), dtype=dtype or _torch.int32, device=device)


def _scratch(nbytes: int, device, stream):
    """A workspace (None for no bytes) of the current stream's memory, which a stream given to the wrapper
    has become; marked as that stream's, so that it is not reused before its work is done."""
    if not nbytes:
        return None, None
    t = _words(nbytes >> 2, device)
    if stream is not None:
        t.record_stream(stream.stream)
    return t, t.data_ptr()


def _matrix(name: str, t, device: int, dims: int = 2):
    """Checks of a tensor with contiguous rows; the row stride (one that passes for a single row)."""
    if t.dim() != dims:
        raise ValueError(f"{name}: expected {dims} dimensions, got {t.dim()}")
    if t.get_device() != device or device < 0:
        raise ValueError(f"{name}: all tensors must be on the same ROCm device")
    shape, steps = t.shape, t.stride()
    width = shape[-1]
    if steps[-1] != 1 and width > 1:
        raise ValueError(f"{name}: rows must be contiguous (column stride 1)")
    return steps[-2] if shape[-2] > 1 else width


def _dense(name: str, t, dtype, shape, device: int):
    """Checks of a dense tensor of `shape`; its address."""
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: expected the shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name}: all tensors must be on the same ROCm device")
    if not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    return t.data_ptr()


def _value_code(name: str, t) -> int:
    code = _out_codes.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: expected float16, bfloat16 or float32, got {t.dtype}")
    return code


def _output(out, shape: tuple, dtype, device):
    if out is None:
        return _torch.empty_strided(shape, (shape[1], 1), dtype=dtype, device=device)
    if out.shape != shape or out.dtype is not dtype or out.device != device \
            or (out.stride(1) != 1 and shape[1] > 1):
        raise ValueError(f"out must be a {shape} {dtype} tensor with contiguous rows")
    return out


def route_tokens(logits, k: int, renormalize: bool = True, valid=None, stream=None) -> Routes:
    """The ``k`` experts with the largest logits for each token (m x experts; float16, bfloat16 or
    float32), their softmax weights, the number of tokens that each got, and the balance loss
    experts * sum_e f_e P_e of the shares f of the choices and the mean probabilities P.

    Equal logits go to the lower index.  An expert at -inf is never chosen; a token with too few
    others gets -1 and weight 0 there, as does one whose ``valid`` (m truth values) is false, which
    counts nowhere.  Weights are probabilities, over their sum with ``renormalize``.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, logits, lambda s: route_tokens(logits, k, renormalize, valid, s))
    device = logits.get_device()
    stride = _matrix("logits", logits, device)
    code = _value_code("logits", logits)
    m, experts = logits.shape
    valid_ptr = None
    if valid is not None:
        valid_ptr = _dense("valid", valid, _torch.bool, (m,), device)
    where = logits.device
    chosen = _torch.empty_strided((m, k), (k, 1), dtype=_torch.int32, device=where)
    weights = _torch.empty_strided((m, k), (k, 1), dtype=_float32, device=where)
    counts = _words(experts, where)
    slopes = _words(experts, where, _float32)
    loss = _torch.empty_strided((), (), dtype=_float32, device=where)
    need = _route_workspace(m, experts)
    workspace, workspace_ptr = _scratch(need, where, stream)
    _call("hadacore_route", device, logits.data_ptr(), stride, code, valid_ptr, m, experts, k,
          renormalize, chosen.data_ptr(), weights.data_ptr(), counts.data_ptr(), loss.data_ptr(),
          slopes.data_ptr(), workspace_ptr, need, _stream_of(stream, device))
    return Routes(chosen, weights, counts, loss, slopes, renormalize)


def route_tokens_gradient(logits, routes: Routes, dweights=None, dloss=None, out=None, stream=None):
    """The logits' gradient, in their type, for the gradients of ``routes.weights`` (m x k) and of
    ``routes.loss`` (a scalar tensor); None is no gradient."""
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, logits, lambda s: route_tokens_gradient(logits, routes,
                                                                          dweights, dloss, out, s))
    device = logits.get_device()
    stride = _matrix("logits", logits, device)
    code = _value_code("logits", logits)
    m, experts = logits.shape
    k = routes.experts.shape[-1]
    chosen = _dense("routes.experts", routes.experts, _torch.int32, (m, k), device)
    weights = _dense("routes.weights", routes.weights, _float32, (m, k), device)
    slopes = _dense("routes.slopes", routes.slopes, _float32, (experts,), device)
    dw = dl = None
    if dweights is not None:
        dw = _dense("dweights", dweights, _float32, (m, k), device)
    if dloss is not None:
        dl = _dense("dloss", dloss, _float32, (), device)
    out = _output(out, (m, experts), logits.dtype, logits.device)
    _call("hadacore_route_gradient", device, logits.data_ptr(), stride, code, chosen, weights, slopes,
          dw, dl, m, experts, k, routes.renormalize, out.data_ptr(), _row_stride(out, experts),
          _stream_of(stream, device))
    return out


def group_tokens(ids, groups: int, stream=None) -> Groups:
    """Slots sorted by group: ``ids`` (tokens, or tokens x choices; int32) holds each slot's group,
    anything outside [0, groups) for none.

    Returns (ends, rows, slots): ``ends`` as the products by expert take them, ``rows`` the place of
    each slot (-1 without a group) and ``slots`` the slot of each place, those without a
    group behind the last end.  Slots of a group keep their order.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, ids, lambda s: group_tokens(ids, groups, s))
    device = ids.get_device()
    if device < 0 or ids.dim() not in (1, 2) or ids.dtype is not _torch.int32 or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous 1-D or 2-D int32 tensor on a ROCm device")
    n, where = ids.numel(), ids.device
    ends, slots = _words(groups, where), _words(n, where)
    rows = _torch.empty_strided(ids.shape, ids.stride(), dtype=_torch.int32, device=where)
    need = _group_workspace(n, groups)
    workspace, workspace_ptr = _scratch(need, where, stream)
    _call("hadacore_group_tokens", device, ids.data_ptr(), n, groups, ends.data_ptr(), rows.data_ptr(),
          slots.data_ptr(), workspace_ptr, need, _stream_of(stream, device))
    return Groups(ends, rows, slots)


def _slots_of(rows, device: int):
    """Tokens and choices of ``rows`` (tokens, or tokens x choices), and its address."""
    if rows.dtype is not _torch.int32 or rows.dim() not in (1, 2) or not rows.is_contiguous():
        raise ValueError("rows must be a contiguous 1-D or 2-D int32 tensor")
    if rows.get_device() != device:
        raise ValueError("rows: all tensors must be on the same ROCm device")
    shape = rows.shape
    return shape[0], shape[1] if len(shape) == 2 else 1, rows.data_ptr()


def dispatch_rows(x, rows, ends, out=None, stream=None):
    """The rows of ``x`` (tokens x width, values of 1, 2 or 4 bytes: codes and their scales too) at
    the places of their slots: (tokens * choices) x width, zeros behind the last end.  ``rows``
    and ``ends`` are ``group_tokens``'.  Its gradient is ``combine_rows`` without weights."""
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, x, lambda s: dispatch_rows(x, rows, ends, out, s))
    device = x.get_device()
    stride = _matrix("x", x, device)
    m, k, rows_ptr = _slots_of(rows, device)
    tokens, width = x.shape
    if tokens != m:
        raise ValueError(f"x has {tokens} rows and rows {m} tokens")
    _check_ends(ends, device)
    size = x.element_size()
    if size not in (1, 2, 4):
        raise TypeError(f"expected values of 1, 2 or 4 bytes, got {x.dtype}")
    if out is None and size == 1:
        out, _ = _padded_rows((m * k, width), x.device)
        if x.dtype is not _torch.uint8:
            out = out.view(x.dtype)
    else:
        out = _output(out, (m * k, width), x.dtype, x.device)
    _call("hadacore_dispatch_rows", device, x.data_ptr(), stride, size, rows_ptr, ends.data_ptr(),
          ends.shape[0], out.data_ptr(), _row_stride(out, width), m, k, width,
          _stream_of(stream, device))
    return out


def combine_rows(y, rows, weights=None, out=None, stream=None):
    """The rows of each token's slots, added by weight: out[t] = sum_j weights[t, j] * y[rows[t, j]]
    (tokens x width, in y's type: float16, bfloat16 or float32), summed in 32 bits.  A slot
    without a row (-1) adds nothing; ``weights`` is float32 of rows' shape, or None for the sum."""
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, y, lambda s: combine_rows(y, rows, weights, out, s))
    device = y.get_device()
    stride = _matrix("y", y, device)
    code = _value_code("y", y)
    m, k, rows_ptr = _slots_of(rows, device)
    places, width = y.shape
    weights_ptr = None if weights is None else _dense("weights", weights, _float32, rows.shape, device)
    out = _output(out, (m, width), y.dtype, y.device)
    _call("hadacore_combine_rows", device, y.data_ptr(), stride, places, code, rows_ptr, weights_ptr,
          out.data_ptr(), _row_stride(out, width), m, k, width, _stream_of(stream, device))
    return out


def combine_rows_gradient(dout, y, rows, ends, weights=None, want_dy: bool = True, stream=None):
    """(dy, dweights) of ``combine_rows`` for the gradient ``dout`` of its output: dy in dout's type,
    zeros behind the last end, and dweights in float32 and rows' shape.  ``y=None`` leaves
    dweights out, ``want_dy=False`` dy: None in their places."""
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, dout, lambda s: combine_rows_gradient(dout, y, rows, ends,
                                                                        weights, want_dy, s))
    device = dout.get_device()
    stride = _matrix("dout", dout, device)
    code = _value_code("dout", dout)
    m, k, rows_ptr = _slots_of(rows, device)
    tokens, width = dout.shape
    if tokens != m:
        raise ValueError(f"dout has {tokens} rows and rows {m} tokens")
    _check_ends(ends, device)
    weights_ptr = None if weights is None else _dense("weights", weights, _float32, rows.shape, device)
    y_ptr, y_stride, dweights, dw_ptr = None, width, None, None
    if y is not None:
        y_stride = _matrix("y", y, device)
        if y.dtype is not dout.dtype or y.shape != (m * k, width):
            raise ValueError(f"y must be a {(m * k, width)} {dout.dtype} tensor")
        y_ptr = y.data_ptr()
        dweights = _torch.empty_strided(rows.shape, rows.stride(), dtype=_float32, device=dout.device)
        dw_ptr = dweights.data_ptr()
    dy = dy_ptr = None
    if want_dy:
        dy = _torch.empty_strided((m * k, width), (width, 1), dtype=dout.dtype, device=dout.device)
        dy_ptr = dy.data_ptr()
    _call("hadacore_combine_gradient", device, dout.data_ptr(), stride, y_ptr, y_stride, code, rows_ptr,
          ends.data_ptr(), ends.shape[0], weights_ptr, dy_ptr, width, dw_ptr, m, k, width,
          _stream_of(stream, device))
    return dy, dweights


def _plan(ends, slots, scales, m: int, device: int):
    """Groups of the adapters, and the addresses of ends, slots and scales."""
    groups, ends_ptr, slots_ptr, scales_ptr = 1, None, None, None
    if ends is not None:
        _check_ends(ends, device)
        groups, ends_ptr = ends.shape[0], ends.data_ptr()
    if slots is not None:
        slots_ptr = _dense("slots", slots, _torch.int32, (m,), device)
    if scales is not None:
        scales_ptr = _dense("scales", scales, _float32, (groups,), device)
    return groups, ends_ptr, slots_ptr, scales_ptr


def adapt_rows(x, down, up, ends=None, slots=None, y=None, scales=None, out=None, dtype=None,
               hidden: bool = False, stream=None):
    """Low-rank adapters, one for each group of tokens: out[t] = y[t] + scales[g] * (x[t] @ down[g]^T)
    @ up[g] for the tokens of group g, and y[t] for those of none.

    ``x`` is tokens x k, ``down`` groups x rank x k and ``up`` groups x rank x n (float16 or bfloat16):
    both weights are stored rank by rank.  ``ends`` and ``slots`` are ``group_tokens``' for one id a
    token; ``slots=None``: the tokens are sorted themselves; ``ends=None``: one adapter (``down``
    and ``up`` without the first dimension, or with one of 1) for all.  ``y`` (tokens x n, x's
    type or float32) may be ``out``; without it the output is of ``dtype`` (default x's).  With
    ``hidden`` returns (out, h), h (tokens x rank, float32) the first products by place, for
    ``adapter_gradient``; its rows behind the last end are not written.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, x, lambda s: adapt_rows(x, down, up, ends, slots, y, scales,
                                                          out, dtype, hidden, s))
    device = x.get_device()
    x_stride = _matrix("x", x, device)
    code = _dtype_code(x)
    if ends is None and down.dim() == 2 and up.dim() == 2:
        down, up = down[None], up[None]
    down_stride, up_stride = _matrix("down", down, device, 3), _matrix("up", up, device, 3)
    m, k = x.shape
    groups, rank, k_down = down.shape
    n = up.shape[2]
    if down.dtype is not x.dtype or up.dtype is not x.dtype:
        raise TypeError(f"down and up must be {x.dtype}, as x, got {down.dtype} and {up.dtype}")
    count, ends_ptr, slots_ptr, scales_ptr = _plan(ends, slots, scales, m, device)
    if k_down != k or up.shape[:2] != (groups, rank) or count != groups:
        raise ValueError(f"x of {tuple(x.shape)}, down of {tuple(down.shape)}, up of {tuple(up.shape)} "
                         f"and {count} groups do not go together")
    y_ptr, y_stride, where = None, n, x.device
    if y is not None:
        y_stride = _matrix("y", y, device)
        if y.shape != (m, n) or (dtype is not None and y.dtype is not dtype):
            raise ValueError(f"y must be a {(m, n)} tensor of the output's type")
        dtype, y_ptr = y.dtype, y.data_ptr()
    elif dtype is None:
        dtype = x.dtype
    if dtype is not x.dtype and dtype is not _float32:
        raise TypeError(f"expected an output of {x.dtype} or float32, got {dtype}")
    if out is None or out is not y:
        out = _output(out, (m, n), dtype, where)
    h_ptr, padded = None, (rank + 15) & ~15
    if hidden:
        h = _torch.empty_strided((m, padded), (padded, 1), dtype=_float32, device=where)
        h_ptr = h.data_ptr()
    need = _adapters_workspace(m, k, n, rank, groups)
    workspace, workspace_ptr = _scratch(need, where, stream)
    _call("hadacore_adapters", device, x.data_ptr(), x_stride, down.data_ptr(), down_stride,
          down.stride(0), up.data_ptr(), up_stride, up.stride(0), scales_ptr, ends_ptr, slots_ptr,
          groups, y_ptr, y_stride, out.data_ptr(), _row_stride(out, n), code, _out_codes[dtype], h_ptr,
          padded, m, k, n, rank, workspace_ptr, need, _stream_of(stream, device))
    if not hidden:
        return out
    return out, h if padded == rank else h.narrow(1, 0, rank)


def adapter_gradient(h, x, ends=None, slots=None, scales=None, out=None, dtype=None, stream=None):
    """The gradient of an adapter's weight: scales[g] * sum over the tokens of group g of h x^T, groups x
    rank x width (rank x width without ``ends``).

    For out = ``adapt_rows(x, down, up, ..., hidden=True)`` with hidden values h and the gradient
    dout: dx and dh are ``adapt_rows(dout, up, down, ..., hidden=True)`` of the same groups, up's gradient
    ``adapter_gradient(h, dout, ...)`` and down's ``adapter_gradient(dh, x, ...)``.  ``dtype`` is x's
    (default) or float32.  A group without tokens gets zeros.
    """
    if _torch is None:
        _init_torch()
    if stream is not None and type(stream) is not _Entered:
        return _on_stream(stream, x, lambda s: adapter_gradient(h, x, ends, slots, scales, out,
                                                                dtype, s))
    device = x.get_device()
    x_stride, h_stride = _matrix("x", x, device), _matrix("h", h, device)
    code = _dtype_code(x)
    m, width = x.shape
    if h.dtype is not _float32 or h.shape[0] != m:
        raise ValueError(f"h must be a float32 tensor of {m} rows")
    rank = h.shape[1]
    groups, ends_ptr, slots_ptr, scales_ptr = _plan(ends, slots, scales, m, device)
    shape = (rank, width) if ends is None else (groups, rank, width)
    if out is None:
        steps = (width, 1) if ends is None else (rank * width, width, 1)
        dtype = dtype or x.dtype
        if dtype is not x.dtype and dtype is not _float32:
            raise TypeError(f"expected an output of {x.dtype} or float32, got {dtype}")
        out = _torch.empty_strided(shape, steps, dtype=dtype, device=x.device)
    elif out.shape != shape or out.device != x.device or (width > 1 and out.stride(-1) != 1) \
            or out.dtype not in (x.dtype, _float32) or (dtype is not None and out.dtype is not dtype):
        raise ValueError(f"out must be a {shape} tensor of the output's type with contiguous rows")
    need = _adapter_gradient_workspace(m, width, rank, groups)
    workspace, workspace_ptr = _scratch(need, x.device, stream)
    _call("hadacore_adapter_gradient", device, h.data_ptr(), h_stride, x.data_ptr(), x_stride, code,
          scales_ptr, ends_ptr, slots_ptr, groups, out.data_ptr(), _row_stride(out, width),
          out.stride(0) if ends is not None else 0, _out_codes[out.dtype], m, width, rank,
          workspace_ptr, need, _stream_of(stream, device))
    return out
