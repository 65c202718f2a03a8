"""ctypes binding of libhadacore (``include/hadacore.h``).

Argument marshalling only: every step of the transform runs in the HIP
kernels of ``libhadacore.so``.  The library is loaded from this package
directory; if it is missing, every call raises (there is no fallback).

The raw entry points take device addresses as integers and keep the C names:
``hadamard_transform``, ``hadamard_transform_strided``, ``hadamard_transform_ws``,
``hadamard_transform_ws_noalloc``, ``hadamard_transform_workspace_size``, ``hadamard_transform_fp8``,
``hadamard_transform_int8``, ``hadamard_transform_fp8_blocks``, ``hadacore_padded_tokens``,
``hadacore_quantize_fp8_columns``, ``hadacore_quantize_fp8_tiles``, ``hadacore_matmul_fp8``,
``hadacore_matmul_fp8_grouped``, ``hadacore_weight_gradient_fp8_grouped``,
``hadacore_stream_copy``, ``hadacore_status_string``, ``hadacore_version``.  ``transform``,
``transform_fp8`` and ``transform_int8`` are convenience wrappers for 2-D torch tensors on a
ROCm device, and so are, for codes with a scale per block of 128, ``transform_fp8_blocks``,
``quantize_fp8_columns``, ``quantize_fp8_tiles``, ``matmul_fp8``, ``grouped_matmul_fp8`` and
``grouped_weight_gradient_fp8``.
"""
from __future__ import annotations

import ctypes
import math
from pathlib import Path

LIBRARY = Path(__file__).resolve().parent / "libhadacore.so"

FP16 = 0
BF16 = 1
FP32 = 2  # output of the FP8 products only
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
    if stream is None:
        stream = _raw_stream(device)
    elif hasattr(stream, "cuda_stream"):
        stream = stream.cuda_stream
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
    if stream is None:
        stream = _raw_stream(device)
    elif hasattr(stream, "cuda_stream"):
        stream = stream.cuda_stream
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
    if stream is None:
        return _raw_stream(device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


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
