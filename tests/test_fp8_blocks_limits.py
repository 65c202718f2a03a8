"""Sizes and strides near the ends of int64 at the FP8 entry points, on the CPU: refused, with
no sum or product of arguments that does not fit."""
from __future__ import annotations

from pathlib import Path

import pytest

from paper_2412_08832_amd import hadacore as H
from test_fp8_blocks_abi import COLUMNS, GRADIENT, GROUPED, MATMUL, ROWS, TILES, _status

# as in test_fp8_blocks_abi: no call here has arguments that validation would accept
cpu_only = pytest.mark.skipif(Path("/dev/kfd").exists(),
                              reason="fake-pointer validation tests run only without a GPU")
LARGEST = 2 ** 63 - 1


def test_padded_tokens_saturate():
    """The largest multiple of 128 where the places do not fit."""
    top = LARGEST // 128 * 128
    assert H.hadacore_padded_tokens(LARGEST, 0) == top
    assert H.hadacore_padded_tokens(LARGEST, 1) == top
    assert H.hadacore_padded_tokens(2 ** 62, 2 ** 62) == top
    assert H.hadacore_padded_tokens(2 ** 60, 2 ** 60) == top
    assert H.hadacore_padded_tokens(2 ** 56, 2 ** 55) == 2 ** 56 + 127 * 2 ** 55
    assert H.hadacore_padded_tokens(2 ** 62, 3) == (2 ** 62 + 381) // 128 * 128
    assert H.hadacore_padded_tokens(5, LARGEST) == 640


ENTRIES = {"rows": (H.hadamard_transform_fp8_blocks, ROWS),
           "columns": (H.hadacore_quantize_fp8_columns, COLUMNS),
           "tiles": (H.hadacore_quantize_fp8_tiles, TILES), "matmul": (H.hadacore_matmul_fp8, MATMUL),
           "grouped": (H.hadacore_matmul_fp8_grouped, GROUPED),
           "gradient": (H.hadacore_weight_gradient_fp8_grouped, GRADIENT)}
NOT_SIZES = {"x", "codes", "codes_t", "scales", "ends", "a", "sa", "b", "sb", "out", "stream", "dtype",
             "scale", "tall"}


@cpu_only
@pytest.mark.parametrize("value", [LARGEST, LARGEST - 15, 2 ** 62, 2 ** 45, -2 ** 63, -2 ** 62])
@pytest.mark.parametrize("entry,name", [(e, n) for e, (_, args) in ENTRIES.items()
                                        for n in args if n not in NOT_SIZES])
def test_extremes_are_refused(entry, name, value):
    call, args = ENTRIES[entry]
    assert _status(call, args, **{name: value}) in (
        "INVALID_VALUE", "INVALID_SIZE", "INVALID_STRIDE", "TOO_LARGE", "OVERLAP", "MISALIGNED")
