"""Refusals of the block quantizers and products, and their references, on the CPU."""
from __future__ import annotations

import math
from pathlib import Path

import numpy as np
import pytest

import blocks_reference as R
from paper_2412_08832_amd import hadacore as H

# as in test_abi: no call here has arguments that validation would accept
cpu_only = pytest.mark.skipif(Path("/dev/kfd").exists(),
                              reason="fake-pointer validation tests run only without a GPU")
X, C, S, T, O, E = (1 << k for k in range(33, 39))  # fake device addresses, far apart

NAMES = {v: k for k, v in H.STATUS_NAMES.items()}


def _status(entry, args, **change):
    values = dict(args)
    values.update(change)
    return H.STATUS_NAMES[entry(*values.values(), check=False)]


ROWS = dict(x=X, x_stride=512, codes=C, codes_stride=512, scales=S, scales_stride=4, m=3, k=512, n=128,
            dtype=H.BF16, scale=1.0, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(k=-128), "INVALID_VALUE"), (dict(n=96), "INVALID_SIZE"),
    (dict(n=1024), "INVALID_SIZE"), (dict(n=0), "INVALID_SIZE"),
    (dict(n=1 << 16, k=1 << 16, x_stride=1 << 16, codes_stride=1 << 16, scales_stride=512), "INVALID_SIZE"),
    (dict(dtype=2), "INVALID_DTYPE"), (dict(scale=math.inf), "INVALID_VALUE"),
    (dict(x_stride=511), "INVALID_STRIDE"), (dict(x_stride=516), "INVALID_STRIDE"),
    (dict(codes_stride=520), "INVALID_STRIDE"), (dict(codes_stride=496), "INVALID_STRIDE"),
    (dict(scales_stride=3), "INVALID_STRIDE"), (dict(x_stride=(1 << 26) + 8), "INVALID_STRIDE"),
    (dict(x=0), "INVALID_VALUE"), (dict(codes=0), "INVALID_VALUE"), (dict(scales=0), "INVALID_VALUE"),
    (dict(x=X + 2), "MISALIGNED"), (dict(x=X + 1, n=1), "MISALIGNED"), (dict(codes=C + 8), "MISALIGNED"),
    (dict(scales=S + 2), "MISALIGNED"), (dict(codes=X + 512), "OVERLAP"), (dict(scales=X + 16), "OVERLAP"),
    (dict(scales=C + 1024), "OVERLAP"), (dict(m=1 << 31), "TOO_LARGE"), (dict(m=0, x=0), "SUCCESS")])
def test_rows_refusals(change, status):
    assert _status(H.hadamard_transform_fp8_blocks, ROWS, **change) == status


COLUMNS = dict(x=X, x_stride=100, ends=E, groups=3, codes=C, codes_stride=512, scales=S,
               scales_stride=4, m=200, k=100, dtype=H.FP16, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(groups=-1), "INVALID_VALUE"), (dict(ends=0), "INVALID_VALUE"),
    (dict(dtype=2), "INVALID_DTYPE"), (dict(x_stride=99), "INVALID_STRIDE"),
    (dict(codes_stride=384), "INVALID_STRIDE"), (dict(codes_stride=520), "INVALID_STRIDE"),
    (dict(scales_stride=3), "INVALID_STRIDE"), (dict(codes=0), "INVALID_VALUE"),
    (dict(x=X + 1), "MISALIGNED"), (dict(codes=C + 4), "MISALIGNED"), (dict(ends=E + 2), "MISALIGNED"),
    (dict(codes=X + 16), "OVERLAP"), (dict(scales=C + 64), "OVERLAP"), (dict(ends=C + 4), "OVERLAP"),
    (dict(m=1 << 30), "TOO_LARGE"), (dict(m=0, groups=0), "SUCCESS"), (dict(k=0), "SUCCESS")])
def test_columns_refusals(change, status):
    assert H.hadacore_padded_tokens(200, 3) == 512
    assert _status(H.hadacore_quantize_fp8_columns, COLUMNS, **change) == status


TILES = dict(x=X, x_stride=200, x_batch=60000, codes=C, codes_stride=208, codes_batch=208 * 300,
             codes_t=T, codes_t_stride=304, codes_t_batch=304 * 200, scales=S, scales_stride=2,
             scales_batch=6, batch=2, m=300, k=200, dtype=H.BF16, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(batch=-1), "INVALID_VALUE"), (dict(dtype=7), "INVALID_DTYPE"),
    (dict(x_stride=199), "INVALID_STRIDE"), (dict(codes_stride=200), "INVALID_STRIDE"),
    (dict(codes_t_stride=300), "INVALID_STRIDE"), (dict(scales_stride=1), "INVALID_STRIDE"),
    (dict(codes_batch=208), "INVALID_STRIDE"), (dict(scales_batch=1), "INVALID_STRIDE"),
    (dict(codes_t_batch=304), "INVALID_STRIDE"), (dict(codes=0), "INVALID_VALUE"),
    (dict(codes_t=T + 8), "MISALIGNED"), (dict(scales=S + 1), "MISALIGNED"), (dict(codes_t=C + 16), "OVERLAP"),
    (dict(scales=X + 4), "OVERLAP"), (dict(m=1 << 30), "TOO_LARGE"), (dict(batch=0), "SUCCESS")])
def test_tiles_refusals(change, status):
    assert _status(H.hadacore_quantize_fp8_tiles, TILES, **change) == status


MATMUL = dict(a=X, a_stride=304, sa=S, sa_stride=3, b=C, b_stride=304, sb=S + 4096, sb_stride=3,
              tall=128, out=O, out_stride=40, dtype=H.FP32, m=7, n=40, k=300, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(n=-1), "INVALID_VALUE"), (dict(k=-1), "INVALID_VALUE"),
    (dict(tall=64), "INVALID_VALUE"), (dict(dtype=3), "INVALID_DTYPE"), (dict(a_stride=300), "INVALID_STRIDE"),
    (dict(a_stride=288), "INVALID_STRIDE"), (dict(b_stride=(1 << 22) + 16), "INVALID_STRIDE"),
    (dict(sa_stride=2), "INVALID_STRIDE"), (dict(sb_stride=2), "INVALID_STRIDE"),
    (dict(out_stride=39), "INVALID_STRIDE"), (dict(a=0), "INVALID_VALUE"), (dict(sb=0), "INVALID_VALUE"),
    (dict(out=0), "INVALID_VALUE"), (dict(a=X + 8), "MISALIGNED"), (dict(sa=S + 2), "MISALIGNED"),
    (dict(out=O + 2), "MISALIGNED"), (dict(out=X + 16), "OVERLAP"), (dict(out=C + 64), "OVERLAP"),
    (dict(out=S + 8), "OVERLAP"), (dict(n=1 << 30, out_stride=1 << 30), "TOO_LARGE"), (dict(m=0), "SUCCESS")])
def test_matmul_refusals(change, status):
    assert _status(H.hadacore_matmul_fp8, MATMUL, **change) == status


@cpu_only
def test_no_groups_need_no_ends():
    """An empty tensor of ends has no address."""
    assert _status(H.hadacore_quantize_fp8_columns, COLUMNS, ends=0, groups=0, m=100) == "SUCCESS"
    assert _status(H.hadacore_matmul_fp8_grouped, GROUPED, ends=0, groups=0, m=0) == "SUCCESS"
    assert _status(H.hadacore_weight_gradient_fp8_grouped, GRADIENT, ends=0, groups=0) == "SUCCESS"
    assert _status(H.hadacore_weight_gradient_fp8_grouped, GRADIENT, ends=0, groups=2) == "INVALID_VALUE"


GROUPED = dict(a=X, a_stride=304, sa=S, sa_stride=3, b=C, b_stride=304, b_batch=304 * 40, sb=S + 4096,
               sb_stride=3, sb_batch=3, ends=E, groups=4, out=O, out_stride=40, dtype=H.FP16, m=7, n=40,
               k=300, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(groups=-1), "INVALID_VALUE"), (dict(ends=0), "INVALID_VALUE"), (dict(ends=E + 1), "MISALIGNED"),
    (dict(b_batch=304 * 40 + 8), "INVALID_STRIDE"), (dict(sb_batch=-3), "INVALID_STRIDE"),
    (dict(b_batch=-304), "INVALID_STRIDE"), (dict(out=C + 304 * 120), "OVERLAP"), (dict(out=E + 4), "OVERLAP"),
    (dict(b_batch=1 << 41), "TOO_LARGE"), (dict(dtype=-1), "INVALID_DTYPE"), (dict(n=0), "SUCCESS")])
def test_grouped_refusals(change, status):
    assert _status(H.hadacore_matmul_fp8_grouped, GROUPED, **change) == status


GRADIENT = dict(a=X, a_stride=512, sa=S, sa_stride=4, b=C, b_stride=512, sb=S + 65536, sb_stride=4, ends=E,
                groups=4, out=O, out_stride=60, out_batch=60 * 40, dtype=H.BF16, places=512, n=40, k=60,
                stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(places=500), "INVALID_SIZE"), (dict(places=-128), "INVALID_VALUE"), (dict(ends=0), "INVALID_VALUE"),
    (dict(out_batch=60 * 39), "INVALID_STRIDE"), (dict(a_stride=496), "INVALID_STRIDE"),
    (dict(sb_stride=3), "INVALID_STRIDE"), (dict(out_stride=59), "INVALID_STRIDE"),
    (dict(ends=E + 2), "MISALIGNED"), (dict(out=O + 1), "MISALIGNED"), (dict(b=O + 16 * 60), "OVERLAP"),
    (dict(groups=0), "SUCCESS")])
def test_gradient_refusals(change, status):
    assert _status(H.hadacore_weight_gradient_fp8_grouped, GRADIENT, **change) == status


def test_padded_tokens():
    """The bound is reached: one token in every group but one, the rest in that."""
    assert H.hadacore_padded_tokens(0, 5) == 0 and H.hadacore_padded_tokens(-1, 5) == 0
    for tokens in (1, 2, 127, 128, 129, 1000):
        for groups in (1, 2, 7, 200):
            used = min(groups, tokens)
            worst = used - 1 + -(-(tokens - used + 1) // 128)
            assert H.hadacore_padded_tokens(tokens, groups) == 128 * worst


def test_reference_codes_are_e4m3():
    """The references' decoder against the oracle's, and a planted mistake is noticed."""
    import oracle
    assert np.array_equal(R.VALUES, oracle.get().decode_e4m3(np.arange(256, dtype=np.uint8)),
                          equal_nan=True)
    y = np.random.default_rng(0).standard_normal((4, 256))
    codes = np.stack([oracle.get().quantize_fp8(b[None])[0][0] for b in y.reshape(-1, 128)])
    scales = (np.abs(y.reshape(-1, 128)).max(axis=1) / 448).astype(np.float32)
    R.check_rows(y, codes.reshape(4, 256), scales)
    codes[3, 7] ^= 0x08
    with pytest.raises(AssertionError):
        R.check_rows(y, codes.reshape(4, 256), scales)
    codes[3, 7] ^= 0x08
    scales[5] *= 1.001
    with pytest.raises(AssertionError):
        R.check_rows(y, codes.reshape(4, 256), scales)
