"""64-bit references of the block quantizers and products, in numpy, and how far a
result may be from them.

Quantizers: as in fp8_compare, a block's scale must be amax / 448 within a few fp32
ulps, and a code the reference's, or, where the fp32 transform can land on the other
side of a rounding boundary, within half an e4m3 step of the reference's value.

Products: with S = sum over blocks of scale * sum |a b|, a full-precision result is
within S (128 * 2^-23 + (blocks + 3) * 2^-24) before its rounding: at most 2^-23 for each
of the 128 additions in a block, a rounding for each block's fma, two for the scales'
product, one to spare.  The FP8 matrix instruction keeps 16 bits below the largest
product of a block at least, so 16-bit outputs may be off by a further 128 * 2^-16 of that
per block.  The rounding to the output type adds half its step.
"""
from __future__ import annotations

import numpy as np

REL_FP32_SLACK = 2.0 ** -17
SCALE_RTOL = 2.0 ** -19
SCALE_ATOL = 2.0 * 2.0 ** -149
BLOCK = 128


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * np.exp2(e.astype(np.float64) - 7))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


VALUES = e4m3_values()


def spacing(v):
    a = np.abs(v)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.floor(np.log2(np.where(a > 0, a, 1.0)))
    return np.where(a < 2.0 ** -6, 2.0 ** -9, np.exp2(e - 3))


def pad_to(x: np.ndarray, axis: int, multiple: int) -> np.ndarray:
    widths = [(0, 0)] * x.ndim
    widths[axis] = (0, -x.shape[axis] % multiple)
    return np.pad(x, widths)


def check_blocks(y: np.ndarray, codes: np.ndarray, scales: np.ndarray, what: str = "") -> None:
    """Blocks y (B, N) in 64 bits against codes (B, N) and scales (B,)."""
    y32 = y.astype(np.float32)
    with np.errstate(all="ignore"):
        amax = np.where(np.isnan(y32).all(axis=1), np.nan,
                        np.where(np.isnan(y32), 0, np.abs(y32)).max(axis=1)).astype(np.float32)
        q = (np.float32(448) / amax).astype(np.float32)
        inv = np.where(np.isfinite(q), q, np.float32(0))
        v = (y32 * inv[:, None]).astype(np.float64)
        want_scale = amax.astype(np.float64) / 448
        got = VALUES[codes]
        near = np.abs(got - v) <= 0.5 * spacing(v) + REL_FP32_SLACK * 448
    both_nan = np.isnan(got) & np.isnan(v)
    bad = ~(near | both_nan)
    assert not bad.any(), f"{what}: {bad.sum()} codes of {bad.size} off, first at {np.argwhere(bad)[0]}"
    s = scales.astype(np.float64)
    with np.errstate(invalid="ignore"):
        close = np.abs(s - want_scale) <= SCALE_RTOL * np.abs(want_scale) + SCALE_ATOL
    close |= (s == want_scale) | (np.isnan(s) & np.isnan(want_scale))
    assert close.all(), f"{what}: {np.count_nonzero(~close)} scales off, first at {np.argwhere(~close)[0]}"


def check_rows(y, codes, scales, what=""):
    """Rows (m, k) with a scale for each 128 columns; the last block may be shorter."""
    m, k = y.shape
    yb = pad_to(y, 1, BLOCK).reshape(-1, BLOCK)
    cb = pad_to(codes, 1, BLOCK).reshape(-1, BLOCK)
    check_blocks(yb, cb, scales.reshape(-1), what)


def check_tiles(w, codes, scales, what=""):
    """A matrix (n, k) with a scale for each tile of 128 x 128."""
    def tiles(x):
        x = pad_to(pad_to(x, 0, BLOCK), 1, BLOCK)
        r, c = x.shape[0] // BLOCK, x.shape[1] // BLOCK
        return x.reshape(r, BLOCK, c, BLOCK).transpose(0, 2, 1, 3).reshape(r * c, -1)
    check_blocks(tiles(w), tiles(codes), scales.reshape(-1), what)


def padded_places(ends, tokens: int):
    """[(group, first token, tokens, first place, blocks)] and the places in all."""
    at, out, low = 0, [], 0
    for g, high in enumerate(ends):
        n = high - low
        blocks = -(-n // BLOCK)
        out.append((g, low, n, at, blocks))
        at += blocks * BLOCK
        low = high
    places = (tokens + 127 * min(len(ends), tokens)) // BLOCK * BLOCK
    return out, places


def widen(codes, scales, tall=1):
    """codes (r, c) times a scale for each `tall` rows and 128 columns."""
    r = np.arange(codes.shape[0]) // tall
    c = np.arange(codes.shape[1]) // BLOCK
    return VALUES[codes] * scales.astype(np.float64)[r][:, c]


def out_step(ref, out):
    """Half the distance between neighbours of the output type at `ref`."""
    digits, least = {"fp32": (23, -149), "fp16": (10, -24), "bf16": (7, -133)}[out]
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.where(ref != 0, np.abs(ref), 2.0 ** least)))
    return 0.5 * np.maximum(np.exp2(e - digits), 2.0 ** least)


def check_product(a, sa, b, sb, got, out: str, tall: int = 128, what: str = "") -> None:
    """got against the product of codes a (m, k), b (n, k) with scales, `tall` rows of b each."""
    va, vb = widen(a, sa), widen(b, sb, tall)
    ref = va @ vb.T
    blocks = max(1, sa.shape[1])
    total = np.abs(va) @ np.abs(vb).T
    tol = total * (128 * 2.0 ** -23 + (blocks + 3) * 2.0 ** -24)
    if out != "fp32":
        for k in range(0, a.shape[1], BLOCK):
            top_a = np.abs(va[:, k:k + BLOCK]).max(axis=1)
            top_b = np.abs(vb[:, k:k + BLOCK]).max(axis=1)
            tol += 128 * 2.0 ** -16 * np.outer(top_a, top_b)
    if out == "fp16":  # what rounds past the largest fp16 is infinite
        over = np.isinf(got) & (np.sign(got) == np.sign(ref)) & (np.abs(ref) + tol >= 65520)
        got, ref = np.where(over, 0, got), np.where(over, 0, ref)
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got.astype(np.float64) - ref) <= tol + out_step(np.abs(ref) + tol, out))
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: "
                           f"{got[tuple(np.argwhere(bad)[0])]} for {ref[tuple(np.argwhere(bad)[0])]}")
    # on the whole the error is far below that bound: the sums' roundings are not all one way
    if ref.size >= 64 and np.linalg.norm(ref):
        rel = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert rel <= {"fp32": 1e-6, "fp16": 4e-4, "bf16": 2.5e-3}[out], f"{what}: rel {rel}"
