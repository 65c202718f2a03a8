"""What the products promise of their sums where terms cancel: outputs in 32 bits add in fp32,
outputs in 16 bits to within 2^-9 of a block's largest product.

With s = a_scale * b_scale and top the largest |A| |B| of a block, the bounds before the
output's rounding are, summed over the blocks (as in blocks_reference):
  - 32 bits: sum of s * sum |a b| * (128 * 2^-23 + (blocks + 3) * 2^-24);
  - 16 bits: that, and 128 * 2^-16 * s * top.
"""
from __future__ import annotations

import numpy as np
import pytest

import blocks_reference as R
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


CODE_OF = {float(v): i for i, v in reversed(list(enumerate(R.VALUES))) if not np.isnan(v)}


def _cancelling(rng, m, n, k):
    """In each block pairs of 448 * 448 and 448 * -448 at random places, integers up to 16
    elsewhere, which e4m3 holds exactly."""
    a = rng.integers(-16, 17, (m, k)).astype(np.float64)
    b = rng.integers(-16, 17, (n, k)).astype(np.float64)
    for low in range(0, k, 128):
        width = min(128, k - low)
        for pair in rng.permutation(width)[:2 * int(rng.integers(1, 4))].reshape(-1, 2):
            at = low + pair
            a[:, at] = 448 * rng.choice([-1.0, 1.0], (m, 1))
            b[:, at] = np.array([448.0, -448.0]) * rng.choice([-1.0, 1.0], (n, 1))
    return a, b


def _upload(values):
    import torch
    codes = np.vectorize(CODE_OF.__getitem__, otypes=[np.uint8])(values)
    pitch = -(-values.shape[1] // 16) * 16
    buf = np.full((values.shape[0], pitch), 0x7F, np.uint8)
    buf[:, :values.shape[1]] = codes
    return torch.from_numpy(buf).cuda()[:, :values.shape[1]]


@pytest.mark.parametrize("variant", ["auto", "tiles-64", "tiles-64x128", "tiles-128", "tiles-256"])
@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("tall", [128, 1])
@pytest.mark.parametrize("m,n,k", [(1, 40, 512), (20, 70, 300), (50, 200, 1024), (300, 270, 640)])
def test_cancelling_products(m, n, k, tall, out, variant, monkeypatch):
    import torch
    if variant == "auto":
        monkeypatch.delenv("HADACORE_VARIANT", raising=False)
    else:
        monkeypatch.setenv("HADACORE_VARIANT", variant)
    rng = np.random.default_rng(m + n + k)
    a, b = _cancelling(rng, m, n, k)
    blocks = -(-k // 128)
    sa = np.exp2(rng.integers(-4, 1, (m, blocks))).astype(np.float32)
    sb = np.exp2(rng.integers(-4, 1, (n if tall == 1 else -(-n // 128), blocks))).astype(np.float32)
    y = H.matmul_fp8(_upload(a), torch.from_numpy(sa).cuda(), _upload(b), torch.from_numpy(sb).cuda(),
                     dtype={"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[out])
    got = y.float().cpu().numpy().astype(np.float64)
    tall_b = sb[np.arange(n) // tall].astype(np.float64)
    ref, bound = np.zeros((m, n)), np.zeros((m, n))
    for i in range(blocks):
        cut = slice(128 * i, 128 * i + 128)
        s = np.outer(sa[:, i].astype(np.float64), tall_b[:, i])
        ref += s * (a[:, cut] @ b[:, cut].T)
        bound += s * (np.abs(a[:, cut]) @ np.abs(b[:, cut]).T) * (128 * 2.0 ** -23 + (blocks + 3) * 2.0 ** -24)
        if out != "fp32":
            bound += 128 * 2.0 ** -16 * s * np.outer(np.abs(a[:, cut]).max(axis=1),
                                                     np.abs(b[:, cut]).max(axis=1))
    assert np.abs(ref).max() + bound.max() < 65504
    off = np.abs(got - ref) - bound - R.out_step(np.abs(ref) + bound, out)
    assert (off <= 0).all(), f"{(off > 0).sum()} of {off.size} past the bound, by {off.max()}"
