"""Adapters take every bit of the hidden values: whole numbers, whose sums are exact in fp32 in any order, so
that the only rounding is the output's and the results are known to the bit."""
from __future__ import annotations

import pytest
import torch

import tokens_reference as R
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _whole(gen, low, high, *shape):
    return torch.randint(low, high, shape, generator=gen)


def _plan(gen, m, groups):
    ends, _, slots = R.group(torch.randint(-1, groups, (m,), generator=gen).int(), groups)
    return ends, slots


@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("m,n,rank,groups", [
    (8, 128, 16, 1), (9, 130, 5, 2), (40, 1024, 16, 3), (300, 256, 24, 3), (90, 200, 64, 2), (300, 384, 64, 1),
    (100, 264, 100, 2), (70, 192, 200, 2), (50, 45, 256, 1)])
def test_output(m, n, rank, groups, dtype, out):
    """x and down of 8 bits: h is a whole number up to 255^2 * 256 < 2^24, mostly of 24 bits, and of a
    single product in every third rank.  Each column takes one rank of it, and y all that the output's type
    holds of it, so that the low bits are left."""
    gen, k = torch.Generator().manual_seed(m + n + rank), 256
    x, down = _whole(gen, 181, 256, m, k), _whole(gen, 181, 256, groups, rank, k)
    down[:, 2::3, 1:] = 0
    sign = 2 * _whole(gen, 0, 2, n) - 1
    up = torch.zeros((groups, rank, n), dtype=torch.int64)
    up[:, torch.arange(n) % rank, torch.arange(n)] = sign
    scale = 2.0 ** -9  # h within fp16's range
    ends, slots = _plan(gen, m, groups)
    part = torch.zeros((m, n), dtype=torch.float64)
    for g, (low, high) in enumerate(R.groups_of(ends, m)):
        t = slots[low:high].long()
        part[t] = scale * ((x[t].double() @ down[g].double().t()) @ up[g].double())
    y = (-part).to(dtype).to(out)
    want = (y.double() + part).to(out)
    assert torch.equal((y.double() + part).float().double(), y.double() + part)
    got = H.adapt_rows(*(t.to(dtype).cuda() for t in (x, down, up)), ends.cuda(), slots.cuda(), y=y.cuda(),
                       scales=torch.full((groups,), scale).cuda())
    assert torch.equal(got.cpu(), want), f"{int((got.cpu() != want).sum())} of {want.numel()}"


@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("m,width,rank,groups", [
    (2, 8, 1, 1), (70, 128, 16, 1), (300, 256, 24, 2), (700, 136, 64, 1), (300, 130, 16, 2), (150, 77, 40, 1),
    (90, 64, 256, 1)])
def test_weight_gradient(m, width, rank, groups, dtype, out):
    """Hidden values of 24 bits; each column has a token with 1 and one with -1 whose values are a few units
    apart, so that sums stay below 2^24 and their low bits are all there is."""
    gen = torch.Generator().manual_seed(m + width + rank)
    ends, slots = _plan(gen, m, groups)
    h = torch.zeros((m, rank), dtype=torch.int64)
    x = torch.zeros((m, width), dtype=torch.int64)
    want = torch.zeros((groups, rank, width), dtype=torch.float64)
    for g, (low, high) in enumerate(R.groups_of(ends, m)):
        h[low:high] = _whole(gen, 2 ** 23, 2 ** 24 - 256, rank) + _whole(gen, 0, 256, high - low, rank)
        if high - low < 2:
            continue
        for c in range(width):
            a, b = (low + torch.randperm(high - low, generator=gen)[:2]).tolist()
            x[slots[a], c], x[slots[b], c] = 1, -1
            want[g, :, c] = (h[a] - h[b]).double()
    got = H.adapter_gradient(h.float().cuda(), x.to(dtype).cuda(), ends.cuda(), slots.cuda(), dtype=out)
    assert torch.equal(got.cpu(), want.to(out)), f"{int((got.cpu() != want.to(out)).sum())} of {want.numel()}"
