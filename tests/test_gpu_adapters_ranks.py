"""A weight's gradient: each rank is a sum of its own, whatever stands in the others."""
from __future__ import annotations

import pytest
import torch

import tokens_reference as R
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
# width: rows of whole 16 bytes and others; rank: one, two and four tiles of 16 in a workgroup, and more of them
SIZES = [(70, 128, 16, 2), (70, 130, 9, 2), (900, 256, 24, 2), (300, 77, 30, 2), (2000, 136, 64, 1), (300, 65, 50, 3),
         (90, 64, 200, 1)]


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _make(m, width, rank, groups, dtype):
    gen = torch.Generator().manual_seed(m + width + rank)
    ends, _, slots = R.group(torch.randint(-1, groups, (m,), generator=gen).int(), groups)
    x, h = torch.randn((m, width), generator=gen).to(dtype), torch.randn((m, rank), generator=gen)
    return gen, h.cuda(), x.cuda(), ends.cuda(), slots.cuda()


@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("m,width,rank,groups", SIZES)
@pytest.mark.parametrize("value", [float("inf"), float("nan"), 2.0 ** 60])
def test_one_rank_in_others(m, width, rank, groups, dtype, out, value):
    """Inf, NaN or a value far past the others' in one rank of one token of each group: every other rank's row
    stays to the bit, and this one's is NaN or infinite (or holds the value)."""
    _, h, x, ends, slots = _make(m, width, rank, groups, dtype)
    clean = H.adapter_gradient(h, x, ends, slots, dtype=out)
    hit = rank // 2
    for low, high in R.groups_of(ends.cpu(), m):
        h[(low + high) // 2, hit] = value
    got = H.adapter_gradient(h, x, ends, slots, dtype=out)
    keep = torch.arange(rank, device="cuda") != hit
    assert torch.equal(got[:, keep], clean[:, keep])
    if value != 2.0 ** 60:
        assert not got[:, hit].isfinite().any()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("m,width,rank,groups", SIZES)
def test_powers_of_two_of_the_ranks(m, width, rank, groups, dtype):
    """h times a power of two for each rank, up to 2^80 apart: the rows of the gradient times the same, exactly."""
    gen, h, x, ends, slots = _make(m, width, rank, groups, dtype)
    # on the CPU: the GPU's pow is a unit off for 15 of these 81
    power = (2.0 ** torch.randint(-40, 41, (rank,), generator=gen)).cuda()
    assert (torch.frexp(power).mantissa == 0.5).all()
    want = H.adapter_gradient(h, x, ends, slots, dtype=F32) * power[:, None]
    assert torch.equal(H.adapter_gradient(h * power, x, ends, slots, dtype=F32), want)
