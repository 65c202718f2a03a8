"""The forms of the kernels that long batches and whole rows take, against 64 bits on the GPU: whole lines of
outputs, every number of tokens to a workgroup, every number of steps of the gradients' ring, and the
streaming forms of the exchange.  The cut of each call is asserted, so that a change of the rules shows here.

Bounds as in tokens_reference: a fp32 sum of n steps is at most n U sum |v| off.
"""
from __future__ import annotations

import pytest
import torch

import tokens_reference as R
from adapters_cut import cuts
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
U = R.U


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _check(name, got, want, off):
    """Within `off` before the rounding to got's type, on the GPU."""
    bound = R.rounded(want, off, got.dtype)
    worst = ((got.double() - want).abs() / bound).max()
    assert bool(worst <= 1), f"{name}: {float(worst)} of its bound"


def _plan(gen, m, groups):
    """Ragged groups, some tokens without one."""
    ids = torch.randint(-1, groups, (m,), generator=gen, device="cuda").int()
    plan = H.group_tokens(ids, groups)
    return plan.ends, plan.slots, R.groups_of(plan.ends.cpu(), m)


FORMS = [  # m, k, n, rank, adapters, unit (0: both products in one launch)
    (1, 64, 128, 16, 1, 0), (16, 96, 1024, 16, 1, 0), (64, 512, 1024, 5, 7, 0), (70, 4096, 2176, 16, 9, 0),
    (300, 64, 128, 16, 2, 16), (300, 512, 1024, 16, 2, 16), (200, 2048, 1024, 30, 7, 16), (513, 72, 640, 200, 2, 16),
    (4200, 64, 4096, 16, 3, 32), (8300, 64, 4096, 9, 3, 64), (16500, 64, 4096, 16, 3, 128), (16500, 40, 4100, 8, 2, 128),
    (4200, 96, 4096, 64, 2, 32), (8300, 64, 4096, 50, 2, 64), (8311, 64, 4097, 64, 3, 64),
    (2100, 64, 4096, 100, 2, 32), (4200, 64, 4096, 100, 2, 64), (4299, 64, 4101, 128, 3, 64),
    (1100, 64, 4096, 160, 2, 32), (1100, 64, 4160, 256, 2, 32), (1133, 64, 4095, 129, 2, 32)]


def test_forms_are_cut_as_listed():
    for (m, k, n, rank, groups, unit), c in zip(FORMS, cuts([f[:5] for f in FORMS])[1]):
        assert (0 if c.fused else c.unit) == unit, (m, k, n, rank, groups)


@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("m,k,n,rank,groups,unit", FORMS)
def test_adapters(m, k, n, rank, groups, unit, dtype, out):
    gen = torch.Generator(device="cuda").manual_seed(m + n + rank)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    x, down, up = normal(m, k).to(dtype), (normal(groups, rank, k) / k ** 0.5).to(dtype), \
        (0.3 * normal(groups, rank, n)).to(dtype)
    y, scales = normal(m, n).to(out), 0.5 + torch.rand(groups, generator=gen, device="cuda")
    ends, slots, spans = _plan(gen, m, groups)
    got, h = H.adapt_rows(x, down, up, ends, slots, y=y, scales=scales, hidden=True)
    for g, (low, high) in enumerate([*spans, (spans[-1][1], m)]):
        t = slots[low:high].long()
        if g == groups:  # no adapter
            assert torch.equal(got[t], y[t])
            continue
        if low == high:
            continue
        xd, dd, ud, s = x[t].double(), down[g].double(), up[g].double(), float(scales[g])
        # the sums over k: steps of a matrix instruction, four or eight waves and up to 16 shares
        want_h, h_off = xd @ dd.t(), (k / 32 + 32 + 8 + 16) * U * (xd.abs() @ dd.abs().t())
        _check(f"h of {g}", h[low:high], want_h, h_off)
        # of h all 24 bits, for fp16 above 2^-35 of the row's largest: three products to a step of 32 ranks
        part = s * (want_h @ ud)
        off = s * ((h_off + (3 * (rank / 32 + 1) + 32 + 3) * U * want_h.abs()) @ ud.abs()) \
            + U * (y[t].double() + part).abs()
        if dtype is F16:
            off += 2.0 ** -35 * s * want_h.abs().amax(1, keepdim=True) * ud.abs().sum(0)
        _check(f"out of {g}", got[t], y[t].double() + part, off)
    place = H.adapt_rows(x, down, up, ends, slots, y=y, scales=scales, out=y)
    assert place is y and torch.equal(y, got)


@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("rank", [16, 24, 32, 64, 72])
@pytest.mark.parametrize("width", [136, 256])
def test_steps_of_the_gradients_ring(width, rank, dtype, out):
    """A group's tokens go through a ring in steps of 32 for each of two waves and a share: none to seven steps."""
    gen = torch.Generator(device="cuda").manual_seed(width + rank)
    x = torch.randn((7300, width), generator=gen, device="cuda").to(dtype)
    h = torch.randn((7300, rank), generator=gen, device="cuda")

    def check(m, ends, slots, spans, scales):
        got = H.adapter_gradient(h[:m], x[:m], ends, slots, scales, dtype=out)
        for g, (low, high) in enumerate(spans):
            t = torch.arange(low, high, device="cuda") if slots is None else slots[low:high].long()
            hd, xd, s = h[low:high].double(), x[t].double(), 1.0 if scales is None else float(scales[g])
            steps = 3 * ((high - low) / 32 + 1) + 32 + 2 + 16 + 2
            off = abs(s) * steps * U * (hd.abs().t() @ xd.abs())
            if dtype is F16 and high > low:
                off += 2.0 ** -35 * abs(s) * hd.abs().amax(0)[:, None] * xd.abs().sum(0)
            _check(f"{m} tokens, group {g}", got if ends is None else got[g], s * (hd.t() @ xd), off)
    for m in (1, 31, 32, 33, 64, 65, 97, 130, 161, 193, 225, 255, 5200, 7300):
        check(m, None, None, [(0, m)], None)
    ends = torch.tensor([0, 1, 34, 34, 98, 300, 1200, 3000], dtype=torch.int32, device="cuda")
    scales = 0.5 + torch.rand(8, generator=gen, device="cuda")
    slots = torch.randperm(3100, generator=gen, device="cuda").int()
    check(3100, ends, slots, R.groups_of(ends.cpu(), 3100), scales)


# 16 MiB and more of rows in whole lines: the streaming forms
LONG = [(4100, 1, 2048, 5), (1100, 2, 4096, 5), (1500, 3, 2048, 4), (700, 7, 2048, 9)]


def _exchange(m, k, width, groups, dtype):
    gen = torch.Generator(device="cuda").manual_seed(m + k)
    ids = torch.randint(-1, groups, (m, k), generator=gen, device="cuda").int()
    plan = H.group_tokens(ids, groups)
    used = int(plan.ends[-1])
    at, token = plan.slots[:used].long(), plan.slots[:used].long() // k

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    assert m * k * width * dtype.itemsize >= 1 << 24
    return plan, used, at, token, normal


@pytest.mark.parametrize("dtype", [torch.uint8, F16, BF16, F32])
@pytest.mark.parametrize("m,k,width,groups", LONG)
def test_long_dispatch(m, k, width, groups, dtype):
    width = width * 2 if dtype.itemsize == 1 else width
    plan, used, _, token, normal = _exchange(m, k, width, groups, dtype)
    x = (100 * normal(m, width)).to(dtype)
    got = H.dispatch_rows(x, plan.rows, plan.ends)
    assert torch.equal(got[:used], x[token]) and not got[used:].any()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("m,k,width,groups", LONG)
def test_long_combine(m, k, width, groups, weighted, dtype):
    plan, used, at, token, normal = _exchange(m, k, width, groups, dtype)
    y = normal(m * k, width).to(dtype)
    y[used:] = float("nan")
    weights = torch.rand((m, k), device="cuda") if weighted else None
    terms = y[:used].double() * (weights.view(-1)[at].double()[:, None] if weighted else 1.0)
    zero = torch.zeros((m, width), dtype=torch.float64, device="cuda")
    want, size = zero.index_add(0, token, terms), zero.index_add(0, token, terms.abs())
    _check("out", H.combine_rows(y, plan.rows, weights), want, k * U * size)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("m,k,width,groups", LONG)
def test_long_combine_gradient(m, k, width, groups, dtype):
    plan, used, at, token, normal = _exchange(m, k, width, groups, dtype)
    y, dout, weights = normal(m * k, width).to(dtype), normal(m, width).to(dtype), torch.rand((m, k), device="cuda")
    y[used:] = float("nan")
    dy, dw = H.combine_rows_gradient(dout, y, plan.rows, plan.ends, weights)
    d, w = dout[token].double(), weights.view(-1)[at].double()[:, None]
    _check("dy", dy[:used], w * d, U * (w * d).abs())
    assert not dy[used:].any()
    product = d * y[:used].double()
    want = torch.zeros(m * k, dtype=torch.float64, device="cuda").index_put((at,), product.sum(1))
    off = torch.zeros_like(want).index_put((at,), (width / 64 + 6 + 3) * U * product.abs().sum(1))
    _check("dweights", dw.view(-1), want, off)
