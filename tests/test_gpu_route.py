"""Routing on the GPU: choices, counts, weights, loss and gradients against 64 bits."""
from __future__ import annotations

import pytest
import torch

import tokens_reference as R
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _logits(m, experts, dtype, seed=0, spread=2.0):
    gen = torch.Generator().manual_seed(seed + 31 * m + experts)
    return (spread * torch.randn((m, experts), generator=gen)).to(dtype)


def _check(logits, k, renormalize, valid=None, gradients=True, device_logits=None, seed=1):
    """Everything about one call; `device_logits`: the same values laid out otherwise."""
    x = logits.cuda() if device_logits is None else device_logits
    v = None if valid is None else valid.cuda()
    got = H.route_tokens(x, k, renormalize=renormalize, valid=v)
    leaf = logits.double().requires_grad_()
    chosen, weights, counts, loss, slopes = R.route(leaf, k, renormalize, valid)
    assert torch.equal(got.experts.cpu(), chosen)
    assert torch.equal(got.counts.cpu(), counts)
    wide = logits.double()
    R.check("weights", got.weights, weights.detach(), R.weight_bound(wide, weights.detach()))
    m = logits.shape[0]
    finite = torch.isfinite(wide)
    spread = float((torch.where(finite, wide, 0).max() - torch.where(finite, wide, 0).min())) if m else 0.0
    # p's own error, and the steps of the sum over the tokens (64 in a lane, 128 lanes, 256 workgroups)
    loss_off = (2 * (spread + 3) + 24 + 64 + 128 + 256 + 2) * R.U * loss.detach().abs()
    R.check("loss", got.loss, loss.detach(), loss_off + 2.0 ** -149)
    R.check("slopes", got.slopes, slopes, 2 * R.U * slopes + 2.0 ** -149)
    again = H.route_tokens(x, k, renormalize=renormalize, valid=v)
    for a, b in zip(got[:5], again[:5]):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
    if not gradients or m == 0:
        return got
    gen = torch.Generator().manual_seed(seed)
    dw, dl = torch.randn((m, k), generator=gen), torch.tensor(0.7)
    for with_w, with_l in ((True, True), (True, False), (False, True)):
        out = H.route_tokens_gradient(x, got, dw.cuda() if with_w else None, dl.cuda() if with_l else None)
        f = ((weights * dw.double()).sum() if with_w else 0.0) + (loss * dl.double() if with_l else 0.0)
        want = torch.zeros_like(wide)
        if f.requires_grad:
            want = torch.autograd.grad(f, leaf, retain_graph=True)[0]
        bound = R.gradient_bound(wide, weights.detach(), dw.double() * with_w, slopes, 0.7 * with_l,
                                 renormalize, chosen)
        assert out.dtype == logits.dtype
        R.check("gradient", out, want, R.rounded(want, bound, logits.dtype))
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,experts,k", [
    (1, 1, 1), (1, 4, 2), (17, 32, 2), (130, 33, 3), (129, 61, 4), (67, 64, 8), (300, 100, 6), (40, 128, 32),
    (33, 200, 8), (260, 256, 8), (35, 257, 5), (50, 512, 8), (21, 700, 7), (18, 1024, 32)])
def test_sizes(m, experts, k, dtype):
    for renormalize in (False, True):
        _check(_logits(m, experts, dtype), k, renormalize)


@pytest.mark.parametrize("m,experts,k", [(5000, 48, 2), (3001, 256, 8), (700, 1000, 4), (20001, 8, 2)])
def test_many_workgroups(m, experts, k):
    valid = torch.rand(m, generator=torch.Generator().manual_seed(3)) > 0.2
    _check(_logits(m, experts, torch.float32), k, True, valid)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_logits_go_to_the_lower_index(dtype):
    logits = _logits(90, 60, dtype).mul(2).round().div(2)
    logits[0] = 0
    logits[1, ::2], logits[1, 1::2] = 0.0, -0.0
    got = _check(logits, 8, True)
    assert got.experts[0].tolist() == list(range(8)) and got.experts[1].tolist() == list(range(8))


@pytest.mark.parametrize("experts,k", [(12, 4), (70, 3), (300, 8)])
def test_masked_experts_and_rows(experts, k):
    """-inf is never chosen; rows without enough others, or any; tokens that are not valid, whatever
    lies there; the lowest finite value is a logit like others."""
    logits = _logits(64, experts, torch.float32)
    logits[:, 5] = -INF
    logits[1, 2:] = -INF
    logits[2] = -INF
    logits[3, : experts - 1] = torch.finfo(torch.float32).min
    logits[4] = torch.finfo(torch.float32).min
    for renormalize in (False, True):
        x, valid = logits.clone(), torch.arange(64) % 7 != 6
        x[3:5] = 0  # the spread of the bound
        _check(x, k, renormalize, valid)
        _check(x, k, renormalize)
        filled = x.clone()
        filled[~valid] = float("nan")
        want = H.route_tokens(x.cuda(), k, renormalize, valid.cuda())
        got = H.route_tokens(filled.cuda(), k, renormalize, valid.cuda())
        dw = torch.ones((64, k), device="cuda")
        for a, b in zip(got[:5], want[:5]):
            assert torch.equal(a, b)
        assert torch.equal(H.route_tokens_gradient(filled.cuda(), got, dw, got.loss),
                           H.route_tokens_gradient(x.cuda(), want, dw, want.loss))
    got = H.route_tokens(logits.cuda(), k, True)
    low = got.weights.cpu()
    assert torch.equal(got.experts.cpu(), R.choose(logits, k))
    assert low[3, 0] == 1 and (low[3, 1:] == 0).all() and (low[4] == 1 / k).all()


def test_nan_and_infinity_stay_in_their_row():
    logits = _logits(20, 40, torch.float32)
    clean = H.route_tokens(logits.cuda(), 3, True)
    logits[4, 7], logits[9, 30] = float("nan"), INF
    got = H.route_tokens(logits.cuda(), 3, True)
    assert got.experts[4, 0] == 7 and got.experts[9, 0] == 30
    keep = torch.ones(20, dtype=torch.bool)
    keep[[4, 9]] = False
    assert torch.equal(got.weights[keep.cuda()], clean.weights[keep.cuda()])
    assert got.weights[4].isnan().all() and got.weights[9].isnan().any() and got.loss.isnan()
    out = H.route_tokens_gradient(logits.cuda(), got, torch.ones((20, 3), device="cuda"))
    assert out[keep.cuda()].isfinite().all() and out[4].isnan().all()


def test_no_tokens_and_none_valid():
    got = H.route_tokens(torch.empty((0, 9), device="cuda"), 2)
    assert got.experts.shape == (0, 2) and (got.counts == 0).all() and got.loss == 0 and (got.slopes == 0).all()
    got = H.route_tokens(torch.randn((5, 9), device="cuda"), 2, valid=torch.zeros(5, dtype=torch.bool, device="cuda"))
    assert (got.experts == -1).all() and (got.weights == 0).all() and (got.counts == 0).all() and got.loss == 0
    assert (H.route_tokens_gradient(torch.randn((5, 9), device="cuda"), got, got.weights, got.loss) == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 5)])
def test_rows_with_gaps_from_any_address(pad, shift, dtype):
    logits = _logits(77, 50, dtype)
    wide = torch.full((77 * (50 + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    view = wide[shift : shift + 77 * (50 + pad)].view(77, 50 + pad)[:, :50]
    view.copy_(logits)
    got = _check(logits, 4, True, device_logits=view)
    out = torch.full_like(wide, 7.0)
    target = out[shift : shift + 77 * (50 + pad)].view(77, 50 + pad)[:, :50]
    dw = torch.randn((77, 4), device="cuda")
    want = H.route_tokens_gradient(view, got, dw, got.loss)
    H.route_tokens_gradient(view, got, dw, got.loss, out=target)
    assert torch.equal(target, want)
    target.fill_(7.0)
    assert (out == 7.0).all()


@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient_against_differences(renormalize):
    """Central differences of the reference's own f in 64 bits at the GPU's gradient: with h = 2^-10 and
    f's third derivatives at most 60 |dw| of the softmax, the cut is below 60 h^2 / 6 sum |d|^3."""
    logits = _logits(6, 20, torch.float32)
    got = H.route_tokens(logits.cuda(), 3, renormalize)
    dw, dl = torch.randn((6, 3), generator=torch.Generator().manual_seed(5)), torch.tensor(0.5)
    grad = H.route_tokens_gradient(logits.cuda(), got, dw.cuda(), dl.cuda()).double().cpu()
    chosen, w, _, _, slopes = R.route(logits.double(), 3, renormalize)

    def f(l):
        p = torch.softmax(l, 1)
        picked = p.gather(1, chosen.long())
        if renormalize:
            picked = picked / picked.sum(1, keepdim=True)
        return float((picked * dw.double()).sum() + 0.5 * (slopes * p.sum(0)).sum())

    gen, h = torch.Generator().manual_seed(6), 2.0 ** -10
    for _ in range(5):
        d = torch.randn((6, 20), generator=gen, dtype=torch.float64)
        slope = (f(logits.double() + h * d) - f(logits.double() - h * d)) / (2 * h)
        bound = R.gradient_bound(logits.double(), w, dw.double(), slopes, 0.5, renormalize, chosen)
        cut = 10 * h * h * float((d.abs() ** 3).sum()) * float(dw.abs().max() + 0.5 * slopes.max())
        assert abs(slope - float((grad * d).sum())) <= float(((bound + R.U * grad.abs()) * d.abs()).sum()) + cut


def test_refusals():
    x = torch.zeros((4, 8), device="cuda")
    r = H.route_tokens(x, 2)
    for bad, kind in ((lambda: H.route_tokens(x.double(), 2), TypeError),
                      (lambda: H.route_tokens(x.cpu(), 2), ValueError),
                      (lambda: H.route_tokens(x[0], 2), ValueError),
                      (lambda: H.route_tokens(x.t(), 2), ValueError),
                      (lambda: H.route_tokens(x, 2, valid=torch.ones(4, device="cuda")), TypeError),
                      (lambda: H.route_tokens(x, 2, valid=torch.ones(3, dtype=torch.bool, device="cuda")), ValueError),
                      (lambda: H.route_tokens_gradient(x, r, torch.zeros((4, 3), device="cuda")), ValueError),
                      (lambda: H.route_tokens_gradient(x, r, torch.zeros((4, 2))), ValueError),
                      (lambda: H.route_tokens_gradient(x, r, out=torch.zeros((4, 9), device="cuda")), ValueError)):
        with pytest.raises(kind):
            bad()
    for k in (0, 9):
        with pytest.raises(H.HadacoreError) as e:
            H.route_tokens(x, k)
        assert e.value.status == 2
    with pytest.raises(H.HadacoreError) as e:
        H.route_tokens(torch.zeros((2, 1025), device="cuda"), 2)
    assert e.value.status == 2
    with pytest.raises(H.HadacoreError) as e:
        H.route_tokens_gradient(x, r, out=x)
    assert e.value.status == 6
    torch.cuda.synchronize()
