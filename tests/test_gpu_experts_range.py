"""The FP8 linear layers where a rotation leaves the type's range: the rotation of n values
of one sign is sqrt(n) times the largest of them, so that fp16 values whose gradients or
products are finite have rotations past 65504.

Bound: as in test_gpu_experts, REL of a product of two coded operands.  Where all terms of a
sum have one sign the codes' errors are below 1/16 each and add up to less than 2/16 + 1/256.
"""
from __future__ import annotations

import pytest

from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu

REL = 0.056
ONE_SIGN = 2 / 16 + 1 / 256
K = 4096


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _normal(seed, *shape):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda")


def _run(x, w, dy, ends=None, rotate=None):
    from paper_2412_08832_amd import experts as E
    x, w, dy = (t.half() for t in (x, w, dy))
    x.requires_grad_()
    w.requires_grad_()
    y = E.train_linear(x, w, ends, rotate)
    y.backward(dy)
    x64, w64, dy64 = (t.detach().double() for t in (x, w, dy))
    if ends is None:
        want = x64 @ w64.t(), dy64 @ w64, dy64.t() @ x64
    else:
        parts = list(zip([0, *ends.tolist()[:-1]], ends.tolist()))
        want = (_cat([x64[a:b] @ w64[e].t() for e, (a, b) in enumerate(parts)]),
                _cat([dy64[a:b] @ w64[e] for e, (a, b) in enumerate(parts)]),
                _stack([dy64[a:b].t() @ x64[a:b] for a, b in parts]))
    assert all(bool((r.abs() < 65504).all()) for r in want), "the true results are finite"
    return dict(zip(("y", "dx", "dw"), zip((y.detach(), x.grad, w.grad), want)))


def _cat(parts):
    import torch
    return torch.cat(parts)


def _stack(parts):
    import torch
    return torch.stack(parts)


def _check(got, want, rel):
    import torch
    assert torch.isfinite(got).all(), f"{int((~torch.isfinite(got)).sum())} values not finite"
    off = float((got.double() - want).norm() / want.norm())
    assert off <= rel, f"relative error {off}"


def _ends(ends):
    import torch
    return None if ends is None else torch.tensor(ends, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("ends", [None, [300, 300, 1000]])
def test_weight_gradients_of_one_sign(ends):
    """dw = 1100 and more everywhere: its rotation would be 70400."""
    import torch
    x, dy = torch.full((1000, K), 1.1), torch.full((1000, 40), 1.0)
    w = _normal(1, *([3] if ends else []), 40, K) / K
    r = _run(x.cuda(), w, dy.cuda() * (2 if ends else 1), _ends(ends))
    _check(*r["dw"], ONE_SIGN)


def test_inputs_of_one_sign():
    """Rows of 2000, whose rotation is 128000."""
    import torch
    x = torch.full((300, K), 2000.0, device="cuda")
    r = _run(x, _normal(2, 64, K) / K, _normal(3, 300, 64) * 1e-2)
    _check(*r["dw"], REL)


@pytest.mark.parametrize("ends", [None, [100, 100, 130]])
def test_input_gradients_of_one_sign(ends):
    """dx = 1100 everywhere."""
    import torch
    w = torch.full((*([3] if ends else []), 2200, K), 0.5, device="cuda")
    r = _run(_normal(4, 130, K) * 0.1, w, torch.ones((130, 2200), device="cuda"), _ends(ends))
    _check(*r["dx"], ONE_SIGN)


@pytest.mark.parametrize("backward", [False, True])
def test_weights_of_one_sign(backward):
    """Weights of 1100, whose rotation is 70400: the layer's outputs stay finite."""
    import torch
    from paper_2412_08832_amd import experts as E
    w = torch.full((130, K), 1100.0, device="cuda").half()
    w[7] *= -1
    x = (_normal(5, 50, K) * 0.05).half()
    want = x.double() @ w.double().t()
    _check(E.linear(x, E.quantize_weights(w, backward=backward)), want, REL)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("scale", [1e-4, 1.0])
def test_small_values_keep_their_precision(dtype, scale):
    """What guards the large values costs the small ones nothing: weights and inputs of 1e-4,
    and gradients of 1e-4 * 1e-4 in bfloat16."""
    import torch
    from paper_2412_08832_amd import experts as E
    t = getattr(torch, dtype)
    x, w = (_normal(6, 200, K) * scale).to(t), (_normal(7, 64, K) * scale).to(t)
    dy = (_normal(8, 200, 64) * (scale if t is torch.bfloat16 else 1.0)).to(t)
    x.requires_grad_()
    w.requires_grad_()
    y = E.train_linear(x, w)
    y.backward(dy)
    x64, w64, dy64 = (v.detach().double() for v in (x, w, dy))
    if t is torch.bfloat16 or scale == 1.0:
        _check(y.detach(), x64 @ w64.t(), REL)
    _check(x.grad, dy64 @ w64, REL)
    _check(w.grad, dy64.t() @ x64, REL)


@pytest.mark.parametrize("ends", [None, [100, 100, 257]])
def test_weight_gradient_in_32_bits(ends):
    """The layer's weight gradient for an optimizer that keeps 32 bits, a sum past fp16's range."""
    import torch
    from paper_2412_08832_amd import experts as E
    x, dy = (_normal(9, 257, K) + 30).half(), (_normal(10, 257, 96) + 30).half()
    got = E.weight_gradient(dy, x, _ends(ends), dtype=torch.float32)
    parts = [(0, 257)] if ends is None else list(zip([0, *ends[:-1]], ends))
    want = _stack([dy[a:b].double().t() @ x[a:b].double() for a, b in parts])
    want = want[0] if ends is None else want
    assert got.dtype == torch.float32 and got.shape == want.shape and float(got.max()) > 65504
    _check(got, want, ONE_SIGN)


@pytest.mark.parametrize("tokens,n,k", [(5, 4, 0), (0, 4, 256), (5, 0, 256)])
@pytest.mark.parametrize("groups", [0, 2])
def test_empty_layers(tokens, n, k, groups):
    """No tokens, no outputs or no columns: zeros, and gradients of the operands' shapes."""
    import torch
    from paper_2412_08832_amd import experts as E
    x = torch.ones((tokens, k), dtype=torch.float16, device="cuda", requires_grad=True)
    w = torch.ones((*([groups] if groups else []), n, k), dtype=torch.float16, device="cuda",
                   requires_grad=True)
    y = E.train_linear(x, w, _ends([tokens // 2, tokens]) if groups else None)
    assert y.shape == (tokens, n) and (y == 0).all()
    y.backward(torch.ones_like(y))
    assert x.grad.shape == x.shape and (x.grad == 0).all()
    assert w.grad.shape == w.shape and (w.grad == 0).all()
