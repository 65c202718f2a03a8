"""The FP8 linear layers' algebra on the CPU, with plain exact products in the kernels' place."""
from __future__ import annotations

import math
from types import SimpleNamespace

import pytest
import torch

from paper_2412_08832_amd import experts as E


def _hadamard(n):
    h = torch.ones((1, 1), dtype=torch.float64)
    while h.shape[0] < n:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)])
    return h / math.sqrt(n)


def _groups(ends):
    return zip([0, *ends.tolist()[:-1]], ends.tolist())


def _transform(x, out=None):
    y = x @ _hadamard(x.shape[-1]).to(x.dtype)
    return y if out is None else out.copy_(y)


def _transform_fp8_blocks(x, n):
    return _transform(x.reshape(-1, n)).view(x.shape), None


def _grouped_matmul(a, sa, b, sb, ends, dtype=None):
    y = a.new_zeros((a.shape[0], b.shape[1]))
    for e, (low, high) in enumerate(_groups(ends)):
        y[low:high] = a[low:high] @ b[e].t()
    return y


def _gradient(dy, sdy, x, sx, ends=None, dtype=None):
    if ends is None:
        return dy @ x.t()
    return torch.stack([dy[:, low:high] @ x[:, low:high].t() for low, high in _groups(ends)])


@pytest.fixture(autouse=True)
def exact_products(monkeypatch):
    """Codes are the values themselves: no gradient passes through the calls, as through the
    kernels' own."""
    def quantize_tiles(w, transposed=False):
        s = w.new_ones((*w.shape[:-2], 1, 1))
        return (w, s, w.transpose(-1, -2).contiguous()) if transposed else (w, s)
    calls = dict(transform=_transform, transform_fp8_blocks=_transform_fp8_blocks,
                 quantize_fp8_tiles=quantize_tiles,
                 quantize_fp8_columns=lambda x, ends=None: (x.t(), None),
                 matmul_fp8=lambda a, sa, b, sb, dtype=None: a @ b.t(),
                 grouped_matmul_fp8=_grouped_matmul, grouped_weight_gradient_fp8=_gradient)
    monkeypatch.setattr(E, "hadacore", SimpleNamespace(
        **{name: torch.no_grad()(call) for name, call in calls.items()}))


def _make(ends):
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((12, 32), generator=gen, dtype=torch.float64)
    w = torch.randn((*([3] if ends else []), 5, 32), generator=gen, dtype=torch.float64)
    dy = torch.randn((12, 5), generator=gen, dtype=torch.float64)
    return x.requires_grad_(), w.requires_grad_(), dy, torch.tensor(ends) if ends else None


def _product(x, w, ends):
    if ends is None:
        return x @ w.t()
    parts = [x[low:high] @ w[e].t() for e, (low, high) in enumerate(_groups(ends))]
    return torch.cat([*parts, x.new_zeros((x.shape[0] - int(ends[-1]), w.shape[1]))])


@pytest.mark.parametrize("rotate", [1, 8, None])
@pytest.mark.parametrize("ends", [None, [4, 4, 11]])
def test_gradients(ends, rotate):
    x, w, dy, ends = _make(ends)
    want = torch.autograd.grad(_product(x, w, ends), (x, w), dy)
    y = E.train_linear(x, w, ends, rotate)
    assert torch.allclose(y, _product(x, w, ends), rtol=1e-12, atol=1e-12)
    got = torch.autograd.grad(y, (x, w), dy)
    for g, r in zip(got, want):
        assert torch.allclose(g, r, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("constant", [True, False])
@pytest.mark.parametrize("ends", [None, [4, 4, 11]])
def test_second_derivatives_are_refused(ends, constant, which):
    """A gradient of the layer is no differentiable function: a loss that holds one has to
    raise, not to lose that term, whether or not the output's gradient requires one itself."""
    x, w, dy, ends = _make(ends)
    y = E.train_linear(x, w, ends)
    f = y.sum() if constant else (y * y).sum()
    grad = torch.autograd.grad(f, (x, w)[which], create_graph=True)[0]
    # the first derivative is there, whole
    ref = _product(x, w, ends)
    want = torch.autograd.grad(ref.sum() if constant else (ref * ref).sum(), (x, w)[which])[0]
    assert torch.allclose(grad.detach(), want, rtol=1e-12, atol=1e-12)
    with pytest.raises(RuntimeError, match="second derivative"):
        (y.sum() + grad.pow(2).sum()).backward()


@pytest.mark.parametrize("wanted", ["x", "w"])
def test_one_gradient_alone(wanted):
    x, w, dy, _ = _make(None)
    leaf = x if wanted == "x" else w
    (w if wanted == "x" else x).requires_grad_(False)
    E.train_linear(x, w).backward(dy)
    want = dy @ w if wanted == "x" else dy.t() @ x
    assert torch.allclose(leaf.grad, want.detach(), rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("k,rotate", [(0, 1), (1, 1), (7, 1), (96, 32), (4096, 4096), (3 << 20, 1 << 15)])
def test_default_rotation(k, rotate):
    assert E.default_rotation(k) == rotate


@pytest.mark.parametrize("ends", [None, [4, 4, 11]])
def test_nothing_to_multiply(ends):
    """Rows without columns: zeros, and empty gradients."""
    x, w, dy, ends = _make(ends)
    x, w = (t.detach()[..., :0].requires_grad_() for t in (x, w))
    y = E.train_linear(x, w, ends)
    assert y.shape == dy.shape and (y == 0).all()
    y.backward(dy)
    assert x.grad.shape == x.shape and w.grad.shape == w.shape
