"""The algebra of routing, exchange, adapters and the mixture on the CPU: plain calls in 64 bits in the
kernels' place, gradients against autograd of the formulas."""
from __future__ import annotations

from types import SimpleNamespace

import pytest
import torch

import tokens_reference as R
from paper_2412_08832_amd import adapters as A
from paper_2412_08832_amd import experts as E
from paper_2412_08832_amd import hadacore as H


def _route_tokens(logits, k, renormalize=True, valid=None):
    return H.Routes(*(t.detach() for t in R.route(logits, k, renormalize, valid)), renormalize)


def _route_gradient(logits, routes, dweights=None, dloss=None):
    p = torch.softmax(logits, 1) * (routes.experts[:, :1] >= 0)
    u = routes.slopes[None] * (0.0 if dloss is None else dloss)
    extra = torch.zeros_like(p)
    if dweights is not None:
        there, index = routes.experts >= 0, routes.experts.clamp(min=0).long()
        if routes.renormalize:
            w = routes.weights
            extra = extra.scatter_add(1, index, there * w * (dweights - (w * dweights).sum(1, keepdim=True)))
        else:
            u = u + extra.scatter_add(1, index, there * dweights)
    return p * (u - (p * u).sum(1, keepdim=True)) + extra


def _dispatch(x, rows, ends):
    return R.dispatch(x, rows, rows.numel())


def _combine(y, rows, weights=None):
    return R.combine(y, rows, weights)[0]


def _combine_gradient(dout, y, rows, ends, weights=None, want_dy=True):
    scaled = torch.ones(rows.shape, dtype=dout.dtype) if weights is None else weights
    dy, dw = dout.new_zeros((rows.numel(), dout.shape[1])), dout.new_zeros(rows.shape)
    for t, j in ((t, j) for t in range(rows.shape[0]) for j in range(rows.shape[1])):
        if rows[t, j] >= 0:
            dy[rows[t, j]] = scaled[t, j] * dout[t]
            dw[t, j] = 0.0 if y is None else dout[t] @ y[rows[t, j]]
    return (dy if want_dy else None), (None if y is None else dw)


def _adapt_rows(x, down, up, ends=None, slots=None, y=None, scales=None, dtype=None, hidden=False):
    down, up = (t if t.dim() == 3 else t[None] for t in (down, up))
    out, _, h, _ = R.adapt(x, down, up, ends, slots, y, scales, 0, 0)
    return (out, h) if hidden else out


def _adapter_gradient(h, x, ends=None, slots=None, scales=None, dtype=None):
    return R.weight_gradient(h, x, ends, slots, scales, torch.bfloat16, torch.float32)[0]


def _linear(x, w, ends, rotate=None):
    parts = [x[low:high] @ w[e].t() for e, (low, high) in enumerate(R.groups_of(ends, x.shape[0]))]
    return torch.cat([*parts, x.new_zeros((x.shape[0] - int(ends[-1]), w.shape[1]))])


@pytest.fixture(autouse=True)
def plain_calls(monkeypatch):
    calls = dict(route_tokens=_route_tokens, route_tokens_gradient=_route_gradient, group_tokens=lambda i, g: H.Groups(*R.group(i, g)),
                 dispatch_rows=_dispatch, combine_rows=_combine, combine_rows_gradient=_combine_gradient,
                 adapt_rows=_adapt_rows, adapter_gradient=_adapter_gradient)
    fake = SimpleNamespace(Routes=H.Routes, Groups=H.Groups, **{n: torch.no_grad()(c) for n, c in calls.items()})
    monkeypatch.setattr(E, "hadacore", fake)
    monkeypatch.setattr(A, "hadacore", fake)
    monkeypatch.setattr(E, "train_linear", _linear)


def _randn(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def _close(got, want):
    assert all(torch.allclose(g, w, rtol=1e-11, atol=1e-12) for g, w in zip(got, want))


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("masked", [False, True])
def test_mixture(renormalize, masked):
    """out and the balance loss of a layer of four experts, two a token, against the formulas."""
    x, logits, w = (t.requires_grad_() for t in (_randn(9, 6), _randn(9, 4, seed=1), _randn(4, 5, 6, seed=2)))
    valid = torch.arange(9) % 4 != 3 if masked else None
    dy = _randn(9, 5, seed=3)
    out, routes = E.mixture(x, logits, w, 2, renormalize, valid)
    got = torch.autograd.grad((out * dy).sum() + 0.3 * routes.loss, (x, logits, w))
    chosen, weights, _, loss, _ = R.route(logits, 2, renormalize, valid)
    y = torch.stack([x @ w[e].t() for e in range(4)], 1)
    want_out = (y.gather(1, chosen.clamp(min=0).long()[..., None].expand(-1, -1, 5)) * weights[..., None]).sum(1)
    assert torch.allclose(out, want_out) and torch.allclose(routes.loss, loss)
    _close(got, torch.autograd.grad((want_out * dy).sum() + 0.3 * loss, (x, logits, w)))


@pytest.mark.parametrize("wanted", ["weights", "loss"])
def test_one_gradient_of_the_routes(wanted):
    logits = _randn(7, 5).requires_grad_()
    routes = E.route(logits, 3)
    _, weights, _, loss, _ = R.route(logits, 3, True)
    f, ref = (routes.loss, loss) if wanted == "loss" else ((routes.weights ** 2).sum(), (weights ** 2).sum())
    _close(torch.autograd.grad(f, logits), torch.autograd.grad(ref, logits))


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("which", ["y", "weights"])
def test_one_gradient_of_the_join(which, weighted):
    if which == "weights" and not weighted:
        return
    groups = H.Groups(*R.group(torch.tensor([[0, 1], [1, -1], [2, 0]], dtype=torch.int32), 3))
    y, w = _randn(6, 4), _randn(3, 2, seed=1) if weighted else None
    leaf = (y if which == "y" else w).requires_grad_()
    out = E.combine(y, groups, w)
    keep = groups.rows >= 0
    ref = (y[groups.rows.clamp(min=0).long()] * keep[..., None] * (1.0 if w is None else w[..., None])).sum(1)
    _close(torch.autograd.grad((out ** 2).sum(), leaf), torch.autograd.grad((ref ** 2).sum(), leaf))


@pytest.mark.parametrize("wanted", ["yxdu", "y", "x", "d", "u", "xu"])
@pytest.mark.parametrize("grouped", [True, False])
def test_adapters(grouped, wanted):
    x, down, up, y = _randn(8, 6), _randn(3, 2, 6, seed=1), _randn(3, 2, 5, seed=2), _randn(8, 5, seed=3)
    scales, dout = torch.tensor([0.5, 2.0, 1.5]), _randn(8, 5, seed=4)
    ids = torch.tensor([0, 2, -1, 0, 2, 2, -1, 0], dtype=torch.int32)
    if not grouped:
        down, up, scales, ids = down[:1], up[:1], scales[:1], torch.zeros(8, dtype=torch.int32)
    groups = H.Groups(*R.group(ids, 3)) if grouped else None
    leaves = {"y": y, "x": x, "d": down, "u": up}
    for name in wanted:
        leaves[name].requires_grad_()
    out = A.adapt(y, x, down, up, groups, scales)
    at = ids.clamp(min=0).long()
    s = torch.where(ids >= 0, scales.double()[at], 0.0)
    ref = y + s[:, None] * torch.einsum("tr,trn->tn", torch.einsum("tk,trk->tr", x, down[at]), up[at])
    assert torch.allclose(out, ref)
    wrt = [leaves[n] for n in wanted]
    _close(torch.autograd.grad(out, wrt, dout), torch.autograd.grad(ref, wrt, dout))


def test_second_derivatives_are_refused():
    """But for y's gradient, which is the output's own."""
    groups = H.Groups(*R.group(torch.tensor([[0, 1], [1, 0]], dtype=torch.int32), 2))
    logits, x, w, y = (t.requires_grad_() for t in (_randn(2, 3), _randn(2, 4), _randn(2, 2), _randn(4, 4)))
    down, up = _randn(1, 2, 4).requires_grad_(), _randn(1, 2, 4).requires_grad_()
    cases = [(lambda: (E.route(logits, 2).weights ** 2).sum(), logits),
             (lambda: (E.dispatch(x, groups) ** 2).sum(), x), (lambda: (E.combine(y, groups, w) ** 2).sum(), y),
             (lambda: (E.combine(y, groups, w) ** 2).sum(), w), (lambda: (A.adapt(x, x.detach(), down, up) ** 2).sum(), up)]
    for f, leaf in cases:
        grad = torch.autograd.grad(f(), leaf, create_graph=True)[0]
        with pytest.raises(RuntimeError, match="second derivative"):
            grad.pow(2).sum().backward()
    out = A.adapt(x, x.detach(), down.detach(), up.detach())
    grad = torch.autograd.grad((out ** 2).sum(), x, create_graph=True)[0]
    _close([torch.autograd.grad(grad.sum(), x)[0]], [2 * torch.ones_like(x)])


def test_scales_with_a_gradient_are_refused():
    with pytest.raises(ValueError):
        A.adapt(_randn(2, 4), _randn(2, 4), _randn(1, 2, 4), _randn(1, 2, 4), scales=torch.ones(1, requires_grad=True))
