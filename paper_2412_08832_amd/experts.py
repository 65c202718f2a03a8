"""Linear layers in FP8 on rotated activations, dense or one weight per expert.

A layer y = x w^T is computed as (x H)(w H)^T, H the Hadamard transform of ``rotate``
columns at a time: H is orthonormal, so y is the same, but the codes are those of rotated
values, as models keep them whose weights have the rotation folded in.  (For its accuracy
alone e4m3 with a scale per 128 values does not need it: the codes keep their relative
precision over 15 binades, so that columns 50 times the others' size cost nothing, and the
example below is 0.029 off without the rotation and 0.037 with it.)  Forward:

    a  = codes of x H          transform_fp8_blocks
    b  = codes of w H          transform, quantize_fp8_tiles
    y  = a b^T                 matmul_fp8, or grouped_matmul_fp8 by expert

Backward, for the output's gradient dy:

    dx = dy w                  transform_fp8_blocks(n=1), the product with w's transposed codes
    dw = dy^T x                quantize_fp8_columns, grouped_weight_gradient_fp8

In dx = (dy (w H)) H and dw = (dy^T (x H)) H the rotations cancel, so neither is made: each
gradient is one product, rounded once.  Between two rotations it would be held in 16 bits,
and values of one sign are up to sqrt(rotate) times larger there, past fp16's range.  The
backward's codes are of w, for which quantize_weights takes one pass more over the weights
(without a rotation they are the forward's).

``python -m paper_2412_08832_amd.experts`` runs a small layer of experts forward and
backward on the GPU and prints its errors against 32 bits, with and without the rotation.

A mixture of experts around such layers: ``route`` chooses each token's experts from a router's
logits (with the balance loss), ``hadacore.group_tokens`` sorts the (token, choice) slots by
expert, ``dispatch`` copies the tokens' rows there and ``combine`` joins the layer's rows by weight,
each with gradients.  ``mixture`` is one layer of it for training, ``serve_mixture`` for serving: that
quantizes every token once and dispatches codes.

    routes = route(logits, k, valid=valid)
    groups = hadacore.group_tokens(routes.experts, experts)
    out = combine(train_linear(dispatch(x, groups), w, groups.ends), groups, routes.weights)
    loss = task_loss(out) + 0.01 * routes.loss

To capture a training step into a graph, let no graph of autograd made outside of the capture live
that has the same leaves (torch would wait for its streams, which a capture cannot).
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import hadacore


class Weights(NamedTuple):
    """Weights laid out for the products: codes of w H, and of w, transposed, for the backward."""
    codes: torch.Tensor
    scales: torch.Tensor
    codes_t: torch.Tensor | None
    scales_t: torch.Tensor | None
    rotate: int


def default_rotation(k: int) -> int:
    """The largest power of two that divides k, at most 32768 (1 for no columns)."""
    return min(k & -k, 1 << 15) or 1


def rotate_rows(x: torch.Tensor, rotate: int) -> torch.Tensor:
    """Each ``rotate`` values of the contiguous tensor ``x`` times H / sqrt(rotate)."""
    if rotate == 1 or x.numel() == 0:
        return x
    return hadacore.transform(x.view(-1, rotate)).view(x.shape)


def quantize_weights(w: torch.Tensor, rotate: int | None = None, backward: bool = True) -> Weights:
    """Weights (n x k, or experts x n x k; float16 or bfloat16) as codes; once for serving,
    every step for training.  ``backward=False`` leaves the transposed codes out."""
    rotate = default_rotation(w.shape[-1]) if rotate is None else rotate
    w, codes_t, scales_t = w.contiguous(), None, None
    if backward:
        codes, scales, codes_t = hadacore.quantize_fp8_tiles(w, transposed=True)
        scales_t = scales.transpose(-1, -2).contiguous()
    if rotate != 1 or not backward:
        # between the rotation and its codes float16 weights are bfloat16, which holds whatever
        # the rotation of finite weights gives (up to sqrt(rotate) times the largest) for two
        # roundings of 2^-9, each a thirtieth of the codes' own
        if rotate != 1 and w.dtype is torch.float16:
            w = w.bfloat16()
        codes, scales = hadacore.quantize_fp8_tiles(rotate_rows(w, rotate))
    return Weights(codes, scales, codes_t, scales_t, rotate)


def _product(a, a_scales, b, b_scales, ends, dtype):
    if ends is None:
        return hadacore.matmul_fp8(a, a_scales, b, b_scales, dtype=dtype)
    return hadacore.grouped_matmul_fp8(a, a_scales, b, b_scales, ends, dtype=dtype)


def linear(x: torch.Tensor, weights: Weights, ends: torch.Tensor | None = None) -> torch.Tensor:
    """x w^T for quantized weights: rows of ``x`` (tokens x k), or, with ``ends``, groups of
    rows sorted by expert, each with its own weight.  No gradient."""
    a, a_scales = hadacore.transform_fp8_blocks(x, n=weights.rotate)
    return _product(a, a_scales, weights.codes, weights.scales, ends, x.dtype)


def weight_gradient(dy: torch.Tensor, x: torch.Tensor, ends: torch.Tensor | None = None,
                    dtype: torch.dtype | None = None) -> torch.Tensor:
    """dy^T x in FP8 (tokens x n, tokens x k), with ``ends`` for each group of rows: the gradient
    of the layer's weights in ``dtype`` (default: x's), float32 for an optimizer that keeps 32 bits."""
    d, d_scales = hadacore.quantize_fp8_columns(dy, ends)
    a, a_scales = hadacore.quantize_fp8_columns(x, ends)
    return hadacore.grouped_weight_gradient_fp8(d, d_scales, a, a_scales, ends,
                                                dtype=x.dtype if dtype is None else dtype)


class _NoSecondDerivative(torch.autograd.Function):
    """The identity, whose gradient raises."""
    @staticmethod
    def forward(ctx, g):
        return g.view_as(g)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the layers have no second derivative: a gradient taken with "
                           "create_graph=True is not to be differentiated")


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, ends, rotate):
        q = quantize_weights(w, rotate, backward=ctx.needs_input_grad[0])
        ctx.weight_dtype = w.dtype
        ctx.save_for_backward(x, ends, q.codes_t, q.scales_t)
        return linear(x, q, ends)

    @staticmethod
    def backward(ctx, dy):
        with torch.no_grad():
            grads = _Linear.gradients(ctx, dy)
        if torch.is_grad_enabled():
            # create_graph=True: the gradients depend on dy and on w or x, through calls that
            # autograd does not see.  once_differentiable would mark them for dy's sake only.
            grads = [g if g is None else _NoSecondDerivative.apply(g.requires_grad_()) for g in grads]
        return *grads, None, None

    @staticmethod
    def gradients(ctx, dy):
        x, ends, codes_t, scales_t = ctx.saved_tensors
        dy = dy.contiguous()
        dx = dw = None
        if ctx.needs_input_grad[0]:
            d, d_scales = hadacore.transform_fp8_blocks(dy, n=1)
            dx = _product(d, d_scales, codes_t, scales_t, ends, x.dtype)
        if ctx.needs_input_grad[1]:
            dw = weight_gradient(dy, x, ends, ctx.weight_dtype)
        return dx, dw


def train_linear(x: torch.Tensor, w: torch.Tensor, ends: torch.Tensor | None = None,
                 rotate: int | None = None) -> torch.Tensor:
    """``linear`` with gradients of ``x`` and ``w`` (both float16 or both bfloat16), whose
    codes are made anew.  First derivatives only: to differentiate a gradient raises."""
    return _Linear.apply(x, w, ends, rotate)


class _First(torch.autograd.Function):
    """What the exchange's functions share: gradients that are not differentiated again."""
    @classmethod
    def backward(cls, ctx, *grads):
        with torch.no_grad():
            out = cls.gradients(ctx, *grads)
        if torch.is_grad_enabled():
            out = [g if g is None else _NoSecondDerivative.apply(g.requires_grad_()) for g in out]
        return tuple(out)


class _Route(_First):
    @staticmethod
    def forward(ctx, logits, k, renormalize, valid):
        routes = hadacore.route_tokens(logits, k, renormalize, valid)
        ctx.renormalize = renormalize
        ctx.mark_non_differentiable(routes.experts, routes.counts, routes.slopes)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, *routes[:5])
        return routes[:5]

    @staticmethod
    def gradients(ctx, _, dweights, __, dloss, ___):
        if dweights is None and dloss is None:
            return None, None, None, None
        logits, *routes = ctx.saved_tensors
        dweights = None if dweights is None else dweights.contiguous()
        return hadacore.route_tokens_gradient(logits, hadacore.Routes(*routes, ctx.renormalize),
                                              dweights, dloss), None, None, None


class _Dispatch(_First):
    @staticmethod
    def forward(ctx, x, rows, ends):
        ctx.save_for_backward(rows)
        return hadacore.dispatch_rows(x, rows, ends)

    @staticmethod
    def gradients(ctx, dxs):
        return hadacore.combine_rows(dxs.contiguous(), *ctx.saved_tensors), None, None


class _Combine(_First):
    @staticmethod
    def forward(ctx, y, weights, rows, ends):
        # y is needed for the weights' gradient, and the weights for y's
        ctx.save_for_backward(y if weights is not None and ctx.needs_input_grad[1] else None, weights, rows, ends)
        return hadacore.combine_rows(y, rows, weights)

    @staticmethod
    def gradients(ctx, dout):
        y, weights, rows, ends = ctx.saved_tensors
        dy, dweights = hadacore.combine_rows_gradient(dout.contiguous(), y, rows, ends, weights,
                                                      want_dy=ctx.needs_input_grad[0])
        return dy, dweights, None, None


def route(logits: torch.Tensor, k: int, renormalize: bool = True,
          valid: torch.Tensor | None = None) -> hadacore.Routes:
    """``hadacore.route_tokens`` with gradients of the logits for ``weights`` and ``loss``."""
    return hadacore.Routes(*_Route.apply(logits.contiguous(), k, renormalize, valid), renormalize)


def dispatch(x: torch.Tensor, groups: hadacore.Groups) -> torch.Tensor:
    """Rows of ``x`` (tokens x width) at the places of their slots, with a gradient."""
    return _Dispatch.apply(x.contiguous(), groups.rows, groups.ends)


def combine(y: torch.Tensor, groups: hadacore.Groups, weights: torch.Tensor | None = None) -> torch.Tensor:
    """The rows of each token's slots joined by weight (tokens x choices, float32; None: their
    sum), with gradients of ``y`` and ``weights``."""
    return _Combine.apply(y.contiguous(), weights, groups.rows, groups.ends)


def _check_router(logits: torch.Tensor, experts: int) -> None:
    """A choice past the last expert would be a slot of no group, whose share of its token is lost."""
    if logits.dim() != 2 or logits.shape[1] != experts:
        raise ValueError(f"logits of {tuple(logits.shape)} for {experts} experts: expected a column for each")


def mixture(x: torch.Tensor, logits: torch.Tensor, w: torch.Tensor, k: int, renormalize: bool = True,
            valid: torch.Tensor | None = None, rotate: int | None = None):
    """(out, routes): each token's ``k`` experts of ``w`` (experts x n x k) by ``logits`` (tokens x
    experts), joined by their weights; with gradients of x, logits (also for ``routes.loss``) and w."""
    _check_router(logits, w.shape[0])
    routes = route(logits, k, renormalize, valid)
    groups = hadacore.group_tokens(routes.experts, w.shape[0])
    return combine(train_linear(dispatch(x, groups), w, groups.ends, rotate), groups, routes.weights), routes


def serve_mixture(x: torch.Tensor, logits: torch.Tensor, weights: Weights, k: int, renormalize: bool = True,
                  valid: torch.Tensor | None = None) -> torch.Tensor:
    """``mixture`` for quantized weights, without gradients: tokens are rotated and quantized once, and
    their codes dispatched."""
    _check_router(logits, weights.codes.shape[0])
    routes = hadacore.route_tokens(logits, k, renormalize, valid)
    groups = hadacore.group_tokens(routes.experts, weights.codes.shape[0])
    a, a_scales = hadacore.transform_fp8_blocks(x, n=weights.rotate)
    y = hadacore.grouped_matmul_fp8(hadacore.dispatch_rows(a, groups.rows, groups.ends),
                                    hadacore.dispatch_rows(a_scales, groups.rows, groups.ends),
                                    weights.codes, weights.scales, groups.ends, dtype=x.dtype)
    return hadacore.combine_rows(y, groups.rows, routes.weights)


def _mixture_example() -> None:
    """A mixture of 8 experts, two a token, its balance loss beside its output."""
    tokens, experts, n, k = 2000, 8, 512, 2048
    x = torch.randn(tokens, k, device="cuda").bfloat16()
    w = (torch.randn(experts, n, k, device="cuda") / k ** 0.5).bfloat16()
    logits, dy = torch.randn(tokens, experts, device="cuda"), torch.randn(tokens, n, device="cuda")
    grads = []
    for plain in (False, True):
        leaves = [t.clone().requires_grad_() for t in ((x.float(), w.float(), logits) if plain else (x, w, logits))]
        if plain:
            p = torch.softmax(leaves[2], 1)
            top = torch.topk(leaves[2], 2, dim=1).indices
            share = p.gather(1, top) / p.gather(1, top).sum(1, keepdim=True)
            all_y = torch.einsum("tk,enk->ten", leaves[0], leaves[1])
            out = (all_y.gather(1, top[..., None].expand(-1, -1, n)) * share[..., None]).sum(1)
            f = torch.bincount(top.view(-1), minlength=experts) / top.numel()
            loss = experts * (f * p.mean(0)).sum()
        else:
            out, routes = mixture(leaves[0], leaves[2], leaves[1], 2)
            loss = routes.loss
        ((out.float() * dy).sum() + loss).backward()
        grads.append([out.detach().float(), *(t.grad.float() for t in leaves), loss.detach()])
    off = [float((a - b).norm() / b.norm()) for a, b in zip(*grads)]
    print(f"mixture: relative error of out {off[0]:.4f}, dx {off[1]:.4f}, dw {off[2]:.4f}, "
          f"d logits {off[3]:.4f}, balance loss {off[4]:.1e}")


def main() -> None:
    torch.manual_seed(0)
    tokens, experts, n, k = 4000, 8, 1024, 4096
    x = torch.randn(tokens, k, device="cuda")
    x[:, torch.randperm(k, device="cuda")[:16]] *= 50
    w = torch.randn(experts, n, k, device="cuda") / k ** 0.5
    dy = torch.randn(tokens, n, device="cuda")
    cuts = torch.sort(torch.randint(0, tokens + 1, (experts - 1,))).values
    ends = torch.cat([cuts, torch.tensor([tokens])]).int().cuda()
    low = [0, *ends.tolist()[:-1]]
    groups = [slice(a, b) for a, b in zip(low, ends.tolist())]
    x16, w16, dy16 = x.bfloat16(), w.bfloat16(), dy.bfloat16()
    want = [torch.cat([x16[s].float() @ w16[e].float().t() for e, s in enumerate(groups)]),
            torch.cat([dy16[s].float() @ w16[e].float() for e, s in enumerate(groups)]),
            torch.stack([dy16[s].float().t() @ x16[s].float() for s in groups])]
    for rotate in (1, default_rotation(k)):
        leaf_x, leaf_w = x16.clone().requires_grad_(), w16.clone().requires_grad_()
        y = train_linear(leaf_x, leaf_w, ends, rotate)
        y.backward(dy16)
        off = [float((g.float() - r).norm() / r.norm())
               for g, r in zip((y.detach(), leaf_x.grad, leaf_w.grad), want)]
        print(f"rotation of {rotate:4d}: relative error of y {off[0]:.4f}, dx {off[1]:.4f}, "
              f"dw {off[2]:.4f}")
    _mixture_example()


if __name__ == "__main__":
    main()
