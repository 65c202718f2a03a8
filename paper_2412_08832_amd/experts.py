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
        raise RuntimeError("the FP8 linear layers have no second derivative: a gradient taken with "
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


if __name__ == "__main__":
    main()
