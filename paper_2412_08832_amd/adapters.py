"""Low-rank adapters of many requests beside a shared projection.

A projection y = x w^T serves every request; a request may bring an adapter of its own,

    out = y + scales[g] * (x down[g]^T) up[g]

for the tokens of adapter g, and y for those without one.  ``down`` is adapters x rank x k and ``up``
adapters x rank x n, in x's type: both rank by rank, so that the same kernels serve forward and
backward.  (A weight kept as n x rank is ``w.t().contiguous()``, once.)  Adapters of smaller ranks
get zero rows.

    groups = hadacore.group_tokens(ids, adapters)          # int32 ids, -1: none; once for all layers
    y = experts.linear(x, weights)                         # FP8, or any projection
    y = adapters.adapt(y, x, down, up, groups, scales)

``adapt`` has gradients of y, x, down and up (first derivatives only, no forward mode); without any to
make it is one call of ``hadacore.adapt_rows``, and ``adapt_rows(..., out=y)`` adds in place.

``python -m paper_2412_08832_amd.adapters`` runs a projection in FP8 with the adapters of a batch of
requests forward and backward on the GPU and prints its errors against 32 bits.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad

from . import hadacore
from .experts import _NoSecondDerivative


class _Adapt(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, x, down, up, ends, slots, scales):
        keep = ctx.needs_input_grad[3]  # the gradient of up takes h
        out = hadacore.adapt_rows(x, down, up, ends, slots, y=y, scales=scales, hidden=keep)
        out, h = out if keep else (out, None)
        ctx.save_for_backward(x, down, up, ends, slots, scales, h)
        return out

    @staticmethod
    def backward(ctx, dout):
        with torch.no_grad():
            grads = _Adapt.gradients(ctx, dout)
        if torch.is_grad_enabled():
            grads = [g if g is None else _NoSecondDerivative.apply(g.requires_grad_()) for g in grads]
        return dout, *grads, None, None, None

    @staticmethod
    def gradients(ctx, dout):
        x, down, up, ends, slots, scales, h = ctx.saved_tensors
        need_x, need_down, need_up = ctx.needs_input_grad[1:4]
        dx = d_down = d_up = None
        # of a projection in 32 bits: rounded to x's type, which the products take; the gradients are
        # rounded to it themselves
        dout = dout.to(x.dtype).contiguous()
        if need_down:
            # without x's gradient only the first of the two products is made
            back = down if need_x else down[..., :0]
            dx, dh = hadacore.adapt_rows(dout, up, back, ends, slots, scales=scales, hidden=True)
            d_down = hadacore.adapter_gradient(dh, x, ends, slots, scales).view(down.shape)
        elif need_x:
            dx = hadacore.adapt_rows(dout, up, down, ends, slots, scales=scales)
        if need_up:
            d_up = hadacore.adapter_gradient(h, dout, ends, slots, scales).view(up.shape)
        return dx if need_x else None, d_down, d_up


def adapt(y: torch.Tensor, x: torch.Tensor, down: torch.Tensor, up: torch.Tensor,
          groups: hadacore.Groups | None = None, scales: torch.Tensor | None = None) -> torch.Tensor:
    """y + scales[g] * (x down[g]^T) up[g] for the tokens of each adapter g; a new tensor of y's type
    (x's, or float32).  ``groups`` is ``hadacore.group_tokens``' of one id a token; None: one
    adapter for all.  ``scales`` (float32, one for each adapter) has no gradient.

    The gradient of a float32 output is y's as it is; for those of x, down and up it is rounded to x's
    type first, as by a cast of the adapters' part before it is added: half a step of that type for
    each value, and float16 has its range (scale the loss as for a float16 layer)."""
    ends, slots = (None, None) if groups is None else (groups.ends, groups.slots)
    if scales is not None and scales.requires_grad and torch.is_grad_enabled():
        raise ValueError("the adapters' scales have no gradient")
    # where forward mode is on, too: the function refuses tensors with tangents, which a call would drop
    if forward_ad._current_level >= 0 or torch.is_grad_enabled() and any(t.requires_grad for t in (y, x, down, up)):
        return _Adapt.apply(y, x.contiguous(), down, up, ends, slots, scales)
    return hadacore.adapt_rows(x, down, up, ends, slots, y=y, scales=scales)


def main() -> None:
    from . import experts
    torch.manual_seed(0)
    tokens, adapters, rank, n, k = 3000, 6, 16, 1024, 4096
    x = torch.randn(tokens, k, device="cuda").bfloat16()
    w = (torch.randn(n, k, device="cuda") / k ** 0.5).bfloat16()
    down = (torch.randn(adapters, rank, k, device="cuda") / k ** 0.5).bfloat16()
    up = (0.2 * torch.randn(adapters, rank, n, device="cuda")).bfloat16()
    scales = 0.5 + torch.rand(adapters, device="cuda")
    dout = torch.randn(tokens, n, device="cuda").bfloat16()
    # requests of a few hundred tokens, some without an adapter
    ids = torch.randint(-1, adapters, (20,), device="cuda").repeat_interleave(150).int()
    groups = hadacore.group_tokens(ids, adapters)
    leaves = [t.clone().requires_grad_() for t in (x, down, up)]
    y = experts.linear(x, experts.quantize_weights(w, backward=False))
    out = adapt(y, *leaves, groups, scales)
    out.backward(dout)
    wide = [t.float().clone().requires_grad_() for t in (x, down, up)]
    s = torch.where(ids >= 0, scales[ids.clamp(min=0).long()], 0.0)[:, None]
    at = ids.clamp(min=0).long()
    h = (wide[0][:, None] @ wide[1][at].transpose(1, 2)).squeeze(1)
    delta = s * (h[:, None] @ wide[2][at]).squeeze(1)
    delta.backward(dout.float())
    got = [(out - y).detach().float(), *(t.grad.float() for t in leaves)]
    want = [delta.detach(), *(t.grad for t in wide)]
    off = [float((g - r).norm() / r.norm()) for g, r in zip(got, want)]
    print(f"relative error of the adapters' part {off[0]:.4f} (rounded beside y), dx {off[1]:.4f}, "
          f"d down {off[2]:.4f}, d up {off[3]:.4f}")


if __name__ == "__main__":
    main()
