"""The adapters' gradients beside a projection in 32 bits: those of a dout rounded to x's type, and y's unrounded."""
from __future__ import annotations

import pytest
import torch

from paper_2412_08832_amd import adapters as A
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_gradient_of_a_wide_output(dtype):
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    gen = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    x, down, up, y = normal(300, 256).to(dtype), normal(3, 8, 256).to(dtype), normal(3, 8, 96).to(dtype), normal(300, 96)
    groups = H.group_tokens(torch.randint(-1, 3, (300,), generator=gen, device="cuda").int(), 3)
    dout = 1000 * normal(300, 96)
    dout[7, 5] = 1e5  # past float16
    grads = []
    for d in (dout, dout.to(dtype).float()):
        leaves = [t.clone().requires_grad_() for t in (y, x, down, up)]
        grads.append(torch.autograd.grad(A.adapt(*leaves, groups), leaves, d))
    assert torch.equal(grads[0][0], dout)
    for a, b in zip(grads[0][1:], grads[1][1:]):
        assert a.dtype == dtype and bool(((a == b) | (a.isnan() & b.isnan())).all())
    assert bool(grads[0][3].isfinite().all()) == (dtype is torch.bfloat16)
