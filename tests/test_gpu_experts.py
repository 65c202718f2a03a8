"""The rotated FP8 linear layers: values and gradients against 64 bits and differences.

Bound of a product's relative error: a code is within 1/16 of its value, evenly, so its
rms error is at most 1/16 / sqrt(3) = 0.036 of it; two operands give 0.051, and the 16-bit
roundings of rotated rows and results less than 0.005 more.
"""
from __future__ import annotations

import pytest

from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu

REL = 0.056


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def _make(tokens, experts, n, k, dtype, ends=None, outliers=True):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(tokens + n + k)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    x = normal(tokens, k)
    if outliers:
        x[:, 3] *= 40
    w = normal(*([experts] if experts else []), n, k) / k ** 0.5
    dy = normal(tokens, n)
    if ends is not None:
        ends = torch.tensor(ends, dtype=torch.int32, device="cuda")
    return x.to(dtype), w.to(dtype), dy.to(dtype), ends


def _expected(x, w, dy, ends):
    import torch
    x, w, dy = x.double().cpu(), w.double().cpu(), dy.double().cpu()
    if ends is None:
        return x @ w.t(), dy @ w, dy.t() @ x
    y, dx, dw = torch.zeros(x.shape[0], w.shape[1]).double(), torch.zeros_like(x), torch.zeros_like(w)
    low = 0
    for e, high in enumerate(ends.tolist()):
        s = slice(low, high)
        y[s], dx[s], dw[e] = x[s] @ w[e].t(), dy[s] @ w[e], dy[s].t() @ x[s]
        low = high
    return y, dx, dw


CASES = [(300, 0, 200, 512, None, None), (1, 0, 64, 128, None, None), (130, 0, 96, 640, 128, None),
         (77, 0, 40, 96, 32, None), (64, 0, 48, 300, 1, None),
         (500, 4, 160, 384, None, [100, 100, 350, 500]), (9, 5, 64, 256, None, [1, 2, 2, 9, 9]),
         (260, 3, 72, 512, 64, [0, 200, 250])]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("tokens,experts,n,k,rotate,ends", CASES)
def test_layer_and_its_gradients(tokens, experts, n, k, rotate, ends, dtype):
    import torch
    from paper_2412_08832_amd import experts as E
    x, w, dy, ends = _make(tokens, experts, n, k, getattr(torch, dtype), ends,
                           outliers=rotate is None)
    want = _expected(x, w, dy, ends)
    x.requires_grad_()
    w.requires_grad_()
    y = E.train_linear(x, w, ends, rotate)
    y.backward(dy)
    for name, got, ref in zip(("y", "dx", "dw"), (y.detach(), x.grad, w.grad), want):
        assert got.shape == ref.shape and _rel(got.cpu(), ref) <= REL, name
    if ends is not None:
        last = int(ends[-1])
        assert (y[last:] == 0).all() and (x.grad[last:] == 0).all()
        for e, (low, high) in enumerate(zip([0, *ends.tolist()[:-1]], ends.tolist())):
            if low == high:
                assert (w.grad[e] == 0).all()
    q = E.quantize_weights(w.detach(), rotate, backward=False)
    assert torch.equal(E.linear(x.detach(), q, ends), y)


@pytest.mark.parametrize("which", ["x", "w"])
@pytest.mark.parametrize("ends", [None, [40, 40, 200]])
def test_gradients_against_differences(which, ends):
    """(f(v + h d) - f(v - h d)) / 2h = <grad, d> for f = <c, y>, which is linear in x and in
    w, so that h may be large.  The codes' error of f is that of a sum of independent terms:
    at most REL |c * y| in the rms, of which four are allowed on either side; the gradient's
    own along d is at most REL |grad| |d|."""
    import torch
    from paper_2412_08832_amd import experts as E
    x, w, c, ends = _make(200, 3 if ends else 0, 96, 512, torch.float16, ends)
    leaf_x, leaf_w = x.clone().requires_grad_(), w.clone().requires_grad_()
    E.train_linear(leaf_x, leaf_w, ends).backward(c)
    v, grad = (x, leaf_x.grad) if which == "x" else (w, leaf_w.grad)
    d = grad.double() / grad.double().norm()
    h = 0.5 * float(v.double().norm())
    values, noise = [], 0.0
    for sign in (1, -1):
        moved = (v.double() + sign * h * d).to(v.dtype)
        y = E.train_linear(*((moved, w) if which == "x" else (x, moved)), ends).double()
        values.append(float((y * c.double()).sum()))
        noise += float((y * c.double()).norm())
    slope = (values[0] - values[1]) / (2 * h)
    expect = float((grad.double() * d).sum())
    assert abs(slope - expect) <= 4 * REL * noise / (2 * h) + REL * float(grad.double().norm())


def test_wrapper_refusals():
    import torch
    a = torch.zeros((4, 256), dtype=torch.uint8, device="cuda")
    b = torch.zeros((130, 256), dtype=torch.uint8, device="cuda")
    sa, sb = torch.ones((4, 2), device="cuda"), torch.ones((2, 2), device="cuda")
    H.matmul_fp8(a, sa, b, sb)
    H.matmul_fp8(a.view(torch.float8_e4m3fn), sa, b, torch.ones((130, 2), device="cuda"))
    ends = torch.tensor([1, 4], dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        H.matmul_fp8(a.to(torch.int8), sa, b, sb)
    with pytest.raises(TypeError):
        H.matmul_fp8(a, sa.double(), b, sb)
    with pytest.raises(TypeError):
        H.matmul_fp8(a, sa, b, sb, dtype=torch.float64)
    with pytest.raises(TypeError):
        H.transform_fp8_blocks(torch.zeros((4, 256), device="cuda"))
    for bad in (lambda: H.matmul_fp8(a, sa, b[:, :128], sb), lambda: H.matmul_fp8(a, sa[:3], b, sb),
                lambda: H.matmul_fp8(a, sa, b, sb.cpu()), lambda: H.matmul_fp8(a[0], sa, b, sb),
                lambda: H.matmul_fp8(a, sa, b, sb, out=torch.zeros((4, 129), device="cuda")),
                lambda: H.matmul_fp8(a, sa, b.t().contiguous().t(), sb),
                # the last row of 250 codes ends where its storage does
                lambda: H.matmul_fp8(a.view(-1)[6:].as_strided((3, 250), (256, 1), 6 + 256),
                                     sa[:3], b[:, :250], sb),
                lambda: H.grouped_matmul_fp8(a, sa, b[None], sb[None], ends),
                lambda: H.grouped_matmul_fp8(a, sa, b[None].expand(2, -1, -1),
                                             sb[None].expand(2, -1, -1), ends.long()),
                lambda: H.quantize_fp8_columns(a.half(), ends.cpu()),
                lambda: H.grouped_weight_gradient_fp8(a, sa, b[:, :128], sb),
                lambda: H.quantize_fp8_tiles(a.half().t()),
                lambda: H.transform_fp8_blocks(a.half(), codes=torch.zeros((4, 255), device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: H.transform_fp8_blocks(a.half(), n=512), 2),
                        (lambda: H.transform_fp8_blocks(a.half()[:, 1:129], n=128), 5),
                        (lambda: H.matmul_fp8(a[:, 8:136], sa[:, :1], b[:, :128], sb[:, :1]), 5)):
        with pytest.raises(H.HadacoreError) as e:
            bad()
        assert e.value.status == status
    torch.cuda.synchronize()
