"""The exchange between tokens and rows sorted by group, on the GPU, against 64 bits."""
from __future__ import annotations

import pytest
import torch

import tokens_reference as R
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _ids(shape, groups, seed=0, none=0.1):
    gen = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, max(groups, 1), shape, generator=gen).to(torch.int32)
    out = torch.rand(shape, generator=gen) < none
    wrong = torch.tensor([-1, groups, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64)
    ids[out] = wrong[torch.randint(0, 4, (int(out.sum()),), generator=gen)].to(torch.int32)
    return ids


def _values(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("shape,groups", [
    ((0,), 3), ((1,), 1), ((5,), 1), ((64,), 0), ((63, 1), 2), ((65, 2), 3), ((17, 2), 32), ((1000, 3), 7),
    ((4096,), 64), ((4097,), 64), ((3000, 4), 61), ((2048, 8), 256), ((5001,), 900), ((5001,), 901),
    ((9001,), 2047), ((9000,), 3201), ((30000,), 4095), ((40000, 5), 8)])
def test_group(shape, groups):
    for none in (0.0, 0.3, 1.0):
        ids = _ids(shape, groups, groups, none)
        if groups == 0 and none < 1:
            ids.fill_(0)
        got = H.group_tokens(ids.cuda(), groups)
        for a, b in zip(got, R.group(ids, groups)):
            assert torch.equal(a.cpu(), b)


def test_group_in_one_run_and_sorted():
    for ids in (torch.full((10000,), 3), torch.arange(10000) // 100, 99 - torch.arange(10000) // 100):
        ids = ids.to(torch.int32)
        for a, b in zip(H.group_tokens(ids.cuda(), 100), R.group(ids, 100)):
            assert torch.equal(a.cpu(), b)


SIZES = [(1, 1, 1), (1, 2, 8), (3, 2, 7), (5, 4, 64), (40, 2, 100), (33, 8, 513), (9, 3, 1000), (64, 2, 2048),
         (7, 5, 2051), (12, 1, 4096), (6, 9, 5003), (2, 32, 300), (300, 2, 16)]


@pytest.mark.parametrize("dtype", [torch.uint8, torch.float8_e4m3fn, *TYPES])
@pytest.mark.parametrize("m,k,width", SIZES)
def test_dispatch(m, k, width, dtype):
    ids = _ids((m, k), 5, m + width)
    ends, rows, _ = R.group(ids, 5)
    x = torch.randint(0, 256, (m, width * dtype.itemsize), dtype=torch.uint8,
                      generator=torch.Generator().manual_seed(m))
    got = H.dispatch_rows(x.cuda().view(dtype), rows.cuda(), ends.cuda())
    assert got.dtype == dtype and got.shape == (m * k, width)
    assert torch.equal(got.contiguous().view(torch.uint8).cpu(), R.dispatch(x, rows, m * k))
    if dtype.itemsize == 1:
        assert got.stride(0) % 16 == 0  # as the products read codes


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("m,k,width", SIZES)
def test_combine(m, k, width, weighted, dtype):
    ends, rows, _ = R.group(_ids((m, k), 4, m + k), 4)
    y = _values((m * k, width), dtype, width)
    y[int(ends[-1]):] = float("nan")  # behind the last end
    w = _values((m, k), torch.float32, 9) if weighted else None
    if weighted:
        w[rows < 0] = float("nan")
    got = H.combine_rows(y.cuda(), rows.cuda(), None if w is None else w.cuda())
    want, size = R.combine(y, rows, w)
    R.check("combine", got, want, R.rounded(want, (k + 1) * R.U * size, dtype))
    assert torch.equal(got, H.combine_rows(y.cuda(), rows.cuda(), None if w is None else w.cuda()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("m,k,width", SIZES)
def test_combine_gradient(m, k, width, weighted, dtype):
    ends, rows, _ = R.group(_ids((m, k), 4, m + k), 4)
    y, dout = _values((m * k, width), dtype, width), _values((m, width), dtype, 1)
    y[int(ends[-1]):] = float("nan")
    w = _values((m, k), torch.float32, 9) if weighted else None
    args = [t.cuda() for t in (rows, ends)]
    dy, dw = H.combine_rows_gradient(dout.cuda(), y.cuda(), *args, None if w is None else w.cuda())
    scaled = torch.ones((m, k), dtype=torch.float64) if w is None else w.double()
    want_y = torch.zeros((m * k, width), dtype=torch.float64)
    want_w, size = torch.zeros((m, k), dtype=torch.float64), torch.zeros((m, k), dtype=torch.float64)
    for t in range(m):
        for j in range(k):
            r = int(rows[t, j])
            if r >= 0:
                want_y[r] = scaled[t, j] * dout[t].double()
                terms = dout[t].double() * y[r].double()
                want_w[t, j], size[t, j] = terms.sum(), terms.abs().sum()
    R.check("dy", dy, want_y, R.rounded(want_y, R.U * want_y.abs(), dtype))
    # a lane's steps (8 of every 512 values at least), the lanes' and the waves'
    R.check("dweights", dw, want_w, R.rounded(want_w, (width / 64 + 8 + 6 + 4) * R.U * size, torch.float32))
    only_y, none = H.combine_rows_gradient(dout.cuda(), None, *args, None if w is None else w.cuda())
    assert none is None and torch.equal(only_y, dy)
    none, only_w = H.combine_rows_gradient(dout.cuda(), y.cuda(), *args, None if w is None else w.cuda(), want_dy=False)
    assert none is None and torch.equal(only_w, dw)


def test_gradient_against_differences():
    """combine is linear in y and in its weights: (f(v + h d) - f(v - h d)) / 2h is <grad, d> up to the
    roundings of the two f, each within the bound of its sums."""
    m, k, width = 20, 3, 200
    ends, rows, _ = (t.cuda() for t in R.group(_ids((m, k), 4, 1), 4))
    y, dout = _values((m * k, width), torch.float32, 2).cuda(), _values((m, width), torch.float32, 3).cuda()
    w = _values((m, k), torch.float32, 4).cuda()
    dy, dw = H.combine_rows_gradient(dout, y, rows, ends, w)
    for name in ("y", "w"):
        v, grad = (y, dy) if name == "y" else (w, dw)
        d, values, noise = torch.randn_like(v), [], 0.0
        for sign in (1, -1):
            moved = v + sign * d
            got = H.combine_rows(moved if name == "y" else y, rows, moved if name == "w" else w)
            values.append(float((got.double() * dout.double()).sum()))
            size = R.combine((moved if name == "y" else y).cpu(), rows.cpu(), (moved if name == "w" else w).cpu())[1]
            # and the rounding of v + d
            noise += (k + 3) * R.U * float((size * dout.double().cpu().abs()).sum())
        slope, expect = (values[0] - values[1]) / 2, float((grad.double() * d.double()).sum())
        assert abs(slope - expect) <= noise + 32 * R.U * float((grad.double() * d.double()).abs().sum()) * width


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.uint8])
def test_rows_with_gaps_from_any_address(dtype):
    """Strided rows from odd addresses; what lies between rows stays."""
    m, k, width, pitch = 30, 2, 301, 333
    ends, rows, _ = (t.cuda() for t in R.group(_ids((m, k), 4, 1), 4))
    x = torch.randint(0, 100, (m, width), generator=torch.Generator().manual_seed(0)).to(dtype)

    def laid(rows_, fill):
        flat = torch.full((rows_ * pitch + 3,), fill, dtype=dtype, device="cuda")
        return flat, flat[3:].view(rows_, pitch)[:, :width]
    _, source = laid(m, 7)
    source.copy_(x)
    flat, target = laid(m * k, 9)
    want = R.dispatch(x, rows.cpu(), m * k)
    H.dispatch_rows(source, rows, ends, out=target)
    assert torch.equal(target.cpu(), want)
    target.fill_(9)
    assert (flat == 9).all()
    if dtype is torch.uint8:
        return
    target.copy_(want)
    flat, back = laid(m, 9)
    H.combine_rows(target, rows, out=back)
    assert torch.equal(back, H.combine_rows(want.cuda(), rows))
    back.fill_(9)
    assert (flat == 9).all()
    dout = source
    for a, b in zip(H.combine_rows_gradient(dout, target, rows, ends),
                    H.combine_rows_gradient(x.cuda(), want.cuda(), rows, ends)):
        assert torch.equal(a, b)


def test_wrong_rows_and_ends_stay_in_bounds():
    """Places past the tensor and ends past the slots: results within what is there."""
    rows = torch.tensor([[0, 99], [2, -5], [2 ** 31 - 1, 3]], dtype=torch.int32, device="cuda")
    ends = torch.tensor([2, 1000], dtype=torch.int32, device="cuda")
    x = torch.randn((3, 40), device="cuda")
    out = H.dispatch_rows(x, rows, ends)
    assert torch.equal(out[0], x[0]) and torch.equal(out[2], x[1]) and torch.equal(out[3], x[2])
    y = torch.randn((6, 40), device="cuda")
    assert torch.equal(H.combine_rows(y, rows), torch.stack([y[0], y[2], y[3]]))
    _, dw = H.combine_rows_gradient(x, y, rows, ends, want_dy=False)
    assert dw[0, 1] == 0 and dw[1, 1] == 0 and dw[2, 0] == 0


def test_nothing_to_move():
    ends = torch.zeros(2, dtype=torch.int32, device="cuda")
    rows = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    assert H.dispatch_rows(torch.empty((0, 8), device="cuda"), rows, ends).shape == (0, 8)
    assert H.combine_rows(torch.empty((0, 8), device="cuda"), rows).shape == (0, 8)
    rows = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    assert (H.combine_rows(torch.empty((0, 8), device="cuda"), rows) == 0).all()
    assert (H.dispatch_rows(torch.ones((3, 8), device="cuda"), rows, ends) == 0).all()
    dy, dw = H.combine_rows_gradient(torch.ones((3, 0), device="cuda"), torch.ones((6, 0), device="cuda"), rows, ends)
    assert dy.shape == (6, 0) and (dw == 0).all()


def test_refusals():
    x = torch.zeros((4, 16), device="cuda")
    ends, rows, _ = H.group_tokens(torch.zeros((4, 2), dtype=torch.int32, device="cuda"), 3)
    y = torch.zeros((8, 16), device="cuda")
    for bad, kind in ((lambda: H.group_tokens(torch.zeros((4, 2), device="cuda"), 3), ValueError),
                      (lambda: H.group_tokens(torch.zeros((4, 2), dtype=torch.int32), 3), ValueError),
                      (lambda: H.dispatch_rows(x.double(), rows, ends), TypeError),
                      (lambda: H.dispatch_rows(x[:3], rows, ends), ValueError),
                      (lambda: H.dispatch_rows(x, rows.long(), ends), ValueError),
                      (lambda: H.dispatch_rows(x, rows, ends.long()), ValueError),
                      (lambda: H.dispatch_rows(x, rows, ends, out=y[:7]), ValueError),
                      (lambda: H.combine_rows(y.to(torch.uint8), rows), TypeError),
                      (lambda: H.combine_rows(y, rows, torch.zeros((4, 3), device="cuda")), ValueError),
                      (lambda: H.combine_rows(y, rows, torch.zeros((4, 2), device="cuda").half()), TypeError),
                      (lambda: H.combine_rows_gradient(x, y[:7], rows, ends), ValueError),
                      (lambda: H.combine_rows_gradient(x, y.half(), rows, ends), ValueError)):
        with pytest.raises(kind):
            bad()
    with pytest.raises(H.HadacoreError) as e:
        H.group_tokens(torch.zeros(4, dtype=torch.int32, device="cuda"), 4096)
    assert e.value.status == 2
    with pytest.raises(H.HadacoreError) as e:
        H.combine_rows(y, rows, out=y[4:])
    assert e.value.status == 6
    torch.cuda.synchronize()
