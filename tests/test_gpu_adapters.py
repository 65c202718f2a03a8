"""Low-rank adapters on the GPU: outputs, hidden values and gradients against 64 bits."""
from __future__ import annotations

import pytest
import torch

import tokens_reference as R
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _make(m, k, n, rank, groups, dtype, out=None, seed=0, idle=True):
    """Inputs on the CPU; some tokens have no adapter and, with `idle`, some adapters no token."""
    gen = torch.Generator().manual_seed(seed + m + k + n + rank)

    def normal(*shape):
        return torch.randn(shape, generator=gen)
    x, down, up = normal(m, k).to(dtype), (normal(groups, rank, k) / max(k, 1) ** 0.5).to(dtype), \
        (0.3 * normal(groups, rank, n)).to(dtype)
    y = normal(m, n).to(out or dtype)
    scales = 0.5 + torch.rand(groups, generator=gen)
    ids = torch.randint(-1, groups - (groups > 2 and idle), (m,), generator=gen).to(torch.int32)
    ends, _, slots = R.group(ids, groups)
    return x, down, up, y, scales, ends, slots


def _cuda(*tensors):
    return [None if t is None else t.cuda() for t in tensors]


def _check(x, down, up, y, scales, ends, slots, out_dtype, on_gpu=None):
    args = _cuda(x, down, up, y, scales, ends, slots) if on_gpu is None else on_gpu
    gx, gd, gu, gy, gs, ge, gl = args
    got, h = H.adapt_rows(gx, gd, gu, ends=ge, slots=gl, y=gy, scales=gs, dtype=out_dtype, hidden=True)
    want, off, want_h, h_off = R.adapt(x, down, up, ends, slots, y, scales, *R.parts(x.dtype, out_dtype))
    assert got.dtype == out_dtype and h.shape == (x.shape[0], down.shape[1])
    R.check("out", got, want, R.rounded(want, off, out_dtype))
    used = x.shape[0] if ends is None else int(ends[-1]) if len(ends) else 0
    R.check("hidden", h[:used], want_h[:used], R.rounded(want_h, h_off, F32)[:used])
    assert torch.equal(got, H.adapt_rows(gx, gd, gu, ends=ge, slots=gl, y=gy, scales=gs, dtype=out_dtype))
    return got, h


SIZES = [  # m, k, n, rank, adapters
    (1, 8, 8, 1, 1), (1, 512, 300, 16, 1), (2, 31, 33, 3, 2), (17, 100, 64, 8, 5), (64, 4096, 513, 16, 32),
    (64, 1000, 1000, 11, 7), (65, 257, 130, 17, 3), (40, 640, 96, 32, 4), (100, 96, 257, 33, 2),
    (70, 300, 1030, 64, 3), (33, 520, 200, 65, 2), (50, 128, 520, 100, 3), (200, 2050, 72, 128, 2),
    (45, 136, 300, 129, 2), (130, 264, 257, 256, 2), (700, 72, 40, 24, 2), (1500, 130, 1100, 16, 3),
    (3000, 64, 2056, 40, 1), (2500, 40, 5000, 5, 2)]


@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("m,k,n,rank,groups", SIZES)
def test_sizes(m, k, n, rank, groups, dtype, out):
    data = _make(m, k, n, rank, groups, dtype, out)
    _check(*data, out)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_without_y_scales_ends_and_slots(dtype):
    x, down, up, y, scales, ends, slots = _make(150, 200, 300, 20, 3, dtype)
    _check(x, down, up, None, scales, ends, slots, dtype)
    _check(x, down, up, None, None, ends, None, F32)
    for d, u in ((down[:1], up[:1]),):
        got, h = _check(x, d, u, y, None, None, None, dtype)
        flat = H.adapt_rows(x.cuda(), d[0].cuda(), u[0].cuda(), y=y.cuda())
        assert torch.equal(got, flat)
        _check(x, d, u, y, scales[:1], None, slots, dtype)


def test_in_place_and_out():
    x, down, up, y, scales, ends, slots = _cuda(*_make(90, 300, 200, 16, 4, BF16))
    want = H.adapt_rows(x, down, up, ends, slots, y, scales)
    out = torch.empty_like(y)
    assert H.adapt_rows(x, down, up, ends, slots, y, scales, out=out) is out and torch.equal(out, want)
    assert H.adapt_rows(x, down, up, ends, slots, y, scales, out=y) is y and torch.equal(y, want)


@pytest.mark.parametrize("ends", [[0, 0, 0], [40, 40, 40], [0, 0, 40], [0, 25, 25], [1, 2, 3], [16, 32, 40], [17, 17, 39]])
def test_groups_of_any_size(ends):
    x, down, up, y, scales, _, _ = _make(40, 136, 200, 16, 3, BF16)
    gen = torch.Generator().manual_seed(5)
    slots = torch.randperm(40, generator=gen).to(torch.int32)
    _check(x, down, up, y, scales, torch.tensor(ends, dtype=torch.int32), slots, BF16)


def test_tokens_without_an_adapter_keep_y():
    """Bit for bit: -0 and NaN among them."""
    for m, n in ((5, 128), (700, 300)):
        x, down, up, y, scales, _, slots = _make(m, 64, n, 8, 2, BF16)
        y[:, 0], y[:, 1] = -0.0, float("nan")
        ends = torch.zeros(2, dtype=torch.int32)
        got = H.adapt_rows(*_cuda(x, down, up), *_cuda(ends, slots), y=y.cuda())
        assert torch.equal(got.view(torch.int16).cpu(), y.view(torch.int16))


def test_no_tokens_groups_or_columns():
    x, down, up, y, scales, ends, slots = _cuda(*_make(10, 64, 48, 8, 2, BF16))
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert H.adapt_rows(x[:0], down, up, ends * 0, none, y[:0]).shape == (0, 48)
    assert torch.equal(H.adapt_rows(x, down[:0], up[:0], none, slots, y), y)
    assert torch.equal(H.adapt_rows(x[:, :0], down[..., :0], up, ends, slots, y), y)
    out, h = H.adapt_rows(x, down, up[..., :0], ends, slots, hidden=True)
    _, want = H.adapt_rows(x, down, up, ends, slots, hidden=True)
    used = int(ends[-1])
    assert out.shape == (10, 0) and torch.equal(h[:used], want[:used])
    g = H.adapter_gradient(want[:0], x[:0], ends * 0, none)
    assert g.shape == (2, 8, 64) and (g == 0).all()
    assert H.adapter_gradient(want, x, none, slots).shape == (0, 8, 64)
    assert H.adapter_gradient(want, x[:, :0], ends, slots).shape == (2, 8, 0)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rows_from_any_address(dtype):
    """Rows with gaps, from addresses that only 2 bytes divide; what lies between rows stays."""
    m, k, n, rank, groups = 50, 203, 301, 12, 3
    data = _make(m, k, n, rank, groups, dtype)
    x, down, up, y, scales, ends, slots = data

    def laid(t, gap):
        rows = t.reshape(-1, t.shape[-1])
        flat = torch.full((rows.shape[0] * (t.shape[-1] + gap) + 1,), float("nan"), dtype=t.dtype, device="cuda")
        view = flat[1:].view(*t.shape[:-1], t.shape[-1] + gap)[..., : t.shape[-1]]
        view.copy_(t)
        return view
    on_gpu = [laid(x, 6), laid(down, 3), laid(up, 5), laid(y, 2), *_cuda(scales, ends, slots)]
    got, h = _check(*data, dtype, on_gpu=on_gpu)
    flat = torch.full((m * (n + 9) + 5,), 3.0, dtype=dtype, device="cuda")
    out = flat[5:].view(m, n + 9)[:, :n]
    H.adapt_rows(*on_gpu[:3], ends=on_gpu[5], slots=on_gpu[6], y=on_gpu[3], scales=on_gpu[4], out=out)
    assert torch.equal(out, got)
    out.fill_(3.0)
    assert (flat == 3.0).all()
    dense = H.adapter_gradient(h.contiguous(), x.cuda(), on_gpu[5], on_gpu[6], dtype=F32)
    assert torch.equal(H.adapter_gradient(h, on_gpu[0], on_gpu[5], on_gpu[6], dtype=F32), dense)
    flat = torch.full((groups * (rank + 1) * (k + 9) + 5,), 3.0, device="cuda")
    out = flat[5:].view(groups, rank + 1, k + 9)[:, :rank, :k]
    H.adapter_gradient(h, on_gpu[0], on_gpu[5], on_gpu[6], out=out)
    assert torch.equal(out, dense)
    out.fill_(3.0)
    assert (flat == 3.0).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_values_stay_with_their_token(dtype):
    """NaN in tokens without an adapter, in y's rows, in one token's x and in one adapter."""
    x, down, up, y, scales, ends, slots = _cuda(*_make(60, 300, 260, 16, 3, dtype))
    clean = H.adapt_rows(x, down, up, ends, slots, y, scales)
    used = int(ends[-1])
    free, one = slots[used:].long(), int(slots[used // 2])
    x2, y2 = x.clone(), y.clone()
    x2[free] = float("nan")
    assert torch.equal(H.adapt_rows(x2, down, up, ends, slots, y, scales), clean)
    x2[one, 299] = float("nan")
    y2[int(slots[0]), 5] = float("inf")
    got = H.adapt_rows(x2, down, up, ends, slots, y2, scales)
    assert got[one].isnan().all() and got[int(slots[0]), 5].isinf()
    keep = torch.ones(60, dtype=torch.bool, device="cuda")
    keep[[one, int(slots[0])]] = False
    assert torch.equal(got[keep], clean[keep])
    d2 = down.clone()
    d2[1] = float("nan")
    got = H.adapt_rows(x, d2, up, ends, slots, y, scales)
    hit = slots[int(ends[0]) : int(ends[1])].long()
    assert got[hit].isnan().all()
    keep = torch.ones(60, dtype=torch.bool, device="cuda")
    keep[hit] = False
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("size", [2.0 ** -12, 1.0, 2.0 ** 7])
def test_fp16_hidden_values_past_fp16(size):
    """h of up to some 2^17 and down to 2^-30: fp32 between the products."""
    x, down, up, y, scales, ends, slots = _make(40, 512, 64, 16, 2, F16, F32)
    x, down = (x * size).to(F16), (down * size * 16).to(F16)
    _check(x, down, (up / 64).to(F16), y, scales, ends, slots, F32)


@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("m,width,rank,groups", [
    (1, 1, 1, 1), (5, 40, 3, 2), (33, 128, 16, 2), (100, 129, 17, 3), (257, 300, 32, 2), (300, 136, 50, 4),
    (280, 257, 64, 1), (90, 70, 100, 2), (600, 200, 256, 2), (1500, 384, 16, 2), (3000, 130, 8, 1), (4100, 64, 40, 3)])
def test_weight_gradient(m, width, rank, groups, dtype, out):
    x, _, _, _, scales, ends, slots = _make(m, width, 8, rank, groups, dtype)
    gen = torch.Generator().manual_seed(m)
    h = torch.randn((m, rank), generator=gen) * torch.exp(3 * torch.randn((m, 1), generator=gen))
    h[int(ends[-1]):] = float("nan")  # not written by adapt_rows
    got = H.adapter_gradient(*_cuda(h, x, ends, slots, scales), dtype=out)
    want, off = R.weight_gradient(h, x, ends, slots, scales, dtype, out)
    assert got.dtype == out
    R.check("gradient", got, want, R.rounded(want, off, out))
    assert torch.equal(got, H.adapter_gradient(*_cuda(h, x, ends, slots, scales), dtype=out))
    if groups == 1:
        h = torch.nan_to_num(h)
        want, off = R.weight_gradient(h, x, None, None, None, dtype, out)
        R.check("one", H.adapter_gradient(h.cuda(), x.cuda(), dtype=out)[None], want, R.rounded(want, off, out))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_gradients_against_the_formula(dtype):
    """The four calls of a training step against autograd of the definition in 64 bits.  dx's bound is that
    of the call; the weights' gradients add that of the hidden values they are made of."""
    x, down, up, y, scales, ends, slots = _make(400, 264, 200, 16, 3, dtype)
    dout = torch.randn((400, 200), generator=torch.Generator().manual_seed(9)).to(dtype)
    leaves = [t.double().requires_grad_() for t in (x, down, up, y)]
    out = leaves[3].clone()
    for g, (low, high) in enumerate(R.groups_of(ends, 400)):
        t = slots[low:high].long()
        out = out.index_add(0, t, float(scales[g]) * (leaves[0][t] @ leaves[1][g].t()) @ leaves[2][g])
    wx, wdown, wup, wy = torch.autograd.grad(out, leaves, dout.double())
    gx, gd, gu, gy, gs, ge, gl, gdo = _cuda(x, down, up, y, scales, ends, slots, dout)
    _, h = H.adapt_rows(gx, gd, gu, ge, gl, gy, gs, hidden=True)
    dx, dh = H.adapt_rows(gdo, gu, gd, ge, gl, scales=gs, hidden=True)
    _, off, want_dh, dh_off = R.adapt(dout, up, down, ends, slots, None, scales, *R.parts(dtype, dtype))
    R.check("dx", dx, wx, R.rounded(wx, off, dtype))
    _, _, want_h, h_off = R.adapt(x, down, up, ends, slots, None, scales, *R.parts(dtype, dtype))
    for name, got, want, hidden, hidden_off, rows in (
            ("down", H.adapter_gradient(dh, gx, ge, gl, gs, dtype=F32), wdown, want_dh, dh_off, x),
            ("up", H.adapter_gradient(h, gdo, ge, gl, gs, dtype=F32), wup, want_h, h_off, dout)):
        _, off = R.weight_gradient(hidden, rows, ends, slots, scales, dtype, F32)
        more, _ = R.weight_gradient(hidden_off, rows.double().abs(), ends, slots, scales, dtype, F32)
        R.check(name, got, want, R.rounded(want, off + more, F32))
    assert torch.equal(wy, dout.double())


WIDTHS = list(range(1, 18)) + [23, 31, 33, 127, 129, 509, 511, 513, 1023, 1025]


def _between(t):
    """The same values on the GPU in rows with NaN before, between and behind them, off 16 bytes."""
    width = t.shape[-1]
    room = torch.full((3 + t[..., 0].numel() * (width + 3) + 3,), float("nan"), dtype=t.dtype, device="cuda")
    rows = room[3:-3].view(*t.shape[:-1], width + 3)
    rows[..., :width] = t.cuda()
    return rows[..., :width], room


@pytest.mark.parametrize("dtype,out", [(F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("m,rank,groups", [(9, 5, 1), (21, 16, 2), (300, 7, 2), (90, 70, 2), (150, 150, 1)])
def test_every_width_of_the_last_columns(m, rank, groups, dtype, out):
    """Rows narrower than a load, and whose last values a load takes from before their place: nothing
    from outside a row gets in, and nothing outside is written."""
    for i, width in enumerate(WIDTHS):
        k, n = width, WIDTHS[(i * 7 + 3) % len(WIDTHS)]
        x, down, up, y, scales, ends, slots = _make(m, k, n, rank, groups, dtype, out, idle=False)
        (gx, _), (gd, _), (gu, _), (gy, room) = (_between(t) for t in (x, down, up, y))
        gs, ge, gl = _cuda(scales, ends, slots)
        got, h = _check(x, down, up, y, scales, ends, slots, out, (gx, gd, gu, gy, gs, ge, gl))
        gap = torch.isnan(room).sum()
        assert H.adapt_rows(gx, gd, gu, ends=ge, slots=gl, y=gy, scales=gs, out=gy) is gy
        assert torch.equal(gy, got) and torch.isnan(room).sum() == gap
        want, off = R.weight_gradient(h.cpu(), x, ends, slots, scales, dtype, F32)
        grad = H.adapter_gradient(h, gx, ge, gl, scales=gs, dtype=F32)
        R.check("gradient", grad, want, R.rounded(want, off, F32))


def test_refusals():
    x, down, up, y, scales, ends, slots = _cuda(*_make(10, 64, 48, 8, 2, BF16))
    h = torch.zeros((10, 8), device="cuda")
    for bad, kind in ((lambda: H.adapt_rows(x.float(), down, up, ends, slots), TypeError),
                      (lambda: H.adapt_rows(x, down.half(), up, ends, slots), TypeError),
                      (lambda: H.adapt_rows(x, down, up, ends, slots, dtype=F16), TypeError),
                      (lambda: H.adapt_rows(x, down, up, ends, slots, y=y.half()), TypeError),
                      (lambda: H.adapt_rows(x, down, up, ends, slots, scales=scales.double()), TypeError),
                      (lambda: H.adapt_rows(x, down, up[:1], ends, slots), ValueError),
                      (lambda: H.adapt_rows(x, down, up, ends[:1], slots), ValueError),
                      (lambda: H.adapt_rows(x, down, up), ValueError),
                      (lambda: H.adapt_rows(x[:, :60], down, up, ends, slots), ValueError),
                      (lambda: H.adapt_rows(x, down, up, ends, slots[:9]), ValueError),
                      (lambda: H.adapt_rows(x, down, up, ends, slots, y=y[:9]), ValueError),
                      (lambda: H.adapt_rows(x, down, up, ends, slots, y=y, dtype=F32), ValueError),
                      (lambda: H.adapt_rows(x, down, up, ends, slots, out=y.float()), ValueError),
                      (lambda: H.adapt_rows(x, down.transpose(1, 2).contiguous().transpose(1, 2), up, ends, slots), ValueError),
                      (lambda: H.adapt_rows(x, down, up, ends.cpu(), slots), ValueError),
                      (lambda: H.adapter_gradient(h.half(), x, ends, slots), ValueError),
                      (lambda: H.adapter_gradient(h[:9], x, ends, slots), ValueError),
                      (lambda: H.adapter_gradient(h, x, ends, slots, dtype=F16), TypeError),
                      (lambda: H.adapter_gradient(h, x, ends, slots, out=h), ValueError)):
        with pytest.raises(kind):
            bad()
    big = torch.zeros((2, 257, 64), dtype=BF16, device="cuda")
    with pytest.raises(H.HadacoreError) as e:
        H.adapt_rows(x, big, big, ends, slots)
    assert e.value.status == 2
    with pytest.raises(H.HadacoreError) as e:
        H.adapt_rows(x, down, up[..., :40], ends, slots, out=x[:, :40])
    assert e.value.status == 6
    torch.cuda.synchronize()
