"""Codes and products of sizes that take a streaming cache policy: the same results as small
calls' bit for bit (quantizers), or 64 bits' (products), and nothing written beside them."""
from __future__ import annotations

import numpy as np
import pytest

import blocks_reference as R
from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _torch_type(out):
    import torch
    return {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}[out]


def _host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _input(shape, gap, dtype, seed):
    """Values whose tiles, rows and columns differ in size; rows `gap` values apart."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    *lead, n, k = shape
    x = torch.randn((*lead, n, k + gap), generator=gen, device="cuda")
    x *= torch.exp2(3 * torch.randn((*lead, n, 1), generator=gen, device="cuda").clamp(-2, 2))
    return x.to(_torch_type(dtype))[..., :k]


# ---- quantizers: strips of less than 2^22 elements take the plain policy ------------

# from 2^22 elements codes are streamed out, past 2^25 the input is streamed in too, both
# where the codes' rows are whole lines, and the second where the input's rows start on 16 bytes
TILES = [((3, 512, 4096), 0), ((1280, 4224), 0), ((2, 4224, 4096), 0), ((2, 4224, 4096), 3),
         ((2, 1031, 4096), 0), ((2, 4300, 4096), 0), ((8448, 4096), 0)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("shape,gap", TILES)
def test_tiles(shape, gap, transposed, dtype):
    import torch
    w = _input(shape, gap, dtype, seed=sum(shape))
    codes, scales, *codes_t = H.quantize_fp8_tiles(w, transposed=transposed)
    for e, matrix in enumerate(w if w.dim() == 3 else w[None]):
        c, s = (codes[e], scales[e]) if w.dim() == 3 else (codes, scales)
        for r in range(0, matrix.shape[0], 896):
            want, want_scales = H.quantize_fp8_tiles(matrix[r:r + 896])
            assert torch.equal(c[r:r + 896], want), f"matrix {e} from row {r}"
            assert torch.equal(s[r // 128:][:want_scales.shape[0]], want_scales)
        cut = slice(matrix.shape[0] // 128 * 128 - 128, matrix.shape[0])
        R.check_tiles(matrix[cut].double().cpu().numpy(), c[cut].cpu().numpy(),
                      s[matrix.shape[0] // 128 - 1:].cpu().numpy(), f"matrix {e}")
    if transposed:
        assert torch.equal(codes.transpose(-1, -2), codes_t[0])


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("n", [1, 8, 64, 128, 2048])
@pytest.mark.parametrize("m,k,gap", [(1100, 4096, 0), (8200, 4224, 0), (8321, 4096, 8)])
def test_rows(m, k, gap, n, dtype):
    import torch
    if k % n:
        k = k // n * n
    x = _input((m, k), gap, dtype, seed=m + n)
    codes, scales = H.transform_fp8_blocks(x, n=n)
    for r in range(0, m, 900):
        want, want_scales = H.transform_fp8_blocks(x[r:r + 900], n=n)
        assert torch.equal(codes[r:r + 900], want) and torch.equal(scales[r:r + 900], want_scales)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("m,k,gap", [(1100, 4096, 0), (8200, 4224, 0), (8321, 4096, 5)])
def test_columns(m, k, gap, dtype):
    import torch
    x = _input((m, k), gap, dtype, seed=m)
    codes, scales = H.quantize_fp8_columns(x)
    for r in range(0, m, 896):
        want, want_scales = H.quantize_fp8_columns(x[r:r + 896])
        assert torch.equal(codes[:, r:r + want.shape[1]], want)
        assert torch.equal(scales[:, r // 128:][:, :want_scales.shape[1]], want_scales)


# ---- products ------------------------------------------------------------------------


def _codes(seed, rows, k, scale_rows=None):
    """e4m3 codes of N(0, 1) values drawn from 2^16 of them, and scales: on the GPU, on the host."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    values = (torch.randn(1 << 16, generator=gen, device="cuda") * 120).clamp(-448, 448)
    table = values.to(torch.float8_e4m3fn).view(torch.uint8)
    pitch = -(-k // 16) * 16
    codes = torch.full((rows, pitch), 0x7F, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // k)
    for r in range(0, rows, step):
        at = torch.randint(0, 1 << 16, (min(step, rows - r), k), generator=gen, device="cuda")
        codes[r:r + step, :k] = table[at]
    scales = torch.exp2(torch.rand((rows if scale_rows is None else scale_rows, -(-k // 128)),
                                   generator=gen, device="cuda") * 4 - 12)
    return codes[:, :k], scales


def _check(a, sa, b, sb, got, out, tall=128, what=""):
    R.check_product(*(t.cpu().numpy() for t in (a, sa, b, sb)), _host(got), out, tall, what)


def _some(n, step):
    return np.unique(np.r_[np.arange(0, n, step), n - 1])


# weights of 2^26 codes and more that one workgroup reads: the three shapes of few rows
FEW = [(1, 3077, 21842, "bf16"), (2, 3077, 21842, "fp16"), (5, 2614, 25674, "fp32"),
       (13, 19413, 3458, "bf16"), (13, 19413, 3458, "fp16"), (8, 8983, 7475, "fp32"),
       (20, 31839, 2109, "bf16"), (17, 31839, 2109, "fp16"), (17, 10807, 6243, "fp32")]


@pytest.mark.parametrize("m,n,k,out", FEW)
def test_few_rows_by_large_weights(m, n, k, out):
    import torch
    a, sa = _codes(m, m, k)
    b, sb = _codes(n, n, k, scale_rows=-(-n // 128))
    buf = torch.full((m + 1, n), 5.0, dtype=_torch_type(out), device="cuda")
    y = H.matmul_fp8(a, sa, b, sb, out=buf[:m])
    assert (buf[m] == 5).all()
    cols = _some(n, 23)
    pick = torch.from_numpy(cols).cuda()
    # the sampled columns as rows of scales of their own
    _check(a, sa, b[pick], sb[pick // 128], y[:, pick], out, 1, f"{m}x{n}x{k}")


@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_few_rows_by_expert(out):
    import torch
    groups, n, k, ends = 24, 1100, 2816, [1] * 5 + [9, 30] + [31] * 10 + [33, 40, 41, 60, 61, 64, 64]
    tokens = 66
    a, sa = _codes(1, tokens, k)
    b, sb = _codes(2, groups * n, k, scale_rows=groups * 9)
    b, sb = b.view(groups, n, k), sb.view(groups, 9, k // 128)
    y = H.grouped_matmul_fp8(a, sa, b, sb, torch.tensor(ends, dtype=torch.int32, device="cuda"),
                             dtype=_torch_type(out))
    low = 0
    for g, high in enumerate(ends):
        if high > low:
            _check(a[low:high], sa[low:high], b[g], sb[g], y[low:high], out, 128, f"group {g}")
        low = high
    assert (y[low:] == 0).all()


# outputs of 128 MiB and more are stored with the streaming policy
LARGE = pytest.mark.parametrize("out", ["bf16", "fp16", "fp32"])


@LARGE
@pytest.mark.parametrize("k", [128, 384, 200])
def test_large_outputs_by_expert(k, out):
    import torch
    n = 8203 if k == 200 else 8200
    ends, tokens = [0, 1000, 1000, 1003, 4600, 8300], 8320
    groups, tiles = len(ends), -(-n // 128)
    a, sa = _codes(3, tokens, k)
    b, sb = _codes(4, groups * n, k, scale_rows=groups * tiles)
    pitch = b.stride(0)
    b = b.as_strided((groups, n, k), (n * pitch, pitch, 1))
    sb = sb.view(groups, tiles, -1)
    buf = torch.full((tokens * n + 64,), 5.0, dtype=_torch_type(out), device="cuda")
    assert buf.numel() * buf.element_size() >= 1 << 27
    y = H.grouped_matmul_fp8(a, sa, b, sb, torch.tensor(ends, dtype=torch.int32, device="cuda"),
                             out=buf[:tokens * n].view(tokens, n))
    assert (buf[tokens * n:] == 5).all()
    low = 0
    for g, high in enumerate(ends):
        if high > low:
            pick = torch.from_numpy(low + _some(high - low, 61)).cuda()
            _check(a[pick], sa[pick], b[g], sb[g], y[pick], out, 128, f"group {g}")
        low = high
    assert (y[low:] == 0).all()


@LARGE
def test_large_gradients(out):
    import torch
    groups, n, k = 6, 3400, 3401
    if out == "fp32":
        n = 1700
    ends, tokens = [200, 200, 328, 457, 457, 900], 1000
    assert groups * n * k * (4 if out == "fp32" else 2) >= 1 << 27
    d = _input((tokens, n), 0, "bf16", 5)
    x = _input((tokens, k), 0, "fp16", 6)
    at = torch.tensor(ends, dtype=torch.int32, device="cuda")
    qd, sd = H.quantize_fp8_columns(d, at)
    qx, sx = H.quantize_fp8_columns(x, at)
    gap = 40  # between the matrices, to be left alone
    buf = torch.full((groups * (n * k + gap),), 5.0, dtype=_torch_type(out), device="cuda")
    g = H.grouped_weight_gradient_fp8(
        qd, sd, qx, sx, at, out=buf.as_strided((groups, n, k), (n * k + gap, k, 1)))
    assert (buf.view(groups, -1)[:, n * k:] == 5).all()
    pick = torch.from_numpy(_some(n, 61)).cuda()
    for e, low, count, place, blocks in R.padded_places(ends, tokens)[0]:
        if count == 0:
            assert (g[e] == 0).all()
            continue
        cut, cuts = slice(place, place + blocks * 128), slice(place // 128, place // 128 + blocks)
        _check(qd[pick, cut], sd[pick, cuts], qx[:, cut], sx[:, cuts], g[e][pick], out, 1, f"group {e}")
