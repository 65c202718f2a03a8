"""A stream given to a wrapper: its outputs and workspace are of that stream's memory, on the GPU's allocator."""
from __future__ import annotations

import pytest
import torch

from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


def _owner(t):
    """The stream of whose memory a tensor is."""
    at = t.data_ptr()
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= at < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("not of torch's memory")


def _calls():
    """Every wrapper, as calls of a stream, and what each gives on the current one."""
    gen = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    m, k, n, e = 9000, 256, 128, 5
    x, w, dy, logits = normal(m, k).bfloat16(), normal(e, n, k).bfloat16(), normal(m, n).bfloat16(), normal(m, e)
    a, sa = H.transform_fp8_blocks(x, 1)
    b, sb = H.quantize_fp8_tiles(w)
    ids = torch.randint(-1, e, (m,), generator=gen, device="cuda").int()
    ends, rows, slots = H.group_tokens(ids, e)
    qx, sqx = H.quantize_fp8_columns(x, ends)
    qd, sqd = H.quantize_fp8_columns(dy, ends)
    down, up = normal(e, 40, k).bfloat16(), normal(e, 40, n).bfloat16()
    weights, h = torch.rand((m,), generator=gen, device="cuda"), normal(m, 40)
    routes = H.route_tokens(logits, 2)
    dw = normal(m, 2)
    wide = normal(4, 1 << 17).bfloat16()
    return [
        lambda s: H.transform(x, stream=s), lambda s: H.transform(wide, stream=s),
        lambda s: H.transform_fp8(x, stream=s), lambda s: H.transform_int8(x, stream=s),
        lambda s: H.transform_fp8_blocks(x, stream=s), lambda s: H.quantize_fp8_columns(x, ends, stream=s),
        lambda s: H.quantize_fp8_tiles(w, transposed=True, stream=s), lambda s: H.matmul_fp8(a, sa, b[0], sb[0], stream=s),
        lambda s: H.grouped_matmul_fp8(a, sa, b, sb, ends, stream=s),
        lambda s: H.grouped_weight_gradient_fp8(qd, sqd, qx, sqx, ends, stream=s),
        lambda s: H.route_tokens(logits, 2, stream=s), lambda s: H.route_tokens_gradient(logits, routes, dw, stream=s),
        lambda s: H.group_tokens(ids, e, stream=s), lambda s: H.dispatch_rows(x, rows, ends, stream=s),
        lambda s: H.combine_rows(x, rows, weights, stream=s),
        lambda s: H.combine_rows_gradient(x, x, rows, ends, weights, stream=s),
        lambda s: H.adapt_rows(x, down, up, ends, slots, hidden=True, stream=s),
        lambda s: H.adapter_gradient(h, x, ends, slots, stream=s)]


def _tensors(result):
    return [t for t in (result if isinstance(result, tuple) else (result,)) if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("form", ["stream", "handle", "default"])
def test_outputs_are_of_the_streams_memory(form, monkeypatch):
    calls = _calls()
    want = [_tensors(call(None)) for call in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    here = torch.cuda.Stream() if form == "default" else torch.cuda.current_stream()
    given = {"stream": side, "handle": side.cuda_stream, "default": 0}[form]
    owner = 0 if form == "default" else side.cuda_stream
    marks, scratch, mark, words = [], [], torch.Tensor.record_stream, H._scratch
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: marks.append((t.data_ptr(), s.cuda_stream)) or mark(t, s),
                        raising=False)

    def spy(*args):
        t, address = words(*args)
        if t is not None:
            scratch.append(_owner(t))
        return t, address
    monkeypatch.setattr(H, "_scratch", spy)
    with torch.cuda.stream(here):
        for i, (call, ref) in enumerate(zip(calls, want)):
            got = _tensors(call(given))
            assert torch.cuda.current_stream() == here
            for t in got:
                assert t.numel() > 0 and _owner(t) == owner, i
                assert (t.data_ptr(), here.cuda_stream) in marks, i
            torch.cuda.synchronize()
            for t, r in zip(got, ref):
                if i == 5:  # places behind the last group are not written
                    continue
                if t.is_floating_point():  # rows of h behind the last end are not written
                    same = (t == r) | (t.isnan() & r.isnan())
                    assert bool(same.all()) or (i == 16 and t is got[1]), i
                else:
                    assert torch.equal(t, r), i
    # routing, grouping, the adapters and their gradient took a workspace each
    assert len(scratch) == 4 and set(scratch) == {owner}


def test_a_freed_block_of_the_current_stream_is_not_taken():
    """What the caller has just freed there may still be in use by its work; the other stream's own is taken."""
    x = torch.randn((1 << 14, 256), device="cuda").bfloat16()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        mine = torch.empty_like(x)
    theirs = torch.empty_like(x)
    wanted, other = mine.data_ptr(), theirs.data_ptr()
    del mine, theirs
    got = H.transform(x, stream=side)
    assert got.data_ptr() == wanted and got.data_ptr() != other
    torch.cuda.synchronize()
    assert torch.equal(got, H.transform(x))
