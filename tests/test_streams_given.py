"""A stream given to a wrapper becomes torch's current one before anything is allocated; without a GPU, by stand-ins
for torch's streams and tensors."""
from __future__ import annotations

import contextlib
import inspect
import types

import pytest

from paper_2412_08832_amd import hadacore as H

WRAPPERS = [H.transform, H.transform_fp8, H.transform_int8, H.transform_fp8_blocks, H.quantize_fp8_columns,
            H.quantize_fp8_tiles, H.matmul_fp8, H.grouped_matmul_fp8, H.grouped_weight_gradient_fp8, H.route_tokens,
            H.route_tokens_gradient, H.group_tokens, H.dispatch_rows, H.combine_rows, H.combine_rows_gradient,
            H.adapt_rows, H.adapter_gradient]


def test_every_wrapper_with_a_stream_is_listed():
    found = {f for n, f in vars(H).items() if inspect.isfunction(f) and not n.startswith(("_", "had"))
             and "stream" in inspect.signature(f).parameters}
    assert found == set(WRAPPERS)


@pytest.mark.parametrize("wrapper", WRAPPERS)
def test_wrappers_enter_the_stream_first(wrapper, monkeypatch):
    """Nothing is asked of the tensors before: any attribute of these raises."""
    stream, calls = object(), []
    monkeypatch.setattr(H, "_on_stream", lambda s, x, call: calls.append((s, x)) or "entered")
    needed = [p for p in inspect.signature(wrapper).parameters.values() if p.default is p.empty]
    tensors = [object() for _ in needed]
    assert wrapper(*tensors, stream=stream) == "entered"
    assert calls[0][0] is stream and calls[0][1] in tensors


class _Stream:
    def __init__(self, cuda_stream, device_index=0):
        self.cuda_stream, self.device_index = cuda_stream, device_index


class _External(_Stream):
    def __init__(self, cuda_stream, device):
        super().__init__(cuda_stream, device)


class _Tensor:
    def __init__(self, device=0):
        self.device, self.marks = device, []

    def get_device(self):
        return self.device

    def record_stream(self, stream):
        self.marks.append(stream.cuda_stream)


@pytest.fixture
def streams(monkeypatch):
    """The handles of torch's current stream, the last one's."""
    current = [5]

    @contextlib.contextmanager
    def stream(s):
        current.append(s.cuda_stream)
        yield
        current.pop()
    cuda = types.SimpleNamespace(Stream=_Stream, ExternalStream=_External, stream=stream,
                                 current_stream=lambda device: _Stream(current[-1], device),
                                 default_stream=lambda device: _Stream(0, device))
    monkeypatch.setattr(H, "_torch", types.SimpleNamespace(cuda=cuda, Tensor=_Tensor))
    return current


@pytest.mark.parametrize("given,handle", [(_Stream(7), 7), (7, 7), (0, 0)])
def test_work_and_memory_are_of_the_stream(streams, given, handle):
    out = (_Tensor(), True, _Tensor())

    def call(entered):
        assert streams[-1] == handle and entered.cuda_stream == handle and entered.stream.cuda_stream == handle
        return out
    assert H._on_stream(given, _Tensor(), call) is out and streams == [5]
    assert out[0].marks == out[2].marks == [5]  # the caller's stream uses them next


@pytest.mark.parametrize("given", [_Stream(5), 5])
def test_the_current_stream_stays(streams, given):
    out = _Tensor()

    def call(entered):
        assert streams == [5] and entered.cuda_stream == 5
        return out
    assert H._on_stream(given, _Tensor(), call) is out and out.marks == []


def test_refusals(streams):
    with pytest.raises(ValueError, match="device 1"):
        H._on_stream(_Stream(7, 1), _Tensor(), lambda s: None)
    # the call refuses a tensor of no GPU by itself
    assert H._on_stream(_Stream(7), _Tensor(-1), lambda s: s) is None and streams == [5]
