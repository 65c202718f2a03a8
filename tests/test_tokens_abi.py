"""Refusals of routing, exchange and adapters, and their size functions, on the CPU."""
from __future__ import annotations

import itertools
from pathlib import Path

import pytest

from paper_2412_08832_amd import hadacore as H

# as in test_abi: no call here has arguments that validation would accept
cpu_only = pytest.mark.skipif(Path("/dev/kfd").exists(),
                              reason="fake-pointer validation tests run only without a GPU")
X, A, B, C, D, E, F, G, W = (1 << k for k in range(33, 42))  # fake device addresses, far apart
BIG = 1 << 30


def _status(entry, args, **change):
    values = dict(args)
    values.update(change)
    return H.STATUS_NAMES[entry(*values.values(), check=False)]


ROUTE = dict(logits=X, stride=40, dtype=H.FP32, valid=0, m=500, experts=40, k=2, renormalize=1, chosen=A,
             weights=B, counts=C, loss=D, slopes=E, workspace=W, bytes=1 << 20, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(experts=0), "INVALID_SIZE"), (dict(experts=1025, stride=1025), "INVALID_SIZE"),
    (dict(k=0), "INVALID_SIZE"), (dict(k=41), "INVALID_SIZE"), (dict(k=33), "INVALID_SIZE"),
    (dict(dtype=3), "INVALID_DTYPE"), (dict(m=BIG), "TOO_LARGE"), (dict(m=BIG // 2), "TOO_LARGE"),
    (dict(stride=39), "INVALID_STRIDE"), (dict(stride=(1 << 26) + 1), "INVALID_STRIDE"),
    (dict(m=1 << 20, stride=1 << 26), "TOO_LARGE"), (dict(logits=0), "INVALID_VALUE"),
    (dict(logits=X + 2), "MISALIGNED"), (dict(dtype=H.BF16, logits=X + 1), "MISALIGNED"),
    (dict(chosen=0), "INVALID_VALUE"), (dict(weights=0), "INVALID_VALUE"), (dict(counts=0), "INVALID_VALUE"),
    (dict(loss=0), "INVALID_VALUE"), (dict(slopes=0), "INVALID_VALUE"), (dict(slopes=E + 2), "MISALIGNED"),
    (dict(m=2, counts=0), "INVALID_VALUE"), (dict(bytes=8), "WORKSPACE"), (dict(workspace=0), "WORKSPACE"),
    (dict(workspace=W + 8), "MISALIGNED"), (dict(weights=A + 4), "OVERLAP"), (dict(chosen=X + 80), "OVERLAP"),
    (dict(valid=A + 1), "OVERLAP"), (dict(workspace=C - 16), "OVERLAP"), (dict(loss=E + 4), "OVERLAP")])
def test_route_refusals(change, status):
    assert _status(H.hadacore_route, ROUTE, **change) == status


ROUTE_GRADIENT = dict(logits=X, stride=40, dtype=H.BF16, chosen=A, weights=B, slopes=E, dweights=F, dloss=D, m=50,
                      experts=40, k=2, renormalize=1, out=G, out_stride=40, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(k=0), "INVALID_SIZE"), (dict(dtype=-1), "INVALID_DTYPE"),
    (dict(stride=39), "INVALID_STRIDE"), (dict(out_stride=39), "INVALID_STRIDE"), (dict(out=0), "INVALID_VALUE"),
    (dict(chosen=0), "INVALID_VALUE"), (dict(weights=0), "INVALID_VALUE"), (dict(slopes=0), "INVALID_VALUE"),
    (dict(dweights=F + 2), "MISALIGNED"), (dict(out=G + 1), "MISALIGNED"), (dict(out=X), "OVERLAP"),
    (dict(out=F + 4), "OVERLAP"), (dict(dloss=G + 80), "OVERLAP"), (dict(m=0, out=0, logits=0, chosen=0), "SUCCESS")])
def test_route_gradient_refusals(change, status):
    assert _status(H.hadacore_route_gradient, ROUTE_GRADIENT, **change) == status


GROUP = dict(ids=X, slots=100000, groups=30, ends=A, rows=B, order=C, workspace=W, bytes=1 << 20, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(slots=-1), "INVALID_VALUE"), (dict(groups=-1), "INVALID_VALUE"), (dict(groups=4096), "INVALID_SIZE"),
    (dict(slots=BIG), "TOO_LARGE"), (dict(ids=0), "INVALID_VALUE"), (dict(ends=0), "INVALID_VALUE"),
    (dict(rows=0), "INVALID_VALUE"), (dict(order=0), "INVALID_VALUE"), (dict(ids=X + 1), "MISALIGNED"),
    (dict(order=C + 2), "MISALIGNED"), (dict(workspace=0), "WORKSPACE"), (dict(bytes=4), "WORKSPACE"),
    (dict(workspace=W + 2), "MISALIGNED"), (dict(rows=X + 4), "OVERLAP"), (dict(order=B + 4), "OVERLAP"),
    (dict(workspace=C + 64), "OVERLAP"), (dict(slots=0, groups=0, ids=0, ends=0, rows=0, order=0), "SUCCESS")])
def test_group_refusals(change, status):
    assert _status(H.hadacore_group_tokens, GROUP, **change) == status


DISPATCH = dict(x=X, stride=100, size=2, rows=A, ends=B, groups=4, out=C, out_stride=100, m=50, k=2, width=100,
                stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(k=0), "INVALID_VALUE"), (dict(width=-1), "INVALID_VALUE"),
    (dict(groups=-1), "INVALID_VALUE"), (dict(size=3), "INVALID_DTYPE"), (dict(size=8), "INVALID_DTYPE"),
    (dict(stride=99), "INVALID_STRIDE"), (dict(out_stride=99), "INVALID_STRIDE"), (dict(x=0), "INVALID_VALUE"),
    (dict(rows=0), "INVALID_VALUE"), (dict(ends=0), "INVALID_VALUE"), (dict(x=X + 1), "MISALIGNED"),
    (dict(ends=B + 2), "MISALIGNED"), (dict(out=X + 200), "OVERLAP"), (dict(out=A), "OVERLAP"),
    (dict(m=BIG), "TOO_LARGE"), (dict(m=1 << 25, width=4096, stride=4096, out_stride=4096, out=0), "INVALID_VALUE"),
    (dict(m=1 << 26, width=4096, stride=4096, out_stride=4096), "OVERLAP"), (dict(m=0), "SUCCESS"),
    (dict(width=0), "SUCCESS")])
def test_dispatch_refusals(change, status):
    assert _status(H.hadacore_dispatch_rows, DISPATCH, **change) == status


COMBINE = dict(y=X, stride=100, places=100, dtype=H.FP16, rows=A, weights=B, out=C, out_stride=100, m=50, k=2,
               width=100, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(places=-1), "INVALID_VALUE"), (dict(m=-1), "INVALID_VALUE"), (dict(dtype=4), "INVALID_DTYPE"),
    (dict(k=-1), "INVALID_VALUE"), (dict(places=BIG), "TOO_LARGE"), (dict(stride=99), "INVALID_STRIDE"),
    (dict(y=0), "INVALID_VALUE"), (dict(rows=0), "INVALID_VALUE"), (dict(weights=B + 2), "MISALIGNED"),
    (dict(dtype=H.FP32, out=C + 2), "MISALIGNED"), (dict(out=X), "OVERLAP"), (dict(out=B + 4), "OVERLAP"),
    (dict(m=0), "SUCCESS"), (dict(width=0), "SUCCESS")])
def test_combine_refusals(change, status):
    assert _status(H.hadacore_combine_rows, COMBINE, **change) == status


COMBINE_GRADIENT = dict(dout=X, stride=100, y=A, y_stride=100, dtype=H.BF16, rows=B, ends=C, groups=4, weights=D,
                        dy=E, dy_stride=100, dweights=F, m=50, k=2, width=100, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(dtype=9), "INVALID_DTYPE"), (dict(stride=99), "INVALID_STRIDE"),
    (dict(y_stride=99), "INVALID_STRIDE"), (dict(dy_stride=99), "INVALID_STRIDE"), (dict(y=0), "INVALID_VALUE"),
    (dict(ends=0), "INVALID_VALUE"), (dict(dweights=F + 1), "MISALIGNED"), (dict(dy=E + 1), "MISALIGNED"),
    (dict(dy=A), "OVERLAP"), (dict(dweights=D), "OVERLAP"), (dict(dweights=E + 40), "OVERLAP"),
    (dict(m=1 << 24, k=1), "TOO_LARGE"), (dict(dy=0, dweights=0), "SUCCESS"), (dict(m=0), "SUCCESS")])
def test_combine_gradient_refusals(change, status):
    assert _status(H.hadacore_combine_gradient, COMBINE_GRADIENT, **change) == status


ADAPT = dict(x=X, x_stride=512, down=A, down_stride=512, down_batch=40 * 512, up=B, up_stride=300, up_batch=40 * 300,
             scales=C, ends=D, slots=E, groups=3, y=F, y_stride=300, out=G, out_stride=300, dtype=H.BF16,
             out_dtype=H.FP32, hidden=0, hidden_stride=48, m=3000, k=512, n=300, rank=40, workspace=W,
             bytes=1 << 30, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(k=-1), "INVALID_VALUE"), (dict(n=-1), "INVALID_VALUE"),
    (dict(groups=-1), "INVALID_VALUE"), (dict(rank=0), "INVALID_SIZE"), (dict(rank=257), "INVALID_SIZE"),
    (dict(groups=4096), "TOO_LARGE"), (dict(m=1 << 27), "TOO_LARGE"),
    (dict(k=(1 << 22) + 1, x_stride=1 << 23, down_stride=1 << 23), "TOO_LARGE"),
    (dict(dtype=H.FP32), "INVALID_DTYPE"), (dict(out_dtype=H.FP16), "INVALID_DTYPE"), (dict(dtype=5), "INVALID_DTYPE"),
    (dict(ends=0), "INVALID_VALUE"), (dict(ends=D + 2), "MISALIGNED"), (dict(slots=E + 1), "MISALIGNED"),
    (dict(scales=C + 2), "MISALIGNED"), (dict(x_stride=511), "INVALID_STRIDE"), (dict(down_stride=511), "INVALID_STRIDE"),
    (dict(up_stride=299), "INVALID_STRIDE"), (dict(y_stride=299), "INVALID_STRIDE"), (dict(out_stride=299), "INVALID_STRIDE"),
    (dict(down_batch=-1), "INVALID_STRIDE"), (dict(up_batch=1 << 42), "TOO_LARGE"), (dict(x=0), "INVALID_VALUE"),
    (dict(up=0), "INVALID_VALUE"), (dict(out=0), "INVALID_VALUE"), (dict(x=X + 1), "MISALIGNED"),
    (dict(out=G + 2), "MISALIGNED"), (dict(hidden=1 << 44, hidden_stride=47), "INVALID_STRIDE"),
    (dict(hidden=1 << 44, hidden_stride=50), "INVALID_STRIDE"), (dict(hidden=(1 << 44) + 4), "MISALIGNED"),
    (dict(workspace=0), "WORKSPACE"), (dict(bytes=100), "WORKSPACE"), (dict(workspace=W + 4), "MISALIGNED"),
    (dict(out=X), "OVERLAP"), (dict(out=B + 4), "OVERLAP"), (dict(out=F + 1200), "OVERLAP"),
    (dict(out=F, out_stride=304), "OVERLAP"), (dict(hidden=G), "OVERLAP"), (dict(workspace=F), "OVERLAP"),
    (dict(m=(1 << 27) - 1, n=1 << 15, x=1 << 50, down=1 << 58, up=1 << 59, y=1 << 51, out=1 << 52, workspace=1 << 53,
          scales=1 << 54, ends=1 << 55, slots=1 << 56, up_stride=1 << 15, up_batch=40 << 15, y_stride=1 << 15, out_stride=1 << 15,
          x_stride=512, bytes=1 << 50), "TOO_LARGE"),
    (dict(m=0, x=0, out=0), "SUCCESS")])
def test_adapters_refusals(change, status):
    assert _status(H.hadacore_adapters, ADAPT, **change) == status


GRADIENT = dict(hidden=X, hidden_stride=48, x=A, x_stride=512, dtype=H.FP16, scales=C, ends=D, slots=E, groups=3, out=F,
                out_stride=512, out_batch=512 * 40, out_dtype=H.FP32, m=9000, width=512, rank=40, workspace=W,
                bytes=1 << 30, stream=0)


@cpu_only
@pytest.mark.parametrize("change,status", [
    (dict(m=-1), "INVALID_VALUE"), (dict(rank=0), "INVALID_SIZE"), (dict(dtype=H.FP32), "INVALID_DTYPE"),
    (dict(out_dtype=H.BF16), "INVALID_DTYPE"), (dict(hidden_stride=39), "INVALID_STRIDE"),
    (dict(x_stride=511), "INVALID_STRIDE"), (dict(out_stride=511), "INVALID_STRIDE"),
    (dict(out_batch=512 * 39), "INVALID_STRIDE"), (dict(ends=0), "INVALID_VALUE"), (dict(hidden=0), "INVALID_VALUE"),
    (dict(x=0), "INVALID_VALUE"), (dict(out=0), "INVALID_VALUE"), (dict(hidden=X + 2), "MISALIGNED"),
    (dict(out=F + 2), "MISALIGNED"), (dict(workspace=0), "WORKSPACE"), (dict(workspace=W + 2), "MISALIGNED"),
    (dict(out=A), "OVERLAP"), (dict(out=X + 16), "OVERLAP"), (dict(workspace=F), "OVERLAP"),
    (dict(groups=0, ends=0), "SUCCESS"), (dict(width=0, x=0, out=0), "SUCCESS")])
def test_adapter_gradient_refusals(change, status):
    assert _status(H.hadacore_adapter_gradient, GRADIENT, **change) == status


def test_sizes_of_workspaces():
    """Every size function over small, large and impossible arguments: a whole number of bytes, 0 for what
    the call rejects."""
    values = [-(1 << 62), -1, 0, 1, 2, 17, 300, 4096, 1 << 22, (1 << 22) + 1, (1 << 27) - 1, BIG, 1 << 62]
    for a, b in itertools.product(values, repeat=2):
        assert H.hadacore_route_workspace_size(a, b) >= 0 and H.hadacore_group_workspace_size(a, b) >= 0
    for m, k, n in itertools.product(values, repeat=3):
        for rank, groups in itertools.product((0, 1, 40, 256, 257), (-1, 0, 1, 9, 4095, 4096)):
            assert H.hadacore_adapters_workspace_size(m, k, n, rank, groups) >= 0
            assert H.hadacore_adapter_gradient_workspace_size(m, n, rank, groups) >= 0
    assert H.hadacore_route_workspace_size(BIG, 8) == H.hadacore_route_workspace_size(8, 1025) == 0
    assert H.hadacore_group_workspace_size(100, 4096) == H.hadacore_group_workspace_size(BIG, 4) == 0
    assert H.hadacore_adapters_workspace_size(1 << 27, 64, 64, 16, 1) == 0
    assert H.hadacore_adapters_workspace_size(5000, 512, 512, 257, 1) == 0
