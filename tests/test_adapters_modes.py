"""Which derivatives the adapters' layer has: reverse mode only; on the CPU, with the calls replaced."""
from __future__ import annotations

import pytest
import torch
from torch.autograd import forward_ad

import tokens_reference as R
from paper_2412_08832_amd import adapters as A
from paper_2412_08832_amd import hadacore as H


def _adapt_rows(x, down, up, ends=None, slots=None, y=None, scales=None, dtype=None, hidden=False):
    out, _, h, _ = R.adapt(x, down, up, ends, slots, y, scales, 0, 0)
    return (out, h) if hidden else out


@pytest.fixture(autouse=True)
def _plain_calls(monkeypatch):
    monkeypatch.setattr(H, "adapt_rows", _adapt_rows)


def _values():
    gen = torch.Generator().manual_seed(0)
    shapes = {"y": (5, 3), "x": (5, 4), "down": (1, 2, 4), "up": (1, 2, 3)}
    return {n: torch.randn(s, generator=gen, dtype=torch.float64) for n, s in shapes.items()}


@pytest.mark.parametrize("dual", ["y", "x", "down", "up"])
def test_tangents_are_refused(dual):
    values = _values()
    with forward_ad.dual_level():
        values[dual] = forward_ad.make_dual(values[dual], torch.ones_like(values[dual]))
        with pytest.raises(NotImplementedError, match="jvp"):
            A.adapt(**values)


def test_without_tangents_the_level_changes_nothing():
    values = _values()
    want = A.adapt(**values)
    with forward_ad.dual_level():
        assert torch.equal(A.adapt(**values), want)


def test_scales_of_a_module_without_gradients():
    """Scales kept as a parameter serve where no gradient is made; where one would be, they are refused."""
    values, scales = _values(), torch.nn.Parameter(torch.full((1,), 2.0, dtype=torch.float64))
    with torch.no_grad():
        assert torch.equal(A.adapt(**values, scales=scales), A.adapt(**values, scales=scales.detach()))
    with pytest.raises(ValueError, match="scales"):
        A.adapt(**values, scales=scales)
