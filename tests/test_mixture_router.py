"""A router has a column for each expert of the mixture: other logits are refused before any work."""
from __future__ import annotations

import pytest
import torch

from paper_2412_08832_amd import experts as E


@pytest.mark.parametrize("columns", [3, 5, 64])
def test_columns_and_experts(columns):
    x, logits = torch.zeros((6, 128)).half(), torch.zeros((6, columns))
    w = torch.zeros((4, 16, 128)).half()
    with pytest.raises(ValueError, match="4 experts"):
        E.mixture(x, logits, w, 2)
    q = E.Weights(w, torch.zeros((4, 1, 1)), None, None, 128)
    with pytest.raises(ValueError, match="4 experts"):
        E.serve_mixture(x, logits, q, 2)


@pytest.mark.parametrize("shape", [(4,), (1, 6, 4)])
def test_dimensions(shape):
    with pytest.raises(ValueError, match="4 experts"):
        E.mixture(torch.zeros((6, 128)).half(), torch.zeros(shape), torch.zeros((4, 16, 128)).half(), 2)
