"""Ends of groups that go down, many of them: the work of a call stays within what valid ends
of as many rows and groups can ask for, and what lies around the output is left alone."""
from __future__ import annotations

import pytest

from paper_2412_08832_amd import hadacore as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    H.library()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("variant", ["auto", "tiles-64", "tiles-64x128", "tiles-128", "tiles-256"])
@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("groups", [2, 65, 2000])
def test_ends_that_go_up_and_down(groups, out, variant, monkeypatch):
    import torch
    if variant == "auto":
        monkeypatch.delenv("HADACORE_VARIANT", raising=False)
    else:
        monkeypatch.setenv("HADACORE_VARIANT", variant)
    m, n, k = 1500, 300, 256
    gen = torch.Generator(device="cuda").manual_seed(groups)

    def codes(rows):
        return (torch.randn((rows, k), generator=gen, device="cuda") * 50).to(torch.float8_e4m3fn)

    a, sa = codes(m), torch.rand((m, 2), generator=gen, device="cuda")
    b, sb = codes(n), torch.rand((3, 2), generator=gen, device="cuda")
    ends = torch.tensor([m, 0] * groups, dtype=torch.int32, device="cuda")[:groups]
    buf = torch.full((m + 2, n), 3.0, dtype=getattr(torch, out), device="cuda")
    H.grouped_matmul_fp8(a, sa, b[None].expand(groups, -1, -1), sb[None].expand(groups, -1, -1), ends,
                         out=buf[1:-1])
    torch.cuda.synchronize()
    assert (buf[0] == 3).all() and (buf[-1] == 3).all()
    # the same shapes with valid ends afterwards: one group has all rows
    ends = torch.full((groups,), m, dtype=torch.int32, device="cuda")
    H.grouped_matmul_fp8(a, sa, b[None].expand(groups, -1, -1), sb[None].expand(groups, -1, -1), ends,
                         out=buf[1:-1])
    want = a.double() * sa.double().repeat_interleave(128, 1)
    want = want @ (b.double() * sb.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)).t()
    assert float((buf[1:-1].double() - want).norm() / want.norm()) <= 2.5e-3
    assert (buf[0] == 3).all() and (buf[-1] == 3).all()
