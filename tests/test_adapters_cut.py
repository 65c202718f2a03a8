"""The adapters' calls are cut within the limits that the kernels and their comments state, on the CPU."""
from __future__ import annotations

import itertools

from adapters_cut import cuts


def test_room_and_units():
    """Every rank, few to many tokens and columns: the second product's LDS, by the pitch of the version that is
    launched, is at most a third of a CU's 160 KiB, and its units are whole tiles."""
    calls = list(itertools.product((1, 17, 512, 1025, 3000, 6000, 8192, 16384, 30000, 70001, (1 << 27) - 1), (512, 4096),
                                   (1, 300, 4096, 1 << 22), range(1, 257), (0, 1, 2, 7, 4095)))
    most, rows = cuts(calls)
    assert 3 * most <= 160 * 1024 and len(rows) == len(calls)
    units = {}
    for (m, k, n, rank, groups), c in zip(calls, rows):
        depth = next(d for d in (32, 64, 128, 256) if rank <= d)
        assert c.unit in (16, 32, 64, 128) and c.room == c.unit * (3 * (depth + 8) * 2 + 8) <= most
        assert 1 <= c.splits <= 16 and c.tiles in (1, 4) and c.ranks == (1 if rank <= 16 else 2 if rank <= 32 else 4)
        assert not c.fused or (rank <= 16 and c.splits == 1)
        units.setdefault(depth, set()).add(c.unit)
    assert units == {32: {16, 32, 64, 128}, 64: {16, 32, 64}, 128: {16, 32, 64}, 256: {16, 32}}
