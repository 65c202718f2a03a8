"""How the library cuts the adapters' calls: its own rules, csrc/adapters_cut.h, compiled for the host."""
from __future__ import annotations

import shutil
import subprocess
import tempfile
from pathlib import Path
from typing import NamedTuple

HERE = Path(__file__).resolve().parent
CSRC = HERE.parent / "paper_2412_08832_amd" / "csrc"


class Cut(NamedTuple):
    fused: int   # both products in one launch
    ranks: int   # tiles of 16 ranks in a workgroup of the first product
    tiles: int   # tiles of 16 tokens there
    splits: int  # shares of its sums
    unit: int    # tokens of a workgroup of the second product
    room: int    # its LDS in bytes


def cuts(calls):
    """(the most LDS, [Cut of each (m, k, n, rank, groups)])."""
    cxx = next(c for c in ("g++", "c++", "clang++", "/opt/rocm/llvm/bin/clang++") if shutil.which(c))
    with tempfile.TemporaryDirectory() as where:
        exe = Path(where) / "cut"
        subprocess.run([cxx, "-std=c++17", "-O1", f"-I{CSRC}", str(HERE / "native" / "adapters_cut_check.cpp"), "-o",
                        str(exe)], check=True, timeout=100)
        lines = "\n".join(" ".join(map(str, c)) for c in calls)
        out = subprocess.run([str(exe)], input=lines, capture_output=True, text=True, check=True, timeout=100).stdout
    most, *rows = out.splitlines()
    return int(most), [Cut(*map(int, r.split())) for r in rows]
