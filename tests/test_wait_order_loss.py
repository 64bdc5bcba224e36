"""The order of loads that the counted waits of the head loss's tiles rely on, read
from the assembly that the compiler makes of them (CPU only).

`s_waitcnt vmcnt(N)` leaves the N newest vector-memory accesses in flight.  In the
tiles of 64 rows the next stage is in LDS behind it if the N = 5 loads of the
stage after it are younger: each stage's loads lie together between two
scheduling barriers, all of them.  The taller tiles wait for every load.
"""
from __future__ import annotations

import os
import re
import subprocess

import pytest

from paper_2608_02703_amd import build


def _kernels(tmp_path):
    """Each kernel as a string: L a load to LDS, r another load, w<N>; a wait, B a
    workgroup's barrier, | a scheduling barrier, : a label, > a branch."""
    try:
        hipcc = build._hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = str(tmp_path / "k_ce_tile.s")
    subprocess.run([hipcc, *build.HIP_FLAGS, f"-I{build.INCLUDE}", "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, "k_ce_tile.hip"), "-o", out], check=True, capture_output=True, text=True)
    kernels, name = {}, None
    with open(out) as f:
        for line in f:
            s = line.strip()
            m = re.match(r"(_ZN\w+k_ce_tile\w+):", line)
            if m:
                name = m.group(1)
                kernels[name] = ""
            elif s.startswith(".section"):
                name = None
            elif name is None:
                continue
            elif s.startswith("; sched_barrier mask(0x00000000)"):
                kernels[name] += "|"
            elif re.match(r"(buffer|global|flat)_load", s):
                kernels[name] += "L" if re.search(r"\blds\b|_lds_", s) else "r"
            elif re.match(r"s_waitcnt vmcnt\(\d+\)", s):
                kernels[name] += f"w{re.search(r'[0-9]+', s).group()};"
            elif s == "s_barrier":
                kernels[name] += "B"
            elif re.match(r"\.LBB", s):
                kernels[name] += ":"
            elif re.match(r"s_c?branch", s):
                kernels[name] += ">"
    return kernels


def test_tiles(tmp_path):
    kernels = _kernels(tmp_path)
    assert len(kernels) == 11
    for name, text in kernels.items():
        _, ti = (int(v) for v in re.findall(r"Li(\d+)", name)[:2])
        loads = ti * 128 // 1024 // 8 + 256 * 128 // 1024 // 8   # of a wave and stage
        ahead = loads if ti == 64 else 0
        assert re.search(rf"\|w{ahead};B\|{'L' * loads}\|", text), f"{name}: {text}"
        assert set(re.findall(r"w(\d+);B", text)) <= {"0", str(ahead)}
