"""The order of loads that the INT8 products' counted waits rely on, read from
the assembly that the compiler makes of them (CPU only).

`s_waitcnt vmcnt(N)` leaves the N newest vector-memory accesses in flight.  The
stage it waits for is in LDS behind it if N younger loads exist, and if no load
of that stage was moved behind one of a later stage: each stage's loads have to
lie between two scheduling barriers (or in blocks of their own), all N of them.
"""
from __future__ import annotations

import os
import re
import subprocess

import pytest

from paper_2608_02703_amd import build


def _kernels(tu, tmp_path):
    """Each kernel as a string: L a load to LDS, r another load, w<N>; a wait, B a
    workgroup's barrier, | a scheduling barrier, : a label, > a branch."""
    try:
        hipcc = build._hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    out = str(tmp_path / (tu + ".s"))
    subprocess.run([hipcc, *build.HIP_FLAGS, f"-I{build.INCLUDE}", "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, tu), "-o", out], check=True, capture_output=True, text=True)
    kernels, name = {}, None
    with open(out) as f:
        for line in f:
            s = line.strip()
            m = re.match(r"(_ZN\w+k_i8_\w+):", line)
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


def _arguments(name):
    return [int(v) for v in re.findall(r"ELi(\d+)", name)]


def test_shares_of_k(tmp_path):
    kernels = _kernels("k_i8_split.hip", tmp_path)
    assert len(kernels) == 6
    for name, text in kernels.items():
        n = 4 * _arguments(name)[0]   # loads of a stage: two 16-row operands of 128 bytes, 1 KB each
        # the loop: the wait, a scheduling barrier, the stage after next, another
        assert re.search(rf"w{n};[:>]*w0;[:>]*\|[:>]*{'L' * n}[:>]*\|", text), f"{name}: {text}"
        # before it the ring's stages, block by block
        assert re.match(rf"[:>]*(L{{{n}}}[:>]+){{2}}", text), f"{name}: {text}"
        assert text.count("L") == 3 * n, f"{name}: {text}"


def test_units_of_channels(tmp_path):
    kernels = _kernels("k_i8_few.hip", tmp_path)
    assert len(kernels) == 6
    for name, text in kernels.items():
        stages = _arguments(name)[0]
        # whole stages of four loads, each begun by the unit's scales or not
        assert all(len(run) in (1, 4, 5) for run in re.findall("L+", text)), f"{name}: {text}"
        assert f"w{4 * (stages - 1)};" in text, f"{name}: {text}"
        # the loop's stage ends at a scheduling barrier, and one follows the wait
        assert re.search(r"LLLL[:>]*\|", text), f"{name}: {text}"
        assert re.search(rf"w{4 * (stages - 1)};[:>]*w0;[:>]*\|", text), f"{name}: {text}"


def test_tiles(tmp_path):
    kernels = _kernels("k_i8_tile.hip", tmp_path)
    assert len(kernels) == 12
    for name, text in kernels.items():
        tm, wm, wn, nsa, nsb = _arguments(name)
        waves = wm * wn
        a, b = tm * 128 // 1024 // waves, 256 * 128 // 1024 // waves   # loads of a wave and stage
        if nsb > nsa:   # b's of a stage in its first step, a's behind the meeting
            loop = rf"\|{'L' * b}\|\|\|w{b};B\|{'L' * a}\|"
        else:
            loop = rf"\|\|\|\|w{(nsa - 2) * (a + b)};B\|{'L' * (a + b)}\|"
        assert re.search(loop, text), f"{name}: {loop} not in {text}"
        # elsewhere (first stages, a tile's last ones) every wait is for all
        assert set(re.findall(r"w(\d+);B", text)) <= {"0", str(b if nsb > nsa else (nsa - 2) * (a + b))}
