"""Which tensors share memory, as BeamStates asks before it takes them (CPU):
against the bytes that each element of either holds."""
from __future__ import annotations

import random

import pytest

from paper_2608_02703_amd.archead import _share_memory

torch = pytest.importorskip("torch")


def _bytes(t):
    at = torch.zeros((), dtype=torch.int64) + t.data_ptr()
    for d, (n, st) in enumerate(zip(t.shape, t.stride())):
        at = at[..., None] + torch.arange(n) * (st * t.element_size())
    at = at.reshape(-1)[:, None] + torch.arange(t.element_size())
    return set(at.reshape(-1).tolist())


def _both(a, b):
    want = bool(_bytes(a) & _bytes(b))
    assert _share_memory(a, b) == want and _share_memory(b, a) == want
    return want


def test_by_hand():
    t = torch.zeros((12, 5, 4), dtype=torch.float16)
    assert _both(t[:8], t[4:]) and not _both(t[:6], t[6:]) and _both(t, t) and _both(t, t[11, 4, 3:])
    kv = torch.zeros((6, 2, 3, 7, 8), dtype=torch.float16)
    assert not _both(kv[:, 0], kv[:, 1]) and _both(kv[:, 0], kv[:, :, 1]) and not _both(kv[..., :3], kv[..., 3:])
    assert not _both(kv[..., 2], kv[..., 5]) and not _both(kv[:, 0, :, :4], kv[:, 0, :, 4:])
    assert _both(kv[:, 0, :, :4], kv[:, 0, :, 3:]) and not _both(kv[::2], kv[1::2])
    u = torch.zeros(4096, dtype=torch.int8)     # states of unlike shape side by side in each row
    rows = u.view(8, 512)
    assert not _both(rows[:, :96].as_strided((8, 3, 32), (512, 32, 1)), rows[:, 96:].as_strided((8, 13, 32), (512, 32, 1)))
    assert not _both(torch.zeros(5).expand(3, 5), torch.zeros(5))
    assert _both(u[:5].expand(3, 5), u[2:9:3]) and not _both(u[:5].expand(3, 5), u[5:9])
    f = torch.zeros(64, dtype=torch.float32)
    assert _both(f, f.view(torch.int8)[3:4]) and not _both(f[1:3], f.view(torch.int8)[:4])


def test_random_views():
    r = random.Random(5)
    base = torch.zeros(700, dtype=torch.int8)
    found = [0, 0]
    for _ in range(3000):
        views = []
        for _ in range(2):
            dt = r.choice([torch.int8, torch.int16, torch.float32])
            buf = base[:700 // 4 * 4].view(dt)
            dims = [(r.randint(1, 4), r.choice([0, 1, 1, 2, 3, 4, 5, 7, 12, 16, 24, 31, 48])) for _ in range(r.randint(0, 3))]
            reach = sum((n - 1) * st for n, st in dims)
            if reach >= buf.numel():
                break
            at = r.randint(0, buf.numel() - 1 - reach)
            views.append(buf.as_strided([n for n, _ in dims], [st for _, st in dims], at))
        if len(views) == 2:
            found[_both(*views)] += 1
    assert min(found) > 100
