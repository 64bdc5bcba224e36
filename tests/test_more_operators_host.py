"""Refusals of the norm's, the adapters' and the head loss's entry points, which
come before any HIP call (CPU).  Every pointer given is a number that no call
follows: each case is refused, or has nothing to do."""
from __future__ import annotations

import pytest

import paper_2608_02703_amd as lib
from paper_2608_02703_amd import archead as ab

torch = pytest.importorskip("torch")

P = 0x10000   # a well aligned address
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def L():
    return ab.lib()


def _norm(L, **kw):
    a = dict(x=P, t=ab.BF16, M=2, d=64, ldx=64, r=P, ldr=64, w=P, wt=ab.BF16, off=0.0, eps=1e-6, total=P, ldt=64, out=P,
             ldo=64, codes=P, ldc=64, scales=P)
    a.update(kw)
    return L.archead_rms_norm(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=0), ab.OK), (dict(M=0, x=None, w=None, codes=None, out=None), ab.OK),
    (dict(t=ab.I8), ab.E_INVALID_ARG), (dict(t=77), ab.E_INVALID_ARG), (dict(wt=ab.F16), ab.E_INVALID_ARG),
    (dict(M=-1), ab.E_INVALID_ARG), (dict(M=2 ** 31), ab.E_INVALID_ARG), (dict(d=0), ab.E_INVALID_ARG),
    (dict(d=16385, ldx=20000, ldr=20000, ldt=20000, ldo=20000, ldc=20000), ab.E_UNSUPPORTED),
    (dict(eps=0.0), ab.E_INVALID_ARG), (dict(eps=-1.0), ab.E_INVALID_ARG), (dict(eps=NAN), ab.E_INVALID_ARG),
    (dict(eps=INF), ab.E_INVALID_ARG), (dict(off=NAN), ab.E_INVALID_ARG), (dict(off=INF), ab.E_INVALID_ARG),
    (dict(ldx=63), ab.E_INVALID_ARG), (dict(ldr=63), ab.E_INVALID_ARG), (dict(ldt=63), ab.E_INVALID_ARG),
    (dict(ldo=63), ab.E_INVALID_ARG), (dict(ldc=63), ab.E_INVALID_ARG), (dict(x=None), ab.E_INVALID_ARG),
    (dict(w=None), ab.E_INVALID_ARG), (dict(out=None, codes=None), ab.E_INVALID_ARG), (dict(scales=None), ab.E_INVALID_ARG),
    (dict(x=P + 1), ab.E_MISALIGNED), (dict(r=P + 1), ab.E_MISALIGNED), (dict(total=P + 1), ab.E_MISALIGNED),
    (dict(out=P + 1), ab.E_MISALIGNED), (dict(w=P + 1), ab.E_MISALIGNED), (dict(wt=ab.F32, w=P + 2), ab.E_MISALIGNED),
    (dict(t=ab.F32, wt=ab.F32, x=P + 2), ab.E_MISALIGNED), (dict(scales=P + 2), ab.E_MISALIGNED),
])
def test_norm_refusals(L, kw, status):
    assert _norm(L, **kw) == status, L.archead_last_error()


def test_python_refuses_host_tensors():
    x, w = torch.zeros(2, 64), torch.ones(64)
    with pytest.raises(ValueError):
        lib.rms_norm(x, w)
    with pytest.raises(ValueError):
        lib.rms_norm_i8(x, w)
