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
    a = dict(x=P, t=ab.BF16, M=2, d=64, ldx=64, r=2 * P, ldr=64, w=P, wt=ab.BF16, off=0.0, eps=1e-6, total=3 * P, ldt=64,
             out=4 * P, ldo=64, codes=P, ldc=64, scales=P)
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
    (dict(total=4 * P), ab.E_INVALID_ARG), (dict(total=P, ldt=65), ab.E_INVALID_ARG), (dict(total=2 * P, ldt=65), ab.E_INVALID_ARG),
    (dict(out=P, ldo=65), ab.E_INVALID_ARG), (dict(out=2 * P, ldo=70), ab.E_INVALID_ARG),
])
def test_norm_refusals(L, kw, status):
    assert _norm(L, **kw) == status, L.archead_last_error()


def test_python_refuses_host_tensors():
    x, w = torch.zeros(2, 64), torch.ones(64)
    with pytest.raises(ValueError):
        lib.rms_norm(x, w)
    with pytest.raises(ValueError):
        lib.rms_norm_i8(x, w)


def _adapters(L, **kw):
    a = dict(y=P, yt=ab.BF16, ldy=32, x=P, xt=ab.BF16, ldx=64, ad=True, ids=P, it=ab.I64, M=2, N=32, K=64, out=2 * P,
             ldo=32, ws=P, wsb=1 << 20)
    d = dict(a=P, b=P, scales=P, ranks=P, n=3, R=16, a_ad=1024, a_row=64, b_ad=512, b_row=16)
    d.update({k: v for k, v in kw.items() if k in d})
    a.update({k: v for k, v in kw.items() if k in a})
    a["ad"] = ab.AdaptersDesc(*d.values()) if a["ad"] else None
    return L.archead_adapters_add(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=0), ab.OK), (dict(N=0), ab.OK), (dict(n=0, out=P), ab.OK), (dict(R=0, out=P, a=None, b=None), ab.OK),
    (dict(K=0, out=P, x=None, ws=None), ab.OK),
    (dict(yt=ab.I8), ab.E_INVALID_ARG), (dict(xt=ab.F32), ab.E_INVALID_ARG), (dict(it=ab.F32), ab.E_INVALID_ARG),
    (dict(ad=False), ab.E_INVALID_ARG), (dict(M=-1), ab.E_INVALID_ARG), (dict(M=2 ** 23 + 1), ab.E_INVALID_ARG),
    (dict(N=2 ** 23 + 1, ldy=2 ** 24, ldo=2 ** 24), ab.E_INVALID_ARG), (dict(K=-1), ab.E_INVALID_ARG),
    (dict(n=-1), ab.E_INVALID_ARG), (dict(n=2 ** 22), ab.E_INVALID_ARG), (dict(R=-1), ab.E_INVALID_ARG),
    (dict(R=257, b_row=300), ab.E_UNSUPPORTED), (dict(ldy=31), ab.E_INVALID_ARG), (dict(ldo=31), ab.E_INVALID_ARG),
    (dict(ldx=63), ab.E_INVALID_ARG), (dict(a_ad=-1), ab.E_INVALID_ARG), (dict(a_row=63), ab.E_INVALID_ARG),
    (dict(b_ad=2 ** 41), ab.E_INVALID_ARG), (dict(b_row=15), ab.E_INVALID_ARG), (dict(y=None), ab.E_INVALID_ARG),
    (dict(x=None), ab.E_INVALID_ARG), (dict(a=None), ab.E_INVALID_ARG), (dict(b=None), ab.E_INVALID_ARG),
    (dict(ids=None), ab.E_INVALID_ARG), (dict(out=None), ab.E_INVALID_ARG), (dict(ws=None), ab.E_INVALID_ARG),
    (dict(out=P, ldo=40), ab.E_INVALID_ARG), (dict(y=P + 1), ab.E_MISALIGNED), (dict(x=P + 1), ab.E_MISALIGNED),
    (dict(a=P + 1), ab.E_MISALIGNED), (dict(b=P + 1), ab.E_MISALIGNED), (dict(out=P + 1), ab.E_MISALIGNED),
    (dict(ids=P + 4), ab.E_MISALIGNED), (dict(scales=P + 2), ab.E_MISALIGNED), (dict(ranks=P + 2), ab.E_MISALIGNED),
    (dict(yt=ab.F32, y=P + 2), ab.E_MISALIGNED), (dict(ws=P + 16), ab.E_MISALIGNED), (dict(wsb=64), ab.E_WORKSPACE),
])
def test_adapters_refusals(L, kw, status):
    assert _adapters(L, **kw) == status, L.archead_last_error()


def test_adapters_workspace_bytes(L):
    f = L.archead_adapters_workspace_bytes
    assert f(0, 64, 16, 2) == f(2, 0, 16, 2) == f(2, 64, 0, 2) == f(2, 64, 16, 0) == f(2, 64, 257, 2) == 0
    assert f(1, 64, 16, 2) % 256 == 0 and f(8192, 4096, 64, 8) < 8192 * 4096 * 2


def test_python_refuses_host_adapters():
    y, x = torch.zeros(2, 8), torch.zeros((2, 4), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lib.adapters_add(y, x, x[None], x[None], torch.zeros(2, dtype=torch.int64))


def _loss(L, gradient=False, **kw):
    a = dict(x=P, ldx=64, w=P, ldw=64, y=P, t=ab.I64)
    s = dict(M=2, V=100, d=64)
    o = dict(dx=P, lddx=64, dw=P, lddw=64) if gradient else dict(loss=P, lse=P)
    g = dict(lse=P, grad=P) if gradient else {}
    e = dict(ws=P, wsb=1 << 30)
    for v in (a, s, o, g, e):
        v.update({k: kw[k] for k in kw if k in v})
    f = L.archead_head_loss_grad if gradient else L.archead_head_loss
    return f(*a.values(), *g.values(), *s.values(), *o.values(), *e.values(), None)


BOTH = [
    (dict(t=ab.F32), ab.E_INVALID_ARG), (dict(M=-1), ab.E_INVALID_ARG), (dict(V=0), ab.E_INVALID_ARG),
    (dict(d=0), ab.E_INVALID_ARG), (dict(M=2 ** 20 + 1), ab.E_UNSUPPORTED), (dict(V=2 ** 22 + 1), ab.E_UNSUPPORTED),
    (dict(d=16385, ldx=20000, ldw=20000, lddx=20000, lddw=20000), ab.E_UNSUPPORTED), (dict(ldx=63), ab.E_INVALID_ARG),
    (dict(ldw=63), ab.E_INVALID_ARG), (dict(x=None), ab.E_INVALID_ARG), (dict(w=None), ab.E_INVALID_ARG),
    (dict(y=None), ab.E_INVALID_ARG), (dict(x=P + 1), ab.E_MISALIGNED), (dict(w=P + 1), ab.E_MISALIGNED),
    (dict(y=P + 4), ab.E_MISALIGNED), (dict(t=ab.I32, y=P + 2), ab.E_MISALIGNED), (dict(ws=None), ab.E_INVALID_ARG),
    (dict(ws=P + 16), ab.E_MISALIGNED), (dict(wsb=1024), ab.E_WORKSPACE), (dict(lse=None), ab.E_INVALID_ARG),
    (dict(lse=P + 2), ab.E_MISALIGNED),
]


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(M=0), ab.OK), (dict(M=0, x=None, w=None, y=None, loss=None, ws=None), ab.OK), (dict(loss=None), ab.E_INVALID_ARG),
    (dict(loss=P + 2), ab.E_MISALIGNED),
])
def test_head_loss_refusals(L, kw, status):
    assert _loss(L, **kw) == status, L.archead_last_error()


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(M=0, dw=None), ab.OK), (dict(M=0, dx=None, dw=None), ab.OK), (dict(dx=None, dw=None), ab.E_INVALID_ARG),
    (dict(grad=None), ab.E_INVALID_ARG), (dict(grad=P + 2), ab.E_MISALIGNED), (dict(lddx=63), ab.E_INVALID_ARG),
    (dict(lddw=63), ab.E_INVALID_ARG), (dict(dx=P + 1), ab.E_MISALIGNED), (dict(dw=P + 1), ab.E_MISALIGNED),
])
def test_head_gradient_refusals(L, kw, status):
    assert _loss(L, gradient=True, **kw) == status, L.archead_last_error()


def test_head_loss_workspace_bytes(L):
    f = L.archead_head_loss_workspace_bytes
    assert f(0, 100, 64, P, 64, 0) == f(2, 0, 64, P, 64, 1) == f(2, 100, 16385, P, 20000, 0) == f(-1, 1, 1, P, 1, 0) == 0
    assert f(2 ** 20 + 1, 1, 1, P, 1, 0) == f(1, 2 ** 22 + 1, 1, P, 1, 0) == 0
    assert f(8, 100, 64, P + 2, 64, 0) > f(8, 100, 64, P, 64, 0)      # rows that have to be copied
    assert f(4096, 151936, 4096, P, 4096, 0) < 4096 * 151936 // 4 and f(4096, 151936, 4096, P, 4096, 1) < 4096 * 151936 * 2 // 3


def test_python_refuses_host_loss():
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lib.head_loss(x, x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        lib.head_loss_grad(x, x, torch.zeros(2, dtype=torch.int64), torch.zeros(2), torch.zeros(2))
