"""Refusals of the 8-bit products' and the beam search's entry points, which
come before any HIP call (CPU).  Every pointer given is a number that no call
follows: each case is refused, or has nothing to do."""
from __future__ import annotations

import ctypes

import pytest

import paper_2608_02703_amd as lib
from paper_2608_02703_amd import archead as ab

torch = pytest.importorskip("torch")

P = 0x10000   # a well aligned address


@pytest.fixture(scope="module")
def L():
    return ab.lib()


def _quantize(L, **kw):
    a = dict(x=P, t=ab.BF16, M=2, d=64, ldx=64, codes=P, ldc=64, scales=P)
    a.update(kw)
    return L.archead_quantize_i8(a["x"], a["t"], a["M"], a["d"], a["ldx"], a["codes"], a["ldc"], a["scales"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=0), ab.OK), (dict(M=0, x=None, codes=None, scales=None), ab.OK),
    (dict(t=ab.I8), ab.E_INVALID_ARG), (dict(t=77), ab.E_INVALID_ARG), (dict(M=-1), ab.E_INVALID_ARG),
    (dict(M=2 ** 31), ab.E_INVALID_ARG), (dict(d=0), ab.E_INVALID_ARG), (dict(d=2 ** 31), ab.E_INVALID_ARG),
    (dict(ldx=63), ab.E_INVALID_ARG), (dict(ldc=63), ab.E_INVALID_ARG), (dict(x=None), ab.E_INVALID_ARG),
    (dict(codes=None), ab.E_INVALID_ARG), (dict(scales=None), ab.E_INVALID_ARG),
    (dict(x=P + 1), ab.E_MISALIGNED), (dict(t=ab.F32, x=P + 2), ab.E_MISALIGNED), (dict(scales=P + 2), ab.E_MISALIGNED),
])
def test_quantize_refusals(L, kw, status):
    assert _quantize(L, **kw) == status, L.archead_last_error()


def _matmul(L, **kw):
    a = dict(a=P, lda=64, sa=P, b=P, ldb=64, sb=P, bias=None, M=2, N=3, K=64, out=P, t=ab.F32, ldo=3)
    a.update(kw)
    return L.archead_matmul_i8(a["a"], a["lda"], a["sa"], a["b"], a["ldb"], a["sb"], a["bias"], a["M"], a["N"], a["K"],
                               a["out"], a["t"], a["ldo"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=0), ab.OK), (dict(N=0), ab.OK), (dict(M=-1), ab.E_INVALID_ARG), (dict(N=-1), ab.E_INVALID_ARG),
    (dict(K=-1), ab.E_INVALID_ARG), (dict(M=2 ** 31), ab.E_INVALID_ARG), (dict(N=2 ** 31), ab.E_INVALID_ARG),
    (dict(K=131072, lda=131072, ldb=131072), ab.E_UNSUPPORTED), (dict(lda=63), ab.E_INVALID_ARG),
    (dict(ldb=63), ab.E_INVALID_ARG), (dict(ldo=2), ab.E_INVALID_ARG), (dict(a=None), ab.E_INVALID_ARG),
    (dict(b=None), ab.E_INVALID_ARG), (dict(sa=None), ab.E_INVALID_ARG), (dict(sb=None), ab.E_INVALID_ARG),
    (dict(out=None), ab.E_INVALID_ARG), (dict(t=ab.I32), ab.E_INVALID_ARG), (dict(sa=P + 2), ab.E_MISALIGNED),
    (dict(sb=P + 1), ab.E_MISALIGNED), (dict(bias=P + 3), ab.E_MISALIGNED), (dict(out=P + 2), ab.E_MISALIGNED),
    (dict(t=ab.F16, out=P + 1), ab.E_MISALIGNED),
])
def test_matmul_refusals(L, kw, status):
    assert _matmul(L, **kw) == status, L.archead_last_error()


def _select(L, **kw):
    a = dict(lg=P, t=ab.F32, B=2, K=4, V=100, ldl=100, scores=P, fin=None, end=-1, n=8, out=P, par=P, tok=P, ended=None,
             ws=P, wsb=1 << 20)
    a.update(kw)
    return L.archead_beam_select(a["lg"], a["t"], a["B"], a["K"], a["V"], a["ldl"], a["scores"], a["fin"], a["end"],
                                 a["n"], a["out"], a["par"], a["tok"], a["ended"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), ab.OK), (dict(B=-1), ab.E_INVALID_ARG), (dict(K=0), ab.E_INVALID_ARG), (dict(K=33), ab.E_INVALID_ARG),
    (dict(B=16384), ab.E_INVALID_ARG), (dict(V=0), ab.E_INVALID_ARG), (dict(V=2 ** 31), ab.E_INVALID_ARG),
    (dict(n=0), ab.E_INVALID_ARG), (dict(n=65), ab.E_INVALID_ARG), (dict(ldl=99), ab.E_INVALID_ARG),
    (dict(end=-2), ab.E_INVALID_ARG), (dict(end=100), ab.E_INVALID_ARG), (dict(fin=P), ab.E_INVALID_ARG),
    (dict(t=ab.I8), ab.E_INVALID_ARG), (dict(lg=None), ab.E_INVALID_ARG), (dict(scores=None), ab.E_INVALID_ARG),
    (dict(out=None), ab.E_INVALID_ARG), (dict(par=None), ab.E_INVALID_ARG), (dict(tok=None), ab.E_INVALID_ARG),
    (dict(ws=None), ab.E_INVALID_ARG), (dict(wsb=64), ab.E_WORKSPACE), (dict(ws=P + 16), ab.E_MISALIGNED),
    (dict(lg=P + 2), ab.E_MISALIGNED), (dict(t=ab.BF16, lg=P + 1), ab.E_MISALIGNED), (dict(scores=P + 2), ab.E_MISALIGNED),
    (dict(out=P + 2), ab.E_MISALIGNED), (dict(par=P + 4), ab.E_MISALIGNED), (dict(tok=P + 4), ab.E_MISALIGNED),
])
def test_select_refusals(L, kw, status):
    assert _select(L, **kw) == status, L.archead_last_error()


def test_beam_workspace_bytes(L):
    assert L.archead_beam_workspace_bytes(0, 5) == 0 and L.archead_beam_workspace_bytes(3, 0) == 0
    small, large = L.archead_beam_workspace_bytes(64, 2048), L.archead_beam_workspace_bytes(64, 2049)
    assert 0 < small < large and small % 256 == 0
    assert L.archead_beam_workspace_bytes(256, 262144) < 256 * 262144 // 16   # far less than the logits


def test_logits_beam_needs_a_handle(L):
    assert L.archead_logits_beam(None, P, 1, 4, 64, P, None, -1, 4, P, P, P, None, P, 1 << 20, None) == ab.E_INVALID_ARG


def _reorder(L, layout=(), **kw):
    names = [n for n, _ in ab.StateLayout._fields_]
    l = dict(zip(names, (2, 3, 16, 96, 48, 16, 96, 48, 16)))
    l.update(layout)
    a = dict(ns=1, src=[P], dst=[2 * P], B=2, K=4, n=4, par=P, t=ab.I64, len=None, lp=True)
    a.update(kw)
    arr = lambda v: None if v is None else (ctypes.c_void_p * max(len(v), 1))(*v)   # noqa: E731
    return L.archead_beam_reorder(ab.StateLayout(*[l[n] for n in names]) if a["lp"] else None, a["ns"], arr(a["src"]),
                                  arr(a["dst"]), a["B"], a["K"], a["n"], a["par"], a["t"], a["len"], None)


@pytest.mark.parametrize("layout,kw,status", [
    ({}, dict(ns=0), ab.OK), ({}, dict(B=0), ab.OK), (dict(positions=0), {}, ab.OK), (dict(n_outer=0), {}, ab.OK),
    (dict(pos_bytes=0), {}, ab.OK), ({}, dict(lp=False), ab.E_INVALID_ARG), ({}, dict(ns=-1), ab.E_INVALID_ARG),
    ({}, dict(B=-1), ab.E_INVALID_ARG), ({}, dict(B=2 ** 25), ab.E_INVALID_ARG), ({}, dict(K=0), ab.E_INVALID_ARG),
    ({}, dict(K=33), ab.E_INVALID_ARG), ({}, dict(n=0), ab.E_INVALID_ARG), ({}, dict(n=65), ab.E_INVALID_ARG),
    ({}, dict(src=None), ab.E_INVALID_ARG), ({}, dict(dst=None), ab.E_INVALID_ARG), ({}, dict(src=[None]), ab.E_INVALID_ARG),
    ({}, dict(dst=[None]), ab.E_INVALID_ARG), ({}, dict(par=None), ab.E_INVALID_ARG), ({}, dict(t=ab.F32), ab.E_INVALID_ARG),
    ({}, dict(par=P + 4), ab.E_MISALIGNED), ({}, dict(t=ab.I32, par=P + 2), ab.E_MISALIGNED),
    ({}, dict(len=P + 1), ab.E_MISALIGNED), (dict(src_row=-96), {}, ab.E_INVALID_ARG),
    (dict(pos_bytes=-1), {}, ab.E_INVALID_ARG), (dict(dst_outer=2 ** 43), {}, ab.E_INVALID_ARG),
    (dict(n_outer=2 ** 31, positions=2 ** 31), {}, ab.E_INVALID_ARG),
    ({}, dict(dst=[P], n=3), ab.E_INVALID_ARG), (dict(dst_row=192), dict(dst=[P]), ab.E_INVALID_ARG),
    ({}, dict(ns=2, src=[P, 3 * P], dst=[P, 4 * P]), ab.E_INVALID_ARG),
])
def test_reorder_refusals(L, layout, kw, status):
    assert _reorder(L, layout, **kw) == status, L.archead_last_error()


def test_python_refuses_host_tensors():
    x = torch.zeros(2, 64)
    c, s = torch.zeros(2, 64, dtype=torch.int8), torch.ones(2)
    with pytest.raises(ValueError):
        lib.quantize_i8(x)
    with pytest.raises(ValueError):
        lib.matmul_i8(c, s, c, s)
    with pytest.raises(ValueError):
        lib.beam_select(x, torch.zeros(1, 2), 2)
    with pytest.raises(ValueError):
        lib.BeamStates([x], 2)


def _layout(s, d, r=0, p=None):
    return dict(zip([n for n, _ in ab.StateLayout._fields_], lib.BeamStates._layout(s, d, r, p)))


def test_state_layouts():
    z = lambda *shape, dtype=torch.int16: torch.zeros(shape, dtype=dtype)   # noqa: E731
    t = z(6, 3, 5, 4)
    assert _layout(t, t) == dict(n_outer=1, positions=1, pos_bytes=120, src_row=120, src_outer=0, src_pos=0, dst_row=120,
                                 dst_outer=0, dst_pos=0)
    l = _layout(t, t, p=2)                      # [rows, heads, positions, dim]
    assert (l["n_outer"], l["positions"], l["pos_bytes"], l["src_outer"], l["src_pos"]) == (3, 5, 8, 40, 8)
    l = _layout(t, t, p=1)                      # [rows, positions, heads, dim]
    assert (l["n_outer"], l["positions"], l["pos_bytes"], l["src_pos"]) == (1, 3, 40, 40)
    u = z(5, 6, 12).transpose(0, 1)             # [rows, positions, width] of [positions, rows, width]
    l = _layout(u, u, p=1)
    assert (l["src_row"], l["src_pos"], l["pos_bytes"]) == (24, 144, 24)
    w = z(6, 3, 5, 8)[..., :4]                  # padded rows of the last dimension
    l = _layout(w, t, p=2)
    assert (l["pos_bytes"], l["src_pos"], l["dst_pos"], l["src_outer"]) == (8, 16, 8, 80)
    h = z(6)                                    # one number a row
    assert _layout(h, h)["pos_bytes"] == 2
    with pytest.raises(ValueError):             # two outer dimensions that do not step as one
        v = z(6, 3, 4, 9, 4)[:, :, :2, :5]
        _layout(v, v, p=3)
    with pytest.raises(ValueError):             # a destination whose rows are one
        _layout(t, z(1, 3, 5, 4).expand(6, 3, 5, 4))
    _layout(z(1, 3, 5, 4).expand(6, 3, 5, 4), t)
