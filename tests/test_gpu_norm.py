"""rms_norm and rms_norm_i8 on the GPU against the oracle in fp64.

Codes and sums have to be equal bit for bit.  A scale is u / n with n and the
quotient off by a few 2^-52: one rounding of 2^-24.  A normed value is t times 1 / n
rounded to fp32: 2^-24 for that, 2^-24 for the product, half its type's eps for the
output (fp16 below its normal range: half its smallest step).  Tolerances are
these, and 2^-20 of them for products of roundings.
"""
from __future__ import annotations

import numpy as np
import pytest

from oracle import norm as oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _np(t):
    return None if t is None else t.detach().cpu().float().numpy()


def _check(x, w, eps, r, offset, codes=None, scales=None, total=None, out=None):
    """x and r as they were before the call."""
    dt = x.dtype
    s, t, n, q, u = oracle.rms_norm(_np(x), _np(w), eps, _np(r), offset)
    if total is not None:
        assert torch.equal(total.cpu().nan_to_num(7.0), torch.from_numpy(s).to(dt).nan_to_num(7.0))
    if codes is not None:
        assert np.array_equal(codes.cpu().numpy(), q)
        want = u.astype(np.float64) / n
        got = scales.cpu().double().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(u))
        fine = ~np.isnan(u)
        assert (np.abs(got - want)[fine] <= 2.0 ** -24 * (1 + 2.0 ** -20) * want[fine] + 2.0 ** -150).all()
    if out is not None:
        bad = np.isnan(u)
        got = out.cpu().double().numpy()
        assert np.isnan(got[bad]).all()
        want = t[~bad].astype(np.float64) / n[~bad, None]
        half = 0.0 if dt == torch.float32 else torch.finfo(dt).eps / 2
        tol = (2.0 ** -23 + half) * (1 + 2.0 ** -20) * np.abs(want) + (2.0 ** -25 if dt == torch.float16 else 2.0 ** -125)
        big = np.abs(want) + tol >= torch.finfo(dt).max
        assert (np.where(big, 0, np.abs(got[~bad] - want) - tol) <= 0).all()


def _rows(M, d, dtype, seed, r=True, w32=False):
    gen = torch.Generator().manual_seed(seed)
    dt = DTYPES[dtype]
    x = (torch.randn((M, d), generator=gen) * torch.exp(torch.randn((M, 1), generator=gen))).to(dt)
    res = (torch.randn((M, d), generator=gen) * 3).to(dt) if r else None
    w = (1 + 0.3 * torch.randn(d, generator=gen)).to(torch.float32 if w32 else dt)
    return x.cuda(), w.cuda(), None if res is None else res.cuda()


SIZES = [(1, 1), (3, 7), (2, 8), (5, 9), (4, 63), (17, 64), (1, 511), (33, 512), (3, 513), (1, 4096), (7, 4097),
         (3, 5003), (2, 8192), (2, 16383), (2, 16384), (1030, 64), (1027, 4100)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("M,d", SIZES)
def test_norm_i8_with_residual(M, d, dtype):
    from paper_2608_02703_amd import rms_norm_i8
    x, w, r = _rows(M, d, dtype, M * 100003 + d, w32=d % 2 == 1)
    codes, scales, total, out = rms_norm_i8(x, w, eps=1e-5, residual=r, normed=True)
    _check(x, w, 1e-5, r, 0.0, codes, scales, total, out)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("M,d", [(1, 64), (5, 515), (2, 4096), (300, 2560)])
def test_norm_alone(M, d, dtype):
    """No residual, an offset, 16-bit rows alone or codes alone."""
    from paper_2608_02703_amd import rms_norm, rms_norm_i8
    x, w, _ = _rows(M, d, dtype, 7 * d + M, r=False)
    _check(x, w, 1e-6, None, 1.0, out=rms_norm(x, w, offset=1.0))
    codes, scales = rms_norm_i8(x, w, offset=1.0)
    _check(x, w, 1e-6, None, 1.0, codes, scales)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,d", [(2060, 16384), (70000, 512), (8200, 4104)])
def test_norm_many_rows(M, d, dtype):
    """Rows taken by workgroups one after another; four groups a thread."""
    from paper_2608_02703_amd import rms_norm_i8
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((M, d), generator=gen, device="cuda").to(DTYPES[dtype])
    r = torch.randn((M, d), generator=gen, device="cuda").to(DTYPES[dtype])
    w = torch.randn(d, generator=gen, device="cuda").to(DTYPES[dtype])
    got = rms_norm_i8(x, w, residual=r, normed=True)
    at = torch.cat([torch.arange(0, M, 997), torch.arange(M - 40, M)]).cuda()
    _check(x[at], w, 1e-6, r[at], 0.0, *[t[at] for t in got])


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_norm_odd_rows(dtype):
    """Zeros, the largest and smallest values, rows that are not finite, weights
    of zero and below."""
    from paper_2608_02703_amd import rms_norm_i8
    info = torch.finfo(DTYPES[dtype])
    n = 600
    gen = torch.Generator().manual_seed(9)
    z = torch.randn(n, generator=gen, dtype=torch.float64)
    rows = [torch.zeros(n, dtype=torch.float64), z.clamp(-1, 1) * info.max, z * info.tiny, z * info.tiny * info.eps * 4,
            z * 1e-3, torch.full((n,), 5.0, dtype=torch.float64)]
    for bad in (float("nan"), float("inf"), -float("inf")):
        rows.append(z.clone())
        rows[-1][n // 3] = bad
    x = torch.stack(rows).to(DTYPES[dtype]).cuda()
    w = torch.randn(n, generator=gen).to(DTYPES[dtype]).clamp(-0.99, 0.99).cuda()
    w[3], w[n - 1] = 0.0, -0.5
    for eps in (1e-6, 1e-30):
        codes, scales, out = rms_norm_i8(x, w, eps=eps, normed=True)
        _check(x, w, eps, None, 0.0, codes, scales, None, out)
    assert torch.isnan(scales[-3:]).all() and torch.isnan(out[-3:]).all() and not codes[-3:].any()
    assert not out[0].any() and not codes[0].any()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("d", [61, 640])
def test_norm_strides_and_places(dtype, d):
    """Rows in wider buffers at odd places, sums in place of x or the residual,
    normed rows in place of x; what lies between rows stays."""
    from paper_2608_02703_amd import rms_norm, rms_norm_i8
    M, ld = 70, d + 13
    x, w, r = _rows(M, d, dtype, 5)

    def wide(t, off):
        buf = torch.full((M * ld + 32,), 99, dtype=t.dtype, device="cuda")
        v = buf[off:].as_strided((M, d), (ld, 1))
        v.copy_(t)
        return buf, v

    for place in ("residual", "x", None):
        (bx, vx), (br, vr) = wide(x, 3), wide(r, 5)
        (bo, vo), (bc, vc) = wide(torch.zeros_like(x), 7), wide(torch.zeros((M, d), dtype=torch.int8, device="cuda"), 1)
        total = {"residual": vr, "x": vx, None: None}[place]
        codes, scales, s, out = rms_norm_i8(vx, w, residual=vr, codes=vc, normed=vo, total=total)
        assert place is None or s is total
        _check(x, w, 1e-6, r, 0.0, codes, scales, s, out)
        for b, v in ((bx, vx), (br, vr), (bo, vo), (bc, vc)):
            v.fill_(99)
            assert (b == 99).all()
    bx, vx = wide(x, 1)
    out = rms_norm(vx, w, out=vx)
    _check(x, w, 1e-6, None, 0.0, out=out)
    vx.fill_(99)
    assert (bx == 99).all()
    y, z = r.clone(), x.clone()
    out, s = rms_norm(z, w, residual=y, total=z, out=y)
    assert s is z and out is y
    _check(x, w, 1e-6, r, 0.0, total=s, out=out)
    y = r.clone()
    out, s = rms_norm(x.clone(), w, residual=y, total=y)
    assert s is y
    _check(x, w, 1e-6, r, 0.0, total=s, out=out)


def test_norm_no_rows_and_reproducible():
    from paper_2608_02703_amd import rms_norm, rms_norm_i8
    x, w, r = _rows(37, 1000, "bf16", 3)
    codes, scales, total, out = rms_norm_i8(x[:0], w, residual=r[:0], normed=True)
    assert codes.shape == (0, 1000) and scales.shape == (0,) and total.shape == out.shape == (0, 1000)
    a, b = rms_norm(x, w, residual=r), rms_norm(x, w, residual=r)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_norm_then_product():
    """The step of an INT8 layer: norm with residual, product, against fp64."""
    from paper_2608_02703_amd import matmul_i8, quantize_i8, rms_norm_i8
    M, d, N = 40, 1024, 300
    x, w, r = _rows(M, d, "bf16", 21)
    weight = torch.randn((N, d), generator=torch.Generator().manual_seed(4)).cuda() / 32
    qw, sw = quantize_i8(weight)
    codes, scales, total = rms_norm_i8(x, w, residual=r)
    y = matmul_i8(codes, scales, qw, sw)
    _, t, n, q, u = oracle.rms_norm(_np(x), _np(w), 1e-6, _np(r))
    want = (q.astype(np.float64) * (u.astype(np.float64) / n)[:, None]) @ \
        (qw.cpu().double().numpy() * sw.cpu().double().numpy()[:, None]).T
    # the exact sum times two scales: a rounding of the scale and three of the product
    assert (np.abs(y.cpu().double().numpy() - want) <= 4 * 2.0 ** -24 * (1 + 2.0 ** -20) * np.abs(want) + 2.0 ** -120).all()


def test_norm_on_a_stream_and_in_a_graph():
    from paper_2608_02703_amd import rms_norm_i8
    x, w, r = _rows(130, 2560, "bf16", 8)
    want = rms_norm_i8(x, w, residual=r, normed=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = rms_norm_i8(x, w, residual=r, normed=True)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = rms_norm_i8(x, w, residual=r, normed=True)
    for seed in range(3):
        nx, _, nr = _rows(130, 2560, "bf16", 50 + seed)
        x.copy_(nx)
        r.copy_(nr)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(rms_norm_i8(x, w, residual=r, normed=True), held))
