"""adapters_add on the GPU against the oracle in fp64.

Products of 16-bit numbers are exact in fp32; an inner sum of K of them in any
order is off by at most K 2^-24 of the sum of their magnitudes, the part sums
and the scale by 17 more.  t goes on in parts of 17 bits at least (24 of bf16 for
fp32 outputs, 22 of fp16): 2^-17 (2^-24, 2^-21).  The outer sum of R products,
in up to three parts each, adds 3 R 2^-24, the power of two nothing, y one
rounding of the result, and the output's type half its eps.
"""
from __future__ import annotations

import numpy as np
import pytest

from oracle import adapters as oracle

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
    return None if t is None else t.detach().cpu().double().numpy()


def _inputs(M, N, K, R, n, dtype="bf16", y="bf16", seed=0, ids=None, none=0.2, ragged=False, scales=True):
    gen = torch.Generator().manual_seed(seed)
    dt = DTYPES[dtype]
    if ids is None:
        ids = torch.randint(0, max(n, 1), (M,), generator=gen)
        ids = torch.where(torch.rand(M, generator=gen) < none, -1, ids)
    return dict(y=(torch.randn((M, N), generator=gen) * 2).to(DTYPES[y]).cuda(),
                x=torch.randn((M, K), generator=gen).to(dt).cuda(),
                a=(torch.randn((n, R, K), generator=gen) / max(K, 1) ** 0.5).to(dt).cuda(),
                b=(torch.randn((n, N, R), generator=gen) * 0.3).to(dt).cuda(), ids=torch.as_tensor(ids).cuda(),
                scales=(torch.randn(n, generator=gen) * 2).cuda() if scales else None,
                ranks=torch.randint(-1, R + 3, (n,), generator=gen, dtype=torch.int32).cuda() if ragged else None)


def _check(i, out, before=None):
    y = i["y"] if before is None else before
    want, bound = oracle.add(_np(y), _np(i["x"]), _np(i["a"]), _np(i["b"]), i["ids"].cpu().numpy(), _np(i["scales"]),
                             None if i["ranks"] is None else i["ranks"].cpu().numpy())
    K, R = i["a"].shape[2], i["a"].shape[1]
    part = 2.0 ** -21 if i["x"].dtype == torch.float16 else 2.0 ** -24 if y.dtype == torch.float32 else 2.0 ** -17
    tol = ((K + 17 + 3 * R) * 2.0 ** -24 + part) * bound + 2.0 ** -24 * (np.abs(want) + bound)
    if y.dtype != torch.float32:
        tol = tol + torch.finfo(y.dtype).eps / 2 * (np.abs(want) + tol) + (2.0 ** -25 if y.dtype == torch.float16 else 0)
    worst = np.abs(_np(out) - want) - tol * (1 + 2.0 ** -20)
    assert (worst <= 0).all(), f"{(worst > 0).sum()} of {worst.size} off, the worst by {worst.max():.3g}"
    bare = (i["ids"] < 0) | (i["ids"] >= i["a"].shape[0])
    assert torch.equal(out[bare], y[bare])


TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("bf16", "f16"), ("f16", "f16"), ("f16", "f32"), ("f16", "bf16")]
SIZES = [(1, 64, 64, 16, 1), (1, 1, 1, 1, 1), (3, 7, 5, 3, 2), (16, 256, 512, 16, 16), (17, 100, 264, 8, 3),
         (64, 300, 128, 32, 70), (65, 513, 1000, 24, 4), (130, 1111, 333, 12, 5), (7, 4096, 4096, 64, 2),
         (40, 250, 2048, 128, 3), (5, 130, 96, 200, 2), (33, 77, 640, 256, 3), (300, 96, 72, 50, 9),
         (600, 300, 128, 16, 200), (1, 64, 16384, 16, 1), (2, 70, 9001, 8, 2)]


@pytest.mark.parametrize("dtype,y", TYPES)
@pytest.mark.parametrize("M,N,K,R,n", SIZES)
def test_adapters(M, N, K, R, n, dtype, y):
    from paper_2608_02703_amd import adapters_add
    i = _inputs(M, N, K, R, n, dtype, y, seed=M * 7 + N, none=0.0 if M == 1 else 0.2, ragged=(M + N) % 2 == 1)
    _check(i, adapters_add(**i))


@pytest.mark.parametrize("ids", ["runs", "one", "none", "far", "every other"])
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
def test_orders_of_ids(ids, idt):
    """Requests one after another, one adapter for all, none at all, ids outside,
    and tokens with and without in turn."""
    from paper_2608_02703_amd import adapters_add
    M, n = 150, 6
    v = {"runs": torch.arange(M) // 29, "one": torch.full((M,), 3), "none": torch.full((M,), -1),
         "far": torch.tensor([0, 5, 6, 7, -2, 2 ** 31 - 1, -2 ** 31, 1] * 19)[:M],
         "every other": torch.where(torch.arange(M) % 2 == 0, torch.arange(M) % n, -7)}[ids].to(idt)
    if idt == torch.int64 and ids == "far":
        v[::8] = 2 ** 40
    i = _inputs(M, 200, 256, 16, n, ids=v)
    _check(i, adapters_add(**i))
    before = i["y"].clone()
    assert adapters_add(**i, out=i["y"]) is i["y"]
    _check(i, i["y"], before)


@pytest.mark.parametrize("dtype,y", [("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("R", [16, 20])
def test_strides_and_places(R, dtype, y):
    """Rows in wider buffers at odd places, adapters that share their factors,
    in place and not; what lies between rows stays."""
    from paper_2608_02703_amd import adapters_add
    M, N, K, n = 70, 131, 100, 5
    i = _inputs(M, N, K, R, n, dtype, y, seed=4, ragged=True)

    def wide(t, off, pad):
        rows, cols = t.shape[:-1].numel(), t.shape[-1]
        buf = torch.full((rows * (cols + pad) + 32,), 99, dtype=t.dtype, device="cuda")
        ld, st = cols + pad, []
        for k in reversed(range(t.dim() - 1)):
            st.insert(0, ld)
            ld *= t.shape[k]
        v = buf[off:].as_strided(t.shape, (*st, 1))
        v.copy_(t)
        return buf, v
    j = dict(i)
    for k, off, pad in (("x", 3, 5), ("a", 1, 3), ("b", 5, 1), ("y", 7, 9)):
        j[k] = wide(i[k], off, pad)[1]
    buf, out = wide(i["y"], 1, 4)
    _check(i, adapters_add(**j, out=out))
    out.fill_(99)
    assert (buf == 99).all()
    buf, y = wide(i["y"], 2, 6)
    j["y"] = y
    _check(i, adapters_add(**j, out=y))
    y.fill_(99)
    assert (buf == 99).all()
    j = dict(i, a=i["a"][:1].expand(n, R, K), b=i["b"][:1].expand(n, N, R))
    _check(j, adapters_add(**j))


def test_what_ranks_leave_out_is_not_used():
    """NaN behind an adapter's rank, in adapters that no token has and in x of tokens without one."""
    from paper_2608_02703_amd import adapters_add
    for R in (24, 21):
        i = _inputs(50, 90, 136, R, 4, ids=torch.arange(50) % 5 % 4, none=0.0)
        i["ids"] = torch.where(i["ids"] == 3, -1, i["ids"])
        i["ranks"] = torch.tensor([R, 0, 7, R], dtype=torch.int32, device="cuda")
        want = adapters_add(**i)
        _check(i, want)
        i["a"][1], i["a"][2, 7:], i["a"][3] = float("nan"), float("inf"), float("nan")
        i["b"][1], i["b"][2, :, 7:], i["b"][3] = float("nan"), float("nan"), float("inf")
        i["x"][i["ids"] < 0] = float("nan")
        assert torch.equal(adapters_add(**i), want)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_large_and_small_values(dtype):
    """Inner sums far above and below fp16's range, and rows that are not finite."""
    from paper_2608_02703_amd import adapters_add
    i = _inputs(40, 64, 512, 16, 3, dtype, "f32", ids=torch.arange(40) % 3)
    i["y"].zero_()
    big = 200.0 if dtype == "f16" else 1e15
    i["x"][::4] *= big
    i["a"][0] *= big
    i["x"][1::4] *= 1e-3
    i["a"][1] *= 1e-3 if dtype == "f16" else 1e-15
    _check(i, adapters_add(**i))
    want = adapters_add(**i)
    i["x"][7, 3], i["x"][8, 5] = float("inf"), float("nan")
    got = adapters_add(**i)
    keep = torch.ones(40, dtype=torch.bool)
    keep[7] = keep[8] = False
    assert torch.equal(got[keep.cuda()], want[keep.cuda()])
    assert not torch.isfinite(got[7]).any() and torch.isnan(got[8]).all()


def test_nothing_to_add():
    from paper_2608_02703_amd import adapters_add
    for M, N, K, R, n in ((0, 8, 8, 4, 2), (3, 0, 8, 4, 2), (3, 8, 0, 4, 2), (3, 8, 8, 0, 2), (3, 8, 8, 4, 0)):
        i = _inputs(M, N, K, R, n, ids=torch.zeros(M, dtype=torch.int64), scales=False)
        assert torch.equal(adapters_add(**i), i["y"])
        adapters_add(**i, out=i["y"])


def test_beside_an_int8_product():
    """A layer's step: norm, 8-bit product, adapters on the same rows in 16 bits."""
    from paper_2608_02703_amd import adapters_add, matmul_i8, quantize_i8, rms_norm_i8
    M, K, N = 48, 512, 320
    gen = torch.Generator().manual_seed(2)
    x, r = (torch.randn((M, K), generator=gen).bfloat16().cuda() for _ in range(2))
    w = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    qw, sw = quantize_i8((torch.randn((N, K), generator=gen) / 16).cuda())
    codes, scales, total, h = rms_norm_i8(x, w, residual=r, normed=True)
    y = matmul_i8(codes, scales, qw, sw)
    i = _inputs(M, N, K, 16, 4, "bf16", "f32", seed=6)
    i.update(x=h, y=y)
    before = y.clone()
    adapters_add(**i, out=y)
    _check(i, y, before)


def test_streams_and_graphs():
    from paper_2608_02703_amd import adapters_add
    i = _inputs(37, 600, 640, 16, 5)
    want = adapters_add(**i)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = adapters_add(**i)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = adapters_add(**i)
    for seed in range(4):
        j = _inputs(37, 600, 640, 16, 5, seed=90 + seed)
        for k in ("x", "ids", "y", "a"):
            i[k].copy_(j[k])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(adapters_add(**i), held)
        _check(i, held)


def test_beyond_32_bit_offsets():
    """Factors and outputs past 2^31 elements."""
    from paper_2608_02703_amd import adapters_add
    M, N, K, R, n = 70, 4096, 64, 8, 3
    step = (1 << 31) // 2 + 8
    i = _inputs(M, N, K, R, n)
    a = torch.empty(2 * step + R * K, dtype=torch.bfloat16, device="cuda").as_strided((n, R, K), (step, K, 1))
    a.copy_(i["a"])
    y = torch.empty((M - 1) * (1 << 25) + N, dtype=torch.bfloat16, device="cuda").as_strided((M, N), (1 << 25, 1))
    y.copy_(i["y"])
    j = dict(i, a=a, y=y)
    _check(i, adapters_add(**j))
    adapters_add(**j, out=y)
    _check(i, y)


@pytest.mark.parametrize("scale", [2.0 ** 117, 2.0 ** -95])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_largest_and_smallest_scales(scale, dtype):
    """Inner sums near the ends of fp32: they keep their bits, and reach the sum finite.
    (Three bf16 parts of 2^-95 are normal numbers down to 2^-14 of it.)"""
    from paper_2608_02703_amd import adapters_add
    i = _inputs(20, 70, 64, 40, 3, dtype, "f32", seed=9)
    i["y"].zero_()
    i["scales"] = torch.tensor([scale, -scale, scale / 2], device="cuda")
    out = adapters_add(**i)
    assert torch.isfinite(out).all()
    _check(i, out)


@pytest.mark.parametrize("dtype,y", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("M,N,K,R,n", [(2100, 40, 100, 256, 2), (2100, 33, 264, 200, 4), (700, 50, 72, 90, 300),
                                       (64, 40, 136, 256, 70), (1100, 30601, 40, 20, 3), (1100, 30600, 33, 70, 16)])
def test_many_tokens(M, N, K, R, n, dtype, y):
    """Enough tokens, or outputs, for the ways that take more ranks or tiles at a time, their ids in runs and not."""
    from paper_2608_02703_amd import adapters_add
    i = _inputs(M, N, K, R, n, dtype, y, seed=M + N, ragged=n % 2 == 0)
    if n <= 4:
        i["ids"][:M // 2] = i["ids"][:M // 2].sort().values
    _check(i, adapters_add(**i))
