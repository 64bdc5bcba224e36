"""quantize_i8 and matmul_i8 on the GPU against the oracle in fp64 and whole
numbers.

Codes and scales have to be equal bit for bit.  A product is the exact integer
sum, rounded to fp32 and multiplied twice in fp32: three roundings of at most
2^-24 of it each, the bias one more of at most 2^-24 of the result, and the
output's own of at most half its type's eps of the result (fp16 below its
normal range: half its smallest step).  Tolerances are these, and 2^-40 for
their products.
"""
from __future__ import annotations

import numpy as np
import pytest

from oracle import int8 as oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _f64(t):
    return t.cpu().to(torch.float64).numpy()


def _check_codes(x, codes, scales):
    q, s = oracle.quantize(_f64(x))
    assert np.array_equal(scales.cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy(), q)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("M,d", [(1, 1), (3, 7), (2, 8), (5, 9), (4, 63), (1, 511), (1, 4096), (7, 4097), (3, 5003),
                                 (2, 16384), (2, 16385), (1, 40001), (1030, 64), (1025, 515), (1024, 4096),
                                 (1027, 4100)])
def test_quantize(M, d, dtype):
    from paper_2608_02703_amd import quantize_i8
    gen = torch.Generator().manual_seed(M * 100003 + d)
    x = torch.randn((M, d), generator=gen) * torch.exp(2 * torch.randn((M, 1), generator=gen))
    x = x.to(DTYPES[dtype]).cuda()
    codes, scales = quantize_i8(x)
    _check_codes(x, codes, scales)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_quantize_halves_and_odd_rows(dtype):
    """Exact halves (scale a power of two), zeros, the smallest and largest
    values, and rows that are not finite."""
    from paper_2608_02703_amd import quantize_i8
    dt = DTYPES[dtype]
    info = torch.finfo(dt)
    halves = torch.arange(-252, 253, dtype=torch.float64) / 2   # -126, -125.5, ..., 126
    rows = [torch.cat([halves * f, torch.tensor([127.0 * f], dtype=torch.float64)]) for f in (1.0, 2.0 ** -6, 8.0)]
    n = rows[0].numel()
    gen = torch.Generator().manual_seed(5)
    r = torch.randn(n, generator=gen, dtype=torch.float64)
    rows += [torch.zeros(n, dtype=torch.float64), r.clamp(-1, 1) * info.max, r * info.tiny,
             r * info.tiny * info.eps * 4, r * 1e-3]
    for bad in (float("nan"), float("inf"), -float("inf")):
        rows.append(r.clone())
        rows[-1][n // 3] = bad
    x = torch.stack(rows).to(dt).cuda()
    codes, scales = quantize_i8(x)
    _check_codes(x, codes, scales)
    assert torch.isnan(scales[-3:]).all() and not codes[-3:].any()


def test_quantize_fp32_next_to_halves():
    """fp32 quotients within a unit of a half, where a rounded quotient would
    fall on it."""
    from paper_2608_02703_amd import quantize_i8
    rng = np.random.default_rng(11)
    rows = []
    for _ in range(64):
        top = np.float32(rng.uniform(1, 2))
        s = np.float32(np.float64(top) / 127)
        h = ((rng.integers(0, 126, 200) + 0.5) * np.float64(s)).astype(np.float32)
        row = np.concatenate([h, np.nextafter(h, np.float32(0)), np.nextafter(h, np.float32(9)), [top]])
        rows.append(row * rng.choice([-1, 1], row.size).astype(np.float32))
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).cuda()
    _check_codes(x, *quantize_i8(x))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("off,ldx,ldc", [(1, 77, 70), (3, 80, 73), (8, 128, 96)])
def test_quantize_strides(dtype, off, ldx, ldc):
    """Rows inside wider buffers at odd places; what lies between the codes'
    rows stays."""
    from paper_2608_02703_amd import quantize_i8
    M, d = 1030, 61
    buf = torch.randn((M, ldx), dtype=torch.float32).to(DTYPES[dtype]).cuda()
    x = buf.reshape(-1)[off:off + (M - 1) * ldx + d].as_strided((M, d), (ldx, 1))
    cbuf = torch.full((M, ldc), 99, dtype=torch.int8, device="cuda")
    codes, scales = quantize_i8(x, codes=cbuf[:, 3:3 + d])
    _check_codes(x, codes, scales)
    assert (cbuf[:, :3] == 99).all() and (cbuf[:, 3 + d:] == 99).all()


# ------------------------------------------------------------------- product
def _operands(M, N, K, seed, bias, lda=None, ldb=None, off=0):
    rng = np.random.default_rng(seed)
    code = lambda r: rng.integers(-128, 128, (r, K)).astype(np.int8)   # noqa: E731
    a, b = code(M), code(N)
    sa, sb = (np.exp(rng.standard_normal(r)).astype(np.float32) * np.float32(0.01) for r in (M, N))
    bi = (rng.standard_normal(N) * 3).astype(np.float32) if bias else None

    def put(t, ld):
        r = t.shape[0]
        flat = torch.full((off + max(r, 1) * ld + 16,), 77, dtype=torch.int8, device="cuda")
        v = flat[off:].as_strided((r, K), (ld, 1))
        v.copy_(torch.from_numpy(t))
        return v
    ta, tb = put(a, lda or K), put(b, ldb or K)
    up = lambda v: None if v is None else torch.from_numpy(v).cuda()   # noqa: E731
    return (a, sa, b, sb, bi), (ta, up(sa), tb, up(sb), up(bi))


def _check_product(host, out, dtype):
    y, p = oracle.matmul(*host)
    got = _f64(out)
    dt = DTYPES[dtype]
    u = 2.0 ** -24
    tol = (3 * u * np.abs(p) + u * np.abs(y)) * (1 + 2.0 ** -20) + 2.0 ** -140
    if dtype != "f32":
        tol = tol + torch.finfo(dt).eps / 2 * (np.abs(y) + tol) + (2.0 ** -25 if dtype == "f16" else 0)
    big = np.abs(y) + tol >= torch.finfo(dt).max   # (fp16: infinity on either side of its border)
    worst = np.where(big, 0, np.abs(got - y) - tol)
    assert (worst <= 0).all(), f"{(worst > 0).sum()} of {worst.size} off, the worst by {worst.max():.3g}"
    assert (np.abs(got[big]) >= torch.finfo(dt).max * 0.999).all()


def _run_product(M, N, K, dtype, bias, seed=0, **kw):
    from paper_2608_02703_amd import matmul_i8
    host, (a, sa, b, sb, bi) = _operands(M, N, K, seed, bias, **kw)
    out = matmul_i8(a, sa, b, sb, bias=bi, out_dtype=DTYPES[dtype])
    assert out.dtype == DTYPES[dtype] and tuple(out.shape) == (M, N)
    _check_product(host, out, dtype)


MS = [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 200, 256, 257, 333, 600]


@pytest.mark.parametrize("M", MS)
def test_matmul_tokens(M):
    _run_product(M, 519, 256, "f32", False, seed=M)


@pytest.mark.parametrize("M", [1, 3, 16, 40, 130, 300])
@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 15, 16, 17, 63, 65, 127, 128, 129, 255, 257, 1000])
def test_matmul_channels(M, N):
    _run_product(M, N, 192, "bf16", N % 2 == 1, seed=N)


@pytest.mark.parametrize("M", [1, 9, 33, 100, 300])
@pytest.mark.parametrize("K", [1, 2, 15, 16, 17, 32, 48, 63, 64, 65, 80, 100, 112, 127, 128, 129, 144, 255, 256, 272, 384,
                               512, 1000, 1024, 1040, 2048, 4096, 4112, 5003, 8192])
def test_matmul_depths(M, K):
    _run_product(M, 131, K, "f32", True, seed=K)


@pytest.mark.parametrize("M", [1, 7, 64, 300])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("off,lda,ldb", [(0, 144, 160), (1, 129, 131), (4, 132, 128), (16, 256, 128), (8, 128, 136)])
def test_matmul_strides(M, dtype, off, lda, ldb):
    _run_product(M, 300, 128, dtype, True, seed=off, lda=lda, ldb=ldb, off=off)


@pytest.mark.parametrize("M", [1, 33, 300])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("N,ldo,off", [(300, 300, 0), (300, 304, 8), (301, 305, 1), (255, 263, 3)])
def test_matmul_output_rows(M, dtype, N, ldo, off):
    """Outputs inside a wider buffer: what lies around them stays."""
    from paper_2608_02703_amd import matmul_i8
    host, (a, sa, b, sb, bi) = _operands(M, N, 128, 3, True)
    flat = torch.full((off + M * ldo + 64,), -7.0, dtype=DTYPES[dtype], device="cuda")
    out = flat[off:].as_strided((M, N), (ldo, 1))
    assert matmul_i8(a, sa, b, sb, bias=bi, out=out) is out
    _check_product(host, out, dtype)
    mask = torch.ones_like(flat, dtype=torch.bool)
    mask[off:].as_strided((M, N), (ldo, 1)).fill_(False)
    assert (flat[mask] == -7.0).all()


# More tiles than CUs, so that workgroups take several and their loads run on
# from one to the next: every tile height, stages of one tile up to more than are
# in flight, K that ends inside a stage.
@pytest.mark.parametrize("K", [16, 128, 256, 272, 400, 640, 1040])
@pytest.mark.parametrize("M,N", [(40, 70001), (120, 66000), (180, 67003), (250, 66500)])
def test_matmul_many_tiles(M, N, K):
    _run_product(M, N, K, "bf16", True, seed=K)


@pytest.mark.parametrize("M,N,K", [(4100, 5003, 640), (2049, 9001, 1152), (700, 30011, 144)])
def test_matmul_many_tiles_of_many_tokens(M, N, K):
    _run_product(M, N, K, "f16", False, seed=M)


# Several units of channels a wave: one stage to a unit and more, both ring
# depths (the second where a is large)
@pytest.mark.parametrize("M,N,K", [(1, 70001, 16), (3, 70001, 256), (8, 40003, 272), (5, 34005, 528), (16, 33001, 1040),
                                   (7, 33001, 2064), (8, 3001, 8192), (2, 2000, 16384), (16, 5000, 4096), (4, 50257, 1536)])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_matmul_few_tokens(M, N, K, dtype):
    _run_product(M, N, K, dtype, M % 2 == 1, seed=N)


# The same with so many channels that b is streamed in units, where a fills half
# of the LDS and more
@pytest.mark.parametrize("M,N,K", [(8, 17003, 8192), (16, 20003, 4096), (2, 16500, 16384), (1, 16401, 272)])
def test_matmul_few_tokens_long_rows(M, N, K):
    _run_product(M, N, K, "bf16", True, seed=K)


# K split over the waves of a workgroup: shares of no stage up to many, K that
# ends inside a stage, in tiles of 16 and of 32 rows, and tiles of the last XCD only
@pytest.mark.parametrize("K", [16, 112, 128, 144, 896, 1024, 1040, 2064, 14336])
@pytest.mark.parametrize("M,N", [(1, 130), (16, 1000), (5, 4099), (17, 1003), (33, 31), (97, 1325), (256, 515)])
def test_matmul_split_depths(M, N, K):
    _run_product(M, N, K, "bf16", True, seed=M + K)


# The same with rows at any byte, and with too few stages for every wave
@pytest.mark.parametrize("K", [1, 15, 17, 127, 255, 257, 513, 1023, 2049, 5003])
@pytest.mark.parametrize("M,N", [(1, 130), (16, 1000), (5, 4099), (3, 16001), (17, 1003), (33, 31), (97, 1325), (256, 515),
                                 (60, 8190)])
def test_matmul_split_depths_at_any_alignment(M, N, K):
    _run_product(M, N, K, "f16", True, seed=M + K)


# Rows at any byte in large tiles: one stage, two, many
@pytest.mark.parametrize("M,N,K", [(2100, 3001, 333), (700, 9003, 129), (1500, 5001, 1001), (513, 12345, 255)])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_matmul_any_alignment_of_many_tiles(M, N, K, dtype):
    _run_product(M, N, K, dtype, True, seed=M)


# Strided operands and outputs inside a wider buffer, streamed in units, in tiles
# of every height and at any byte
@pytest.mark.parametrize("M,N,K,lda,ldb", [(3, 40003, 144, 160, 192), (40, 40003, 144, 160, 192),
                                           (120, 66001, 128, 144, 160), (180, 67003, 64, 80, 112),
                                           (250, 66001, 128, 176, 128), (700, 9003, 130, 133, 141)])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_matmul_strided_rows_of_many_channels(M, N, K, lda, ldb, dtype):
    from paper_2608_02703_amd import matmul_i8
    host, (a, sa, b, sb, bi) = _operands(M, N, K, M, True, lda=lda, ldb=ldb, off=16)
    ldo, off = N + 5, 3
    flat = torch.full((off + M * ldo + 64,), -7.0, dtype=DTYPES[dtype], device="cuda")
    out = flat[off:].as_strided((M, N), (ldo, 1))
    matmul_i8(a, sa, b, sb, bias=bi, out=out)
    _check_product(host, out, dtype)
    mask = torch.ones_like(flat, dtype=torch.bool)
    mask[off:].as_strided((M, N), (ldo, 1)).fill_(False)
    assert (flat[mask] == -7.0).all()


# As in use: captured with the quantisation, where b is streamed in units and where
# workgroups take several tiles
@pytest.mark.parametrize("M,N", [(4, 30000), (16, 30000), (64, 70000), (200, 70000)])
def test_matmul_of_many_channels_in_a_graph(M, N):
    from paper_2608_02703_amd import matmul_i8, quantize_i8
    K = 256
    wq, ws = quantize_i8(torch.randn((N, K), device="cuda").to(torch.bfloat16))
    x = torch.randn((M, K), device="cuda").to(torch.bfloat16)
    run = lambda: matmul_i8(*quantize_i8(x), wq, ws)   # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(3):
        x.copy_(torch.randn((M, K), device="cuda").to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, run())


# Rows of b, of a or of the output at offsets that pass 32 bits, in every way that
# the product is made
@pytest.mark.parametrize("M,N,K,lda,ldb,ldo", [
    (3, 2100, 128, 128, 1 << 21, 2100), (40, 2100, 128, 128, 1 << 21, 60000000), (3, 17000, 128, 128, 1 << 18, 1100000000),
    (40, 70000, 128, 128, 65536, 60000000), (600, 2100, 128, 1 << 22, 128, 2100), (40, 2100, 100, 100, (1 << 21) + 1, 2100),
    (40, 70001, 100, 60000001, 65537, 60000000), (2000, 4000, 130, 2200001, 131, 4001)])
def test_matmul_far_rows(M, N, K, lda, ldb, ldo):
    from paper_2608_02703_amd import matmul_i8
    rng = np.random.default_rng(M + N)
    host, dev = [], []
    for rows, ld in ((M, lda), (N, ldb)):
        codes = rng.integers(-128, 128, (rows, K)).astype(np.int8)
        scale = (rng.random(rows) * 0.01).astype(np.float32)
        view = torch.empty((rows - 1) * ld + K, dtype=torch.int8, device="cuda").as_strided((rows, K), (ld, 1))
        view.copy_(torch.from_numpy(codes))
        host += [codes, scale]
        dev += [view, torch.from_numpy(scale).cuda()]
    out = torch.empty((M - 1) * ldo + N, dtype=torch.bfloat16, device="cuda").as_strided((M, N), (ldo, 1))
    matmul_i8(*dev, out=out)
    _check_product((*host, None), out, "bf16")


def test_quantize_far_rows():
    from paper_2608_02703_amd import quantize_i8
    for d in (300, 5001):
        ld = 1200000000
        x = torch.empty(2 * ld + d, dtype=torch.float16, device="cuda").as_strided((3, d), (ld, 1))
        x.copy_(torch.randn((3, d)))
        codes = torch.empty(2 * ld + d, dtype=torch.int8, device="cuda").as_strided((3, d), (ld, 1))
        scales = quantize_i8(x, codes=codes)[1]
        _check_codes(x, codes, scales)


@pytest.mark.parametrize("M,N,K", [(1, 20000, 1024), (40, 3000, 4096), (200, 70000, 512), (40, 3000, 4095), (300, 20000, 500)])
def test_two_products_at_once(M, N, K):
    """On two streams, of the same operands and of one operand with itself."""
    from paper_2608_02703_amd import matmul_i8
    _, (a, sa, b, sb, bi) = _operands(M, N, K, 5, True)
    want, own = matmul_i8(a, sa, b, sb, bias=bi), matmul_i8(a, sa, a, sa)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append((matmul_i8(a, sa, b, sb, bias=bi), matmul_i8(a, sa, a, sa)))
    torch.cuda.synchronize()
    for x, y in got:
        assert torch.equal(x, want) and torch.equal(y, own)


@pytest.mark.parametrize("M,N", [(1, 33), (20, 33), (70, 260), (300, 260)])
def test_matmul_largest_sums(M, N):
    """K at its limit with all codes -128: 131071 * 2^14 < 2^31."""
    from paper_2608_02703_amd import matmul_i8
    for K in (131071, 131056):
        a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
        b = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
        b[::2] = 127
        out = matmul_i8(a, torch.ones(M, device="cuda"), b, torch.ones(N, device="cuda"))
        want = torch.full((N,), float(np.float32(K * 16384)))
        want[::2] = float(np.float32(-K * 127 * 128))
        assert torch.equal(out.cpu(), want.expand(M, N))


def test_matmul_empty_and_zero_depth():
    from paper_2608_02703_amd import matmul_i8
    z = lambda *s: torch.zeros(s, dtype=torch.int8, device="cuda")   # noqa: E731
    one = lambda n: torch.ones(n, device="cuda")   # noqa: E731
    assert tuple(matmul_i8(z(0, 64), one(0), z(5, 64), one(5)).shape) == (0, 5)
    assert tuple(matmul_i8(z(5, 64), one(5), z(0, 64), one(0)).shape) == (5, 0)
    bias = torch.randn(7, device="cuda")
    assert torch.equal(matmul_i8(z(3, 0), one(3), z(7, 0), one(7), bias=bias), bias.expand(3, 7))
    assert not matmul_i8(z(3, 0), one(3), z(7, 0), one(7)).any()


def test_matmul_scales_that_are_not_finite_stay_in_their_rows():
    from paper_2608_02703_amd import matmul_i8
    for M in (4, 40, 300):
        host, (a, sa, b, sb, _) = _operands(M, 70, 128, 9, False)
        ref = matmul_i8(a, sa, b, sb)
        sa[2] = float("nan")
        out = matmul_i8(a, sa, b, sb)
        assert torch.isnan(out[2]).all()
        out[2] = ref[2]
        assert torch.equal(out, ref)


@pytest.mark.parametrize("M", [1, 16, 64, 200, 512])
def test_matmul_streams_and_graphs(M):
    """On a side stream, and captured with its quantisation: replays on new
    inputs, eager work between them."""
    from paper_2608_02703_amd import matmul_i8, quantize_i8
    N, K = 1040, 512
    w = torch.randn((N, K), device="cuda").to(torch.bfloat16)
    wq, ws = quantize_i8(w)
    x = torch.randn((M, K), device="cuda").to(torch.bfloat16)
    call = lambda t: matmul_i8(*quantize_i8(t), wq, ws, out_dtype=torch.bfloat16)   # noqa: E731
    ref = call(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call(x)
    side.synchronize()
    assert torch.equal(got, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = call(x)
    for seed in range(4):
        x.copy_(torch.randn((M, K), generator=torch.Generator().manual_seed(seed)))
        g.replay()
        want = call(x)
        torch.cuda.synchronize()
        assert torch.equal(held, want)


@pytest.mark.parametrize("M", [1, 4, 16, 17, 48, 64, 65, 128, 333])
def test_int8_head(M):
    """An INT8 head made of a dense one at the widths of a real head: the whole
    path against the oracle's on the same codes."""
    from paper_2608_02703_amd import matmul_i8, quantize_i8
    V, d = 5003, 2560
    gen = torch.Generator().manual_seed(M)
    w = (torch.randn((V, d), generator=gen) * 0.02).to(torch.bfloat16).cuda()
    x = torch.randn((M, d), generator=gen).to(torch.bfloat16).cuda()
    wq, ws = quantize_i8(w)
    xq, xs = quantize_i8(x)
    _check_codes(x, xq, xs)
    out = matmul_i8(xq, xs, wq, ws)
    _check_product((xq.cpu().numpy(), xs.cpu().numpy(), wq.cpu().numpy(), ws.cpu().numpy(), None), out, "f32")


def test_int8_head_against_the_dense_one():
    """Logits of the INT8 head go to the fidelity metrics: the rounding's error
    is at most half a step of either operand in every product."""
    from paper_2608_02703_amd import logit_fidelity, matmul_i8, quantize_i8
    gen = torch.Generator().manual_seed(1)
    w = (torch.randn((4096, 512), generator=gen) * 0.05).cuda()
    x = torch.randn((9, 512), generator=gen).cuda()
    wq, ws = quantize_i8(w)
    xq, xs = quantize_i8(x)
    ref = x @ w.T
    test = matmul_i8(xq, xs, wq, ws)
    kl, sq, ref_idx, rank = logit_fidelity(ref, test)
    bound = (xs[:, None] / 2 * w.abs().sum(1) + ws / 2 * (xq.float().abs() * xs[:, None]).sum(1)[:, None]).square().sum(1)
    assert (sq <= bound * 1.01).all() and torch.isfinite(kl).all()
    assert torch.equal(ref_idx, ref.argmax(1))


def test_refuses_mismatched_tensors():
    from paper_2608_02703_amd import matmul_i8, quantize_i8
    q = torch.zeros((4, 64), dtype=torch.int8, device="cuda")
    s = torch.ones(4, device="cuda")
    for bad in (lambda: matmul_i8(q, s[:3], q, s), lambda: matmul_i8(q, s, q[:, :32], s),
                lambda: matmul_i8(q, s, q, s, bias=s[:2]), lambda: matmul_i8(q, s, q.t(), s),
                lambda: matmul_i8(q, s, q, s, out=torch.empty((4, 5), device="cuda")),
                lambda: quantize_i8(torch.zeros(64, device="cuda")),
                lambda: quantize_i8(torch.zeros((4, 64), device="cuda"), codes=q[:, :32])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: matmul_i8(q.float(), s, q, s), lambda: matmul_i8(q, s.double(), q, s),
                lambda: matmul_i8(q, s, q, s, out_dtype=torch.float64), lambda: quantize_i8(q),
                lambda: matmul_i8(q, s, q, s, out=torch.empty((4, 4), device="cuda"), out_dtype=torch.bfloat16)):
        with pytest.raises(TypeError):
            bad()
