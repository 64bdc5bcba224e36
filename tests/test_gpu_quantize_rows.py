"""quantize_i8 at the ends of its range: scales whose half is no fp32 number,
rows in four groups a thread and longer, more rows than a launch has groups of
threads for.  Codes and scales have to be the oracle's bit for bit."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import int8 as oracle
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _check(x, codes, scales, step=1 << 22):
    """Against the oracle, some rows at a time."""
    rows = max(step // x.shape[1], 1)
    for m in range(0, x.shape[0], rows):
        q, s = oracle.quantize(x[m:m + rows].cpu().to(torch.float64).numpy())
        assert np.array_equal(scales[m:m + rows].cpu().numpy(), s, equal_nan=True), m
        assert np.array_equal(codes[m:m + rows].cpu().numpy(), q), m


@pytest.mark.parametrize("d", [130, 700])
def test_scales_whose_half_is_no_number(d):
    """Scales in [2^-126, 2^-125) are multiples of 2^-149, the odd ones' halves
    are not: elements next to such halves."""
    from paper_2608_02703_amd import quantize_i8
    rng = np.random.default_rng(d)
    rows, odd = [], 0
    for _ in range(400):
        top = np.float32(127 * 2.0 ** -126 * rng.uniform(1, 2))
        s = int(float(np.float32(np.float64(top) / 127)) * 2.0 ** 149)
        odd += s % 2
        n = rng.integers(0, 127, d - 1) * s + s // 2 + rng.integers(-1, 3, d - 1)
        rows.append(np.append(n * 2.0 ** -149 * rng.choice([-1, 1], d - 1), float(top)).astype(np.float32))
    assert odd > 100
    x = torch.from_numpy(np.stack(rows)).cuda()
    _check(x, *quantize_i8(x))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_smallest_scales(dtype):
    """Rows whose largest element runs from nothing to 2^-115."""
    from paper_2608_02703_amd import quantize_i8
    gen = torch.Generator().manual_seed(7)
    size = 2.0 ** -(149 - 34 * torch.rand((2000, 1), generator=gen, dtype=torch.float64))
    x = ((torch.rand((2000, 300), generator=gen, dtype=torch.float64) * 2 - 1) * size).to(DTYPES[dtype]).cuda()
    _check(x, *quantize_i8(x))


# 2^25 elements and more in rows longer than 512: an odd length just above it, one
# that is no multiple of a thread's groups, one that is read again in part
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("M,d", [(65537, 513), (8193, 4099), (840, 40003)])
def test_many_elements(M, d, dtype):
    from paper_2608_02703_amd import quantize_i8
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((M, d), generator=gen, device="cuda") * torch.exp(torch.randn((M, 1), generator=gen, device="cuda"))
    x = x.to(DTYPES[dtype])
    x[M // 2, d - 1] = float("nan")
    x[M - 1] = 0
    _check(x, *quantize_i8(x))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_many_elements_inside_wider_rows(dtype):
    from paper_2608_02703_amd import quantize_i8
    M, d, ldx, ldc = 33000, 1019, 1031, 1025
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((M, ldx), generator=gen, device="cuda").to(DTYPES[dtype])[:, 5:5 + d]
    buf = torch.full((M, ldc), 99, dtype=torch.int8, device="cuda")
    codes, scales = quantize_i8(x, codes=buf[:, 3:3 + d])
    _check(x, codes, scales)
    assert (buf[:, :3] == 99).all() and (buf[:, 3 + d:] == 99).all()


# more rows than a launch has groups of threads: a workgroup to a row, 16 lanes to one
@pytest.mark.parametrize("M,d", [((1 << 21) + 3, 2057), ((1 << 25) + 21, 11)])
def test_more_rows_than_groups(M, d):
    from paper_2608_02703_amd import quantize_i8
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((M, d), generator=gen, device="cuda", dtype=torch.bfloat16)
    say(f"{M} rows of {d}")
    codes, scales = quantize_i8(x)
    torch.cuda.synchronize()
    few = 1000
    for m in (0, M - few):   # the oracle's
        _check(x[m:m + few], codes[m:m + few], scales[m:m + few])
    step = (1 << 26) // d
    for m in range(0, M, step):   # and the same formulas in 64 bits there
        v = x[m:m + step].double()
        s = (v.abs().amax(1) / 127).float()
        assert torch.equal(scales[m:m + step], s), m
        assert torch.equal(codes[m:m + step], torch.round(v / s.double()[:, None]).to(torch.int8)), m
