"""adapters_add where the inner sums of one token are of very different size, at
the end of fp32 and beyond."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import adapters as oracle
from tests.test_gpu_adapters import TYPES, _check, _inputs, _np

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,y", TYPES)
@pytest.mark.parametrize("M,R,n,ragged", [(20, 8, 2, False), (20, 5, 2, False), (70, 16, 3, False), (70, 40, 2, True),
                                          (300, 64, 2, False), (2100, 200, 3, True)])
def test_ranks_of_different_size(M, R, n, ragged, dtype, y):
    """Rows of a from 2^12 down to 2^-20, and each output of one rank alone: every inner sum keeps its
    own bits, however large the token's others are."""
    from paper_2608_02703_amd import adapters_add
    N, K = 2 * R + 3, 72
    i = _inputs(M, N, K, R, n, dtype, y, seed=M + R, ragged=ragged)
    i["y"].zero_()
    a = torch.randn((n, R, K), generator=torch.Generator().manual_seed(R))
    i["a"] = (a * torch.exp2(12 - 32 * (torch.arange(R) * 5 % R) / max(R - 1, 1))[:, None]).to(i["x"].dtype).cuda()
    at = torch.arange(N, device="cuda")
    i["b"][:] = 0
    i["b"][:, at, at % R] = (1 + at / N).to(i["x"].dtype)
    if y == "f16":
        i["scales"] = torch.tensor([0.5, -0.25, 0.125], device="cuda")[:n]
    out = adapters_add(**i)
    if y == "f16":   # outputs with a sum beyond its range
        want, _ = oracle.add(*(_np(i[k]) for k in ("y", "x", "a", "b")), i["ids"].cpu().numpy(), _np(i["scales"]),
                             i["ranks"].cpu().numpy() if ragged else None)
        far = torch.from_numpy(np.abs(want) >= 65504).cuda()
        assert (out.abs()[far] >= 65504 - 32).all()
        fits = ~far.any(0)
        assert fits.sum() >= N // 2
        i["y"], i["b"], out = i["y"][:, fits], i["b"][:, fits], out[:, fits]
    _check(i, out)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_inner_sums_at_the_end_of_fp32(dtype, y):
    """(2 - 2^-12) 2^127, which the operands' type would round to infinity: times 2^-7 it is finite."""
    from paper_2608_02703_amd import adapters_add
    i = _inputs(20, 70, 64, 40, 3, dtype, y, seed=9, none=0.0)
    i["y"].zero_()
    i["x"].zero_()
    i["x"][:, :2] = 1
    i["a"].zero_()
    up = 15 if dtype == "f16" else 127
    i["a"][:, :3, 0] = (2 - 2.0 ** -7) * 2.0 ** up
    i["a"][:, :3, 1] = (2.0 ** -7 - 2.0 ** -12) * 2.0 ** up
    i["scales"] = torch.tensor([1.0, -1.0, 0.5], device="cuda") * 2.0 ** (127 - up)
    i["b"] = i["b"].clamp(-1, 1) / 128
    out = adapters_add(**i)
    assert torch.isfinite(out).all()
    _check(i, out)


@pytest.mark.parametrize("dtype,y", TYPES)
def test_infinite_inner_sums(dtype, y):
    """They go on as infinities of their sign, whatever bits b has."""
    from paper_2608_02703_amd import adapters_add
    i = _inputs(30, 64, 40, 8, 2, dtype, y, seed=3, none=0.0, scales=False)
    i["x"][:, 3] = 0
    i["x"][4:8, 3] = torch.tensor([1, -1, 1, -1], device="cuda") * float("inf")
    i["a"][:, :, 3] = 1
    i["b"][:] = i["b"][:, :, :1]   # of one sign over the ranks
    i["b"][:, ::7] = 0.25          # one bit
    out = adapters_add(**i).float()
    b = i["b"][i["ids"].long(), :, 0].float()
    assert (b != 0).all()
    assert torch.equal(out[4:8], torch.sign(b[4:8]) * i["x"][4:8, 3:4].float())
    out[4:8] = 0
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("dtype,y", [("f16", "f32"), ("f16", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("R", [7, 20, 64, 100])
def test_some_adapters_of_different_ranks(R, dtype, y):
    """Enough tokens and outputs for several tiles at a time, of which those of one adapter have ranks
    of very different size."""
    from paper_2608_02703_amd import adapters_add
    M, N, K, n = 1100, 30601, 40, 3
    i = _inputs(M, N, K, R, n, dtype, y, seed=R, ragged=R == 20)
    i["ids"][:M // 2] = i["ids"][:M // 2].sort().values
    i["y"].zero_()
    i["a"][1, ::2] = (i["a"][1, ::2].double() * 2.0 ** -20).to(i["a"].dtype)
    i["b"][1, ::5, 1::2] = 0
    _check(i, adapters_add(**i))


@pytest.mark.parametrize("dtype,y", TYPES)
def test_infinite_factors(dtype, y):
    """An infinity in b stays in its row of outputs and in its adapter's tokens."""
    from paper_2608_02703_amd import adapters_add
    i = _inputs(40, 70, 64, 12, 3, dtype, y, seed=4)
    want = adapters_add(**i)
    i["b"][1, 17, 3] = float("inf")
    out = adapters_add(**i)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[i["ids"] == 1, 17] = True
    assert not torch.isfinite(out[hit]).any() and torch.equal(out[~hit], want[~hit])


@pytest.mark.parametrize("dtype,y", [("f16", "f32"), ("f16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("span", [6, 10, 13, 16, 20])
@pytest.mark.parametrize("R", [16, 50])
def test_ranks_within_a_span(R, span, dtype, y):
    """Rows of a over 2^-6 to 2^-20, below and above where fp16's parts end, outputs of one rank alone."""
    from paper_2608_02703_amd import adapters_add
    M, N, K, n = 400, 3 * R, 256, 3
    i = _inputs(M, N, K, R, n, dtype, y, seed=span)
    i["y"].zero_()
    i["a"] = (i["a"].double() * torch.exp2(-span * (torch.arange(R, device="cuda") * 7 % R) / (R - 1))[:, None]).to(i["a"].dtype)
    at = torch.arange(N, device="cuda")
    i["b"][:] = 0
    i["b"][:, at, at % R] = (1 + at / N).to(i["b"].dtype)
    _check(i, adapters_add(**i))
