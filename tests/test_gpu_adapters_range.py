"""adapters_add with inner sums at the end of fp32 and beyond."""
from __future__ import annotations

import pytest

from tests.test_gpu_adapters import TYPES, _check, _inputs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


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
