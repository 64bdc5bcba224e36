"""rms_norm and rms_norm_i8 at eps so small that 1 / n leaves fp32's range."""
from __future__ import annotations

import pytest

from tests.test_gpu_norm import DTYPES, _check

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("d", [5, 64, 256, 257, 1000, 4099])
@pytest.mark.parametrize("eps", [1e-20, 1e-60, 1e-61, 1e-76, 1e-78, 1e-90, 1e-150, 5e-324])
def test_rows_of_zeros_and_smallest_numbers(dtype, d, eps):
    """out = t / n to its bits where n is below fp32's numbers; a row of zeros gives zeros, codes 0 and
    a finite scale."""
    from paper_2608_02703_amd import rms_norm, rms_norm_i8
    dt = DTYPES[dtype]
    step = torch.finfo(dt).tiny * torch.finfo(dt).eps   # the smallest number
    gen = torch.Generator().manual_seed(d)
    rows = [torch.zeros(d, dtype=torch.float64) for _ in range(4)]
    rows[1][d // 2] = step
    rows += [k * torch.randint(-9, 10, (d,), generator=gen).double() * step for k in (1, 3000)]
    rows += [torch.randn(d, generator=gen).double() * k for k in (1e-30, 1.0)]
    rows[2][d - 1] = -0.0
    x = torch.stack(rows).to(dt).cuda()
    w = torch.randn(d, generator=gen).to(dt).cuda()
    zero = [r for r in range(len(rows)) if not x[r].any()]
    some = [r for r in range(len(rows)) if r not in zero]
    codes, scales, out = rms_norm_i8(x, w, eps=eps, normed=True)
    _check(x[some], w, eps, None, 0.0, codes[some], scales[some], None, out[some])
    assert not out[zero].any() and not codes[zero].any() and torch.isfinite(scales).all() and (scales > 0).all()
    assert torch.equal(rms_norm(x, w, eps=eps), out)


@pytest.mark.parametrize("w", [1e30, 3e38])
def test_large_weights_of_smallest_rows(w):
    """t = s w reaches far above s, and so does out."""
    from paper_2608_02703_amd import rms_norm_i8
    x = torch.full((3, 300), 2.0 ** -149, device="cuda")
    x[1, ::2] *= -5
    x[2] *= 2.0 ** 60
    weight = torch.full((300,), w, device="cuda")
    weight[::3] = 1.0
    for eps in (1e-300, 1e-89):
        codes, scales, out = rms_norm_i8(x, weight, eps=eps, normed=True)
        _check(x, weight, eps, None, 0.0, codes, scales, None, out)
