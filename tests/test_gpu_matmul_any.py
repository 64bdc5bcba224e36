"""matmul_i8 for rows at any byte with more than one tile of 64 x 64 to a compute
unit and too few of 128 x 128 (those and other sizes are in
test_gpu_matmul_i8.py, whose bounds these are): several stages of 128 k, K that
ends inside one or at its first byte, every output type, bias, odd rows."""
from __future__ import annotations

import pytest

from tests.test_gpu_matmul_i8 import DTYPES, _check_product, _operands

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("M,N,K", [(1, 50000, 1001), (16, 33001, 257), (100, 30000, 129), (65, 16500, 333), (64, 17001, 255),
                                   (130, 12003, 384)])
def test_tiles_of_64(M, N, K, dtype):
    from paper_2608_02703_amd import matmul_i8
    host, (a, sa, b, sb, bi) = _operands(M, N, K, K, True, lda=K + 2, ldb=K + 5, off=3)
    ldo, off = N + 3, 1
    flat = torch.full((off + M * ldo + 64,), -7.0, dtype=DTYPES[dtype], device="cuda")
    out = flat[off:].as_strided((M, N), (ldo, 1))
    matmul_i8(a, sa, b, sb, bias=bi, out=out)
    _check_product(host, out, dtype)
    mask = torch.ones_like(flat, dtype=torch.bool)
    mask[off:].as_strided((M, N), (ldo, 1)).fill_(False)
    assert (flat[mask] == -7.0).all()
    host, dev = (*host[:4], None), (a, sa, b, sb)
    _check_product(host, matmul_i8(*dev, out_dtype=DTYPES[dtype]), dtype)
