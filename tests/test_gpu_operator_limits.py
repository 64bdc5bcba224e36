"""The INT8 products, the rounding and the beam selection at the largest sizes that
they take, against the formulas in 64 bits on the GPU, some rows at a time."""
from __future__ import annotations

import math

import pytest

from tests.gpu_util import say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

MOST = 2 ** 31 - 1   # elements of a row, rows, tokens of a vocabulary


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _parts(n, step=1 << 26):
    return [slice(i, min(i + step, n)) for i in range(0, n, step)]


def test_quantize_the_longest_row():
    from paper_2608_02703_amd import quantize_i8
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, MOST), generator=gen, device="cuda", dtype=torch.bfloat16)
    x[0, MOST - 1] = -50.0
    say("quantize 1 x 2^31 - 1")
    codes, scales = quantize_i8(x)
    torch.cuda.synchronize()
    s = torch.tensor(50.0 / 127, dtype=torch.float64).float()
    assert scales.cpu().item() == s.item()
    for p in _parts(MOST):
        assert torch.equal(codes[0, p], torch.round(x[0, p].double() / s.double().item()).to(torch.int8)), p


def test_matmul_of_the_most_channels():
    """K = 1: every output is one product, three roundings to fp32 at most of it
    (of exactly known operands: the same operations in fp32) and one to bf16."""
    from paper_2608_02703_amd import matmul_i8
    gen = torch.Generator(device="cuda").manual_seed(2)
    b = torch.randint(-128, 128, (MOST, 1), generator=gen, device="cuda", dtype=torch.int8)
    sb = torch.rand(MOST, generator=gen, device="cuda")
    a = torch.tensor([[-77]], dtype=torch.int8, device="cuda")
    sa = torch.tensor([0.375], device="cuda")
    say("matmul 1 x 2^31 - 1 x 1")
    out = matmul_i8(a, sa, b, sb, out_dtype=torch.bfloat16)
    torch.cuda.synchronize()
    for p in _parts(MOST):   # (an integer times 0.375 is exact in fp32, the fma with no bias rounds once)
        want = (b[p, 0].double() * (-77 * 0.375) * sb[p].double()).float().to(torch.bfloat16)
        assert torch.equal(out[0, p], want), p


def test_select_from_the_largest_vocabulary():
    from paper_2608_02703_amd import beam_select
    lg = torch.full((2, MOST), -5.0, dtype=torch.bfloat16, device="cuda")
    at = [[MOST - 1, 7, 2 ** 30 + 13], [MOST - 2, 0, 2 ** 31 - 4096]]
    up = [[20.0, 18.0, 16.0], [21.0, 19.5, 17.0]]
    for k in range(2):
        for v, u in zip(at[k], up[k]):
            lg[k, v] = u
    scores = torch.tensor([[-1.0, -1.5]], device="cuda")
    say("select from 2 x 2^31 - 1")
    out, parents, tokens = beam_select(lg, scores, 8)
    torch.cuda.synchronize()
    want = []
    for k, c in enumerate((-1.0, -1.5)):
        top = max(up[k])
        s = sum(math.exp(u - top) for u in up[k]) + (MOST - 3) * math.exp(-5.0 - top)
        want += [(c - math.log(s) + (u - top), k, v) for u, v in zip(up[k], at[k])]
        # of the rest, all equal, the lowest tokens
        want += [(c - math.log(s) + (-5.0 - top), k, v) for v in range(10) if v not in at[k]]
    want.sort(key=lambda w: (-w[0], w[1], w[2]))
    assert parents[0].tolist() == [w[1] for w in want[:8]]
    assert tokens[0].tolist() == [w[2] for w in want[:8]]
    # 2^-23 D + 2^-22 + 31 2^-24 of a logsumexp, D = sum p |l - max| below log V, and the scores' own rounding
    bound = 2.0 ** -23 * math.log(MOST) + 2.0 ** -22 + 31 * 2.0 ** -24
    for got, w in zip(out[0].tolist(), want):
        assert abs(got - w[0]) <= bound + 2.0 ** -24 * abs(w[0]) * 1.001
