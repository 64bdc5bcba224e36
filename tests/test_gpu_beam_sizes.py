"""beam_select over rows of the type's lowest value and logits whose
scores coincide, against the formula in 64
bits and the oracle under the bounds of test_gpu_beam.py."""
from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_beam import DTYPES, _case, check

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _score(lg, cum):
    """fp64 scores of one beam, with the distance to the row's largest first."""
    lg = lg.astype(np.float64)
    d = lg - lg.max()
    return cum + (d - np.log(np.exp(d).sum()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 40, 6000, 70000])
def test_rows_of_the_lowest_value(V, dtype):
    """A mask of the type's lowest value that leaves nothing: every token is as
    likely as any other, and the row's logsumexp is log V away from it, which is
    lost in a difference of numbers of its size."""
    from paper_2608_02703_amd import beam_select
    low = torch.finfo(DTYPES[dtype]).min
    lg, scores = _case(1, 4, V, dtype, V)
    lg = lg.clone()
    lg[1] = low
    lg[2] = low
    lg[2, V - 2:] = low / 2
    scores[:] = torch.tensor([-0.5, -0.25, -0.125, -3.0])
    n = 16
    got = beam_select(lg, scores, n)
    host = lg.cpu().to(torch.float64).numpy()
    s = np.stack([_score(host[k], float(scores[0, k])) for k in range(4)]).reshape(-1)
    order = np.lexsort((np.arange(s.size), -s))[:n]
    assert np.array_equal((got[1] * V + got[2])[0].cpu().numpy(), order)
    # (the bound of the file with the checks: 2^-23 D + 2^-22 + 31 2^-24 of a logsumexp with D below log V)
    bound = 2.0 ** -23 * np.log(V) + 2.0 ** -22 + 31 * 2.0 ** -24
    v = got[0][0].cpu().numpy().astype(np.float64)
    assert (np.abs(v - s[order]) <= bound + 2.0 ** -24 * np.abs(s[order]) * 1.001).all()
    check(lg, scores, n, got)


def test_logits_that_differ_by_less_than_a_score_shows():
    """Scores are fp64: logits of one beam whose scores coincide there go by
    their tokens."""
    from paper_2608_02703_amd import beam_select
    lg = torch.full((2, 9000), -3.0, device="cuda")
    lg[:, 100], lg[:, 4000], lg[:, 8000] = 1e-18, 3e-18, -1e-18
    lg[:, 6000] = 1.0
    scores = torch.tensor([[-1.25, -1.5]], device="cuda")
    _, parents, tokens = beam_select(lg, scores, 8)
    assert parents[0].tolist() == [0, 1, 0, 0, 0, 1, 1, 1]
    assert tokens[0].tolist() == [6000, 6000, 100, 4000, 8000, 100, 4000, 8000]
