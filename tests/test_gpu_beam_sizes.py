"""beam_select and PackedHead.logits_beam over many beams and large vocabularies
(more chunks and spans than a thread of the choice keeps), rows of the type's
lowest value, and BeamStates of very many blocks and sequences, against the
oracle under the bounds of test_gpu_beam.py."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import beam as oracle
from tests.test_gpu_beam import DTYPES, _case, check

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


# chunks of 512 logits: above 4096 of a sequence they are read twice; above 256
# spans of 2048 a row, so are their sums
LARGE = [(1, 16, 140001), (1, 32, 70001), (2, 9, 262143), (1, 2, 524391), (1, 5, 600001), (1, 1, 2200000)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("B,K,V", LARGE)
def test_select_of_many_chunks(B, K, V, dtype):
    """The best pairs anywhere, in the last chunks and in the last spans."""
    from paper_2608_02703_amd import beam_select
    lg, scores = _case(B, K, V, dtype, V)
    check(lg, scores, 2 * K, beam_select(lg, scores, 2 * K))
    lg = lg.clone()
    scores = scores / 100
    lg[K - 1::K, V - 70:] += 12       # the last beam's last chunk
    lg[K - 1::K, -1500] += 13
    lg[:, 524288 if V > 524289 else V // 2] += 12
    for n in (1, 16, 64):
        check(lg, scores, n, beam_select(lg, scores, n))
    allowed = torch.rand(V, generator=torch.Generator().manual_seed(K)) < 0.7   # bans, an ended beam, one not in use
    lg.masked_fill_(~allowed.cuda(), -float("inf"))
    fin = torch.zeros((B, K), dtype=torch.bool, device="cuda")
    fin[:, 0] = K > 1
    if K > 2:
        scores[0, 1] = -float("inf")
    got = beam_select(lg, scores, 32, finished=fin, end_token=V - 3)
    check(lg, scores, 32, got, finished=fin, end_token=V - 3)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("B,K,V", LARGE)
def test_select_ties_of_many_chunks(B, K, V, dtype):
    """Equal scores on both sides of what a thread keeps, few and very many."""
    from paper_2608_02703_amd import beam_select
    scores = torch.full((B, K), -1.25, device="cuda")
    lg = torch.zeros((B * K, V), dtype=DTYPES[dtype], device="cuda")
    check(lg, scores, 8, beam_select(lg, scores, 8), exact=True)
    at = torch.arange(7, V, V // 9)   # a few in every row
    lg[:, at.cuda()] = 3.0
    check(lg, scores, 64, beam_select(lg, scores, 64), exact=True)
    lg[: (K - 1), at.cuda()] = 0      # of the first sequence, those of its last beam alone
    check(lg, scores, 16, beam_select(lg, scores, 16), exact=True)


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


@pytest.mark.parametrize("V", [151936, 262144])
@pytest.mark.parametrize("B,K,n", [(1, 4, 8), (4, 8, 16), (16, 16, 16)])
def test_logits_beam_of_large_vocabularies(V, B, K, n):
    from paper_2608_02703_amd import PackedHead, beam_select
    from synth import make_head, make_x
    from tests.gpu_util import torch_x
    ph = PackedHead.from_arrays(_large_head(V))
    try:
        x = torch_x(make_x("tiny", B * K))
        scores = -torch.rand((B, K), generator=torch.Generator().manual_seed(n)).cuda()
        fin = torch.zeros((B, K), dtype=torch.bool, device="cuda")
        fin[0, -1] = True
        lg = ph.logits(x)
        got = ph.logits_beam(x, scores, n, finished=fin, end_token=V - 1)
        want = beam_select(lg, scores, n, finished=fin, end_token=V - 1)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        few = min(B, 2)   # (the oracle over the first sequences)
        check(lg[:few * K], scores[:few], n, [t[:few] for t in got], finished=fin[:few], end_token=V - 1)
    finally:
        ph.close()


_HEADS = {}


def _large_head(V):
    from synth import make_head
    if V not in _HEADS:
        _HEADS.clear()
        _HEADS[V] = make_head("tiny", V=V)
    return _HEADS[V]


# more blocks of a row, and more sequences, than a launch has in one dimension
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,K,shape,p", [(1, 4, (70001, 3, 16), 2), (40000, 2, (2, 5), 1), (33000, 3, (7,), None)])
def test_reorder_of_very_many_blocks(B, K, shape, p, in_place):
    from paper_2608_02703_amd import BeamStates
    gen = torch.Generator().manual_seed(B)
    states = [torch.randint(-99, 99, (B * K, *shape), generator=gen, dtype=torch.int8).cuda() for _ in range(2)]
    out = None if in_place else [torch.full_like(s, 5) for s in states]
    q = torch.randint(0, K, (B, K), generator=gen).cuda()
    rows = (q + K * torch.arange(B, device="cuda")[:, None]).view(-1)
    want = [s[rows] for s in states]
    got = BeamStates(states, K, out, pos_dim=p).reorder(q)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    some = oracle.reorder(states[0][:2 * K].cpu().numpy(), states[0][:2 * K].cpu().numpy(), q[:2].cpu().numpy(), K) \
        if not in_place and B > 1 else None
    assert some is None or np.array_equal(got[0][:2 * K].cpu().numpy(), some)
