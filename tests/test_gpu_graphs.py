"""The packed head's calls captured into HIP graphs: every replay gives what an
eager call gives for the inputs as they are then, bit for bit, on every kernel,
with eager work between the replays, two graphs in one workspace, and where the
waves that need t = x V_c^T, x B_w^T never wait for it (then each computes what
has not arrived, in another order of its sum, so the logits' tolerance of
gpu_util applies)."""
from __future__ import annotations

import pytest

from synth import make_head
from tests.gpu_util import LOGIT_TOL, say

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

PATHS = [("gemv", 1), ("gemv", 6), ("dec", 8), ("dec", 40), ("mid", 24), ("mid", 45), ("tiled", 24), ("tiled", 200)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.fixture(scope="module")
def head():
    from paper_2608_02703_amd import PackedHead
    ph = PackedHead.from_arrays(make_head("tiny"))
    yield ph
    ph.close()


@pytest.fixture(autouse=True)
def _reset(head):
    from paper_2608_02703_amd import archead as ab
    yield
    head.force_path("auto")
    head.set_launch(ab.LAUNCH_T_SPIN_LIMIT, -1)


def _x(M, seed):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn((M, 512), generator=gen) * (1 + seed % 3)).to(torch.bfloat16).cuda()


def _capture(call, pool=None):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, pool=pool):
        held = call()
    return g, held


def _replays(call, x, same):
    g, held = _capture(call)
    for seed in range(1, 6):
        x.copy_(_x(x.shape[0], seed))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = call()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert same(a, b), seed


def _equal(a, b):
    return torch.equal(a, b)


def _close(a, b):
    return bool(((a - b).abs() <= 2 * LOGIT_TOL * (1 + b.abs())).all())


@pytest.mark.parametrize("path,M", PATHS)
def test_logits(head, path, M):
    head.force_path(path)
    x = _x(M, 0)
    say(f"{path} M={M}")
    _replays(lambda: [head.logits(x)], x, _equal)


@pytest.mark.parametrize("path,M", PATHS[:6])
def test_logits_whose_waves_do_not_wait(head, path, M):
    from paper_2608_02703_amd import archead as ab
    head.force_path(path)
    head.set_launch(ab.LAUNCH_T_SPIN_LIMIT, 0)
    x = _x(M, 0)
    _replays(lambda: [head.logits(x)], x, _close)


@pytest.mark.parametrize("path,M", PATHS)
def test_cross_entropy_and_argmax(head, path, M):
    head.force_path(path)
    x = _x(M, 0)
    y = torch.arange(M, device="cuda") * 37 % 8192
    _replays(lambda: [*head.logits_ce(x, y), *head.logits_argmax(x)], x, _equal)


@pytest.mark.parametrize("M,k", [(1, 4), (1, 20), (8, 10), (300, 7)])
def test_topk(head, M, k):
    x = _x(M, 0)
    _replays(lambda: [*head.logits_topk(x, k)], x, _equal)


@pytest.mark.parametrize("M", [1, 5, 24, 200])
def test_without_a_workspace(head, M):
    x = _x(M, 0)
    out = torch.empty((M, 8192), device="cuda")
    g, _ = _capture(lambda: head.logits_noalloc(x, out=out))
    for seed in range(1, 5):
        x.copy_(_x(M, seed))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, head.logits(x))


@pytest.mark.parametrize("B,K,n", [(1, 1, 4), (1, 4, 8), (2, 8, 8), (12, 4, 4)])
def test_logits_beam(head, B, K, n):
    x = _x(B * K, 0)
    scores = -torch.rand((B, K), generator=torch.Generator().manual_seed(n)).cuda()
    fin = torch.zeros((B, K), dtype=torch.bool, device="cuda")
    fin[0, -1] = K > 1
    _replays(lambda: [*head.logits_beam(x, scores, n, finished=fin, end_token=3)], x, _equal)


@pytest.mark.parametrize("path,M", [("gemv", 1), ("dec", 8), ("mid", 24)])
def test_two_graphs_of_one_workspace(head, path, M):
    head.force_path(path)
    ws = torch.empty(head.workspace_bytes(M), dtype=torch.uint8, device="cuda")
    xs = [_x(M, i) for i in range(2)]
    graphs = [_capture(lambda x=x: head.logits(x, ws=ws)) for x in xs]
    for seed in range(1, 5):
        for i, (g, held) in enumerate(graphs):
            xs[i].copy_(_x(M, 10 * seed + i))
            g.replay()
            torch.cuda.synchronize()
            got = held.clone()
            assert torch.equal(got, head.logits(xs[i]))


@pytest.mark.parametrize("M", [1, 70, 300])
def test_fidelity_to_a_dense_head(head, M):
    gen = torch.Generator().manual_seed(M)
    dense = (torch.randn((8192, 512), generator=gen) * 0.05).to(torch.bfloat16).cuda()
    x = _x(M, 0)
    _replays(lambda: [*head.logit_fidelity_head(x, dense)], x, _equal)
