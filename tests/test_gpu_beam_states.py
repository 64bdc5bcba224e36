"""What BeamStates takes and refuses of tensors in the same memory."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def test_refuses_destinations_that_overlap_in_part():
    from paper_2608_02703_amd import BeamStates
    t = torch.zeros((12, 5, 16), device="cuda")
    s = torch.zeros((8, 5, 16), device="cuda")
    for bad in (lambda: BeamStates([t[:8], t[4:12]], 4), lambda: BeamStates([t[..., :8], t[..., 7:]], 4),
                lambda: BeamStates([t, t[:, 4:]], 4, pos_dim=1), lambda: BeamStates([t[:4], t[8:], t[4:][:4], t[7:11]], 4),
                lambda: BeamStates([s, s], 4, [t[:8], t[4:]])):
        with pytest.raises(ValueError, match="destinations share memory"):
            bad()


@pytest.mark.parametrize("in_place", [False, True])
def test_takes_states_that_lie_among_each_other(in_place):
    """Keys and values, layers, and states of unlike width of one buffer."""
    from paper_2608_02703_amd import BeamStates
    B, K, L, H, T, D = 2, 3, 4, 2, 9, 8
    gen = torch.Generator().manual_seed(1)
    a = torch.randn((B * K, L, 2, H, T, D), generator=gen).cuda()
    b = torch.randn((B * K, 40), generator=gen).cuda()
    views = lambda a, b: [a[:, i, j] for i in range(L) for j in range(2)], lambda a, b: [b[:, :7], b[:, 7:9], b[:, 9:]]   # noqa: E731
    q = torch.tensor([[2, 0, 0], [1, 1, 0]], device="cuda")
    rows = (q + K * torch.arange(B, device="cuda")[:, None]).view(-1)
    for view in views:
        x, y = a.clone(), b.clone()
        u, v = torch.zeros_like(x), torch.zeros_like(y)
        BeamStates(view(x, y), K, None if in_place else view(u, v)).reorder(q)
        new = (x, y) if in_place else (u, v)
        for got, old in zip(view(*new), view(a, b)):
            assert torch.equal(got, old[rows])


def test_takes_two_buffers_that_lie_among_each_other():
    """A cache whose rows hold the states before and after a step; sources may
    be the same memory."""
    from paper_2608_02703_amd import BeamStates
    K = 4
    both = torch.randn((2 * K, 2, 5, 16), generator=torch.Generator().manual_seed(2)).cuda()
    old = both.clone()
    q = torch.tensor([[3, 0, 3, 1], [2, 2, 1, 0]], device="cuda")
    rows = (q + K * torch.arange(2, device="cuda")[:, None]).view(-1)
    BeamStates([both[:, 0]], K, [both[:, 1]]).reorder(q)
    assert torch.equal(both[:, 1], old[rows, 0]) and torch.equal(both[:, 0], old[:, 0])
    out = [torch.zeros((2 * K, 5, 16), device="cuda") for _ in range(2)]
    for got in BeamStates([both[:, 0]] * 2, K, out).reorder(q):
        assert torch.equal(got, old[rows, 0])
    for bad in (lambda: BeamStates([both[:, 0]], K, [both[:, 0]]), lambda: BeamStates([both[:, 0, 1:]], K, [both[:, 0, :4]]),
                lambda: BeamStates([out[0], both[:, 0]], K, [both[:, 1], out[0]])):
        with pytest.raises(ValueError, match="out shares memory"):
            bad()
