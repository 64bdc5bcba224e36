"""head_loss and head_loss_grad where logits are far from zero: near-certain
targets, and finite logits up to the ends of fp32.

The inputs make every logit exact: its products have at most 16 bits, and those
that are added lie within fp32's 24.
"""
from __future__ import annotations

import math

import pytest

from oracle import loss as oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U, R = 2.0 ** -24, 2.0 ** -8
LOWEST = -float(torch.finfo(torch.bfloat16).max)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("V", [1, 300, 1000, 40000])
@pytest.mark.parametrize("c", [0.0, 7.3, -100.3, 1e4, -1e9, 2.4e38, -2.4e38, -LOWEST, LOWEST])
def test_equal_logits(c, V):
    """loss = log V wherever they lie: every exponential is 1 and their sum exact, so there is the
    log's two units, and where one tile meets another nothing."""
    from paper_2608_02703_amd import head_loss
    x, w = torch.zeros((70, 64)), torch.zeros((V, 64))
    x[:, 5], w[:, 5] = 1, c
    loss, lse = head_loss(x.bfloat16().cuda(), w.bfloat16().cuda(), (torch.arange(70) % V).cuda())
    c = float(torch.tensor(c).bfloat16())
    assert ((loss.double() - math.log(V)).abs() <= 4 * U * math.log(V)).all()
    assert ((lse.double() - (c + math.log(V))).abs() <= 4 * U * math.log(V) + U * abs(c + math.log(V))).all()


@pytest.mark.parametrize("M", [3, 128, 700])
def test_near_certain_targets(M):
    """The target's logit in 15 .. 120, all others 0: loss = log(1 + (V - 1) e^-t) from log sums that
    are 1 and more, so it is never below 0, and 0 where all others are less than 2^-25 together.
    Otherwise an exponential is off by 2 t U (its argument's roundings), 4 U (itself) and 2 U (products), the sum
    by U (1 + s) for each addition (64 in a lane at most, 1 over the lanes, 8 over the waves, 6 over the tiles), the
    log by two of its units and the loss by a last rounding."""
    from paper_2608_02703_amd import head_loss
    V, d = 999, 64
    gen = torch.Generator().manual_seed(M)
    k = 640 + M % 300
    targets = torch.full((M,), k)
    x, w = torch.zeros((M, d)), torch.zeros((V, d))
    # t = x0 + x1 93 / 128, in steps of 2^-17 and below 2^7
    w[k, 0], w[k, 1] = 1.0, 93 / 128
    x[:, 0] = torch.rand(M, generator=gen) * 104 + 15
    x[:, 1] = torch.rand(M, generator=gen).clamp(min=2.0 ** -3)
    x, w = x.bfloat16(), w.bfloat16()
    t = x.double() @ w[k].double()
    assert torch.equal(t.float().double(), t) and t.min() >= 15 and t.max() <= 121
    loss, lse = head_loss(x.cuda(), w.cuda(), targets.cuda())
    loss, lse = loss.cpu().double(), lse.cpu().double()
    s = (V - 1) * torch.exp(-t)
    want = torch.log1p(s)
    assert (loss >= 0).all()
    assert not loss[s < 2.0 ** -26].any()
    tol = U * ((2 * t + 6) * s + 79 * (1 + s) + 5 * want)
    assert ((loss - want).abs() <= tol).all()
    assert ((lse - (t + want)).abs() <= tol + 2 * U * (t + want)).all()


@pytest.mark.parametrize("M", [5, 200, 700])
@pytest.mark.parametrize("low", [LOWEST, -2.4e38, -1e38])
def test_rows_of_the_lowest_value(M, low):
    """Padding rows of the head whose logits are the lowest finite values, whole waves and tiles of
    columns of them: as if they were not there, and their gradient 0."""
    from paper_2608_02703_amd import head_loss, head_loss_grad
    V, d = 1500, 64
    gen = torch.Generator().manual_seed(M)
    w = (torch.randn((V, d), generator=gen) / 4).bfloat16()
    x = torch.randn((M, d), generator=gen).bfloat16()
    x[:, 0], w[:, 0] = 1, 0
    lost = torch.zeros(V, dtype=torch.bool)
    lost[0:40] = lost[64:128] = lost[256:512] = lost[600:680] = lost[1400:] = True
    w[lost] = 0
    w[lost, 0] = low
    there = torch.nonzero(~lost).reshape(-1)
    y = torch.randint(0, len(there), (M,), generator=gen)
    grad = torch.randn(M, generator=gen).cuda()
    x, w, targets = x.cuda(), w.cuda(), there[y].cuda()
    loss, lse = head_loss(x, w, targets)
    o = oracle.head_loss(x, w[there.cuda()], y.cuda(), grad)
    # a logit by d U of its magnitudes; exponentials and sums as for rows that are all there
    steps, e = 100, d * U * o["reach"]
    tol = 2 * e + U * (steps + 3 * (o["lse"].abs() + o["loss"].abs()))
    assert ((loss - o["loss"]).abs() <= tol).all() and ((lse - o["lse"]).abs() <= tol).all()
    dx, dw = head_loss_grad(x, w, targets, lse, grad)
    assert not dw[lost.cuda()].any()
    tg = 2 * e + U * (o["far"] + steps + 4 * o["lse"].abs())
    least = 2.0 ** -126 * (1 + grad.abs().max().item())
    tx = (tg[:, None] + R + V * U) * o["dx_mag"] + least * w[there.cuda()].double().abs().sum(0)
    off = (dx[:, 1:] - o["dx"][:, 1:]).abs() - (tx + R * (o["dx"].abs() + tx))[:, 1:]   # (column 0 has the lowest values times 0)
    assert (off <= 2.0 ** -133).all() and torch.isfinite(dx).all()
    tw = (tg.max() + R + M * U) * o["dw_mag"] + least * x.double().abs().sum(0)
    assert ((dw[there.cuda()] - o["dw"]).abs() <= tw + R * (o["dw"].abs() + tw) + 2.0 ** -133).all()


@pytest.mark.parametrize("top", [3e38, 2.4e38, 1.0, -2.4e38, -2.9e38])
def test_one_logit_far_above_the_others(top):
    """Whose probability is 1 then, wherever it lies: G = grad (1 - [v = y]) there, -grad at other targets."""
    from paper_2608_02703_amd import head_loss, head_loss_grad
    M, V, d, k = 40, 700, 64, 333
    x, w = torch.zeros((M, d)).bfloat16().cuda(), torch.zeros((V, d)).bfloat16().cuda()
    x[:, 0], w[:, 0], w[k, 0] = 1, LOWEST, top
    targets = torch.arange(M, device="cuda") * 7
    targets[::3] = k
    grad = torch.ones(M, device="cuda") / 4
    loss, lse = head_loss(x, w, targets)
    high = w[k, 0].double()
    want = high - w[targets, 0].double()
    fits = want <= torch.finfo(torch.float32).max
    assert (lse.double() == high).all() and not loss[::3].any()
    assert ((loss.double() - want).abs() <= U * want)[fits].all() and torch.isinf(loss[~fits]).all()
    dx, dw = head_loss_grad(x, w, targets, lse, grad)
    others = int((targets != k).sum())
    expect = torch.zeros((V, d), device="cuda")
    expect[k, 0] = others / 4
    expect[targets[targets != k], 0] = -0.25
    assert torch.equal(dw.float(), expect)
    assert not dx[::3].any() and not dx[:, 1:].any()
    if high - LOWEST <= torch.finfo(torch.float32).max:   # (the sum, in units of the largest grad)
        got, want = dx[targets != k, 0].double(), (high - LOWEST) / 4
        assert ((got - want).abs() <= (R + 2 * U) * want).all()
