"""head_loss and head_loss_grad on the GPU against the oracle in fp64.

A logit is a sum of d exact products in fp32, off by at most e = d 2^-24 times
the sum of their magnitudes; lse by as much, by the exponentials' two units and their
argument's rounding (a e^-a < 1 units of 2^-24), by the sum's (in a lane, over a
tile's waves and lanes, over the tiles: 100 + V / 2^14 steps of 2^-24) and by the
last additions' 3 2^-24 of the values.  So G is off by p (2 e + 2^-24 (far + 100 + V / 2^14
+ 4 |lse|)) of its grad, far the largest of lse - logit (the exponent's rounding), by its
rounding to bf16 (2^-8 of it), and the sums of V (M) products by as many steps of 2^-24, and the
output's rounding 2^-8.  (bf16 has 8 bits of significand: steps of 2^(e-7) from 2^e on, so
half a step is up to 2^-8 of a value.)  Exponentials, and entries of G, below the normal
numbers of fp32 and bf16 (2^-126) count as 0: that adds 2^-126 (1 + |grad|) to every
entry of G, times the other operand's sum of magnitudes.
"""
from __future__ import annotations

import pytest

from oracle import loss as oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U, R = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _inputs(M, V, d, seed=0, ignored=0.2, sharp=1.0, t64=True):
    gen = torch.Generator().manual_seed(seed + 1000003 * M + 1009 * V + d)
    w = (torch.randn((V, d), generator=gen) * 2 / d ** 0.5).bfloat16()
    targets = torch.randint(0, V, (M,), generator=gen)
    x = ((torch.randn((M, d), generator=gen) + 2 * torch.rand((M, 1), generator=gen) * w[targets].float()) * sharp).bfloat16()
    lost = torch.rand(M, generator=gen) < ignored
    targets = torch.where(lost, torch.tensor([-100, V, -1, 2 ** 31 - 1])[torch.arange(M) % 4], targets)
    grad = torch.randn(M, generator=gen) / max(M, 1)
    return x.cuda(), w.cuda(), targets.to(torch.int64 if t64 else torch.int32).cuda(), grad.cuda()


def _tols(o, V, d):
    e = d * U * o["reach"]
    steps = 100 + V / 2 ** 14
    return 2 * e + U * (steps + 3 * (o["lse"].abs() + o["loss"].abs())), e + U * (steps + 3 * o["lse"].abs()), \
        2 * e + U * (o["far"] + steps + 4 * o["lse"].abs())


def _within(got, want, tol, what):
    off = (got.double() - want).abs() - tol * (1 + 2.0 ** -10)
    assert not (off > 0).any() and not torch.isnan(off).any(), \
        f"{what}: {int((off > 0).sum())} of {off.numel()} off, the worst by {off.max().item():.3g}"


def _check(x, w, targets, grad, loss, lse, dx=None, dw=None):
    (M, d), V = x.shape, w.shape[0]
    o = oracle.head_loss(x, w, targets, grad if dx is not None or dw is not None else None)
    tl, te, tg = _tols(o, V, d)
    _within(loss, o["loss"], tl, "loss")
    _within(lse, o["lse"], te, "lse")
    out = (targets < 0) | (targets >= V)
    assert not loss[out].any() and not lse[out].any()
    worst = tg.max().item() if M else 0.0
    least = 2.0 ** -126 * (1 + grad[~out].abs().max().item()) if (~out).any() else 0.0
    tiny_x, tiny_w = least * w.double().abs().sum(0), least * x[~out].double().abs().sum(0)
    if dx is not None:
        tol = (tg[:, None] + R + V * U) * o["dx_mag"] + tiny_x
        _within(dx, o["dx"], tol + R * (o["dx"].abs() + tol) + 2.0 ** -133, "dx")
        assert not dx[out].any()
    if dw is not None:
        tol = (worst + R + M * U) * o["dw_mag"] + tiny_w
        _within(dw, o["dw"], tol + R * (o["dw"].abs() + tol) + 2.0 ** -133, "dw")


def _step(x, w, targets, grad, **kw):
    from paper_2608_02703_amd import head_loss, head_loss_grad
    loss, lse = head_loss(x, w, targets)
    return (loss, lse, *head_loss_grad(x, w, targets, lse, grad, **kw))


SIZES = [(1, 1, 1), (1, 300, 64), (2, 7, 3), (3, 257, 70), (5, 255, 63), (64, 1000, 128), (65, 511, 100), (128, 512, 64),
         (129, 2050, 192), (257, 700, 65), (300, 5000, 320), (7, 256, 1000), (33, 20011, 520), (600, 333, 448)]


@pytest.mark.parametrize("M,V,d", SIZES)
def test_step(M, V, d):
    i = _inputs(M, V, d, ignored=0.0 if M == 1 else 0.2, t64=(M + V) % 2 == 0)
    _check(*i, *_step(*i))


@pytest.mark.parametrize("M,V,d", [(200, 3001, 256), (64, 700, 192)])
@pytest.mark.parametrize("sharp", [30.0, 0.01])
def test_sharp_and_flat(M, V, d, sharp):
    """Tokens whose probability is nearly 1, and nearly equal logits."""
    i = _inputs(M, V, d, sharp=sharp)
    _check(*i, *_step(*i))


@pytest.mark.parametrize("M,V,d", [(4096, 33000, 64), (2100, 70000, 128), (2100, 40000, 128), (5, 9001, 16383), (300, 8200, 16384)])
def test_several_pieces(M, V, d):
    i = _inputs(M, V, d)
    _check(*i, *_step(*i))


@pytest.mark.parametrize("M,d", [(40, 256), (300, 1100)])
def test_one_of_the_gradients(M, d):
    i = _inputs(M, 900, d)
    loss, lse, dx, dw = _step(*i)
    _, _, a, none = _step(*i, dw=False)
    _, _, no, b = _step(*i, dx=False)
    assert none is None and no is None and torch.equal(a, dx) and torch.equal(b, dw)


@pytest.mark.parametrize("d", [64, 67, 200])
def test_strides(d):
    """Rows in wider buffers at odd places; what lies between outputs' rows stays."""
    M, V, ld = 90, 600, d + 9
    i = _inputs(M, V, d)

    def wide(t, off, ld):
        buf = torch.full((t.shape[0] * ld + 64,), 9.0, dtype=t.dtype, device="cuda")
        v = buf[off:].as_strided(t.shape, (ld, 1))
        v.copy_(t)
        return buf, v
    want = _step(*i)
    _check(*i, *want)
    for off, ld in ((1, d + 9), (3, d + 8), (8, (d + 15) // 8 * 8)):
        x, w = wide(i[0], off, ld)[1], wide(i[1], off, ld)[1]
        (bx, dx), (bw, dw) = wide(i[0], off + 1, ld), wide(i[1], off, ld)
        got = _step(x, w, *i[2:], dx=dx, dw=dw)
        assert got[2] is dx and got[3] is dw
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for b, v in ((bx, dx), (bw, dw)):
            v.fill_(9.0)
            assert (b == 9).all()


def test_tokens_without_a_target_add_nothing():
    """Whatever their rows and weights hold; none, one and all of them."""
    x, w, targets, grad = _inputs(150, 800, 128, ignored=0.5)
    want = _step(x, w, targets, grad)
    out = (targets < 0) | (targets >= 800)
    x[out], grad[out] = float("nan"), float("inf")
    assert all(torch.equal(a, b) for a, b in zip(_step(x, w, targets, grad), want))
    targets[:] = -100
    loss, lse, dx, dw = _step(x, w, targets, grad)
    assert not loss.any() and not lse.any() and not dx.any() and not dw.any()
    x, w, targets, grad = _inputs(150, 800, 128, ignored=0.0)
    targets[:149] = -1
    got = _step(x, w, targets, grad)
    _check(x, w, targets, grad, *got)
    empty = _step(x[:0], w, targets[:0], grad[:0])
    assert empty[0].shape == (0,) and empty[2].shape == (0, 128) and not empty[3].any()


def test_rows_that_are_not_finite():
    """A token's NaN stays with its loss and row; -inf logits count for nothing."""
    x, w, targets, grad = _inputs(70, 500, 64, ignored=0.0)
    want = _step(x, w, targets, grad)
    x[5, 3] = float("nan")
    loss, lse, dx, dw = _step(x, w, targets, grad)
    keep = torch.arange(70, device="cuda") != 5
    assert torch.isnan(loss[5]) and torch.isnan(lse[5]) and torch.isnan(dx[5]).all() and torch.isnan(dw).all()
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip((loss, lse, dx), want))
    x, w, targets, grad = _inputs(40, 300, 64, ignored=0.0)
    x[:, 0] = x[:, 0].abs() + 0.5
    targets.clamp_(min=20)
    w[:20, 0] = float("-inf")
    from paper_2608_02703_amd import head_loss
    loss, lse = head_loss(x, w, targets)
    o = oracle.head_loss(x, w[20:], targets - 20)
    tl, te, _ = _tols(o, 300, 64)
    _within(loss, o["loss"], tl, "loss")
    _within(lse, o["lse"], te, "lse")


def test_against_differences():
    """Directional derivatives of the oracle's loss, by central differences in fp64:
    off by h^2 / 6 of the third derivative, which is at most 8 |u w|^3 with logits
    along u of at most |u w|; and by dx's own bound."""
    M, V, d = 20, 300, 96
    x, w, targets, grad = _inputs(M, V, d)
    _, _, dx, dw = _step(x, w, targets, grad)
    o = oracle.head_loss(x, w, targets, grad)
    gen = torch.Generator().manual_seed(3)
    total = lambda x, w: (oracle.head_loss(x, w, targets)["loss"] * grad.double()).sum()   # noqa: E731
    h = 1e-4
    for k in range(4):
        u, v = (torch.randn(s, generator=gen, dtype=torch.float64).cuda() for s in ((M, d), (V, d)))
        X, W = x.double(), w.double()
        for diff, got, mag, reach in (
                (total(X + h * u, W) - total(X - h * u, W), (dx.double() * u).sum(), (o["dx_mag"] * u.abs()).sum(),
                 (u @ W.t().contiguous()).abs().max()),
                (total(X, W + h * v) - total(X, W - h * v), (dw.double() * v).sum(), (o["dw_mag"] * v.abs()).sum(),
                 (X @ v.t().contiguous()).abs().max())):
            tol = h * h / 6 * 8 * reach ** 3 * grad.abs().double().sum() + 2.1 * R * mag + 1e-9
            assert (diff / (2 * h) - got).abs() <= tol


def test_norm_head_and_packed_head():
    """A training step's end: last norm, loss, gradient through torch's norm; the
    loss agrees with that of the packed head built from the same dense one up to
    its logits' difference."""
    from paper_2608_02703_amd import build_head, head_loss, rms_norm
    V, d, M = 1024, 256, 48
    x, w, targets, grad = _inputs(M, V, d, ignored=0.0)
    weight = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    h, total = rms_norm(x, weight, residual=x.clone())
    loss, lse = head_loss(h, w, targets)
    _check(h, w, targets, grad, loss, lse)
    ph = build_head(w.float(), h.float(), rc=32, rr=16, g=32)
    lg = ph.logits(h)
    ce, _ = ph.logits_ce(h, targets)
    dense = h.float() @ w.float().t()
    gap = (lg - dense).abs().amax(1)
    assert ((ce - loss).abs() <= 2 * gap + 1e-3).all()
    ph.close()


def test_repeatable_streams_and_graphs():
    from paper_2608_02703_amd import head_loss, head_loss_grad
    x, w, targets, grad = _inputs(130, 1500, 192)
    want = _step(x, w, targets, grad)
    assert all(torch.equal(a, b) for a, b in zip(_step(x, w, targets, grad), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _step(x, w, targets, grad)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, lse = head_loss(x, w, targets)
        dx, dw = head_loss_grad(x, w, targets, lse, grad)
    for seed in range(4):   # other numbers of live tokens, none among them
        nx, _, nt, ng = _inputs(130, 1500, 192, seed=seed, ignored=(0.0, 0.5, 1.1, 0.9)[seed])
        x.copy_(nx)
        targets.copy_(nt)
        grad.copy_(ng)
        graph.replay()
        torch.cuda.synchronize()
        want = _step(x, w, targets, grad)
        assert all(torch.equal(a, b) for a, b in zip((loss, lse, dx, dw), want))


@pytest.mark.parametrize("M", [87, 300])
def test_a_mean_loses_no_more_than_its_outputs_do(M):
    """grad 1 / M, which bf16 does not hold: G is in units of it, its entry at a target
    -(1 - p), off by half a step of 2^-8 at most, and by p where it
    rounds to 1; its others are off by 2^-8 p each.
    The rest are the sums' errors and two products' by the unit, and half a step of the output."""
    V, d = 4096, 128
    x, w, targets, _ = _inputs(M, V, d, ignored=0.0)
    x = (x.float() * 0.5).bfloat16()
    grad = torch.full((M,), 1 / M, device="cuda")
    loss, lse, dx, dw = _step(x, w, targets, grad)
    o = oracle.head_loss(x, w, targets, grad)
    tg = _tols(o, V, d)[2]
    xs, ws = x.double(), w.double()
    p = torch.exp(xs @ ws.t().contiguous() - o["lse"][:, None])
    off = R * p
    off[torch.arange(M), targets] = p[torch.arange(M), targets].clamp(max=2.0 ** -9)
    off *= grad[0].double() * (1 + 2.0 ** -7)

    def half_step(v):   # of bf16 at v
        return torch.ldexp(torch.ones_like(v), torch.frexp(v)[1] - 9)
    least = 2.0 ** -120
    tx = off @ ws.abs() + (tg[:, None] + (V + 2) * U) * o["dx_mag"] + least
    _within(dx, o["dx"], tx + half_step(o["dx"].abs() + tx), "dx")
    tw = off.t().contiguous() @ xs.abs() + (tg.max() + (M + 2) * U) * o["dw_mag"] + least
    _within(dw, o["dw"], tw + half_step(o["dw"].abs() + tw), "dw")


@pytest.mark.parametrize("odd", [0.0, float("inf"), 2.0 ** -140, 2.0 ** 100])
def test_grads_of_any_size(odd):
    """All zero, one without a bound, all below the normal numbers, and large ones."""
    x, w, targets, _ = _inputs(40, 300, 64, ignored=0.0)
    grad = torch.full((40,), 0.5 if odd == float("inf") else odd, device="cuda")
    if odd == float("inf"):
        grad[3] = odd
    loss, lse, dx, dw = _step(x, w, targets, grad)
    if odd == float("inf"):
        assert not torch.isfinite(dx[3]).any() and torch.isfinite(dx[:3]).all() and torch.isfinite(dx[4:]).all()
        assert not torch.isfinite(dw).all()
    else:
        _check(x, w, targets, grad, loss, lse, dx, dw)
