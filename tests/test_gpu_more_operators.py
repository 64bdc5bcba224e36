"""The norm, adapters and head loss together, as a program runs them, and at
their limits: large sizes, calls at once on several streams, graphs that take turns."""
from __future__ import annotations

import pytest

from oracle import loss as oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _layer(M, K, N, n, seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)   # noqa: E731
    from paper_2608_02703_amd import quantize_i8
    return dict(x=r(M, K).bfloat16().cuda(), res=r(M, K).bfloat16().cuda(), w=(1 + 0.1 * r(K)).bfloat16().cuda(),
                q=quantize_i8((r(N, K) / K ** 0.5).cuda()), a=(r(n, 16, K) / K ** 0.5).bfloat16().cuda(),
                b=(r(n, N, 16) * 0.2).bfloat16().cuda(), ids=torch.randint(-1, n, (M,), generator=gen).cuda())


def _run_layer(s):
    """norm with residual -> 8-bit product -> adapters on the same rows -> beam selection."""
    from paper_2608_02703_amd import adapters_add, beam_select, matmul_i8, rms_norm_i8
    codes, scales, total, h = rms_norm_i8(s["x"], s["w"], residual=s["res"], normed=True)
    y = matmul_i8(codes, scales, *s["q"])
    adapters_add(y, h, s["a"], s["b"], s["ids"], out=y)
    M = y.shape[0]
    return (total, y, *beam_select(y, torch.zeros((M // 4, 4), device="cuda"), 4))


def test_a_decoding_step():
    s = _layer(48, 1024, 5000, 6, 1)
    total, y, scores, parents, tokens = _run_layer(s)
    h = (s["x"].double() + s["res"].double())
    h = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * s["w"].double()
    W = s["q"][0].double() * s["q"][1].double()[:, None]
    want = h @ W.t().contiguous()
    for k in range(6):
        at = s["ids"] == k
        want[at] += (h[at] @ s["a"][k].double().t().contiguous()) @ s["b"][k].double().t().contiguous()
    # rows to 8 bits: half a step of max|h| / 127 an element; their 16-bit form 2^-8 of it for the adapters
    step = h.abs().amax(1, keepdim=True) / 254
    tol = step * W.abs().sum(1) + 0.05
    assert ((y.double() - want).abs() <= tol).all()
    lp = torch.log_softmax(y.double(), 1).view(12, 4 * 5000)
    assert torch.allclose(scores.double(), lp.topk(4, 1).values, atol=1e-5)


def test_a_step_replayed_and_two_graphs_in_turn():
    s, t = _layer(64, 512, 3000, 5, 2), _layer(64, 512, 3000, 5, 3)
    _run_layer(s), _run_layer(t)
    graphs, held = [], []
    for v in (s, t):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held.append(_run_layer(v))
        graphs.append(g)
    for seed in range(3):
        for v, k in ((s, 10), (t, 20)):
            n = _layer(64, 512, 3000, 5, seed + k)
            for name in ("x", "res", "a", "ids"):
                v[name].copy_(n[name])
        for i in (0, 1, 1, 0):
            graphs[i].replay()
        torch.cuda.synchronize()
        for v, h in ((s, held[0]), (t, held[1])):
            assert all(torch.equal(a, b) for a, b in zip(_run_layer(v), h))


def test_calls_at_once_on_two_streams():
    from paper_2608_02703_amd import head_loss, head_loss_grad
    s, t = _layer(72, 768, 4000, 4, 5), _layer(72, 768, 4000, 4, 6)   # 18 sequences of four beams
    gen = torch.Generator().manual_seed(9)
    loss_in = [((torch.randn((300, 256), generator=gen)).bfloat16().cuda(), (torch.randn((5000, 256), generator=gen) / 8).bfloat16().cuda(),
                torch.randint(-1, 5000, (300,), generator=gen).cuda(), torch.rand(300, generator=gen).cuda()) for _ in range(2)]

    def step(x, w, y, g):
        loss, lse = head_loss(x, w, y)
        return (loss, *head_loss_grad(x, w, y, lse, g))
    want = [_run_layer(s)[:2], _run_layer(t)[:2], step(*loss_in[0]), step(*loss_in[1])]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for k, (stream, v) in enumerate(zip(streams, (s, t))):
            with torch.cuda.stream(stream):
                got[k].append((_run_layer(v)[:2], step(*loss_in[k])))
    torch.cuda.synchronize()
    for k in range(2):
        for layer, st in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(layer, want[k]))
            assert all(torch.equal(a, b) for a, b in zip(st, want[2 + k]))


def test_a_head_past_32_bit_offsets():
    """A head and a gradient of more than 2^32 bytes, rows sampled."""
    from paper_2608_02703_amd import head_loss, head_loss_grad
    M, V, d = 70, 1_100_001, 2048
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = torch.empty((V, d), dtype=torch.bfloat16, device="cuda")
    for v in range(0, V, 65536):
        w[v:v + 65536] = torch.randn((min(65536, V - v), d), generator=gen, device="cuda") / 32
    x = torch.randn((M, d), generator=gen, device="cuda").bfloat16()
    y = torch.randint(0, V, (M,), generator=gen, device="cuda")
    y[:3] = torch.tensor([V - 1, V - 2, -100], device="cuda")
    g = torch.full((M,), 1 / M, device="cuda")
    loss, lse = head_loss(x, w, y)
    dx, dw = head_loss_grad(x, w, y, lse, g)
    xs = x.double()
    want = torch.full((M,), float("-inf"), dtype=torch.float64, device="cuda")
    full = torch.zeros((M, d), dtype=torch.float64, device="cuda")
    for v in range(0, V, 65536):
        want = torch.logaddexp(want, torch.logsumexp(xs @ w[v:v + 65536].double().t().contiguous(), 1))
    live = y >= 0
    assert torch.allclose(lse[live].double(), want[live], atol=1e-4)
    for v in range(0, V, 65536):
        wp = w[v:v + 65536].double()
        p = torch.exp(xs @ wp.t().contiguous() - want[:, None])
        at = torch.nonzero((y >= v) & (y < v + len(wp))).reshape(-1)
        p[at, y[at] - v] -= 1
        p = p * (g.double() * live)[:, None]
        full += p @ wp
        if v == 0 or v + 65536 >= V:
            rows = p.t().contiguous() @ xs
            err = (dw[v:v + 65536].double() - rows).norm() / rows.norm()
            assert err < 2.0 ** -7   # two roundings of 2^-8, of the entries of G and of dw
    assert (dx.double() - full).norm() / full.norm() < 2.0 ** -7 and not dx[2].any()


def test_many_tokens_of_a_small_head():
    """More tokens than a workgroup of the gathering takes at once, most without a target."""
    from paper_2608_02703_amd import head_loss, head_loss_grad
    M, V, d = 300_000, 260, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((M, d), generator=gen, device="cuda").bfloat16()
    w = (torch.randn((V, d), generator=gen, device="cuda") / 4).bfloat16()
    y = torch.randint(0, V, (M,), generator=gen, device="cuda")
    y[torch.rand(M, generator=gen, device="cuda") < 0.9] = -1
    g = torch.rand(M, generator=gen, device="cuda") / M
    loss, lse = head_loss(x, w, y)
    dx, dw = head_loss_grad(x, w, y, lse, g)
    o = oracle.head_loss(x, w, y, g)
    assert torch.allclose(loss.double(), o["loss"], atol=1e-4) and torch.allclose(lse.double(), o["lse"], atol=1e-4)
    for got, want in ((dx, o["dx"]), (dw, o["dw"])):
        assert (got.double() - want).norm() / want.norm() < 2.0 ** -7
    assert not dx[y < 0].any()
