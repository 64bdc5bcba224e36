"""beam_select, PackedHead.logits_beam and BeamStates on the GPU against the
oracle.

Choices within a beam are integer decisions on the logits and have to be the
oracle's exactly.  Between beams they go by scores, which differ from the
oracle's by the error of the beams' logsumexp: with D = sum_v p_v |l_v - max|,
an exponent is off by at most 2 * 2^-24 |l - max| (its difference and its
product with log2 e, each rounded), its exponential by 2^-22 of it at most,
32 of them are added in fp32 (31 * 2^-24), the rest in fp64.  So a logsumexp
is off by at most e = 2^-23 D + 2^-22 + 31 * 2^-24, and out_scores by one fp32
rounding more.  Choices may differ from the oracle's only where scores lie
within 2 e.  Equal rows have equal logsumexps, so equal scores are exact ties.
"""
from __future__ import annotations

import numpy as np
import pytest

from oracle import beam as oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def _error(lg):
    """e of the file's head, over all rows."""
    with np.errstate(invalid="ignore"):
        m = lg.max(axis=1, keepdims=True)
        d = np.where(np.isfinite(lg) & np.isfinite(m), np.abs(lg - m), 0.0)
        p = np.where(np.isfinite(lg) & np.isfinite(m), np.exp(-d), 0.0)
        D = (p * d).sum(1) / np.maximum(p.sum(1), 1e-300)
    return 2.0 ** -23 * D.max(initial=0.0) + 2.0 ** -22 + 31 * 2.0 ** -24


def check(logits, scores, n, got, finished=None, end_token=-1, exact=False):
    lg = logits.detach().cpu().to(torch.float64).numpy()
    sc = scores.cpu().numpy()
    fin = None if finished is None else finished.cpu().numpy()
    vals, parents, tokens = (t.cpu().numpy() for t in got[:3])
    assert vals.dtype == np.float32 and parents.dtype == tokens.dtype == np.int64
    ov, op, ot, oe = oracle.select(lg, sc, n, fin, end_token)
    B, K = sc.shape
    e = _error(lg)
    s = oracle.scores_of(lg, sc, fin, end_token)
    V = s.shape[2]
    if exact:
        assert np.array_equal(parents, op) and np.array_equal(tokens, ot)
    for b in range(B):
        some = int((op[b] >= 0).sum())
        assert (parents[b, :some] >= 0).all() and (parents[b, some:] == -1).all()
        assert (tokens[b, some:] == -1).all() and np.isneginf(vals[b, some:]).all()
        mine = [s[b, k, v] for k, v in zip(parents[b, :some], tokens[b, :some])]
        assert len(set(zip(parents[b], tokens[b]))) >= some
        for j in range(some):
            assert abs(vals[b, j] - mine[j]) <= e + 2.0 ** -24 * abs(mine[j]) * 1.001, (b, j)
            assert j == 0 or mine[j] <= mine[j - 1] + 2 * e
        for k in range(K):   # the first tokens of the beam, in its own order
            t = tokens[b, :some][parents[b, :some] == k]
            want = np.lexsort((np.arange(V), -s[b, k]))[:len(t)]
            assert np.array_equal(t, want), (b, k)
            rest = np.delete(s[b, k], want)
            if some and rest.size:
                assert rest.max() <= min(mine) + 2 * e
    if len(got) > 3:
        ended = got[3].cpu().numpy()
        want = (tokens == end_token) & (tokens >= 0)
        if fin is not None:
            want |= (parents >= 0) & np.take_along_axis(fin.astype(bool), np.maximum(parents, 0), 1)
        assert np.array_equal(ended, want)


def _case(B, K, V, dtype, seed, sigma=3.0, pad=0):
    gen = torch.Generator().manual_seed(seed)
    lg = (torch.randn((B * K, V + pad), generator=gen) * sigma).to(DTYPES[dtype]).cuda()[:, :V]
    scores = -torch.rand((B, K), generator=gen).cumsum(1) * 3
    return lg, scores.cuda()


SHAPES = [(1, 1, 1, 1), (1, 1, 3, 5), (2, 3, 7, 4), (1, 4, 511, 8), (3, 4, 512, 8), (2, 5, 513, 10), (1, 8, 2047, 16),
          (2, 8, 2048, 16), (2, 32, 2049, 64), (1, 4, 8191, 8), (1, 2, 8193, 64), (7, 1, 1000, 3), (4, 2, 50257, 4),
          (1, 16, 33000, 32), (33, 3, 700, 6), (2, 4, 151936, 8)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("B,K,V,n", SHAPES)
def test_select(B, K, V, n, dtype):
    from paper_2608_02703_amd import beam_select
    lg, scores = _case(B, K, V, dtype, B * 1000 + V)
    check(lg, scores, n, beam_select(lg, scores, n))


# Sequences around the spans that one launch reads, with beams that are not read
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("B,K,V,n", [(1, 1, 65536, 4), (1, 1, 65537, 4), (3, 2, 32767, 8), (3, 3, 20480, 6), (2, 4, 16384, 8),
                                     (2, 4, 16385, 8), (2, 16, 4096, 32), (2, 17, 2048, 17), (5, 32, 2048, 64), (2, 32, 2049, 8),
                                     (40, 5, 9000, 10)])
def test_select_of_few_spans(B, K, V, n, dtype):
    from paper_2608_02703_amd import beam_select
    lg, scores = _case(B, K, V, dtype, K * V)
    check(lg, scores, n, beam_select(lg, scores, n))
    if K > 1:
        scores[:, K // 2] = -torch.inf
        fin = torch.zeros((B, K), dtype=torch.bool, device="cuda")
        fin[:, K - 1] = True
        check(lg, scores, n, beam_select(lg, scores, n, finished=fin, end_token=V - 1), finished=fin, end_token=V - 1)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("pad", [1, 2, 3, 5, 8])
def test_select_row_strides(dtype, pad):
    from paper_2608_02703_amd import beam_select
    lg, scores = _case(2, 4, 4097, dtype, pad, pad=pad)
    check(lg, scores, 8, beam_select(lg, scores, 8))
    lg = lg[:, 1:]   # rows that begin off any alignment
    check(lg, scores, 8, beam_select(lg, scores, 8))


@pytest.mark.parametrize("n", [1, 7, 16, 64])
@pytest.mark.parametrize("K,V", [(1, 300), (4, 5000), (16, 33000)])
def test_select_ties(K, V, n):
    """Equal logits and equal beams: ties by beam, then token, however many."""
    from paper_2608_02703_amd import beam_select
    scores = torch.full((2, K), -1.25, device="cuda")
    lg = torch.full((2 * K, V), 0.5, device="cuda")
    check(lg, scores, n, beam_select(lg, scores, n), exact=True)
    gen = torch.Generator().manual_seed(n)
    lg = torch.randint(-3, 3, (1, V), generator=gen).float().expand(2 * K, V).contiguous().cuda()
    check(lg, scores, n, beam_select(lg, scores, n), exact=True)
    lg = torch.zeros((2 * K, V), device="cuda")   # -0 and 0 are equal
    lg[:, ::2] = -0.0
    check(lg, scores, n, beam_select(lg, scores, n), exact=True)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("order", ["up", "down", "block", "steps"])
def test_select_sorted_logits(order, dtype):
    """Logits whose largest lie together: more pairs above the floor than are
    ranked one against all."""
    from paper_2608_02703_amd import beam_select
    K, V = 4, 20000
    r = torch.arange(V).float()
    row = {"up": r / 2000, "down": -r / 2000, "block": torch.where((r > 9000) & (r < 10300), 3.0 + r / 1e4, -2.0),
           "steps": (r / 700).floor()}[order]
    lg = row.expand(K, V).to(DTYPES[dtype]).contiguous().cuda()
    scores = torch.tensor([[0.0, -0.5, -1.0, -1.0]], device="cuda")
    for n in (1, 8, 64):
        check(lg, scores, n, beam_select(lg, scores, n))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_select_masks(dtype):
    """Rows with nothing left, NaN, +inf, the type's lowest value, few tokens
    allowed; beams not in use."""
    from paper_2608_02703_amd import beam_select
    low = torch.finfo(DTYPES[dtype]).min
    for V in (40, 6000):
        lg, scores = _case(3, 8, V, dtype, V)
        lg = lg.clone()
        lg[0] = -float("inf")
        lg[1, V // 2] = float("nan")
        lg[2, V - 1] = float("inf")
        lg[3] = low
        lg[4, : V - 3] = low
        lg[5, 3:] = -float("inf")
        lg[6, 0] = -float("inf")
        lg[8:16] = -float("inf")                 # a sequence without any candidate
        lg[16:24, 2:] = -float("inf")            # fewer candidates than places
        scores[0, 7] = -float("inf")
        scores[2, 1:] = -float("inf")
        scores[2, 2] = float("nan")
        for n in (1, 8, 16, 64):
            check(lg, scores, n, beam_select(lg, scores, n))
            check(lg, scores, n, beam_select(lg, scores, n, end_token=1), end_token=1)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("kind", [torch.bool, torch.uint8])
def test_select_finished(dtype, kind):
    """Ended beams offer their end token alone; what their logits hold does
    not matter."""
    from paper_2608_02703_amd import beam_select
    B, K, V = 5, 6, 3001
    lg, scores = _case(B, K, V, dtype, 8)
    fin = torch.zeros((B, K), dtype=kind, device="cuda")
    fin[0, 2] = fin[1, :5] = fin[2] = fin[3, 0] = 1
    scores[3, 0] = -float("inf")
    scores[4, 3] = 2.0
    lg = lg.clone()
    lg[2], lg[K:K + 2] = float("nan"), float("inf")
    for n in (1, 6, 12, 64):
        for end in (0, V - 1):
            check(lg, scores, n, beam_select(lg, scores, n, finished=fin, end_token=end), finished=fin, end_token=end)


def test_select_first_step():
    """One beam in use, the others at -inf: the K best of that beam."""
    from paper_2608_02703_amd import beam_select
    lg, scores = _case(3, 4, 9000, "f32", 2)
    scores[:] = -float("inf")
    scores[:, 0] = 0
    got = beam_select(lg, scores, 4)
    check(lg, scores, 4, got)
    assert not got[1].any()
    top = torch.sort(lg[::4], dim=1, descending=True, stable=True).indices[:, :4]
    assert torch.equal(got[2], top)


def test_select_large_offsets_and_far_scores():
    from paper_2608_02703_amd import beam_select
    lg, scores = _case(2, 4, 10000, "f32", 4)
    for shift in (1e4, -3e5):
        check(lg + shift, scores, 8, beam_select(lg + shift, scores, 8))
    check(lg, scores * 1000, 8, beam_select(lg, scores * 1000, 8))


@pytest.mark.parametrize("V", [3000, 40000])
def test_select_far_rows(V):
    """Rows of logits at offsets that pass 32 bits."""
    from paper_2608_02703_amd import beam_select
    lg, scores = _case(2, 3, V, "f32", V)
    ld = 450000000
    far = torch.empty(5 * ld + V, dtype=torch.float32, device="cuda").as_strided((6, V), (ld, 1))
    far.copy_(lg)
    check(far, scores, 6, beam_select(far, scores, 6))


def test_two_selections_at_once():
    from paper_2608_02703_amd import beam_select
    cases = [_case(2, 4, V, "f32", V) for V in (5000, 60000)]
    want = [beam_select(lg, scores, 8) for lg, scores in cases]
    torch.cuda.synchronize()
    got = []
    for lg, scores in cases * 4:
        with torch.cuda.stream(torch.cuda.Stream()):
            got.append(beam_select(lg, scores, 8))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(x, y) for x, y in zip(g, want[i % 2]))


def test_select_is_reproducible_and_needs_no_clean_workspace():
    from paper_2608_02703_amd import beam_select, lib
    lg, scores = _case(4, 8, 30000, "bf16", 6, sigma=1.0)
    first = beam_select(lg, scores, 16)
    ws = torch.empty(lib().archead_beam_workspace_bytes(32, 30000), dtype=torch.uint8, device="cuda")
    for fill in (0, 127, 255):
        ws.fill_(fill)
        again = beam_select(lg, scores, 16, ws=ws)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_select_over_its_own_inputs():
    """n == K with out_scores = scores and out_finished = finished."""
    from paper_2608_02703_amd import beam_select, lib
    from paper_2608_02703_amd.archead import F32
    B, K, V = 3, 5, 4000
    lg, scores = _case(B, K, V, "f32", 12)
    fin = torch.zeros((B, K), dtype=torch.uint8, device="cuda")
    fin[1, 1] = fin[2, 0] = 1
    want = beam_select(lg, scores, K, finished=fin, end_token=17)
    par, tok = (torch.empty((B, K), dtype=torch.int64, device="cuda") for _ in range(2))
    ws = torch.empty(lib().archead_beam_workspace_bytes(B * K, V), dtype=torch.uint8, device="cuda")
    st = lib().archead_beam_select(lg.data_ptr(), F32, B, K, V, V, scores.data_ptr(), fin.data_ptr(), 17, K,
                                   scores.data_ptr(), par.data_ptr(), tok.data_ptr(), fin.data_ptr(), ws.data_ptr(),
                                   ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert st == 0
    for a, b in zip((scores, par, tok, fin.bool()), want):
        assert torch.equal(a, b)


def test_select_streams_and_graphs():
    from paper_2608_02703_amd import beam_select
    lg, scores = _case(2, 4, 20000, "f32", 3)
    want = beam_select(lg, scores, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = beam_select(lg, scores, 8)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):   # two graphs of one pool
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=graphs[0][0].pool() if graphs else None):
            held = beam_select(lg, scores, 8)
        graphs.append((g, held))
    for seed in range(4):
        lg.copy_(torch.randn(lg.shape, generator=torch.Generator().manual_seed(seed)) * 2)
        for g, held in graphs:
            g.replay()
            want = beam_select(lg, scores, 8)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_select_refusals():
    from paper_2608_02703_amd import ArcheadError, beam_select
    lg, scores = _case(2, 4, 100, "f32", 1)
    fin = torch.zeros((2, 4), dtype=torch.bool, device="cuda")
    for bad in (lambda: beam_select(lg[:7], scores, 4), lambda: beam_select(lg, scores.t(), 4),
                lambda: beam_select(lg, scores, 0), lambda: beam_select(lg, scores, 65),
                lambda: beam_select(lg, scores, 4, finished=fin[:1], end_token=1),
                lambda: beam_select(lg, scores.view(-1), 4)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: beam_select(lg.double(), scores, 4), lambda: beam_select(lg, scores.half(), 4),
                lambda: beam_select(lg, scores, 4, finished=fin.int(), end_token=1)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: beam_select(lg, scores, 4, finished=fin), lambda: beam_select(lg, scores, 4, end_token=100),
                lambda: beam_select(lg, scores, 4, ws=torch.empty(256, dtype=torch.uint8, device="cuda")),
                lambda: beam_select(torch.zeros((33, 5), device="cuda"), torch.zeros((1, 33), device="cuda"), 2)):
        with pytest.raises(ArcheadError):
            bad()


# --------------------------------------------------------------- reordering
def _values(shape, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    t = torch.randint(-2 ** 31, 2 ** 31 - 1, shape, generator=gen)
    return t.to(dtype) if not dtype.is_floating_point else (t % 4093).to(dtype)


def _want(s, d, parents, beams, lengths, p):
    """The oracle's destination; positions of the tensors in dimension p."""
    sn, dn = s.cpu(), d.cpu()
    if p is not None:
        sn, dn = sn.movedim(p, 1), dn.movedim(p, 1)
    else:
        sn, dn = sn[:, None], dn[:, None]
    out = oracle.reorder(sn.numpy(), dn.numpy(), parents.cpu().numpy(), beams,
                         None if lengths is None else lengths.cpu().numpy())
    t = torch.from_numpy(out)
    return t.movedim(1, p) if p is not None else t[:, 0]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("idx", [torch.int32, torch.int64])
@pytest.mark.parametrize("B,K", [(1, 1), (1, 4), (3, 2), (2, 7), (2, 8), (1, 9), (2, 16), (1, 32)])
def test_reorder_any_parents(B, K, idx, in_place):
    """Random parents, cycles, everything from one beam, unchanged, and places
    without a parent."""
    from paper_2608_02703_amd import BeamStates
    gen = torch.Generator().manual_seed(B * 64 + K)
    choices = [torch.randint(0, K, (B, K), generator=gen), torch.arange(K).flip(0).expand(B, K),
               torch.roll(torch.arange(K), 1).expand(B, K), torch.zeros((B, K), dtype=torch.int64),
               torch.full((B, K), K - 1), torch.arange(K).expand(B, K),
               torch.rand((B, K), generator=gen).argsort(1),
               torch.where(torch.rand((B, K), generator=gen) < 0.4, -1, torch.randint(0, K, (B, K), generator=gen)),
               torch.randint(-3, K + 3, (B, K), generator=gen)]
    for i, p in enumerate(choices):
        p = p.to(idx).contiguous().cuda()
        states = [_values((B * K, 3, 37, 16), torch.int16, 10 * i + j).cuda() for j in range(3)]
        out = None if in_place else [torch.full_like(s, -5) for s in states]
        want = [_want(s, s if in_place else d, p, K, None, None) for s, d in zip(states, out or states)]
        before = [s.clone() for s in states]
        got = BeamStates(states, K, out).reorder(p)
        for s, b, g, w in zip(states, before, got, want):
            assert torch.equal(g.cpu(), w), i
            assert in_place or torch.equal(s, b)


@pytest.mark.parametrize("K,n", [(1, 5), (1, 64), (4, 8), (8, 3), (32, 64)])
def test_reorder_to_another_number_of_beams(K, n):
    from paper_2608_02703_amd import BeamStates
    B = 3
    p = torch.randint(0, K, (B, n), generator=torch.Generator().manual_seed(n)).cuda()
    s = _values((B * K, 40, 24), torch.float32, 3).cuda()
    d = torch.zeros((B * n, 40, 24), device="cuda")
    want = _want(s, d, p, K, None, None)
    assert torch.equal(BeamStates([s], K, [d], n).reorder(p)[0].cpu(), want)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", [torch.int8, torch.float16, torch.float32, torch.int64])
@pytest.mark.parametrize("shape,p", [((5, 33, 64), 2), ((33, 5, 64), 1), ((33, 3), 1), ((2, 50, 5), 2), ((1, 1, 1), 2),
                                     ((7, 130), 2), ((600, 16), 1)])
def test_reorder_lengths(shape, p, dtype, in_place):
    """Leading positions only: lengths of 0, 1, part, all, and out of range;
    everything behind them stays."""
    from paper_2608_02703_amd import BeamStates
    B, K = 6, 4
    T = shape[p - 1]
    lengths = torch.tensor([0, 1, T // 2, T, T + 9, -4], dtype=torch.int32).cuda()
    q = torch.randint(0, K, (B, K), generator=torch.Generator().manual_seed(T)).cuda()
    states = [_values((B * K, *shape), dtype, j).cuda() for j in range(2)]
    out = None if in_place else [_values(s.shape, dtype, 7).cuda() for s in states]
    want = [_want(s, d, q, K, lengths, p) for s, d in zip(states, out or states)]
    for g, w in zip(BeamStates(states, K, out, pos_dim=p).reorder(q, lengths), want):
        assert torch.equal(g.cpu(), w)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", ["kv_views", "rows_second", "padded", "odd_bytes", "offset", "mixed"])
def test_reorder_strides(name, in_place):
    """Views: keys and values of one buffer, rows in the second dimension,
    padded rows, odd sizes and addresses, states of several shapes."""
    from paper_2608_02703_amd import BeamStates
    B, K = 2, 5
    R = B * K

    def make(seed):
        if name == "kv_views":
            kv = _values((R, 2, 3, 21, 32), torch.float16, seed).cuda()
            return [kv[:, 0], kv[:, 1]], 0, 2, kv
        if name == "rows_second":
            t = _values((21, R, 6, 8), torch.float16, seed).cuda()
            return [t], 1, 0, t
        if name == "padded":
            t = _values((R, 3, 21, 40), torch.float16, seed).cuda()
            return [t[..., :24]], 0, 2, t
        if name == "odd_bytes":
            t = _values((R, 3, 21, 7), torch.int8, seed).cuda()
            return [t], 0, 2, t
        if name == "offset":
            t = _values((R * 3 * 21 * 16 + 5,), torch.int16, seed).cuda()
            return [t[5:].view(R, 3, 21, 16)], 0, 2, t
        ts = [_values((R, h, 21, d), dt, seed + d).cuda() for h, d, dt in
              ((3, 16, torch.float16), (3, 16, torch.float16), (1, 5, torch.int8), (2, 4, torch.float32))]
        return ts, 0, 2, None
    states, r, p, whole = make(1)
    out, _, _, dwhole = (None, r, p, whole) if in_place else make(50)
    q = torch.randint(0, K, (B, K), generator=torch.Generator().manual_seed(3)).cuda()
    lengths = torch.tensor([21, 13], dtype=torch.int32).cuda()
    at = lambda t: t.movedim(r, 0).movedim((p if p > r else p + 1), 1)   # noqa: E731  rows, positions first
    want = [oracle.reorder(at(s).cpu().numpy(), at(d).cpu().numpy(), q.cpu().numpy(), K, lengths.cpu().numpy())
            for s, d in zip(states, out or states)]
    expected = None
    if dwhole is not None and name in ("padded", "offset"):
        expected = dwhole.clone()
    got = BeamStates(states, K, out, row_dim=r, pos_dim=p).reorder(q, lengths)
    for g, w in zip(got, want):
        assert torch.equal(at(g).cpu(), torch.from_numpy(w))
    if name == "padded":
        assert torch.equal(dwhole[..., 24:], expected[..., 24:])
    if name == "offset":
        assert torch.equal(dwhole[:5], expected[:5])


def test_reorder_many_states_and_graph():
    """More states than one launch takes, captured and replayed with other
    parents, in place: each replay moves the rows once more."""
    from paper_2608_02703_amd import BeamStates
    B, K = 2, 4
    states = [_values((B * K, 33, 8), torch.float16, j).cuda() for j in range(150)]
    ref = [s.cpu() for s in states]
    p = torch.zeros((B, K), dtype=torch.int64, device="cuda")
    p.copy_(torch.arange(K))
    plan = BeamStates(states, K)
    plan.reorder(p)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plan.reorder(p)
    for seed in range(4):
        q = torch.randint(0, K, (B, K), generator=torch.Generator().manual_seed(seed))
        p.copy_(q)
        g.replay()
        torch.cuda.synchronize()
        rows = (q + K * torch.arange(B)[:, None]).view(-1)
        ref = [t[rows] for t in ref]
        assert all(torch.equal(s.cpu(), t) for s, t in zip(states, ref))


@pytest.mark.parametrize("in_place", [False, True])
def test_reorder_beyond_the_caches(in_place):
    """More bytes than the caches hold (another kind of stores)."""
    from paper_2608_02703_amd import BeamStates
    B, K, T = 2, 3, 1001
    gen = torch.Generator(device="cuda").manual_seed(4)
    states = [torch.randint(0, 99, (B * K, 8, T, 4096), generator=gen, device="cuda", dtype=torch.int8)
              for _ in range(2)]
    out = None if in_place else [torch.full_like(s, 7) for s in states]
    p = torch.tensor([[2, 0, 2], [1, 2, 0]], device="cuda")
    lengths = torch.tensor([T, 650], dtype=torch.int32, device="cuda")
    old = [s.clone() for s in states]
    for s, g in zip(old, BeamStates(states, K, out, pos_dim=2).reorder(p, lengths)):
        for b in range(B):
            n = int(lengths[b])
            for j in range(K):
                assert torch.equal(g[b * K + j, :, :n], s[b * K + int(p[b, j]), :, :n])
                rest = s[b * K + j, :, n:]
                assert torch.equal(g[b * K + j, :, n:], rest if in_place else torch.full_like(rest, 7))


def test_reorder_far_rows():
    """Rows whose offsets pass 32 bits."""
    from paper_2608_02703_amd import BeamStates
    K, T, D = 4, 9, 64
    far = 1300 * 2 ** 20   # bytes between rows
    buf = torch.zeros(far * (K - 1) + T * D, dtype=torch.int8, device="cuda")
    s = buf.as_strided((K, T, D), (far, D, 1))
    s.copy_(_values((K, T, D), torch.int8, 5))
    old = s.cpu()
    p = torch.tensor([[3, 0, 3, 1]], device="cuda")
    BeamStates([s], K, pos_dim=1).reorder(p)
    assert torch.equal(s.cpu(), old[p[0].cpu()])


def test_reorder_refusals():
    from paper_2608_02703_amd import BeamStates
    s = torch.zeros((8, 5, 16), device="cuda")
    for bad in (lambda: BeamStates([s], 3), lambda: BeamStates([s], 0), lambda: BeamStates([s], 33),
                lambda: BeamStates([s], 4, out_beams=5), lambda: BeamStates([s], 4, [s]),
                lambda: BeamStates([s[:4]], 4, [s[2:6]]), lambda: BeamStates([s, s], 4),
                lambda: BeamStates([s], 4, [torch.zeros((8, 5, 17), device="cuda")]),
                lambda: BeamStates([s], 4, [torch.zeros((8, 5, 16), device="cuda").half()]),
                lambda: BeamStates([s], 4, []), lambda: BeamStates([s], 4, row_dim=3),
                lambda: BeamStates([s], 4, pos_dim=0), lambda: BeamStates([s, s[:4]], 4),
                lambda: BeamStates([s], 4).reorder(torch.zeros((2, 3), dtype=torch.int64, device="cuda")),
                lambda: BeamStates([s], 4).reorder(torch.zeros((2, 4), dtype=torch.int64)),
                lambda: BeamStates([s], 4).reorder(torch.zeros((2, 4), dtype=torch.int64, device="cuda"),
                                                   torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        BeamStates([s], 4).reorder(torch.zeros((2, 4), device="cuda"))
    empty = torch.zeros((8, 0, 16), device="cuda")
    p = torch.zeros((2, 4), dtype=torch.int64, device="cuda")
    assert BeamStates([empty], 4).reorder(p)[0] is empty
    assert BeamStates([], 4).reorder(p) == []


# ----------------------------------------------------------- used together
@pytest.mark.parametrize("B,K,n", [(1, 1, 1), (1, 4, 8), (2, 8, 8), (10, 5, 10), (40, 4, 8)])
def test_logits_beam_is_the_selection_over_the_heads_logits(B, K, n):
    """Every kernel that serves the head's logits (1 to 160 tokens)."""
    from paper_2608_02703_amd import PackedHead, beam_select
    from synth import make_head, make_x
    from tests.gpu_util import torch_x
    ph = PackedHead.from_arrays(make_head("tiny"))
    x = torch_x(make_x("tiny", B * K))
    scores = -torch.rand((B, K), generator=torch.Generator().manual_seed(n)).cuda()
    fin = torch.zeros((B, K), dtype=torch.bool, device="cuda")
    fin[0, -1] = True
    lg = ph.logits(x)
    got = ph.logits_beam(x, scores, n, finished=fin, end_token=5)
    want = beam_select(lg, scores, n, finished=fin, end_token=5)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    check(lg, scores, n, got, finished=fin, end_token=5)
    assert len(ph.logits_beam(x, scores, n)) == 3


def test_logits_beam_refusals():
    from paper_2608_02703_amd import ArcheadError, PackedHead
    from synth import make_head
    ph = PackedHead.from_arrays(make_head("tiny"))
    x = torch.zeros((4, 512), dtype=torch.bfloat16, device="cuda")
    s = torch.zeros((1, 4), device="cuda")
    with pytest.raises(ValueError):
        ph.logits_beam(x[:, :256], s, 4)
    with pytest.raises(ValueError):
        ph.logits_beam(x[:3], s, 4)
    with pytest.raises(TypeError):
        ph.logits_beam(x.float(), s, 4)
    with pytest.raises(ArcheadError):
        ph.logits_beam(x, s, 4, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ArcheadError):
        ph.logits_beam(x, s, 4, end_token=8192)


@pytest.mark.parametrize("kind", ["packed", "int8"])
def test_beam_search_end_to_end(kind):
    """A whole search over a toy model (the hidden state of a row is a function
    of its last token and step): logits of a packed or an INT8 head,
    selection, histories and states reordered in place, against the oracle
    taking the same steps on the same logits."""
    from paper_2608_02703_amd import BeamStates, PackedHead, beam_select, matmul_i8, quantize_i8
    from synth import make_head
    V, d, B, K, steps, end = 8192, 512, 3, 4, 7, 11
    gen = torch.Generator().manual_seed(2)
    embed = torch.randn((V, d), generator=gen).to(torch.bfloat16).cuda()
    if kind == "packed":
        ph = PackedHead.from_arrays(make_head("tiny"))
        bias = None
    else:
        wq, ws = quantize_i8((torch.randn((V, d), generator=gen) * 0.2).cuda())
        bias = torch.zeros(V, device="cuda")
        bias[end] = 14.0   # so that some hypotheses end
    scores = torch.full((B, K), -float("inf"), device="cuda")
    scores[:, 0] = 0
    fin = torch.zeros((B, K), dtype=torch.bool, device="cuda")
    history = torch.full((B * K, steps), -9, dtype=torch.int64, device="cuda")
    cache = torch.zeros((B * K, 2, steps, 16), dtype=torch.float16, device="cuda")
    plan, kv = BeamStates([history], K, pos_dim=1), BeamStates([cache], K, pos_dim=2)
    last = torch.arange(B * K, device="cuda") % K
    h_ref = history.cpu().numpy().copy()
    c_ref = cache.cpu().numpy().copy()
    for t in range(steps):
        x = embed[(last.clamp_min(0) * 7 + t) % V]
        lg = ph.logits(x) if kind == "packed" else matmul_i8(*quantize_i8(x), wq, ws, bias=bias)
        got = ph.logits_beam(x, scores, K, fin, end) if kind == "packed" else beam_select(lg, scores, K, fin, end)
        check(lg, scores, K, got, finished=fin, end_token=end)
        scores, parents, tokens, fin = got
        length = torch.full((B,), t, dtype=torch.int32, device="cuda")
        plan.reorder(parents, length)
        kv.reorder(parents, length)
        last = tokens.view(-1)
        history[:, t] = last
        cache[:, :, t] = (last % 97).to(torch.float16)[:, None, None]
        p = parents.cpu().numpy()
        h_ref = oracle.reorder(h_ref, h_ref, p, K, [t] * B)
        h_ref[:, t] = last.cpu().numpy()
        c_ref = oracle.reorder(c_ref.swapaxes(1, 2), c_ref.swapaxes(1, 2), p, K, [t] * B).swapaxes(1, 2)
        c_ref[:, :, t] = (last.cpu().numpy() % 97)[:, None, None]
        assert np.array_equal(history.cpu().numpy(), h_ref)
        assert np.array_equal(cache.cpu().numpy(), c_ref)
        assert (scores[:, :-1] >= scores[:, 1:]).all()
    if kind == "int8":
        assert fin.any()
