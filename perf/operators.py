"""Workloads of the operators around a head's logits that a generating
program runs: products of 8-bit integers (an INT8 head, and the layers below
it), the rounding of rows to 8 bits that feeds them, the choice of a beam
search's next hypotheses from their logits, and the reordering of the states
that the chosen ones continue.

  quantize   ``quantize_i8``: rows to int8 codes and one fp32 scale a row
  matmul     ``matmul_i8``: int8 [M, K] x int8 [N, K], a scale per row of each
  select     ``beam_select``: the n best (beam, token) pairs of every sequence
  reorder    ``BeamStates.reorder``: cache rows gathered by the chosen beams

With ``own`` false ``run`` computes them from elementary torch operations;
with ``own`` true it calls ``paper_2608_02703_amd``.  Sizes are those of this
repository's heads (``synth.CONFIGS``) and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4, "i8": 1}
_TINY = 2.0 ** -126     # smallest scale of a row
_MAX_CACHE = 48 * 16 * 8 * 1500 * 128 * 2   # bytes of the largest reorder case's destination
_MAX_LOGITS = 32 * 8 * 262144
_MAX_MACS = 4096 * 151936 * 4096
_MAX_QUANT = 151936 * 4096


def listed():
    return [
        # the hidden state of one decoded token, before an INT8 product
        dict(name="quantize_m1", op="quantize", M=1, d=4096, dtype="bf16"),
        # a ragged batch of wide fp32 rows whose length is odd
        dict(name="quantize_m777_odd", op="quantize", M=777, d=5003, dtype="f32"),
        # a head's rows rounded once when a model is loaded
        dict(name="quantize_head", op="quantize", M=151936, d=4096, dtype="bf16"),
        # one stream: logits of an INT8 head
        dict(name="matmul_m1", op="matmul", M=1, N=151936, K=4096, out="f32", bias=False),
        # four sequences of four beams on the largest vocabulary
        dict(name="matmul_m16", op="matmul", M=16, N=262144, K=2560, out="bf16", bias=False),
        # a prompt on a head with a bias and an odd vocabulary
        dict(name="matmul_m333_odd", op="matmul", M=333, N=50257, K=1536, out="f16", bias=True),
        # logits of a prefill-sized batch
        dict(name="matmul_m4096", op="matmul", M=4096, N=151936, K=4096, out="bf16", bias=False),
        # one sequence of four beams on a small vocabulary: launches and latency
        dict(name="select_b1k4", op="select", B=1, K=4, V=8192, n=8, dtype="f32", done=0, banned=0.0),
        # eight sequences of four beams, eight candidates each
        dict(name="select_b8k4", op="select", B=8, K=4, V=151936, n=8, dtype="f32", done=0, banned=0.0),
        # a full batch: ended beams among the live ones, tokens that a grammar
        # bans, an odd vocabulary in bf16
        dict(name="select_b32k8_bf16", op="select", B=32, K=8, V=262143, n=16, dtype="bf16", done=1,
             banned=0.2),
        # a short decoder's small cache, reordered where it lies; beams that
        # live on keep their rows
        dict(name="reorder_small_inplace", op="reorder", B=1, K=4, n=4, L=8, H=8, T=64, D=64, used=57,
             dtype="bf16", inplace=True),
        # the keys and values of 24 layers, into a second cache
        dict(name="reorder_cache", op="reorder", B=2, K=8, n=8, L=48, H=8, T=2048, D=128, used=1500,
             dtype="bf16", inplace=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["quantize", "matmul", "matmul", "select", "reorder"])
        if op == "quantize":
            case = dict(op=op, M=_log_int(rng, 1, 65536), d=_log_int(rng, 64, 16384),
                        dtype=rng.choice(["bf16", "f16", "f32"]))
            if case["M"] * case["d"] <= _MAX_QUANT:
                return case
        elif op == "matmul":
            K = _log_int(rng, 64, 16384)
            if rng.random() < 0.75:
                K = (K + 127) // 128 * 128
            case = dict(op=op, M=_log_int(rng, 1, 4096), N=_log_int(rng, 1024, 262144), K=K,
                        out=rng.choice(["f32", "bf16", "f16"]), bias=rng.random() < 0.3)
            if case["M"] * case["N"] * K <= _MAX_MACS and case["N"] * K <= _MAX_QUANT:
                return case
        elif op == "select":
            K = rng.choice([1, 2, 3, 4, 5, 8, 16])
            case = dict(op=op, B=_log_int(rng, 1, 64), K=K, V=_log_int(rng, 1000, 262144),
                        n=rng.choice([K, 2 * K]), dtype=rng.choice(["f32", "bf16", "f16"]),
                        done=rng.choice([0, 0, K // 3]), banned=rng.choice([0.0, 0.0, 0.3]))
            if case["B"] * K * case["V"] <= _MAX_LOGITS:
                return case
        else:
            K = rng.choice([2, 3, 4, 5, 8, 16])
            n = K
            inplace = rng.random() < 0.4
            if not inplace and rng.random() < 0.25:
                K, n = 1, K   # a prompt's cache, once for every beam
            T = _log_int(rng, 16, 4096)
            case = dict(op=op, B=_log_int(rng, 1, 8), K=K, n=n, L=rng.randint(2, 60), H=rng.choice([1, 2, 4, 8]),
                        T=T, D=rng.choice([64, 80, 96, 128, 256]), used=rng.randint(T // 2, T),
                        dtype=rng.choice(["bf16", "f16", "f32", "i8"]), inplace=inplace)
            size = case["L"] * case["B"] * n * case["H"] * T * case["D"] * _BYTES[case["dtype"]]
            if size <= _MAX_CACHE:
                return case


# ------------------------------------------------------------------ inputs
def _pattern(case):
    """One sequence's parents up to the beams' numbering, by the case alone:
    good beams are continued more than once, others not at all.  In place the
    beams that live on keep their rows."""
    K, n = case["K"], case["n"]
    r = random.Random(1000 * K + n)
    if case["inplace"]:
        live = max(1, (2 * K + 1) // 3)
        return [i if i < live else r.randrange(live) for i in range(n)]
    return [min(int(r.expovariate(2.0 / K)), K - 1) for _ in range(n)]


def _lengths(case):
    """Positions in use of each sequence."""
    B, used = case["B"], case["used"]
    return [max(1, used - b * used // (3 * B)) for b in range(B)]


def _randn(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dev = "cuda"
    if case["op"] == "quantize":   # hidden states or weights with a few large channels
        d = case["d"]
        channel = torch.exp(0.5 * _randn(d, gen))
        channel[torch.randint(0, d, (4,), generator=gen, device=dev)] *= 8
        x = torch.empty((case["M"], d), dtype=_DTYPES[case["dtype"]], device=dev)
        for m in range(0, case["M"], 16384):
            x[m:m + 16384] = _randn((min(16384, case["M"] - m), d), gen) * channel
        return dict(x=x)
    if case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        code = lambda r: torch.randint(-127, 128, (r, K), generator=gen, device=dev, dtype=torch.int8)  # noqa: E731
        scale = lambda r, s: _randn(r, gen).abs() * s + s / 4   # noqa: E731
        return dict(a=code(M), b=code(N), a_scales=scale(M, 0.02), b_scales=scale(N, 0.0005),
                    bias=_randn(N, gen) if case["bias"] else None)
    if case["op"] == "select":
        B, K, V = case["B"], case["K"], case["V"]
        lg = _randn((B * K, V), gen) * 2.5
        lg[:, torch.randint(0, V, (40,), generator=gen, device=dev)] += 6   # what the context asks for
        if case["banned"]:
            lg.masked_fill_(torch.rand(V, generator=gen, device=dev) < case["banned"], -math.inf)
        scores = (_randn((B, K), gen) * 4).abs().cumsum(1).neg()
        done = torch.zeros((B, K), dtype=torch.bool, device=dev)
        if case["done"]:
            at = torch.rand((B, K), generator=gen, device=dev).argsort(1)[:, :case["done"]]
            done.scatter_(1, at, True)
        return dict(logits=lg.to(_DTYPES[case["dtype"]]), scores=scores, finished=done if case["done"] else None,
                    end=V // 2 if case["done"] else -1)
    B, K, n = case["B"], case["K"], case["n"]
    base = torch.tensor(_pattern(case), device=dev)
    if K == n:   # the beams under other numbers in every sequence
        to = torch.rand((B, K), generator=gen, device=dev).argsort(1)
        parents = torch.empty((B, n), dtype=torch.int64, device=dev).scatter_(1, to, to[:, base])
    else:
        parents = base.expand(B, n).contiguous()
    shape = (case["H"], case["T"], case["D"])
    dt = _DTYPES[case["dtype"]]

    def cache(rows):
        if dt == torch.int8:
            return torch.randint(-127, 128, (rows, *shape), generator=gen, device=dev, dtype=dt)
        return torch.randn((rows, *shape), generator=gen, device=dev, dtype=dt)
    src = [cache(B * K) for _ in range(case["L"])]
    dst = src if case["inplace"] else [torch.zeros((B * n, *shape), dtype=dt, device=dev) for _ in src]
    return dict(src=src, dst=dst, parents=parents,
                lengths=torch.tensor(_lengths(case), dtype=torch.int32, device=dev))


def prepare(case, seed):
    state = dict(case=case, **_inputs(case, seed))
    if own and case["op"] == "reorder":   # a program describes its caches once
        from paper_2608_02703_amd import BeamStates
        state["plan"] = BeamStates(state["src"], case["K"], None if case["inplace"] else state["dst"], case["n"],
                                   pos_dim=2)
    return state


# ------------------------------------------------------------- plain forms
def _quantize(x):
    # 64 bits: quotients next to a half go to the same side whatever divides
    x = x.double()
    scale = (x.abs().amax(1) / 127).float().clamp_min(_TINY)
    return torch.round(x / scale.double()[:, None]).to(torch.int8), scale


def _matmul(a, b, a_scales, b_scales, bias, dtype):
    y = (a.float() @ b.float().T) * a_scales[:, None] * b_scales
    return (y if bias is None else y + bias).to(dtype)


def _select(logits, scores, n, finished, end):
    # 64 bits: scores of different beams that are nearly equal keep their order
    B, K = scores.shape
    V = logits.shape[1]
    s = logits.double().view(B, K, V)
    top = s.amax(2, keepdim=True)
    s = s - (top + (s - top).exp().sum(2, keepdim=True).log())
    cum = scores.double()[:, :, None]
    s = torch.where((s > -math.inf) & cum.isfinite(), s + cum, -math.inf)
    if finished is not None:
        f = finished[:, :, None]
        at_end = torch.arange(V, device=s.device) == end
        s = torch.where(f, torch.where(at_end & cum.isfinite(), cum, -math.inf), s)
    best, at = torch.sort(s.view(B, K * V), dim=1, descending=True, stable=True)
    best, at = best[:, :n], at[:, :n]
    some = best > -math.inf
    parents, tokens = torch.where(some, at // V, -1), torch.where(some, at % V, -1)
    out = [best.float(), parents, tokens]
    if finished is not None:
        out.append(some & ((tokens == end) | finished.gather(1, parents.clamp_min(0))))
    return tuple(out)


def _reorder(src, dst, parents, lengths, K):
    B, n = parents.shape
    rows = (parents + K * torch.arange(B, device=parents.device)[:, None]).view(-1)
    used = torch.arange(src[0].shape[2], device=rows.device) < lengths.repeat_interleave(n)[:, None]
    return [d.copy_(torch.where(used[:, None, :, None], s[rows], d)) for s, d in zip(src, dst)]


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        import paper_2608_02703_amd as lib
        if op == "quantize":
            return lib.quantize_i8(state["x"])
        if op == "matmul":
            return lib.matmul_i8(state["a"], state["a_scales"], state["b"], state["b_scales"], bias=state["bias"],
                                 out_dtype=_DTYPES[case["out"]])
        if op == "select":
            return lib.beam_select(state["logits"], state["scores"], case["n"], finished=state["finished"],
                                   end_token=state["end"])
        return state["plan"].reorder(state["parents"], state["lengths"])
    if op == "quantize":
        return _quantize(state["x"])
    if op == "matmul":
        return _matmul(state["a"], state["b"], state["a_scales"], state["b_scales"], state["bias"],
                       _DTYPES[case["out"]])
    if op == "select":
        return _select(state["logits"], state["scores"], case["n"], state["finished"], state["end"])
    return _reorder(state["src"], state["dst"], state["parents"], state["lengths"], case["K"])


# ----------------------------------------------------- work and exact values
def work(case):
    op = case["op"]
    if op == "quantize":
        n = case["M"] * case["d"]
        return {"bytes": n * (_BYTES[case["dtype"]] + 1) + 4 * case["M"], "flops": 4 * n}
    if op == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + 4 * (M + N) + (4 * N if case["bias"] else 0) + M * N * _BYTES[case["out"]],
                "flops": 2 * M * N * K}
    if op == "select":   # the logits of an ended beam say nothing
        live = case["B"] * (case["K"] - case["done"]) * case["V"]
        return {"bytes": live * _BYTES[case["dtype"]] + case["B"] * (5 * case["K"] + 21 * case["n"]), "flops": 4 * live}
    p = _pattern(case)
    moved = [(i, q) for i, q in enumerate(p) if not (case["inplace"] and i == q)]
    rows = len(moved) + len({q for _, q in moved})
    row = case["L"] * case["H"] * case["D"] * _BYTES[case["dtype"]]
    return {"bytes": sum(_lengths(case)) * row * rows + 8 * case["B"] * case["n"], "flops": 0}


def exact(case, seed):
    op = case["op"]
    i = _inputs(case, seed)
    if op == "reorder":
        parents, lengths, found = i["parents"].tolist(), i["lengths"].tolist(), []
        for s, d in zip(i["src"], i["dst"]):
            new = d.to(torch.float64)
            for b, (p, used) in enumerate(zip(parents, lengths)):
                for j, q in enumerate(p):
                    new[b * case["n"] + j, :, :used] = s[b * case["K"] + q, :, :used].to(torch.float64)
            found.append(new)
        return found
    if op == "quantize":
        codes, scales = [], []
        for x in i["x"].split(16384):
            x = x.to(torch.float64)
            s = torch.maximum(x.max(1).values, -x.min(1).values).div(127.0).to(torch.float32)
            s = torch.where(s < _TINY, torch.full_like(s, _TINY), s).to(torch.float64)
            q = x / s.unsqueeze(1)
            low = q.floor()
            up = (q - low > 0.5) | ((q - low == 0.5) & (low.remainder(2) == 1))   # halves to even
            codes.append((low + up).to(torch.int8))
            scales.append(s)
        return torch.cat(codes), torch.cat(scales)
    if op == "matmul":
        a = i["a"].to(torch.float64) * i["a_scales"].to(torch.float64).unsqueeze(1)
        parts = []
        for n in range(0, case["N"], 32768):
            b = i["b"][n:n + 32768].to(torch.float64) * i["b_scales"][n:n + 32768].to(torch.float64).unsqueeze(1)
            y = torch.matmul(a, b.t().contiguous())
            parts.append(y if i["bias"] is None else y + i["bias"][n:n + 32768].to(torch.float64))
        return torch.cat(parts, 1)
    B, K, V, n = case["B"], case["K"], case["V"], case["n"]
    scores = torch.full((B, n), -math.inf, dtype=torch.float64)
    parents = torch.full((B, n), -1, dtype=torch.int64)
    tokens = parents.clone()
    ended = torch.zeros((B, n), dtype=torch.bool)
    for b in range(B):
        lg = i["logits"][b * K:(b + 1) * K].to(torch.float64)
        s = i["scores"][b].to(torch.float64).unsqueeze(1) + torch.log_softmax(lg, 1)
        s = torch.nan_to_num(s, nan=-math.inf)
        if i["finished"] is not None:
            f = i["finished"][b]
            s[f] = -math.inf
            s[f, i["end"]] = i["scores"][b][f].to(torch.float64)
        s = s.reshape(-1)
        floor = torch.topk(s, min(n, s.numel())).values[-1]
        at = torch.nonzero((s >= floor) & (s > -math.inf)).reshape(-1)
        order = sorted(zip((-s[at]).tolist(), at.tolist()))[:n]
        for j, (v, q) in enumerate(order):
            scores[b, j], parents[b, j], tokens[b, j] = -v, q // V, q % V
            if i["finished"] is not None:
                ended[b, j] = q % V == i["end"] or bool(i["finished"][b, q // V])
    out = [scores, parents, tokens]
    if i["finished"] is not None:
        out.append(ended)
    return tuple(t.cuda() for t in out)
