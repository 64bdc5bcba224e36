"""Workloads of the operators that stand right before, beside and behind a
head or an INT8 layer:

  norm      ``rms_norm`` / ``rms_norm_i8``: the residual's addition, the root-mean-square norm, and its
            rows in 16 bits (for a packed head) or rounded to 8 bits with a scale each (for ``matmul_i8``)
  adapters  ``adapters_add``: low-rank adapters of many requests at once, added to a shared projection's output
  loss      ``head_loss``: softmax cross entropy of a dense bf16 head over its whole vocabulary, no logits kept
  step      ``head_loss`` and ``head_loss_grad``: the same with the gradients of the hidden states and of the head

With ``own`` false ``run`` computes them from elementary torch operations;
with ``own`` true it calls ``paper_2608_02703_amd``.  Sizes are those of this
repository's heads (``synth.CONFIGS``) and generic ones.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_TINY = 2.0 ** -126     # smallest step of a row's codes
_EPS = 1e-6
_MAX_NORM = 16384 * 8192
_MAX_LOSS = 4096 * 151936 * 4096
_MAX_ADAPTED = 8192 * (4096 + 14336)


def listed():
    return [
        # the hidden state of one decoded token, between two INT8 layers
        dict(name="norm_m1", op="norm", M=1, d=4096, dtype="bf16", residual=True, codes=True, normed=False, offset=0.0),
        # a ragged batch of wide fp32 rows whose length is odd
        dict(name="norm_m777_odd", op="norm", M=777, d=5003, dtype="f32", residual=False, codes=True, normed=True,
             offset=0.0),
        # the last norm before a packed head, weights held as w - 1
        dict(name="norm_m4096_final", op="norm", M=4096, d=2560, dtype="bf16", residual=True, codes=False, normed=True,
             offset=1.0),
        # a long prompt: 8 bits for the projection, 16 for the adapters beside it
        dict(name="norm_m16384", op="norm", M=16384, d=8192, dtype="bf16", residual=True, codes=True, normed=True,
             offset=0.0),
        # sixteen sequences that decode, each with an adapter of its own
        dict(name="adapters_m16", op="adapters", M=16, K=4096, N=4096, R=16, n=16, dtype="bf16", y="bf16",
             layout="mixed", none=0.0, ragged=False),
        # a full decoding batch: 32 adapters of several ranks, some tokens without one
        dict(name="adapters_m256", op="adapters", M=256, K=4096, N=14336, R=32, n=32, dtype="bf16", y="bf16",
             layout="mixed", none=0.2, ragged=True),
        # adapters of an odd vocabulary beside an INT8 head's fp32 logits
        dict(name="adapters_m333_odd", op="adapters", M=333, K=1536, N=50257, R=12, n=5, dtype="f16", y="f32",
             layout="runs", none=0.1, ragged=True),
        # prompts of eight requests, one after another
        dict(name="adapters_m8192", op="adapters", M=8192, K=4096, N=14336, R=64, n=8, dtype="bf16", y="bf16",
             layout="runs", none=0.0, ragged=False),
        # the loss of a few tokens on the small head: launches and latency
        dict(name="loss_m8", op="loss", M=8, V=8192, d=512, ignored=0.0),
        # evaluation of a ragged batch on an odd vocabulary
        dict(name="loss_m333_odd", op="loss", M=333, V=50257, d=1536, ignored=0.1),
        # a training step on answers alone: the prompts' tokens have no target
        dict(name="step_m1024_answers", op="step", M=1024, V=262144, d=2560, ignored=0.4, head=True),
        # a training step of the largest batch
        dict(name="step_m4096", op="step", M=4096, V=151936, d=4096, ignored=0.0, head=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _even(rng, x, to):
    """x, three times in four as the next multiple of `to`."""
    return (x + to - 1) // to * to if rng.random() < 0.75 else x


def draw(rng):
    while True:
        op = rng.choice(["norm", "adapters", "loss", "step"])
        if op == "norm":
            codes = rng.random() < 0.7
            case = dict(op=op, M=_log_int(rng, 1, 16384), d=_even(rng, _log_int(rng, 64, 16384), 64),
                        dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), residual=rng.random() < 0.7, codes=codes,
                        normed=not codes or rng.random() < 0.3, offset=rng.choice([0.0, 0.0, 1.0]))
            if case["M"] * case["d"] <= _MAX_NORM:
                return case
        elif op == "adapters":
            case = dict(op=op, M=_log_int(rng, 1, 8192), K=_even(rng, _log_int(rng, 256, 16384), 64),
                        N=_even(rng, _log_int(rng, 256, 65536), 64), R=rng.choice([4, 8, 12, 16, 24, 32, 50, 64, 128]),
                        n=rng.randint(1, 40), dtype=rng.choice(["bf16", "bf16", "f16"]),
                        y=rng.choice(["bf16", "f16", "f32"]), layout=rng.choice(["mixed", "runs"]),
                        none=rng.choice([0.0, 0.0, 0.3]), ragged=rng.random() < 0.5)
            if case["M"] * (case["K"] + case["N"]) <= _MAX_ADAPTED and case["n"] * case["R"] <= 2048:
                return case
        else:
            case = dict(op=op, M=_log_int(rng, 1, 8192), V=_log_int(rng, 1000, 262144),
                        d=_even(rng, _log_int(rng, 128, 8192), 64), ignored=rng.choice([0.0, 0.0, 0.2, 0.6]))
            if op == "step":
                case["head"] = rng.random() < 0.7
            if case["M"] * case["V"] * case["d"] <= _MAX_LOSS and case["V"] * case["d"] <= 151936 * 8192 \
                    and case["M"] * case["V"] <= 4096 * 262144:
                return case


# ------------------------------------------------------------------ inputs
def _randn(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _live(case):
    """Tokens of a loss that have a target."""
    return case["M"] - int(case["M"] * case["ignored"])


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dev, M = "cuda", case["M"]
    if case["op"] == "norm":   # hidden states with a few large channels
        d, dt = case["d"], _DTYPES[case["dtype"]]
        channel = torch.exp(0.5 * _randn(d, gen))
        channel[torch.randint(0, d, (4,), generator=gen, device=dev)] *= 8
        return dict(x=(_randn((M, d), gen) * channel).to(dt),
                    residual=(_randn((M, d), gen) * channel * 3).to(dt) if case["residual"] else None,
                    weight=(1 - case["offset"] + 0.3 * _randn(d, gen)).to(dt))
    if case["op"] == "adapters":
        n, R, K, N, dt = case["n"], case["R"], case["K"], case["N"], _DTYPES[case["dtype"]]
        if case["layout"] == "runs":   # requests one after another
            ids = torch.randint(0, n, (M,), generator=gen, device=dev).sort().values
        else:
            ids = torch.randint(0, n, (M,), generator=gen, device=dev)
            if M == n:
                ids = torch.rand(n, generator=gen, device=dev).argsort()
        if case["none"]:   # tokens of requests without an adapter
            ids = torch.where(torch.rand(M, generator=gen, device=dev) < case["none"], -1, ids)
        ranks = None
        if case["ragged"]:
            ranks = torch.randint(1, R + 1, (n,), generator=gen, device=dev, dtype=torch.int32)
            ranks[0] = R
        return dict(x=_randn((M, K), gen).to(dt), y=(_randn((M, N), gen) * 2).to(_DTYPES[case["y"]]),
                    a=(_randn((n, R, K), gen) / math.sqrt(K)).to(dt), b=(_randn((n, N, R), gen) * 0.3).to(dt),
                    ids=ids.to(torch.int32), ranks=ranks,
                    scales=0.5 + torch.rand(n, generator=gen, device=dev))
    V, d = case["V"], case["d"]
    w = torch.empty((V, d), dtype=torch.bfloat16, device=dev)
    spread = 2 / math.sqrt(d)
    for v in range(0, V, 32768):
        w[v:v + 32768] = _randn((min(32768, V - v), d), gen) * spread
    targets = torch.randint(0, V, (M,), generator=gen, device=dev)
    # hidden states that lean towards their token, as a trained model's do
    lean = 2.5 * torch.rand((M, 1), generator=gen, device=dev)
    x = (_randn((M, d), gen) + lean * w[targets].float()).to(torch.bfloat16)
    live = _live(case)
    order = torch.rand(M, generator=gen, device=dev).argsort()
    targets[order[live:]] = -100
    return dict(x=x, w=w, targets=targets, grad=torch.full((M,), 1.0 / max(live, 1), device=dev))


def prepare(case, seed):
    return dict(case=case, **_inputs(case, seed))


# ------------------------------------------------------------- plain forms
def _norm(x, residual, weight, offset, codes, normed):
    dt = x.dtype
    s = x.float()
    if residual is not None:
        s = s + residual.float()
    t = s * (offset + weight.float())
    # 64 bits: quotients next to a half go to the same side whatever divides
    rs = (s.double().square().mean(1) + _EPS).rsqrt()
    out = []
    if codes:
        step = (t.abs().amax(1).double() / 127).float().clamp_min(_TINY).double()
        out += [torch.round(t.double() / step[:, None]).to(torch.int8), (step * rs).float()]
    if residual is not None:
        out.append(s.to(dt))
    if normed:
        out.append((t * rs.float()[:, None]).to(dt))
    return tuple(out)


def _adapters(y, x, a, b, ids, scales, ranks):
    # every token's products with every adapter, those of others made zero
    n, R, K = a.shape
    t = (x.float() @ a.reshape(n * R, K).float().T).view(-1, n, R)
    at = torch.arange(n, device=x.device)
    t = torch.where(ids[:, None, None] == at[:, None], t * scales[:, None], 0.0)
    if ranks is not None:
        t = torch.where(torch.arange(R, device=x.device) < ranks[:, None], t, 0.0)
    up = b.permute(0, 2, 1).reshape(n * R, -1).float()
    return (y.float() + t.view(-1, n * R) @ up).to(y.dtype)


def _loss(x, w, targets, grad, head):
    V = w.shape[0]
    live = (targets >= 0) & (targets < V)
    y = torch.where(live, targets, 0)[:, None]
    x, wf = torch.where(live[:, None], x.float(), 0.0), w.float()
    p = x @ wf.T
    top = p.amax(1, keepdim=True)
    at = p.gather(1, y)
    lse = top + (p - top).exp().sum(1, keepdim=True).log()
    loss = torch.where(live, (lse - at)[:, 0], 0.0)
    if grad is None:
        return loss, torch.where(live, lse[:, 0], 0.0)
    p = p.sub_(lse).exp_()
    p.scatter_(1, y, p.gather(1, y) - 1)
    p *= torch.where(live, grad, 0.0)[:, None]
    dx = (p @ wf).to(w.dtype)
    return (loss, dx, (p.T @ x).to(w.dtype)) if head else (loss, dx)


def run(state):
    s, case, op = state, state["case"], state["case"]["op"]
    if own:
        import paper_2608_02703_amd as lib
        if op == "norm":
            if case["codes"]:
                return lib.rms_norm_i8(s["x"], s["weight"], eps=_EPS, residual=s["residual"], offset=case["offset"],
                                       normed=case["normed"])
            out = lib.rms_norm(s["x"], s["weight"], eps=_EPS, residual=s["residual"], offset=case["offset"])
            return out[::-1] if isinstance(out, tuple) else (out,)   # the sums first, as for 8 bits
        if op == "adapters":
            return lib.adapters_add(s["y"], s["x"], s["a"], s["b"], s["ids"], scales=s["scales"], ranks=s["ranks"])
        loss, lse = lib.head_loss(s["x"], s["w"], s["targets"])
        if op == "loss":
            return loss, lse
        dx, dw = lib.head_loss_grad(s["x"], s["w"], s["targets"], lse, s["grad"], dw=case["head"])
        return (loss, dx, dw) if case["head"] else (loss, dx)
    if op == "norm":
        return _norm(s["x"], s["residual"], s["weight"], case["offset"], case["codes"], case["normed"])
    if op == "adapters":
        return _adapters(s["y"], s["x"], s["a"], s["b"], s["ids"], s["scales"], s["ranks"])
    return _loss(s["x"], s["w"], s["targets"], s["grad"] if op == "step" else None, case.get("head"))


# ----------------------------------------------------- work and exact values
def work(case):
    op, M = case["op"], case["M"]
    if op == "norm":
        n, size = M * case["d"], _BYTES[case["dtype"]]
        each = size * (1 + 2 * case["residual"] + case["normed"]) + case["codes"]
        return {"bytes": n * each + size * case["d"] + 4 * M * case["codes"], "flops": 6 * n}
    if op == "adapters":   # the adapters that some token has, at most (ranks at their mean)
        K, N, R = case["K"], case["N"], case["R"]
        used, rank = min(case["n"], M), (R + 1) / 2 if case["ragged"] else R
        with_one = M * (1 - case["none"])
        return {"bytes": int(used * rank * (K + N) * 2 + with_one * K * 2 + 2 * M * N * _BYTES[case["y"]] + 4 * M),
                "flops": int(2 * with_one * rank * (K + N))}
    V, d, live = case["V"], case["d"], _live(case)
    if op == "loss":
        return {"bytes": 2 * d * (V + live) + 16 * M, "flops": 2 * live * V * d}
    return {"bytes": 2 * d * (V + live + M + (V if case["head"] else 0)) + 16 * M,
            "flops": (6 if case["head"] else 4) * live * V * d}


def exact(case, seed):
    i = _inputs(case, seed)
    f64 = torch.float64
    if case["op"] == "norm":
        x, w = i["x"].to(torch.float32), i["weight"].to(torch.float32).add(case["offset"])
        if case["residual"]:
            x = torch.add(x, i["residual"].to(torch.float32))
        t = torch.mul(x, w).to(f64)
        x = x.to(f64)
        inv = 1.0 / torch.sqrt(torch.einsum("md,md->m", x, x) / case["d"] + _EPS)
        out = []
        if case["codes"]:
            u = torch.maximum(t.max(1).values, -t.min(1).values).div(127.0).to(torch.float32)
            u = torch.where(u < _TINY, torch.full_like(u, _TINY), u).to(f64)
            q = t / u.unsqueeze(1)
            low = q.floor()
            up = (q - low > 0.5) | ((q - low == 0.5) & (low.remainder(2) == 1))   # halves to even
            out += [(low + up).to(torch.int8), u * inv]
        if case["residual"]:
            out.append(x)
        if case["normed"]:
            out.append(t * inv.unsqueeze(1))
        return tuple(out)
    if case["op"] == "adapters":
        y = i["y"].to(f64)
        for k in range(case["n"]):
            rows = torch.nonzero(i["ids"] == k).reshape(-1)
            r = case["R"] if i["ranks"] is None else int(i["ranks"][k])
            t = torch.mm(i["x"][rows].to(f64), i["a"][k, :r].to(f64).t().contiguous())
            y[rows] += torch.mm(t, i["b"][k, :, :r].to(f64).t().contiguous()) * i["scales"][k].to(f64)
        return y
    M, V, d = case["M"], case["V"], case["d"]
    rows = torch.nonzero(i["targets"] >= 0).reshape(-1)
    x, y = i["x"][rows].to(f64), i["targets"][rows]
    lse = torch.full((len(rows),), -math.inf, dtype=f64, device=x.device)
    at = torch.zeros_like(lse)
    pieces = [(v, i["w"][v:v + 16384].to(f64)) for v in range(0, V, 16384)]
    for v, w in pieces:
        lg = torch.mm(x, w.t().contiguous())
        lse = torch.logaddexp(lse, torch.logsumexp(lg, 1))
        here = torch.nonzero((y >= v) & (y < v + len(w))).reshape(-1)
        at[here] = lg[here, y[here] - v]
    full = torch.zeros((2, M), dtype=f64, device=x.device)
    full[0, rows], full[1, rows] = lse - at, lse
    if case["op"] == "loss":
        return full[0], full[1]
    dx, dw = torch.zeros((M, d), dtype=f64, device=x.device), []
    g = i["grad"][rows].to(f64)
    for v, w in pieces:
        p = torch.exp(torch.mm(x, w.t().contiguous()) - lse.unsqueeze(1))
        here = torch.nonzero((y >= v) & (y < v + len(w))).reshape(-1)
        p[here, y[here] - v] -= 1
        p = p * g.unsqueeze(1)
        dx[rows] += torch.mm(p, w)
        if case["head"]:
            dw.append(torch.mm(p.t().contiguous(), x))
    return (full[0], dx, torch.cat(dw)) if case["head"] else (full[0], dx)
