"""Oracle of a dense head's softmax cross entropy and its gradients, in fp64
(torch, on the inputs' device), with what rounding errors are relative to."""
from __future__ import annotations

import torch


def head_loss(x, w, targets, grad=None):
    """x [M, d], w [V, d], targets [M], grad [M] or None -> dict of fp64 tensors:
    loss, lse [M]; reach [M], the largest sum of magnitudes of a token's
    logits; with grad also dx [M, d], dw [V, d], and their sums of magnitudes
    dx_mag and dw_mag, G's entries taken as |grad| (p + [v = y]).  Tokens without a
    target are left out."""
    f64 = torch.float64
    V = w.shape[0]
    y = targets.to(torch.int64)
    at = torch.nonzero((y >= 0) & (y < V)).reshape(-1)
    xs, ws, ys = x[at].to(f64), w.to(f64), y[at]
    wt = ws.t().contiguous()
    lg = xs @ wt
    lse = torch.logsumexp(lg, 1)
    M, d = x.shape
    one = lambda v: torch.zeros(M, dtype=f64, device=x.device).index_copy_(0, at, v)   # noqa: E731
    out = dict(loss=one(lse - lg.gather(1, ys[:, None])[:, 0]), lse=one(lse))
    out["reach"] = one((xs.abs() @ wt.abs()).amax(1)) if len(at) else one(lse)
    out["far"] = one((lse[:, None] - lg).amax(1)) if len(at) else one(lse)
    if grad is not None:
        p = torch.exp(lg - lse[:, None])
        g = grad[at].to(f64)[:, None]
        hot = torch.zeros_like(p).scatter_(1, ys[:, None], 1.0)
        G, mag = g * (p - hot), g.abs() * (p + hot)
        rows = lambda v: torch.zeros((M, d), dtype=f64, device=x.device).index_copy_(0, at, v)   # noqa: E731
        out["dx"], out["dx_mag"] = rows(G @ ws), rows(mag @ ws.abs())
        out["dw"], out["dw_mag"] = G.t().contiguous() @ xs, mag.t().contiguous() @ xs.abs()
    return out
