"""The oracles of the norm, the adapters and the head loss against closed forms,
hand-made examples and each other (CPU)."""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import adapters, norm

torch = pytest.importorskip("torch")


def test_norm_by_hand():
    x = np.array([[3.0, -4.0], [0, 0]], np.float32)
    s, t, n, codes, u = norm.rms_norm(x, np.array([1.0, 0.5], np.float32), 0.0 + 1e-12)
    assert np.array_equal(s, x) and t.tolist() == [[3.0, -2.0], [0.0, 0.0]]
    assert math.isclose(n[0], math.sqrt(12.5), rel_tol=1e-12) and math.isclose(n[1], 1e-6, rel_tol=1e-9)
    assert codes.tolist() == [[127, -85], [0, 0]] and u[0] == np.float32(3 / 127) and u[1] == np.float32(2.0 ** -126)


def test_norm_adds_the_residual_and_the_offset():
    x, r = np.array([[1.0, 2.0]], np.float32), np.array([[0.5, -2.0]], np.float32)
    s, t, n, _, _ = norm.rms_norm(x, np.array([0.5, 1.0], np.float32), 1.0, r, 1.0)
    assert s.tolist() == [[1.5, 0.0]] and t.tolist() == [[2.25, 0.0]] and math.isclose(n[0], math.sqrt(2.125))


def test_norm_codes_stand_for_the_normed_row():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((7, 300)).astype(np.float32)
    w = rng.standard_normal(300).astype(np.float32)
    s, t, n, codes, u = norm.rms_norm(x, w, 1e-6)
    y = t.astype(np.float64) / n[:, None]
    step = u.astype(np.float64) / n
    assert (np.abs(codes * step[:, None] - y) <= step[:, None] * 0.500001).all()
    x[3, 5] = np.nan
    assert np.isnan(norm.rms_norm(x, w, 1e-6)[4][3])


def test_adapters_by_hand():
    y = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]])
    x = np.array([[1.0, 1.0, 0.0]] * 3)
    a = np.array([[[1.0, 2.0, 9.0], [0.0, 1.0, 9.0]], [[2.0, 0.0, 0.0], [5.0, 5.0, 5.0]]])
    b = np.array([[[1.0, 0.0], [0.0, -1.0]], [[1.0, 7.0], [3.0, 7.0]]])
    out, bound = adapters.add(y, x, a, b, [0, -1, 1], scales=[2.0, 0.5], ranks=[2, 1])
    assert out.tolist() == [[1 + 2 * 3, 2 - 2 * 1], [3.0, 4.0], [5 + 0.5 * 2, 6 + 0.5 * 6]]
    assert bound.tolist() == [[6.0, 2.0], [0.0, 0.0], [1.0, 3.0]]
    assert adapters.add(y, x, a, b, [2, 5, -7])[0].tolist() == y.tolist()


def test_head_loss_by_autograd_and_by_hand():
    from oracle import loss
    torch.manual_seed(1)
    x, w = torch.randn(5, 6, dtype=torch.float64), torch.randn(9, 6, dtype=torch.float64)
    y, g = torch.tensor([0, 8, -100, 3, 9]), torch.randn(5, dtype=torch.float64)
    o = loss.head_loss(x, w, y, g)
    xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
    lg = xa @ wa.t()
    live = torch.tensor([0, 1, 3])
    each = torch.nn.functional.cross_entropy(lg[live], y[live], reduction="none")
    (each * g[live]).sum().backward()
    assert torch.allclose(o["loss"][live], each.detach()) and not o["loss"][[2, 4]].any() and not o["lse"][[2, 4]].any()
    assert torch.allclose(o["dx"], xa.grad) and torch.allclose(o["dw"], wa.grad)
    assert (o["dx"].abs() <= o["dx_mag"] + 1e-12).all() and (o["dw"].abs() <= o["dw_mag"] + 1e-12).all()
    even = loss.head_loss(torch.zeros(1, 4, dtype=torch.float64), torch.ones(8, 4, dtype=torch.float64), torch.tensor([2]))
    assert math.isclose(float(even["loss"]), math.log(8))
