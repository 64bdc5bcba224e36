"""The oracles of the 8-bit products and of beam search against closed forms
and hand-made examples (CPU)."""
from __future__ import annotations

from fractions import Fraction

import numpy as np

from oracle import beam, int8


def _nearest(x, s):
    q = Fraction(float(x)) / Fraction(float(s))
    low = q.numerator // q.denominator
    rest = q - low
    return low + (rest > Fraction(1, 2) or (rest == Fraction(1, 2) and low % 2 == 1))


def test_quantize_against_exact_fractions():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((6, 40)) * 10.0 ** rng.integers(-30, 30, (6, 1))).astype(np.float32)
    x[0] = 0
    x[1, :4] = [127, 0.5, 1.5, -2.5]
    x[1, 4:] = 3
    q, s = int8.quantize(x)
    assert s[0] == np.float32(2.0 ** -126) and not q[0].any()
    assert s[1] == 1 and q[1, :4].tolist() == [127, 0, 2, -2]
    for r in range(1, 6):
        assert abs(float(s[r]) * 127 / np.abs(x[r]).max() - 1) < 1e-6
        assert [int(v) for v in q[r]] == [_nearest(v, s[r]) for v in x[r]]


def test_quantize_marks_rows_that_are_not_finite():
    x = np.ones((3, 4), np.float32)
    x[0, 1], x[1, 2] = np.nan, -np.inf
    q, s = int8.quantize(x)
    assert np.isnan(s[:2]).all() and not q[:2].any() and (q[2] == 127).all()


def test_matmul_by_hand():
    a, b = np.array([[1, -2, 3]], np.int8), np.array([[4, 5, -6], [-128, 127, 0]], np.int8)
    y, p = int8.matmul(a, np.array([0.5], np.float32), b, np.array([2, 0.25], np.float32), np.array([1, -1], np.float32))
    assert p.tolist() == [[-24.0, -47.75]] and y.tolist() == [[-23.0, -48.75]]


def test_select_by_hand():
    lg = np.log(np.array([[0.5, 0.25, 0.25], [0.125, 0.125, 0.75]]))
    vals, parents, tokens, ended = beam.select(lg, np.array([[0.0, 0.0]]), 4, end_token=2)
    assert parents.tolist() == [[1, 0, 0, 0]] and tokens.tolist() == [[2, 0, 1, 2]]
    assert ended.tolist() == [[True, False, False, True]]
    assert np.allclose(np.exp(vals), [[0.75, 0.5, 0.25, 0.25]])


def test_select_leaves_out_what_is_no_candidate():
    lg = np.zeros((5, 2))
    lg[0] = -np.inf
    lg[1, 0] = np.nan
    lg[2, 1] = np.inf
    lg[4, 1] = -np.inf
    vals, parents, tokens, ended = beam.select(lg, np.array([[0, 0, 0, -np.inf, -1.0]]), 2)
    assert parents.tolist() == [[4, -1]] and tokens.tolist() == [[0, -1]]
    assert vals.tolist() == [[-1.0, -np.inf]]


def test_select_ended_beams_keep_their_score():
    vals, parents, tokens, ended = beam.select(np.zeros((2, 4)), np.array([[-5.0, -0.5]]), 2,
                                               finished=np.array([[False, True]]), end_token=3)
    assert parents.tolist() == [[1, 0]] and tokens.tolist() == [[3, 0]]
    assert vals[0, 0] == -0.5 and ended.tolist() == [[True, False]]


def test_reorder_by_hand():
    s = np.arange(8).reshape(4, 2)
    p = np.array([[1, 0], [-1, 1]])
    assert beam.reorder(s, s, p, 2).tolist() == [[2, 3], [0, 1], [4, 5], [6, 7]]
    assert beam.reorder(s, s, p, 2, lengths=[1, 0]).tolist() == [[2, 1], [0, 3], [4, 5], [6, 7]]
