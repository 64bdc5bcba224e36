"""archead_beam_reorder refuses states whose rows, blocks and positions reach past
what 64-bit offsets hold, before any HIP call (CPU; every pointer given is a
number that no call follows)."""
from __future__ import annotations

import pytest

from paper_2608_02703_amd import archead as ab
from tests.test_operators_host import L, _reorder  # noqa: F401  (L: a fixture)

BIG = 2 ** 42


@pytest.mark.parametrize("layout,kw", [
    (dict(src_row=BIG), dict(B=2 ** 24, K=32, n=32)), (dict(dst_row=BIG), dict(B=2 ** 24, K=32, n=32)),
    (dict(dst_row=BIG), dict(B=2 ** 20, K=1, n=64)), (dict(src_row=BIG), dict(B=2 ** 20, K=2, n=1)),
    (dict(n_outer=2 ** 22, src_outer=BIG), {}), (dict(n_outer=2 ** 22, dst_outer=BIG), {}),
    (dict(positions=2 ** 22, src_pos=BIG), {}), (dict(positions=2 ** 22, dst_pos=BIG), {}),
    (dict(n_outer=2 ** 20, positions=2 ** 20, pos_bytes=16, src_outer=BIG, src_pos=BIG, src_row=BIG), dict(B=2 ** 19)),
])
def test_reaches_past_64_bits(L, layout, kw):   # noqa: F811
    assert _reorder(L, layout, **kw) == ab.E_INVALID_ARG
    assert b"2^62" in L.archead_last_error()


@pytest.mark.parametrize("layout,kw", [(dict(src_row=BIG, dst_row=BIG), dict(B=0)), (dict(src_row=BIG), dict(ns=0, B=2 ** 17)),
                                       (dict(n_outer=1, src_outer=BIG, positions=0, dst_pos=BIG), {})])
def test_strides_without_steps(L, layout, kw):   # noqa: F811
    assert _reorder(L, layout, **kw) == ab.OK
