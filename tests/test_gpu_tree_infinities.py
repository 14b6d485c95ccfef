"""Infinities and NaN among the V values of a bf16 cache: every row that sees one has
it in that column (opposite ones: NaN), and no other column changes.  Bound: that of
test_gpu_tree.py.
"""
import math

import pytest
import torch

from test_gpu_tree import close, room, run, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("t,H,L", [(1, 4, 300), (5, 4, 300), (12, 4, 130), (30, 8, 700), (40, 8, 64), (64, 8, 1000)])
def test_infinite_values_of_a_bf16_cache(wq, room, hd, t, H, L):
    def spoil(q, kn, vn, k, v):
        v[0, 20, 0, 17] = math.inf
        v[0, L - 1, 0, 40] = -math.inf
        v[0, 3, 0, 0], v[0, 50, 0, 0] = math.inf, -math.inf
        v[0, 60, 0, 63] = math.nan
        v[0, 10, 0, 5], v[0, 11, 0, 5] = math.inf, math.inf
        v[0, 9, 0, 33], vn[0, 0, 0, 33] = -math.inf, math.inf
    o, ref, tol = run(wq, room, 2, t, H, 1, hd, 16, [L, 70], seed=51, spoil=spoil)
    inf = math.inf
    assert (ref[0, :, :, 17] == inf).all() and (ref[0, :, :, 40] == -inf).all() and (ref[0, :, :, 5] == inf).all()
    assert ref[0, :, :, 0].isnan().all() and ref[0, :, :, 63].isnan().all() and ref[0, :, :, 33].isnan().all()
    assert torch.isfinite(ref[1]).all() and int(torch.isfinite(ref[0, 0, 0]).sum()) == hd - 6
    close(o, ref, tol)
