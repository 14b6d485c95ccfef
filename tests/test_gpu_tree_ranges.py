"""Tree attention with values far from 1: small V rows, in the cache and among the
drafts, beside drafts with high scores; masked drafts of any finite size.  The result
scales with V, so its error has to as well.  Bound: that of test_gpu_tree.py, in which
every term is relative to V's size.
"""
import math

import pytest
import torch

from test_gpu_tree import close, room, run, wq  # noqa: F401

pytestmark = pytest.mark.gpu


def towards(q, kn, j, score, scale):
    """Draft j's key along the query of the same draft (one query head a kv head), with this score (natural units)."""
    d = q[:, j].float()
    kn[:, j] = (d * (score / scale / d.pow(2).sum(-1, keepdim=True))).to(torch.bfloat16)


def small(score, size, hd):
    def spoil(q, kn, vn, k, v):
        for j in range(q.shape[1]):
            towards(q, kn, j, score, hd ** -0.5)
        for x in (v, vn):
            x.copy_(((x.float() + 0.5) * size).to(torch.bfloat16))
    return spoil


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -7, 1e-3, 2.0 ** -13, 1000.0])
@pytest.mark.parametrize("score", [8.0, 10.0])
def test_small_values_beside_a_high_draft(wq, room, bits, size, score):
    # 232 heads of one row: one split a sequence on 152 SMs
    close(*run(wq, room, 29, 1, 8, 8, 64, bits, [1500] * 28 + [77], seed=41, spoil=small(score, size, 64)))
    close(*run(wq, room, 1, 3, 2, 2, 128, bits, [2500], seed=42, spoil=small(score, size, 128)))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("size", [1.0, 1e-3, 2.0 ** -13])
def test_small_values_many_drafts(wq, room, bits, size):
    close(*run(wq, room, 2, 40, 2, 2, 128, bits, [700, 1500], seed=43, spoil=small(9.0, size, 128)))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("ratio", [2.0 ** -12, 2.0 ** 12])
@pytest.mark.parametrize("t", [1, 24])
def test_drafts_of_another_size_than_the_context(wq, room, bits, ratio, t):
    def spoil(q, kn, vn, k, v):
        for j in range(t):
            towards(q, kn, j, -8.0 if ratio > 1 else 8.0, 64 ** -0.5)
        vn.copy_((vn.float() * ratio).to(torch.bfloat16))
    close(*run(wq, room, 2, t, 4, 4, 64, bits, [300, 1200], seed=44, spoil=spoil))


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("t,H", [(12, 2), (40, 8)])
@pytest.mark.parametrize("size", [3e38, 1e20, 1e9])
def test_masked_drafts_of_any_size(wq, room, bits, t, H, size):
    """Drafts that only themselves see, or no one, with finite K and V of any size."""
    def spoil(q, kn, vn, k, v):
        vn[0, 5], vn[1, 7] = size, -size
        kn[0, 6], kn[1, 7] = -size, size
        vn[1, 0] = (vn[1, 0].float() / size).to(torch.bfloat16)

    vis = torch.ones((2, t, t), dtype=torch.bool).tril()
    vis[0, :, 5:7] = False
    vis[0, 5, 5] = True
    vis[1, :, 7] = False
    o, ref, tol = run(wq, room, 2, t, H, 1, 128, bits, [200, 90], vis=vis, seed=45, spoil=spoil)
    assert float(ref[0, 5].abs().max()) > 1e6 and float(ref[0, 7:].abs().max()) < 100 and float(ref[1].abs().max()) < 100
    close(o, ref, tol)
