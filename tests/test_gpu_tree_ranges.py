"""Tree attention with values far from 1: small V rows, in the cache and among the
drafts, beside drafts with high scores; masked drafts of any finite size; V rows of
zeros.  The result scales with V, so its error has to as well.  Bound: that of test_gpu_tree.py, in which
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


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("size", [1.0, 1e-3, 2.0 ** -13])
@pytest.mark.parametrize("t,H", [(1, 2), (30, 2)])
def test_zero_rows_beside_small_values(wq, room, bits, size, t, H):
    """Rows of zeros among the cached V (attended to more than the others) and among the drafts'."""
    def spoil(q, kn, vn, k, v):
        for x in (v, vn):
            x.copy_(((x.float() + 0.5) * size).to(torch.bfloat16))
        for j in range(t):
            towards(q, kn, j, 7.0 if j % 3 else -3.0, 64 ** -0.5)
        k[:, 5], k[:, 700] = kn[:, 0], kn[:, t // 2]
        v[:, 5], v[:, 700], v[:, 300:310], vn[:, t // 2] = 0, 0, 0, 0
    close(*run(wq, room, 2, t, H, H, 64, bits, [1500, 600], seed=46, spoil=spoil))
    # one split a sequence, a row of zeros in every 16 positions of a tile
    def sixteenths(q, kn, vn, k, v):
        spoil(q, kn, vn, k, v)
        for p in range(5, 128, 16):
            k[:, p], v[:, p] = kn[:, 1 % t], 0
    close(*run(wq, room, 29, t, 12 * H, 12 * H, 64, bits, [800] * 28 + [701], seed=48, spoil=sixteenths))
    # every V row of the cache, or of the drafts, is zeros
    def empty(which):
        def f(q, kn, vn, k, v):
            (v if which else vn).zero_()
            (vn if which else v).copy_(((vn if which else v).float() * size).to(torch.bfloat16))
        return f
    for which in (0, 1):
        close(*run(wq, room, 1, t, H, H, 64, bits, [400], seed=47, spoil=empty(which)))


def test_a_row_of_zeros_is_marked(wq):
    """Scale 1 and zero -0 (any other row's is +0): what attention knows it by."""
    rows = torch.randn((1, 4, 1, 64)).to(torch.bfloat16)
    rows[0, 1] = 0
    rows[0, 2] = rows[0, 2].abs()  # zero point 0
    rows[0, 3] = 1e-9              # below the smallest scale: held as zeros
    for bits in (8, 4):
        c = wq.kv_cache(1, 1, 4, 64, bits)
        wq.kv_append(c, rows.cuda(), rows.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"))
        for m in (c.k_meta, c.v_meta):
            m = (m.cpu().flatten().long() & 0xffffffff).tolist()
            assert m[1] == m[3] == 0x80003c00 and m[0] >> 31 == 0 and m[2] >> 16 == 0
        k, v = wq.kv_read(c, torch.zeros(1, dtype=torch.int32, device="cuda"), 4, dtype=torch.float32)
        assert (k[0, 1] == 0).all() and (v[0, 3] == 0).all() and not torch.signbit(k[0, 1]).any()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("ratio", [2.0 ** 7, 2.0 ** 10, 2.0 ** 16, 2.0 ** 20])
@pytest.mark.parametrize("t", [1, 30])
def test_large_rows_that_hardly_count(wq, room, bits, ratio, t):
    """One V row far larger than the others and hardly attended to, and a row of zeros attended to more than all others:
    in whole tiles and in ragged ones, alone and with other tiles in a range."""
    def spoil(q, kn, vn, k, v):
        for j in range(t):
            q[:, j] = q[:, 0]
        for x in (v, vn):
            x.copy_(((x.float() + 0.5) * 2.0 ** -5).to(torch.bfloat16))
        d = q[:, 0].float()
        for p, score in ((70, -25.0), (v.shape[1] - 3, -25.0), (300, 9.0)):
            k[:, p] = (d * (score * 8 / d.pow(2).sum(-1, keepdim=True))).to(torch.bfloat16)
        v[:, 70], v[:, -3] = (v[:, 70].float() * ratio).to(torch.bfloat16), (v[:, -3].float() * -ratio).to(torch.bfloat16)
        v[:, 300] = 0
    close(*run(wq, room, 20, t, 24, 24, 64, bits, [800] * 19 + [701], seed=49, spoil=spoil))
    close(*run(wq, room, 1, t, 2, 2, 64, bits, [1000], seed=50, spoil=spoil))
    close(*run(wq, room, 1, t, 8, 8, 64, bits, [333], seed=51, spoil=spoil))
