"""Attention over pages where a row's scores are far from zero: softmax does not change when all of them are shifted, so neither
may the result, in either kernel."""
import math

import pytest
import torch

from paged_util import attn_ref, check, fill_pool, i32, pool_values, status
from paper_2606_04238_gb300 import wq
from test_gpu_paged import BF, ragged, randn

pytestmark = pytest.mark.gpu


def shifted(nq, n, hd, bits, level, page=32, h=8, kv=2, seed=0):
    """One sequence (q, cu, tables, pool) whose position j has scores of about -level[j]: channel 3 of K times channel 3 of q."""
    cu, tables, n_pages = ragged([nq], [n], page, seed)
    k, v = (randn(n_pages, kv, page, hd, seed=seed + s) for s in (1, 2))
    k *= 3
    level = torch.as_tensor(level, device="cuda", dtype=torch.float32).expand(n)
    at = torch.arange(n, device="cuda")
    b = 16.0
    k[tables[0].long().repeat_interleave(page)[:n], :, at % page, 3] = (level * hd ** 0.5 / b)[:, None]
    pool = wq.kv_pool(n_pages, kv, page, hd, bits)
    fill_pool(pool, k.to(BF), v.to(BF))
    q = randn(nq, h, hd, seed=seed + 5) * 0.3
    q[..., 3] = -b
    return q.to(BF), cu, tables, pool


LEVELS = [-90.0, 90.0, 200.0, 1000.0]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq,n", [(1, 300), (3, 300), (17, 17), (20, 1500), (150, 150), (300, 700)])
@pytest.mark.parametrize("level", LEVELS)
def test_all_scores_far_from_zero(level, nq, n, hd, bits):
    """Also the first rows of a prompt, which see one position or a few."""
    q, cu, tables, pool = shifted(nq, n, hd, bits, level, seed=nq)
    o = wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq)
    check(o, *attn_ref(q, cu, [n], tables, pool, hd ** -0.5), f"{level} {nq} {hd} {bits}")
    assert status() == 0


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq", [3, 30, 260])
@pytest.mark.parametrize("first,last", [(130.0, 120.0), (120.0, 130.0), (200.0, 100.0), (127.0, 125.0)])
def test_scores_around_the_least_power(first, last, nq, hd, bits):
    """Scores on both sides of 2^-126, from `first` at position 0 on to `last` (in powers of two): none of them is lost."""
    n = 400
    level = torch.linspace(first, last, n) * math.log(2)
    q, cu, tables, pool = shifted(nq, n, hd, bits, level, seed=nq)
    o = wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq)
    check(o, *attn_ref(q, cu, [n], tables, pool, hd ** -0.5), f"{first} {nq} {hd} {bits}")


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("level", LEVELS)
def test_the_same_rows_through_both_kernels(level, hd, bits):
    """max_q says which kernel runs, not what comes out: either way within the bound."""
    nq, n = 3, 200
    q, cu, tables, pool = shifted(nq, n, hd, bits, level, seed=9)
    ref, bound = attn_ref(q, cu, [n], tables, pool, hd ** -0.5)
    padded = torch.cat([q, torch.zeros((497, *q.shape[1:]), dtype=BF, device="cuda")])
    for most in (3, 4, 5, 500):
        check(wq.attn_paged(padded, i32(*cu), i32(n), tables, pool, max_q=most)[:nq], ref, bound, f"{most}")
    assert status() == 0


@pytest.mark.parametrize("level", [90.0, 500.0])
def test_low_scores_beside_others(level):
    """A batch of both kinds: one sequence with low scores beside one around zero, decode steps and chunks."""
    h, kv, hd, page = 8, 2, 128, 32
    nq, lens = [1, 1, 40, 200], [333, 90, 41, 450]
    for bits in (16, 8, 4):
        cu, tables, n_pages = ragged(nq, lens, page, 4)
        k, v = (randn(n_pages, kv, page, hd, seed=s) for s in (1, 2))
        for b in (1, 3):
            k[tables[b, :-(-lens[b] // page)].long(), :, :, 3] = level * hd ** 0.5 / 16
        pool = wq.kv_pool(n_pages, kv, page, hd, bits)
        fill_pool(pool, k.to(BF), v.to(BF))
        q = randn(cu[-1], h, hd, seed=6) * 0.3
        q[..., 3] = -16
        q = q.to(BF)
        o = wq.attn_paged(q, i32(*cu), i32(*lens), tables, pool, max_q=200)
        check(o, *attn_ref(q, cu, lens, tables, pool, hd ** -0.5), f"{bits}")


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq", [3, 150])
@pytest.mark.parametrize("level", [1e5, 1e6, 1e7, -1e7])
def test_scores_of_millions(level, nq, hd, bits):
    """Up to 2^24 (times log2 e) fp32's steps make a mean of what is seen: no infinity, no NaN, nothing beyond the largest V."""
    n = 300
    q, cu, tables, pool = shifted(nq, n, hd, bits, level / 16, seed=nq)
    q[..., 3] *= 16
    o = wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq).double()
    kind = 2.0 ** -8 if bits == 16 else 2.0 ** -10  # roundings of p and V, and the store's
    V = pool_values(pool)[1][tables[0].long()].transpose(1, 2).reshape(-1, 2, hd)[:n].abs().amax(0).repeat_interleave(4, 0)
    assert bool((o.abs() <= V * (1 + kind) * (1 + 2.0 ** -8)).all()) and status() == 0
