"""Attention over pages where infinities of K make a row's scores -inf: alone they leave softmax without a value (NaN), beside
finite ones they count for nothing.  Rows of zeros are those of sequences that are not served, no others."""
import math

import pytest
import torch

from paged_util import attn_ref, check, fill_pool, i32, status
from paper_2606_04238_gb300 import wq
from test_gpu_paged import BF, ragged, randn

pytestmark = pytest.mark.gpu


def lowest(nq, n, upto, hd, page=16, h=8, kv=2):
    """(q, cu, tables, pool, k, v): the first `upto` positions have infinite keys, whose products with q are -inf."""
    cu, tables, n_pages = ragged([nq], [n], page, 1)
    k, v = (randn(n_pages, kv, page, hd, seed=s) for s in (1, 2))
    at = torch.arange(upto, device="cuda")
    k[tables[0].long().repeat_interleave(page)[:upto], :, at % page, 3] = math.inf
    pool = wq.kv_pool(n_pages, kv, page, hd, 16)
    fill_pool(pool, k.to(BF), v.to(BF))
    q = randn(nq, h, hd, seed=5)
    q[..., 3] = -1
    return q.to(BF), cu, tables, pool, k, v


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq,n", [(1, 1), (1, 3000), (3, 300), (150, 150), (30, 2000), (300, 700)])
def test_all_scores_infinite(nq, n, hd):
    q, cu, tables, pool, *_ = lowest(nq, n, n, hd)
    assert bool(wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq).isnan().all())
    # infinities of V as well: still no value
    pool.v.fill_(math.inf)
    assert bool(wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq).isnan().all())
    # a sequence that is not served
    assert bool((wq.attn_paged(q, i32(*cu), i32(-1), tables, pool, max_q=nq) == 0).all())
    assert status() == 0


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq,n", [(3, 300), (150, 300), (30, 2000)])
def test_some_scores_infinite(nq, n, hd):
    """Rows that see a position with a finite score are those of the finite positions alone."""
    upto, page = 208, 16
    q, cu, tables, pool, *_ = lowest(nq, n, upto, hd)
    o = wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq)
    rows = max(0, nq - (n - upto))  # rows that see infinite ones only
    assert bool(o[:rows].isnan().all())
    ref, bound = attn_ref(q[rows:], [0, nq - rows], [n - upto], tables[:, upto // page:], pool, hd ** -0.5)
    check(o[rows:], ref, bound)
    assert status() == 0
