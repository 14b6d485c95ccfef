"""Attention over pages at the most positions that a table may have, 2^31 - 1024: requests may share pages, and a table may
name one page over and over, so that no pool's size keeps such lengths away.

All entries of the table but the last name one page, whose scores lie so far below the last one's that they count for nothing
(2^31 times e^-60 is below 2^-55): the rows are those of the last page alone.
"""
import pytest
import torch

from paged_util import attn_ref, check, fill_pool, i32, status
from paper_2606_04238_gb300 import wq
from test_gpu_paged import BF, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("nq", [1, 3])
@pytest.mark.parametrize("less", [0, 1, 100])
def test_the_longest_table(nq, bits, less):
    h, kv, hd, page = 8, 1, 64, 256
    pages = (2 ** 31 - 1024) // page
    k, v = (randn(2, kv, page, hd, seed=s) for s in (1, 2))
    k[0, ..., 3], k[1, ..., 3] = 60 * hd ** 0.5 / 16, 0
    pool = wq.kv_pool(2, kv, page, hd, bits)
    fill_pool(pool, k.to(BF), v.to(BF))
    tables = torch.zeros((1, pages), dtype=torch.int32, device="cuda")
    tables[0, -1] = 1
    q = randn(nq, h, hd, seed=5) * 0.3
    q[..., 3] = -16
    q = q.to(BF)
    n = pages * page - less
    o = wq.attn_paged(q, i32(0, nq), i32(n), tables, pool, max_q=nq)
    check(o, *attn_ref(q, [0, nq], [page - less], i32(1).view(1, 1), pool, hd ** -0.5))
    assert status() == 0
