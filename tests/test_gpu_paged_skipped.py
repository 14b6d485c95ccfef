"""A decoder layer's step over pages with a token whose position the table of angles does not have: what comes out does not
hang on what the workspace and the pages held before."""
import pytest
import torch

from paged_util import i32, status
from paper_2606_04238_gb300 import wq
from test_gpu_paged_decoder import B, P, PAGE, Batch
from test_gpu_tree_decoder import D, HD, _layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [[3, 1, 2, 5], [3, 90, 2, 40]])
def test_a_position_outside_the_table(new, bits):
    layer, m = _layer(wq, 21), sum(new)
    table = wq.rope_table(P * PAGE, HD)
    g = torch.Generator(device="cuda").manual_seed(7)
    x, before = (torch.randn((m, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    results = []
    for used in (False, True):
        torch.manual_seed(3)
        torch.cuda.manual_seed(3)
        batch = Batch(bits)
        ws = wq.decoder_paged_workspace(B, m, layer)
        cu, lens, pos, slots = batch.plan([0] * B, new, m)
        step = lambda x, p: wq.decoder_paged_forward(x, cu, lens, p, slots, layer, batch.pool, batch.tables, table,  # noqa: E731
                                                     max_q=max(new), ws=ws)
        if used:  # an earlier step leaves its queries in the workspace and its rows in the pages
            step(before, pos)
            assert status() == 0
        p = pos.clone()
        p[[1, int(cu[1]), int(cu[2])]] = i32(P * PAGE, -1, 2 ** 31 - 1)
        y = step(x, p)
        assert status() == -1 and status() == 0
        keys, values = wq.paged_read(batch.pool, slots)
        results.append((y, keys, values))
        for t in (keys, values):
            there = (t != 0).flatten(1).any(1)
            want = torch.ones(m, dtype=torch.bool, device="cuda")
            want[[1, int(cu[1]), int(cu[2])]] = False
            assert torch.equal(there, want)
        assert bool(y.isfinite().all())
    for a, b in zip(*results):
        assert torch.equal(a, b)
