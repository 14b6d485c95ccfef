"""Rotary positions of many tokens (wq_qkv_rope): the form with 128 threads a token, which
takes more than two tokens an SM, and the border to the other; head counts of one and of
several passes through the registers.  Bound: that of test_gpu_kv.py's test_rope.
"""
import pytest
import torch

from test_gpu_kv import _rope64, wq  # noqa: F401

pytestmark = pytest.mark.gpu


def check(wq, m, H, kv, hd, d, norm):
    g = torch.Generator().manual_seed(m + H + hd)
    qkv = torch.randn((m, (H + 2 * kv) * hd), generator=g)
    x = (torch.randn((m, d), generator=g) * 3).to(torch.bfloat16) if d else None
    pos = torch.randint(0, 5000, (m,), generator=g, dtype=torch.int32)
    table = wq.rope_table(5000, hd)
    got = wq.qkv_rope(qkv.cuda(), pos.cuda(), table, H, kv, x=None if x is None else x.cuda(), head_norm=norm)
    for a, r in zip(got, _rope64(qkv, x, pos, table, H, kv, norm)):
        tol = 2.0 ** -18 * r.abs().amax(-1, keepdim=True) + r.abs() * 2.0 ** -8 * 1.01
        assert a.shape == r.shape and bool(((a.double().cpu() - r).abs() <= tol).all())
    assert wq.device_status() == 0


@pytest.mark.parametrize("H,kv,hd", [(1, 1, 64), (24, 4, 128), (40, 8, 128), (64, 8, 64), (80, 2, 128)])
@pytest.mark.parametrize("over", [0, 1])
@pytest.mark.parametrize("d", [0, 2880])
def test_either_side_of_the_border(wq, H, kv, hd, over, d):
    check(wq, 2 * torch.cuda.get_device_properties(0).multi_processor_count + over, H, kv, hd, d, True)


@pytest.mark.parametrize("H,kv,hd,d,norm", [(40, 8, 128, 5120, True), (64, 8, 64, 2880, True), (3, 1, 128, 8, False)])
def test_many_tokens(wq, H, kv, hd, d, norm):
    check(wq, 1220, H, kv, hd, d, norm)


@pytest.mark.parametrize("hd", [64, 128])
def test_skipped_positions_among_many(wq, hd):
    m, H, kv = 700, 8, 2
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn((m, (H + 2 * kv) * hd), generator=g)
    pos = torch.randint(0, 64, (m,), generator=g, dtype=torch.int32)
    bad = torch.zeros(m, dtype=torch.bool)
    bad[[0, 333, 699]] = True
    table = wq.rope_table(64, hd)
    out = [torch.full((m, n, hd), 7.0, dtype=torch.bfloat16, device="cuda") for n in (H, kv, kv)]
    wq.qkv_rope(qkv.cuda(), torch.where(bad, 64, pos).cuda(), table, H, kv, q=out[0], k=out[1], v=out[2])
    assert wq.device_status() == -1 and wq.device_status() == 0
    for a, r in zip(out, _rope64(qkv, None, pos, table, H, kv, True)):
        a = a.double().cpu()
        assert (a[bad] == 7).all()
        tol = 2.0 ** -18 * r.abs().amax(-1, keepdim=True) + r.abs() * 2.0 ** -8 * 1.01
        assert bool(((a - r).abs() <= tol)[~bad].all())
