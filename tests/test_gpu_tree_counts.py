"""Tree attention with far fewer drafts than the call has places for: the calls whose
row blocks, counted with every place filled, are more than the CTAs that the device
holds at once, and counted with the drafts that exist are fewer, so that contexts are
split although the full call's would not be.  Outputs are filled beforehand: every
row has to be written, padding drafts with zeros.  Bound: that of test_gpu_tree.py.
"""
import math

import pytest
import torch

from test_gpu_tree import close, reference, tree, visible, wq  # noqa: F401

pytestmark = pytest.mark.gpu


def row_blocks(kv, rep, counts):
    return kv * sum(max(1, (c * rep + 127) // 128) for c in counts)


def call(wq, t, H, kv, hd, bits, lens, counts, seed, cap=None, bad=()):
    """Output (filled with NaN before), reference and bound; the sequences of `bad` have a length out of range."""
    b, L = len(lens), cap or max(1, max(lens))
    ctas = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    real = [0 if i in bad else c for i, c in enumerate(counts or [t] * b)]
    assert row_blocks(kv, H // kv, [t] * b) >= ctas > row_blocks(kv, H // kv, [c for i, c in enumerate(real) if i not in bad])
    g = torch.Generator().manual_seed(seed)
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)
    q, kn, vn, k, v = bf(b, t, H, hd), bf(b, t, kv, hd), bf(b, t, kv, hd), bf(b, L, kv, hd), bf(b, L, kv, hd)
    parents = tree(b, t, seed)
    cache = wq.kv_cache(b, kv, L, hd, bits)
    zero = torch.zeros(b, dtype=torch.int32, device="cuda")
    wq.kv_append(cache, k.cuda(), v.cuda(), zero)
    kr, vr = wq.kv_read(cache, zero, L, dtype=torch.float32)
    given = [L + 1 if i in bad else n for i, n in enumerate(lens)]
    o = torch.full((b, t, H, hd), math.nan, dtype=torch.bfloat16, device="cuda")
    ws = wq.attn_tree_workspace(b, t, H, kv, hd, L)
    ws.fill_(0xff)  # NaN wherever a partial result is read that no one wrote
    wq.attn_tree(q.cuda(), kn.cuda(), vn.cuda(), cache, torch.tensor(given, dtype=torch.int32, device="cuda"),
                 mask=wq.tree_mask(parents).cuda(), o=o, ws=ws,
                 counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"))
    assert wq.device_status() == (-1 if bad else 0)
    ref, tol = reference(q, kn, vn, kr.double().cpu().transpose(1, 2), vr.double().cpu().transpose(1, 2), lens, real,
                         visible(parents), hd ** -0.5)
    for i in bad:
        ref[i] = math.nan  # skipped: as it was filled
    return o.cpu().double(), ref, tol


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd", [64, 128])
def test_few_drafts_of_many_places(wq, bits, hd):
    close(*call(wq, 128, 64, 8, hd, bits, [700, 90, 333, 650, 1], [16, 9, 16, 1, 12], 31))
    close(*call(wq, 128, 64, 8, hd, bits, [700, 90, 0, 650, 400], [0, 40, 16, 0, 128], 32))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_one_long_sequence_among_short_ones(wq, bits):
    close(*call(wq, 61, 64, 8, 64, bits, [3000] + [100] * 9, [32] * 10, 33))
    g = torch.Generator().manual_seed(34)
    lens = [int(x) for x in torch.randint(200, 771, (20,), generator=g)]
    counts = [int(x) for x in torch.randint(10, 21, (20,), generator=g)]
    close(*call(wq, 20, 64, 8, 64, bits, lens, counts, 35))


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("counts", [None, [4] * 40])
def test_skipped_sequences_beside_valid_ones(wq, bits, counts):
    """40 x 8 heads of one row block each, three sequences of a length out of range."""
    lens = [(97 * i) % 450 + 50 for i in range(40)]
    lens[3] = 700  # the one that is split
    close(*call(wq, 5, 16, 8, 64, bits, lens, counts, 36, cap=700, bad=(0, 7, 39)))


def test_roomy_cache(wq):
    """Lengths far below the cache's positions."""
    close(*call(wq, 128, 64, 8, 64, 8, [300, 20, 0, 640, 511], [7, 30, 3, 16, 128], 37, cap=5000))
