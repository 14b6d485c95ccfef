"""Attention of drafted trees over a 16-, 8- or 4-bit cache (wq_attn_tree)
against the same in 64 bits on the values the cache holds.

Bound, per output element, of what the kernel rounds (bf16 has 8 significant bits:
round to nearest is within 2^-8 of the value): each probability to bf16 (2^-11 over
a quantized cache, whose drafts are bf16 too), so at most 2^-8 sum_j p_j |v_j|; the
bf16 store, 2^-8 |o|; fp32 scores and exponents, some 2^-15 of sum_j p_j |v_j|; and
binary16's smallest steps: p_j times its row's scale s_j is within 2^-25 of the
largest such product, and what it multiplies is at most the row's range r_j over s_j,
so each of the n terms is within 2^-25 max_i p_i r_i (a row's scales differ from
r / qmax by less than 2, a draft's by less than 4).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wq():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_04238_gb300 import wq as mod
    mod.device_status()
    return mod


def words(vis):
    """int32 [b, t, ceil(t / 32)] of bool [b, t, t]."""
    b, t, _ = vis.shape
    w = (t + 31) // 32
    out = torch.zeros((b, t, w), dtype=torch.int64)
    for j in range(t):
        out[:, :, j // 32] |= vis[:, :, j].long() << (j % 32)
    return torch.where(out >= 2 ** 31, out - 2 ** 32, out).to(torch.int32)


def tree(b, t, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.stack([torch.tensor([int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(t)],
                                     dtype=torch.int32) for _ in range(b)])


def visible(parents):
    b, t = parents.shape
    vis = torch.zeros((b, t, t), dtype=torch.bool)
    for s in range(b):
        for i in range(t):
            j = i
            while j >= 0:
                vis[s, i, j] = True
                j = int(parents[s, j])
    return vis


def reference(q, kn, vn, k, v, lens, counts, vis, scale):
    """fp64 output and error bound.  k, v: fp64 cached values [b, h, L, hd]."""
    b, t, H, hd = q.shape
    kv = kn.shape[2]
    rep = H // kv
    o = torch.zeros((b, t, H, hd), dtype=torch.float64)
    tol = torch.full_like(o, 1e-30)
    for s in range(b):
        n, m = int(lens[s]), int(counts[s])
        if m == 0:
            continue
        for g in range(kv):
            hs = slice(g * rep, (g + 1) * rep)
            keys = torch.cat([k[s, g, :n], kn[s, :m, g].double()])
            vals = torch.cat([v[s, g, :n], vn[s, :m, g].double()])
            x = torch.einsum("thd,jd->thj", q[s, :m, hs].double(), keys) * scale
            see = torch.cat([torch.ones((m, n), dtype=torch.bool), vis[s, :m, :m]], 1)[:, None]
            x = torch.where(see, x, torch.full_like(x, -math.inf))
            top = x.amax(-1, keepdim=True)
            p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
            p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
            safe = torch.where(see.unsqueeze(-1), vals, torch.zeros((), dtype=torch.float64))
            out = torch.einsum("thj,thjd->thd", p, safe.expand(m, rep, n + m, hd)) if not torch.isfinite(vals).all() \
                else torch.einsum("thj,jd->thd", p, vals)
            mag = torch.einsum("thj,jd->thd", p, vals.abs().nan_to_num(0, 0, 0))
            span = 2 * vals.abs().nan_to_num(0, 0, 0).amax(-1)  # a row's range, at most
            big = 4 * (p * span).amax(-1, keepdim=True)
            o[s, :m, hs] = out
            tol[s, :m, hs] = (2.0 ** -8 + 2.0 ** -15) * mag + 2.0 ** -8 * 1.01 * out.abs().nan_to_num(0, 0, 0) + \
                (n + m) * 2.0 ** -25 * big + 1e-30
    return o, tol


# Short caches run on the mma.sync kernel, roomy ones on the tcgen05 kernel: every test takes both.
ROOMY = 800_000


@pytest.fixture(params=["short", "roomy"])
def room(request):
    """Positions of a cache beyond the filled ones, so that the call takes the other kernel."""
    def capacity(b, kv, t, H, filled):
        tiles = (t * (H // kv) + 15) // 16
        return filled if request.param == "short" else max(filled, ROOMY // (b * kv * tiles) + 1)
    return capacity


def run(wq, room, b, t, H, kv, hd, bits, lens, counts=None, vis=None, parents=None, seed=0, max_len=None, scale=None,
        vscale=1.0, spoil=None):
    g = torch.Generator().manual_seed(seed)
    L = max_len or max(1, max(lens))
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)
    q, kn, vn = bf(b, t, H, hd) * 1.5, bf(b, t, kv, hd), bf(b, t, kv, hd)
    k, v = bf(b, L, kv, hd), bf(b, L, kv, hd)
    if vscale != 1.0:  # rows of very different sizes
        v = (v.float() * torch.exp(torch.randn((b, L, kv, 1), generator=g) * math.log(vscale))).to(torch.bfloat16)
    lens_t = torch.tensor(lens, dtype=torch.int32)
    counts_t = None if counts is None else torch.tensor(counts, dtype=torch.int32)
    mask = None
    if parents is not None:
        mask, vis = wq.tree_mask(parents), visible(parents)
        assert torch.equal(mask, words(vis))
    elif vis is not None:
        mask = words(vis)
    else:
        vis = torch.ones((t, t), dtype=torch.bool).tril().expand(b, t, t)
    if spoil:
        spoil(q, kn, vn, k, v)
    cache = wq.kv_cache(b, kv, room(b, kv, t, H, L), hd, bits)
    zero = torch.zeros(b, dtype=torch.int32, device="cuda")
    wq.kv_append(cache, k.cuda(), v.cuda(), zero)
    kr, vr = wq.kv_read(cache, zero, L, dtype=torch.float32)
    dev = lambda x: None if x is None else x.cuda()
    o = wq.attn_tree(q.cuda(), kn.cuda(), vn.cuda(), cache, lens_t.cuda(), mask=dev(mask), counts=dev(counts_t), scale=scale)
    assert wq.device_status() == 0
    ref, tol = reference(q, kn, vn, kr.double().cpu().transpose(1, 2), vr.double().cpu().transpose(1, 2), lens,
                         counts or [t] * b, vis, hd ** -0.5 if scale is None else scale)
    return o.cpu().double(), ref, tol


def close(o, ref, tol):
    assert o.shape == ref.shape
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(o)) and torch.equal(ref.isnan(), o.isnan())
    assert torch.equal(o[~fine & ~ref.isnan()], ref[~fine & ~ref.isnan()])
    d = (o - ref).abs()[fine] - tol[fine]
    assert not d.numel() or float(d.max()) <= 0, f"beyond the bound by {float(d.max()):.3e}"


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,kv,t", [(4, 1, 1), (8, 2, 5), (5, 1, 3), (2, 2, 33), (32, 2, 7), (8, 1, 61)])
def test_trees(wq, room, bits, hd, H, kv, t):
    lens = [0, 1, 15, 16, 17, 31, 33, 127, 129, 300]
    b = len(lens)
    counts = [max(1, t - i % 3) for i in range(b)]
    close(*run(wq, room, b, t, H, kv, hd, bits, lens, counts, parents=tree(b, t, t), seed=t + hd + bits, max_len=301))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_one_token_long_contexts(wq, room, bits):
    close(*run(wq, room, 2, 1, 8, 2, 128, bits, [4097, 9001], seed=1))
    close(*run(wq, room, 1, 1, 8, 1, 64, bits, [20000], seed=2))


@pytest.mark.parametrize("bits,hd,H,kv", [(16, 128, 8, 2), (8, 128, 10, 2), (4, 128, 8, 1), (8, 64, 16, 2), (4, 64, 8, 2),
                                          (16, 64, 8, 1)])
def test_many_drafts(wq, room, bits, hd, H, kv):
    close(*run(wq, room, 2, 128, H, kv, hd, bits, [777, 1500], [128, 101], parents=tree(2, 128, 3), seed=3))
    close(*run(wq, room, 1, 64, H, kv, hd, bits, [2048], seed=4))  # a chain: mask None


@pytest.mark.parametrize("bits,hd", [(16, 128), (8, 64), (4, 128)])
def test_more_row_blocks_than_ctas(wq, room, bits, hd):
    """45 x 8 heads of up to three drafts, lengths and counts of zero among them: a CTA takes several."""
    g = torch.Generator().manual_seed(3)
    lens = [int(x) for x in torch.randint(0, 700, (45,), generator=g)]
    counts = [int(x) for x in torch.randint(0, 4, (45,), generator=g)]
    lens[0], lens[7], lens[8], lens[44], counts[44], counts[5], counts[6] = 0, 0, 0, 640, 0, 0, 0
    close(*run(wq, room, 45, 3, 16, 8, hd, bits, lens, counts=counts, parents=tree(45, 3, 1), seed=21))


@pytest.mark.parametrize("bits,hd", [(16, 64), (8, 128), (4, 64)])
def test_uneven_row_blocks(wq, room, bits, hd):
    """Two to four row blocks a head, 2 to 32 tiles each: the ends of some and the begins of the next go to one CTA."""
    lens = [3832, 2316, 1272, 1492, 3947, 2660, 1, 2751]
    counts = [33, 42, 50, 50, 48, 60, 46, 41]
    close(*run(wq, room, 8, 61, 64, 8, hd, bits, lens, counts=counts, parents=tree(8, 61, 2), seed=22))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_rows_that_see_nothing(wq, room, bits):
    b, t = 3, 20
    vis = torch.rand((b, t, t), generator=torch.Generator().manual_seed(5)) < 0.2
    vis[:, 4] = False
    vis[1] = False
    o, ref, tol = run(wq, room, b, t, 8, 2, 128, bits, [0, 0, 40], vis=vis, seed=5)
    close(o, ref, tol)
    assert (o[0, 4] == 0).all() and (o[1] == 0).all() and (o[2, 4] != 0).any()
    o, ref, tol = run(wq, room, b, t, 8, 2, 128, bits, [7, 0, 40], [0, 20, 3], vis=vis, seed=6)  # no drafts, padding drafts
    close(o, ref, tol)
    assert (o[0] == 0).all() and (o[2, 3:] == 0).all()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("t,H", [(12, 4), (40, 8)])
def test_masked_and_unused_places_hold_anything(wq, room, bits, t, H):
    """NaN and infinities in drafts a row does not see, in padding drafts and behind the length."""
    def spoil(q, kn, vn, k, v):
        for x in (k, v):
            x[0, 200:] = math.nan
            x[1, 90:] = math.inf
        kn[0, 5], vn[0, 5] = math.nan, math.inf
        kn[1, 3], vn[1, 7] = -math.inf, math.nan
        q[0, t - 2:], kn[0, t - 2:], vn[0, t - 2:] = math.nan, math.nan, math.nan

    vis = torch.ones((2, t, t), dtype=torch.bool).tril()
    vis[0, :, 5] = False
    vis[1, :, 3] = False
    vis[1, :, 7] = False
    o, ref, tol = run(wq, room, 2, t, H, 1, 128, bits, [200, 90], [t - 2, t], vis=vis, seed=7, spoil=spoil, max_len=210)
    assert torch.isfinite(ref).all()
    close(o, ref, tol)


@pytest.mark.parametrize("bits", [16, 8])
def test_seen_infinities_reach_only_their_rows(wq, room, bits):
    t = 20
    def spoil(q, kn, vn, k, v):
        vn[0, 5, 0, 17] = math.inf
        vn[0, 9, 0, 64] = math.nan

    vis = torch.ones((1, t, t), dtype=torch.bool).tril()
    vis[0, 12:15, 5] = False
    vis[0, 13:, 9] = False
    o, ref, tol = run(wq, room, 1, t, 4, 1, 128, bits, [50], vis=vis, seed=8, spoil=spoil)
    assert torch.isinf(ref[0, 6, :, 17]).all() and torch.isnan(ref[0, 10, :, 64]).all() and torch.isfinite(ref[0, 13]).all()
    close(o, ref, tol)


@pytest.mark.parametrize("bits", [8, 4])
def test_rows_of_very_different_scales(wq, room, bits):
    close(*run(wq, room, 2, 6, 8, 2, 128, bits, [500, 77], vscale=100.0, seed=9))
    close(*run(wq, room, 1, 40, 8, 1, 64, bits, [500], vscale=100.0, seed=10))


def test_nan_row_of_a_quantized_cache(wq, room):
    def spoil(q, kn, vn, k, v):
        k[0, 30, 0, 4] = math.nan
    o, ref, _ = run(wq, room, 2, 4, 4, 1, 64, 8, [60, 30], seed=11, spoil=spoil)
    assert o[0].isnan().all() and torch.isfinite(o[1]).all()


@pytest.mark.parametrize("scale", [1.0, 0.02])
def test_scale_and_peaked_scores(wq, room, scale):
    close(*run(wq, room, 1, 9, 8, 2, 128, 16, [333], scale=scale, seed=12))
    close(*run(wq, room, 1, 30, 8, 2, 128, 8, [333], scale=scale, seed=13))


def test_query_rows_of_any_size(wq, room):
    """Rows of q from 2^-60 to 2^60: scores far below and (clipped to one key) far above 1."""
    def spoil(q, kn, vn, k, v):
        for i in range(q.shape[1]):
            q[0, i] = (q[0, i].float() * 2.0 ** (-60 + 20 * (i % 4))).to(torch.bfloat16)
    for bits in (16, 8, 4):
        close(*run(wq, room, 1, 8, 4, 1, 128, bits, [100], seed=14, spoil=spoil))


def test_lengths_out_of_range(wq):
    x = torch.zeros((3, 2, 1, 64), dtype=torch.bfloat16, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for cap, lens, counts in ((8, i32(-1, 9, 8), None), (8, i32(0, 0, 0), i32(-1, 3, 2)),
                              (300_000, i32(-1, 300_001, 8), None), (300_000, i32(0, 0, 0), i32(-1, 3, 2))):
        c = wq.kv_cache(3, 1, cap, 64, 8)
        o = torch.full_like(x, 3.0)
        wq.attn_tree(x, x, x, c, lens, counts=counts, o=o)
        assert wq.device_status() == -1 and wq.device_status() == 0
        assert (o[:2] == 3).all() and (o[2] == 0).all()


@pytest.mark.parametrize("L", [5000, 90_000])
def test_workspace_of_a_larger_call_other_stream_and_repeats(wq, L):
    b, t, H, kv, hd = 2, 9, 8, 2, 128
    ws = wq.attn_tree_workspace(8, 64, H, kv, hd, L)
    g = torch.Generator(device="cuda").manual_seed(15)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    c = wq.kv_cache(b, kv, L, hd, 8)
    wq.kv_append(c, bf(b, 5000, kv, hd), bf(b, 5000, kv, hd), torch.zeros(b, dtype=torch.int32, device="cuda"))
    q, kn, vn = bf(b, t, H, hd), bf(b, t, kv, hd), bf(b, t, kv, hd)
    lens = torch.tensor([4999, 3000], dtype=torch.int32, device="cuda")
    first = wq.attn_tree(q, kn, vn, c, lens, ws=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            again = wq.attn_tree(q, kn, vn, c, lens, ws=ws)
    side.synchronize()
    assert torch.equal(first, again)
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(q)
    with torch.cuda.graph(graph):
        wq.attn_tree(q, kn, vn, c, lens, ws=ws, o=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)


def test_offsets_past_32_bits(wq):
    """The last sequence and head of a cache of 2.5 GB a tensor."""
    b, kv, L, hd = 10, 8, 120_001, 128
    c = wq.kv_cache(b, kv, L, hd, 16)
    g = torch.Generator(device="cuda").manual_seed(16)
    c.k[-1, -1].normal_(generator=g)
    c.v[-1, -1].normal_(generator=g)
    q = torch.randn((b, 2, kv, hd), generator=g, device="cuda").to(torch.bfloat16)
    kn = torch.zeros((b, 2, kv, hd), dtype=torch.bfloat16, device="cuda")
    lens = torch.full((b,), L, dtype=torch.int32, device="cuda")
    o = wq.attn_tree(q, kn, kn, c, lens)
    ref, tol = reference(q[-1:, :, -1:].cpu(), kn[-1:, :, -1:].cpu(), kn[-1:, :, -1:].cpu(), c.k[-1:, -1:].double().cpu(),
                         c.v[-1:, -1:].double().cpu(), [L], [2], torch.ones((1, 2, 2), dtype=torch.bool).tril(), hd ** -0.5)
    close(o[-1:, :, -1:].cpu().double(), ref, tol)


def test_small_workspace_is_refused(wq):
    c = wq.kv_cache(1, 2, 8192, 128, 8)
    x = torch.zeros((1, 1, 8, 128), dtype=torch.bfloat16, device="cuda")
    n = torch.zeros((1, 1, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(wq.WQError) as e:
        wq.attn_tree(x, n, n, c, torch.zeros(1, dtype=torch.int32, device="cuda"),
                     ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -7


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("t", [2, 30])
def test_a_nan_query_gives_nan_rows(wq, room, bits, t):
    """Also where every score of a row is NaN; the other rows are as without it."""
    def spoil(q, kn, vn, k, v):
        q[0, 1, 0, 3] = math.nan
    o, ref, tol = run(wq, room, 1, t, 4, 1, 128, bits, [300], seed=17, spoil=spoil)
    assert ref[0, 1, 0].isnan().all() and torch.isfinite(ref[0, 0]).all() and torch.isfinite(ref[0, 1, 1]).all()
    close(o, ref, tol)


def test_zero_scale_is_the_mean(wq, room):
    close(*run(wq, room, 1, 24, 4, 1, 64, 8, [100], scale=0.0, seed=18))
    close(*run(wq, room, 1, 24, 4, 1, 64, 16, [100], scale=-0.1, seed=19))
    close(*run(wq, room, 1, 24, 4, 1, 64, 4, [100], scale=-0.1, seed=20))
