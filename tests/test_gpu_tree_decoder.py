"""The verify step of a decoder layer (wq_decoder_tree_forward): a chain of drafts
against the same tokens decoded one by one, a tree against its paths, and the
cache after the accepted path is appended.

Tolerance: the two ways differ by bf16 roundings of q, of the probabilities, of o,
x1 and h, each some 2^-9 / sqrt(3) of its tensor, and what they flip further on;
1e-2 in the 2-norm is about four times their sum.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

D, INTER, H, KV, HD, R = 512, 1024, 8, 2, 64, 8


@pytest.fixture(scope="module")
def wq():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_04238_gb300 import wq as mod
    mod.device_status()
    return mod


def _layer(wq, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = lambda n, k, s=0.03: torch.randn((n, k), generator=g, device="cuda") * s
    bf = lambda n, k: w(n, k, 0.01).to(torch.bfloat16)
    mlp = wq.MLPLayer(wq.pack(w(INTER, D), 128, 2), wq.pack(w(INTER, D), 128, 2), wq.pack(w(D, INTER), 128, 4),
                      bf(2 * R, D), bf(INTER, R), bf(INTER, R), 2.0)
    return wq.DecoderLayer(wq.pack(w((H + 2 * KV) * HD, D), 128, 4), wq.pack(w(D, H * HD), 64, 4), mlp, H, KV, HD)


def _rel(a, b):
    a, b = a.double(), b.double()
    return float((a - b).norm() / b.norm())


def _setup(wq, bits, b, ctx, lens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    c = wq.kv_cache(b, KV, ctx, HD, bits)
    wq.kv_append(c, bf(b, max(lens), KV, HD), bf(b, max(lens), KV, HD), torch.zeros(b, dtype=torch.int32, device="cuda"))
    return c, bf


@pytest.mark.parametrize("b,t", [(1, 4), (3, 5), (2, 40)])
def test_chain_is_sequential_decoding(wq, b, t):
    lens = [33, 64, 7][:b]
    layer = _layer(wq, 1)
    c, bf = _setup(wq, 16, b, 128, lens, 2)
    x = bf(b, t, D)
    lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pos = lens_t[:, None] + torch.arange(t, dtype=torch.int32, device="cuda")
    y, kn, vn = wq.decoder_tree_forward(x, lens_t, pos, layer, c, wq.rope_table(128, HD))
    kc, vc = c.k.clone(), c.v.clone()
    for i in range(t):
        yi = wq.decoder_layer_forward(x[:, i].contiguous(), lens_t + i, layer, kc, vc)
        assert _rel(y[:, i], yi) < 1e-2
    wq.kv_append(c, kn, vn, lens_t)
    for s in range(b):
        n = lens[s]
        assert torch.equal(c.k[s, :, :n], kc[s, :, :n])
        for mine, theirs in ((c.k, kc), (c.v, vc)):
            a, r = mine[s, :, n:n + t].float(), theirs[s, :, n:n + t].float()
            # fp32 sums in another order (the projections' calls differ by up to 3e-6 of the result's norm, some 2^-15 of
            # the head's largest value, which a rotation may cancel): the same bf16 value, or rarely its neighbour
            tol = r.abs() * 2.0 ** -7 + r.abs().amax(-1, keepdim=True) * 2.0 ** -15
            assert float((a != r).float().mean()) < 0.01 and bool(((a - r).abs() <= tol).all())
    assert wq.device_status() == 0


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_tree_is_its_paths(wq, bits):
    """Every leaf's path, run as a chain of its own, gives the tree's outputs; then the path is kept."""
    parents = torch.tensor([[-1, 0, 0, 1, 2, 4, -1, 6]], dtype=torch.int32)
    b, t, lens = 1, 8, [50]
    layer = _layer(wq, 3)
    c, bf = _setup(wq, bits, b, 96, lens, 4)
    x = bf(b, t, D)
    table = wq.rope_table(96, HD)
    lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    depth = [0] * t
    for i in range(t):
        depth[i] = 0 if parents[0, i] < 0 else depth[int(parents[0, i])] + 1
    pos = (lens_t[:, None] + torch.tensor([depth], dtype=torch.int32, device="cuda")).contiguous()
    ws = wq.decoder_tree_workspace(b, t, layer, 96)
    y, kn, vn = wq.decoder_tree_forward(x, lens_t, pos, layer, c, table, mask=wq.tree_mask(parents).cuda(), ws=ws)
    for leaf in (3, 5, 7):
        path = []
        i = leaf
        while i >= 0:
            path.insert(0, i)
            i = int(parents[0, i])
        yp, kp, vp = wq.decoder_tree_forward(x[:, path].contiguous(), lens_t, pos[:, path].contiguous(), layer, c, table)
        assert _rel(y[:, path], yp) < 1e-2
    # keep the path 0, 2, 4, 5 and decode on: the same as a cache that was given the rows in order
    path = torch.tensor([[0, 2, 4, 5]], dtype=torch.int32, device="cuda")
    other = wq.KVCache(c.k.clone(), c.v.clone(), None if bits == 16 else c.k_meta.clone(),
                       None if bits == 16 else c.v_meta.clone(), HD, bits)
    wq.kv_append(c, kn, vn, lens_t, index=path)
    keep = path[0].long()
    wq.kv_append(other, kn[:, keep].contiguous(), vn[:, keep].contiguous(), lens_t)
    assert torch.equal(c.k, other.k) and torch.equal(c.v, other.v)
    nxt = bf(b, 1, D)
    p1 = lens_t[:, None] + 4
    y1, _, _ = wq.decoder_tree_forward(nxt, lens_t + 4, p1, layer, c, table, ws=ws)
    y2, _, _ = wq.decoder_tree_forward(nxt, lens_t + 4, p1, layer, other, table)
    assert torch.equal(y1, y2) and wq.device_status() == 0


def test_padding_drafts_do_not_change_the_others(wq):
    layer = _layer(wq, 5)
    b, t, lens = 2, 6, [20, 31]
    c, bf = _setup(wq, 8, b, 64, lens, 6)
    x = bf(b, t, D)
    lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pos = lens_t[:, None] + torch.arange(t, dtype=torch.int32, device="cuda")
    counts = torch.tensor([6, 4], dtype=torch.int32, device="cuda")
    y, kn, _ = wq.decoder_tree_forward(x, lens_t, pos, layer, c, wq.rope_table(64, HD), counts=counts)
    x2 = x.clone()
    x2[1, 4:] = 1.0
    y2, _, _ = wq.decoder_tree_forward(x2, lens_t, pos, layer, c, wq.rope_table(64, HD), counts=counts)
    assert torch.equal(y[0], y2[0]) and torch.equal(y[1, :4], y2[1, :4])
