"""The verify step of a decoder layer (wq_decoder_tree_forward) with heads of 128 and more
tokens than the batched-decode kernels take: a batch of trees against the same step of
each of its paths as a chain of its own over the same cache.

Tolerance: that of test_gpu_tree_decoder.py, whose roundings these are.
"""
import pytest
import torch

from test_gpu_tree import tree
from test_gpu_tree_decoder import _rel, wq  # noqa: F401

pytestmark = pytest.mark.gpu

D, INTER, H, KV, HD, R = 1024, 1536, 10, 2, 128, 8


def _layer(wq, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = lambda n, k, s=0.03: torch.randn((n, k), generator=g, device="cuda") * s
    bf = lambda n, k: w(n, k, 0.01).to(torch.bfloat16)
    mlp = wq.MLPLayer(wq.pack(w(INTER, D), 128, 2), wq.pack(w(INTER, D), 128, 2), wq.pack(w(D, INTER), 128, 4),
                      bf(2 * R, D), bf(INTER, R), bf(INTER, R), 2.0)
    return wq.DecoderLayer(wq.pack(w((H + 2 * KV) * HD, D), 128, 4), wq.pack(w(D, H * HD), 64, 4), mlp, H, KV, HD)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("b,t,ctx", [(2, 7, 600), (6, 61, 900), (3, 128, 300)])
def test_batch_of_trees_is_its_paths(wq, bits, b, t, ctx):
    lens = [ctx - 137 * i for i in range(b)]
    counts = [t - (5 * i) % 4 for i in range(b)]
    layer = _layer(wq, 7)
    g = torch.Generator(device="cuda").manual_seed(8)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    c = wq.kv_cache(b, KV, ctx + t, HD, bits)
    wq.kv_append(c, bf(b, ctx, KV, HD), bf(b, ctx, KV, HD), i32([0] * b))
    parents = tree(b, t, 9)
    depth = torch.zeros((b, t), dtype=torch.int32)
    for s in range(b):
        for i in range(t):
            p = int(parents[s, i])
            depth[s, i] = 0 if p < 0 else depth[s, p] + 1
    x, table, lens_t = bf(b, t, D), wq.rope_table(ctx + t, HD), i32(lens)
    pos = (lens_t[:, None] + depth.cuda()).contiguous()
    y, kn, vn = wq.decoder_tree_forward(x, lens_t, pos, layer, c, table, mask=wq.tree_mask(parents).cuda(), counts=i32(counts))
    assert wq.device_status() == 0 and torch.isfinite(y).all()
    for s in range(b):
        for leaf in {counts[s] - 1, counts[s] // 2}:
            path, i = [], leaf
            while i >= 0:
                path.insert(0, i)
                i = int(parents[s, i])
            one = wq.KVCache(c.k[s:s + 1].clone(), c.v[s:s + 1].clone(), None if bits == 16 else c.k_meta[s:s + 1].clone(),
                             None if bits == 16 else c.v_meta[s:s + 1].clone(), HD, bits)
            yp, kp, vp = wq.decoder_tree_forward(x[s:s + 1, path].contiguous(), lens_t[s:s + 1].contiguous(),
                                                 pos[s:s + 1, path].contiguous(), layer, one, table)
            assert _rel(y[s, path], yp[0]) < 1e-2
            assert _rel(kn[s, path], kp[0]) < 1e-2 and _rel(vn[s, path], vp[0]) < 1e-2
