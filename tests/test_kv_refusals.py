"""What the KV-cache and tree-attention calls refuse on the host, before any launch."""
import ctypes

import pytest

OK, ARG, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3, -4, -7


@pytest.fixture(scope="module")
def L():
    from paper_2606_04238_gb300 import _build
    _build.build()
    from paper_2606_04238_gb300 import wq
    return wq.lib()


def cache(**kw):
    from paper_2606_04238_gb300 import wq
    f = dict(k=256, v=512, k_meta=768, v_meta=1024, batch=2, n_kv=2, max_len=64, head_dim=128, bits=8)
    f.update(kw)
    return ctypes.byref(wq._KVCache(**f))


def strides(*v):
    return (ctypes.c_int64 * 3)(*v)


BAD_CACHES = [(dict(bits=2), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(max_len=0), SHAPE),
              (dict(batch=0), SHAPE), (dict(n_kv=-1), SHAPE), (dict(k=None), ARG), (dict(v=264), ALIGN),
              (dict(k_meta=None), ARG), (dict(v_meta=1028), ALIGN), (dict(batch=1 << 20, n_kv=1 << 20), SHAPE)]


def append(L, c=None, k=256, v=512, dtype=0, n_src=4, ks=(1024, 256, 128), vs=(1024, 256, 128), start=256, counts=None,
           index=None, n=4):
    return L.wq_kv_append(cache() if c is None else c, k, v, dtype, n_src, strides(*ks), strides(*vs), start, counts, index, n, None)


def read(L, c=None, start=256, counts=None, n=4, k=256, v=512, dtype=0):
    return L.wq_kv_read(cache() if c is None else c, start, counts, n, k, v, dtype, None)


def tree(L, c=None, q=256, kn=512, vn=768, t=4, h=8, lens=256, counts=None, mask=None, scale=0.1, o=256, ws=256, nb=1 << 30):
    return L.wq_attn_tree(q, kn, vn, t, h, cache() if c is None else c, lens, counts, mask, scale, o, ws, nb, None)


def rope(L, qkv=256, x=None, m=3, d=0, pos=256, table=512, n_pos=8, h=4, kv=2, hd=128, flags=8, q=256, k=512, v=768):
    return L.wq_qkv_rope(qkv, x, m, d, pos, table, n_pos, h, kv, hd, flags, q, k, v, None)


@pytest.mark.parametrize("kw,st", BAD_CACHES)
@pytest.mark.parametrize("call", [append, read, tree])
def test_bad_caches(L, call, kw, st):
    assert call(L, c=cache(**kw)) == st and L.wq_last_error()
    assert call(L, c=ctypes.cast(None, ctypes.POINTER(type(cache()._obj)))) == ARG


def test_bf16_cache_needs_no_scales(L):
    assert append(L, c=cache(bits=16, k_meta=None, v_meta=None), n=0) == OK


@pytest.mark.parametrize("kw,st", [
    (dict(dtype=2), ARG), (dict(n=-1), ARG), (dict(n=5), SHAPE), (dict(n_src=-1), SHAPE), (dict(k=None), ARG),
    (dict(start=None), ARG), (dict(v=520), ALIGN), (dict(ks=(1024, 252, 128)), ALIGN),
    (dict(dtype=1, vs=(1022, 256, 128)), ALIGN), (dict(n=1 << 28, n_src=1 << 28), SHAPE), (dict(n=0), OK)])
def test_append(L, kw, st):
    assert append(L, **kw) == st


@pytest.mark.parametrize("kw,st", [(dict(dtype=-1), ARG), (dict(n=-2), ARG), (dict(k=None), ARG), (dict(start=None), ARG),
                                   (dict(v=8), ALIGN), (dict(n=1 << 28), SHAPE), (dict(n=0), OK)])
def test_read(L, kw, st):
    assert read(L, **kw) == st


@pytest.mark.parametrize("kw,st", [
    (dict(t=-1), UNSUPPORTED), (dict(t=129), UNSUPPORTED), (dict(h=7), UNSUPPORTED), (dict(h=0), UNSUPPORTED),
    (dict(h=34), UNSUPPORTED), (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(q=None), ARG),
    (dict(lens=None), ARG), (dict(o=None), ARG), (dict(ws=None), ARG), (dict(kn=520), ALIGN), (dict(ws=264), ALIGN),
    (dict(t=0), OK)])
def test_tree(L, kw, st):
    assert tree(L, **kw) == st


@pytest.mark.parametrize("kw,st", [
    (dict(m=-1), ARG), (dict(flags=1), ARG), (dict(hd=32), UNSUPPORTED), (dict(h=0), SHAPE), (dict(kv=0), SHAPE),
    (dict(x=256, d=12), SHAPE), (dict(x=256, d=0), SHAPE), (dict(n_pos=0), SHAPE), (dict(qkv=None), ARG),
    (dict(pos=None), ARG), (dict(table=None), ARG), (dict(q=260), ALIGN), (dict(x=260, d=8), ALIGN), (dict(m=0), OK)])
def test_rope(L, kw, st):
    assert rope(L, **kw) == st


def test_decoder_tree(L):
    from paper_2606_04238_gb300 import wq
    q = lambda n, k, bits, group=128: wq._QWeight(256, 256, n, k, group, bits)
    d, inter, h, kv, hd = 512, 1024, 4, 2, 128

    def layer(qkv_n=(h + 2 * kv) * hd):
        mlp = wq._MLPLayer(q(inter, d, 2), q(inter, d, 2), q(d, inter, 4), None, None, None, 0, 0.0)
        return wq._DecoderLayer(q(qkv_n, d, 4), q(d, h * hd, 4), mlp, h, kv, hd, 1e6)

    def call(ly=None, c=None, t=4, x=256, lens=256, pos=256, table=256, flags=0, ws=None):
        ly = layer() if ly is None else ly
        return L.wq_decoder_tree_forward(x, t, lens, pos, ctypes.byref(ly), cache() if c is None else c, table, 64, None, None, flags,
                                         256, 512, 768, ws, 0, None)

    assert call(ly=layer(qkv_n=512)) == SHAPE
    assert call(c=cache(n_kv=4)) == SHAPE and call(c=cache(head_dim=64)) == SHAPE and call(c=cache(bits=5)) == UNSUPPORTED
    assert call(t=129) == UNSUPPORTED and call(t=-1) == UNSUPPORTED and call(c=cache(batch=1000), t=17) == SHAPE
    assert call(flags=2) == ARG and call(x=None) == ARG and call(pos=None) == ARG and call(table=None) == ARG
    assert call(t=0) == OK


def test_tree_mask():
    import torch
    from paper_2606_04238_gb300 import wq
    m = wq.tree_mask(torch.tensor([[-1, 0, 0, 1, -1], [-1, -1, 1, 2, 3]], dtype=torch.int32))
    assert m.flatten().tolist() == [1, 3, 5, 11, 16, 1, 2, 6, 14, 30]
    chain = wq.tree_mask((torch.arange(40, dtype=torch.int32) - 1)[None])
    assert chain.shape == (1, 40, 2) and chain[0, 31].tolist() == [-1, 0] and chain[0, 39].tolist() == [-1, 255]
    with pytest.raises(AssertionError):
        wq.tree_mask(torch.tensor([[0]], dtype=torch.int32))
