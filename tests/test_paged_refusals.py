"""What the calls on pages refuse on the host, before any launch."""
import ctypes

import pytest

from test_kv_refusals import ALIGN, ARG, BAD_CACHES, L, OK, SHAPE, UNSUPPORTED, WORKSPACE, cache  # noqa: F401


def pool(**kw):
    f = dict(batch=8, max_len=32)
    f.update(kw)
    return cache(**f)


def plan(L, lens=256, keep=None, n_new=512, batch=2, page=32, tables=256, max_pages=4, free=512, n_pages=8, n_free=256, out=512,
         m=4, cu=256, kv_lens=512, pos=256, slots=512):
    return L.wq_page_plan(lens, keep, n_new, batch, page, tables, max_pages, free, n_pages, n_free, out, m, cu, kv_lens, pos,
                          slots, None)


def put(L, c=None, qkv=256, dtype=1, x=None, m=3, d=0, pos=256, table=512, n_pos=8, qw=None, kw=None, h=4, flags=8, slots=256, q=256):
    return L.wq_qkv_paged(qkv, dtype, x, m, d, pos, table, n_pos, qw, kw, h, flags, pool() if c is None else c, slots, q, None)


def read(L, c=None, slots=256, m=3, k=256, v=512, dtype=0):
    return L.wq_paged_read(pool() if c is None else c, slots, m, k, v, dtype, None)


def attn(L, c=None, q=256, m=4, max_q=2, h=8, batch=2, cu=256, lens=512, tables=256, max_pages=4, scale=0.1, o=256, ws=256, nb=1 << 40):
    return L.wq_attn_paged(q, m, max_q, h, pool() if c is None else c, batch, cu, lens, tables, max_pages, scale, o, ws, nb, None)


@pytest.mark.parametrize("kw,st", [b for b in BAD_CACHES if "max_len" not in b[0]] + [
    (dict(max_len=0), SHAPE), (dict(max_len=8), UNSUPPORTED), (dict(max_len=48), UNSUPPORTED), (dict(max_len=512), UNSUPPORTED),
    (dict(batch=1 << 24, n_kv=1, max_len=128), SHAPE)])
@pytest.mark.parametrize("call", [put, read, attn])
def test_bad_pools(L, call, kw, st):
    assert call(L, c=pool(**kw)) == st and L.wq_last_error()
    assert call(L, c=ctypes.cast(None, ctypes.POINTER(type(cache()._obj)))) == ARG


@pytest.mark.parametrize("kw,st", [
    (dict(page=8), UNSUPPORTED), (dict(page=100), UNSUPPORTED), (dict(batch=-1), ARG), (dict(batch=2049), SHAPE), (dict(m=-1), ARG),
    (dict(m=(1 << 18) + 1), SHAPE), (dict(max_pages=0), SHAPE), (dict(max_pages=1 << 26), SHAPE), (dict(n_pages=0), SHAPE),
    (dict(n_pages=1 << 26), SHAPE), (dict(batch=2048, max_pages=1 << 22), SHAPE), (dict(lens=None), ARG), (dict(n_new=None), ARG),
    (dict(tables=None), ARG), (dict(free=None), ARG), (dict(n_free=None), ARG), (dict(out=None), ARG), (dict(cu=None), ARG),
    (dict(kv_lens=None), ARG), (dict(pos=None), ARG), (dict(slots=None), ARG), (dict(batch=0), OK)])
def test_plan(L, kw, st):
    assert plan(L, **kw) == st


@pytest.mark.parametrize("kw,st", [
    (dict(dtype=2), ARG), (dict(m=-1), ARG), (dict(flags=1), ARG), (dict(flags=0, qw=256), ARG), (dict(h=0), SHAPE),
    (dict(h=1 << 16), SHAPE), (dict(x=256, d=12), SHAPE), (dict(n_pos=0), SHAPE), (dict(qkv=None), ARG), (dict(slots=None), ARG),
    (dict(q=None), ARG), (dict(table=None), ARG), (dict(qkv=264), ALIGN), (dict(kw=260), ALIGN), (dict(table=516), ALIGN),
    (dict(m=0), OK), (dict(m=0, pos=None, table=None, n_pos=0), OK)])
def test_put(L, kw, st):
    assert put(L, **kw) == st


@pytest.mark.parametrize("kw,st", [(dict(dtype=-1), ARG), (dict(m=-1), ARG), (dict(m=1 << 28), SHAPE), (dict(slots=None), ARG),
                                   (dict(k=None), ARG), (dict(v=520), ALIGN), (dict(m=0), OK)])
def test_read(L, kw, st):
    assert read(L, **kw) == st


@pytest.mark.parametrize("kw,st", [
    (dict(h=0), UNSUPPORTED), (dict(h=7), UNSUPPORTED), (dict(h=34), UNSUPPORTED), (dict(batch=-1), ARG), (dict(batch=2049), SHAPE),
    (dict(m=-1), ARG), (dict(m=(1 << 18) + 1), SHAPE), (dict(max_pages=0), SHAPE), (dict(max_pages=1 << 26), SHAPE),
    (dict(scale=float("inf")), ARG), (dict(scale=float("nan")), ARG), (dict(max_q=0), ARG), (dict(max_q=5), ARG), (dict(q=None), ARG),
    (dict(cu=None), ARG), (dict(lens=None), ARG), (dict(tables=None), ARG), (dict(o=None), ARG), (dict(ws=None), ARG),
    (dict(q=264), ALIGN), (dict(o=258), ALIGN), (dict(ws=264), ALIGN), (dict(m=0), OK), (dict(batch=0), OK)])
def test_attn(L, kw, st):
    assert attn(L, **kw) == st


def test_workspaces_of_no_sizes(L):
    for bad in ((0, 1, 8, 2, 64), (1, 0, 8, 2, 64), (1, 1, 7, 2, 64), (1, 1, 8, 0, 64)):
        assert L.wq_attn_paged_workspace_bytes(*bad) == 0
    assert L.wq_decoder_paged_workspace_bytes(1, 1, None) == 0


def test_a_layer_is_needed(L):
    assert L.wq_decoder_paged_forward(256, 1, 1, 1, 256, 256, 256, 256, None, None, None, pool(), 256, 4, 256, 8, 0, 256, 256, 1 << 30,
                                      None) == ARG


def test_outputs_over_their_inputs(L):
    row = 8 * 128 * 2  # bytes of q and o; of qkv 12 heads of fp32
    for o in (1 << 16, (1 << 16) + 16, (1 << 16) + 4 * row - 16, (1 << 16) - 4 * row + 16):
        assert attn(L, q=1 << 16, o=o) == ARG and b"over" in L.wq_last_error()
    for q in (1 << 16, (1 << 16) + 3 * 12 * 128 * 4 - 16, (1 << 16) - 3 * row + 16):
        assert put(L, qkv=1 << 16, h=8, q=q) == ARG and b"over" in L.wq_last_error()
