"""Calls on pages whose outputs lie over what other threads of the same call may still read (or write): refused on the host,
before any launch.  What a plan reads before it writes may be an output as well."""
import pytest

from test_kv_refusals import ARG, L  # noqa: F401
from test_paged_refusals import attn, plan, pool, put, read

M, H, KV, HD, PAGE, PAGES = 3, 4, 2, 128, 32, 8
ROWS = PAGES * KV * PAGE
MB = 1 << 20


def refused(L, st):
    return st == ARG and b"over" in L.wq_last_error()


def edges(at, size, mine, step=16):
    """Places of an array of `mine` bytes that shares its first, its last and some other bytes with [at, at + size)."""
    return sorted({at, (at + size - 1) // step * step, (at - mine) // step * step + step, at + size // 2 // step * step})


def a_pool(bits=8):
    return pool(k=16 * MB, v=20 * MB, k_meta=24 * MB, v_meta=28 * MB, bits=bits)


HELD = [("k", 16 * MB, ROWS * HD), ("v", 20 * MB, ROWS * HD), ("k_meta", 24 * MB, ROWS * 4), ("v_meta", 28 * MB, ROWS * 4)]
PUT = dict(qkv=MB, x=2 * MB, pos=3 * MB, table=4 * MB, qw=5 * MB, kw=6 * MB, slots=7 * MB, d=2560, n_pos=8)


@pytest.mark.parametrize("name,at,size", [("qkv", MB, M * (H + 2 * KV) * HD * 4), ("x", 2 * MB, M * 2560 * 2), ("pos", 3 * MB, M * 4),
                                          ("table", 4 * MB, 8 * HD * 4), ("qw", 5 * MB, HD * 2), ("kw", 6 * MB, HD * 2),
                                          ("slots", 7 * MB, M * 4), *HELD])
def test_queries_over_inputs(L, name, at, size):  # noqa: F811
    for q in edges(at, size, M * H * HD * 2):
        assert refused(L, put(L, c=a_pool(), q=q, **PUT)), (name, hex(q))


@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_read_over_one_another_and_the_pool(L, dtype):  # noqa: F811
    mine = M * KV * HD * (2 + 2 * dtype)
    for v in edges(MB, mine, mine):
        assert refused(L, read(L, c=a_pool(), slots=7 * MB, k=MB, v=v, dtype=dtype))
    for _, at, size in HELD + [("slots", 7 * MB, M * 4)]:
        for p in edges(at, size, mine):
            for kw in (dict(k=p, v=MB), dict(k=MB, v=p)):
                assert refused(L, read(L, c=a_pool(), slots=7 * MB, dtype=dtype, **kw))


def test_attention_over_inputs(L):  # noqa: F811
    kw = dict(q=MB, m=4, h=8, batch=2, cu=2 * MB, lens=3 * MB, tables=4 * MB, max_pages=4, ws=8 * MB)
    mine = 4 * 8 * HD * 2
    for _, at, size in HELD + [("q", MB, mine), ("cu", 2 * MB, 12), ("lens", 3 * MB, 8), ("tables", 4 * MB, 32)]:
        for o in edges(at, size, mine):
            assert refused(L, attn(L, c=a_pool(), o=o, **kw))


WRITTEN = dict(tables=(MB, 2 * 4 * 4), free=(2 * MB, 8 * 4), cu=(3 * MB, 3 * 4), kv_lens=(4 * MB, 2 * 4), pos=(5 * MB, 4 * 4),
               slots=(6 * MB, 4 * 4), out=(7 * MB, 4))


@pytest.mark.parametrize("one", WRITTEN)
@pytest.mark.parametrize("other", WRITTEN)
def test_a_plan_over_itself(L, one, other):  # noqa: F811
    if one == other:
        return
    at, size = WRITTEN[one]
    for p in edges(at, size, WRITTEN[other][1], step=4):
        kw = {n: a for n, (a, _) in WRITTEN.items()}
        kw[other] = p
        assert refused(L, plan(L, lens=9 * MB, n_new=10 * MB, n_free=11 * MB, **kw))


@pytest.mark.gpu
def test_outputs_in_the_workspace():
    import torch

    from paged_util import i32
    from paper_2606_04238_gb300 import wq
    ws, c = wq.attn_paged_workspace(1, 1, H, KV, HD), wq.kv_pool(PAGES, KV, PAGE, HD, 8)
    q = torch.zeros((1, H, HD), dtype=torch.bfloat16, device="cuda")
    o = ws[-2 * q.numel():].view(torch.bfloat16).view(1, H, HD)
    with pytest.raises(wq.WQError) as e:
        wq.attn_paged(q, i32(0, 1), i32(5), i32(0).view(1, 1), c, o=o, ws=ws)
    assert e.value.status == ARG
