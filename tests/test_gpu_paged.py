"""The operators on pages against plain forms: step plans against a loop, rows written and read against the quantizer's
definition, attention against fp64 with bounds element by element."""
import math
import random

import pytest
import torch

from paged_util import attn_ref, check, fill_pool, i32, plan_loop, pool_values, status
from paper_2606_04238_gb300 import wq

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(*shape, seed=0, dtype=torch.float32):
    return torch.randn(shape, generator=gen(seed), device="cuda").to(dtype)


# ---- plans ---------------------------------------------------------------------

def run_plan(lens, keep, n_new, tables, free, n_free, page, m, in_place=False):
    t, f, nf, le = i32(*sum(tables, [])).view(len(lens), -1), i32(*free), i32(n_free), i32(*lens)
    out = nf if in_place else i32(-7)
    cu, kv, pos, slots = wq.page_plan(le, i32(*n_new), t, f, nf, page, m, keep=None if keep is None else i32(*keep),
                                      n_free_out=None if in_place else out, kv_lens=le if in_place else None)
    assert in_place or (nf.item() == n_free and le.tolist() == lens)
    return cu.tolist(), kv.tolist(), pos.tolist(), slots.tolist(), t.tolist(), f.tolist(), out.item()


def a_batch(rng, batch, page, max_pages, spare):
    """Requests that hold distinct pages, and a stack of what is left."""
    lens = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, max_pages * page), max_pages * page]) for _ in range(batch)]
    lens = [min(x, max_pages * page) for x in lens]
    have = [-(-x // page) for x in lens]
    ids = list(range(sum(have) + spare))
    rng.shuffle(ids)
    tables, at = [], 0
    for h in have:
        tables.append(ids[at:at + h] + [-1] * (max_pages - h))
        at += h
    return lens, tables, ids[at:] + [-1] * at, spare


@pytest.mark.parametrize("seed", range(12))
@pytest.mark.parametrize("batch,page,max_pages", [(1, 16, 1), (3, 16, 5), (40, 32, 9), (513, 256, 3), (700, 64, 4), (2048, 16, 6)])
def test_plan_is_the_loop(batch, page, max_pages, seed):
    rng = random.Random(1000 * batch + seed)
    lens, tables, free, n_free = a_batch(rng, batch, page, max_pages, rng.choice([0, 1, batch, 4 * batch]))
    keep = [rng.choice([x, x, 0, max(0, x - rng.randint(0, 7)), rng.randint(0, x)]) for x in lens] if seed % 3 else list(lens)
    new = [rng.choice([0, 1, 1, rng.randint(0, 2 * page)]) for _ in lens]
    new = [min(n, max_pages * page - k) for n, k in zip(new, keep)]
    m = max(1, sum(new) + rng.choice([0, 5, 700]))
    want = plan_loop(lens, keep, new, tables, free, n_free, page, m)
    got = run_plan(lens, keep if seed % 3 else None, new, tables, free, n_free, page, m, in_place=seed % 2 == 1)
    for name, g, w in zip(("cu", "kv_lens", "positions", "slots", "tables", "free", "n_free"), got, want):
        assert g == (list(w) if isinstance(w, (list, tuple)) else w), name
    assert status() == 0 and not want[-1]


def test_plan_of_requests_out_of_range():
    page, P = 16, 4
    lens = [5, -1, 65, 10, 10, 3, 0, 20]
    keep = [5, 0, 65, 11, -1, 3, 0, 20]
    new = [1, 1, 0, 1, 1, -2, 65, 1]
    tables = [[8 * b + i for i in range(P)] for b in range(8)]
    free = list(range(32, 64)) + [0] * 0 + [7] * 32
    want = plan_loop(lens, keep, new, tables, free, 32, page, 100)
    got = run_plan(lens, keep, new, tables, free, 32, page, 100)
    assert got == tuple(list(w) if isinstance(w, list) else w for w in want[:-1])
    assert want[-1] and status() == -1 and status() == 0


def test_plan_of_more_tokens_than_rows():
    lens, new = [3, 3, 3, 3], [2, 5, 0, 1]
    tables, free = [[0, -1], [1, -1], [2, -1], [3, -1]], [4, 5, 6, 7]
    want = plan_loop(lens, lens, new, tables, free, 4, 16, 4)
    assert run_plan(lens, None, new, tables, free, 4, 16, 4) == tuple(list(w) if isinstance(w, list) else w for w in want[:-1])
    assert want[1] == [5, -1, 3, -1] and want[0] == [0, 2, 4, 4, 4] and status() == -1


def test_plan_without_pages_left():
    # requests 1 and 2 want more than there is with those before them; 3 wants none
    lens, new = [16, 16, 16, 15], [1, 20, 1, 1]
    tables, free = [[0, -1, -1], [1, -1, -1], [2, -1, -1], [3, -1, -1]], [4, 5, -1, -1, -1, -1]
    want = plan_loop(lens, lens, new, tables, free, 2, 16, 30)
    got = run_plan(lens, None, new, tables, free, 2, 16, 30)
    assert got == tuple(list(w) if isinstance(w, list) else w for w in want[:-1])
    assert got[1] == [17, -1, -1, 16] and got[6] == 1 and status() == 0


def test_plan_of_a_stack_out_of_range():
    got = run_plan([0], None, [1], [[9]], [99, 0], 1, 16, 2)  # a page that the pool does not have
    assert got[3] == [-1, -1] and status() == -1
    for n in (-3, 5):
        run_plan([0], None, [1], [[9]], [0, 1], n, 16, 2)
        assert status() == -1
    # pages given back beyond the pool (twice) stay off the stack's end
    got = run_plan([32, 32], [0, 0], [0, 0], [[0, 1], [0, 1]], [1, 0, 7], 2, 16, 2)
    assert got[5] == [1, 0, 0] and got[6] == 3 and status() == -1


def test_steps_of_a_batch_in_a_graph():
    """A captured plan, replayed: lens, tables and the stack live on the device and every page stays owned once."""
    page, P, B, m = 16, 8, 5, 64
    n_pages = 24
    lens, tables, free, n_free = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B, P), -1, dtype=torch.int32, device="cuda"), \
        torch.arange(n_pages, dtype=torch.int32, device="cuda"), i32(n_pages)
    keep, new = lens.clone(), i32(*[0] * B)
    out = [torch.empty(s, dtype=torch.int32, device="cuda") for s in (B + 1, m, m)]
    step = lambda: wq.page_plan(lens, new, tables, free, n_free, page, m, keep=keep, cu=out[0], kv_lens=lens, positions=out[1],  # noqa: E731
                                slots=out[2])
    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    rng = random.Random(5)
    L, T, F, nf = [0] * B, tables.tolist(), free.tolist(), n_pages
    for _ in range(30):
        K = [rng.choice([x, x, 0, max(0, x - 3)]) for x in L]
        N = [min(rng.choice([1, 1, 0, 13]), P * page - k) for k in K]
        keep.copy_(i32(*K))
        new.copy_(i32(*N))
        g.replay()
        cu, kv, pos, slots, T, F, nf, _ = plan_loop(L, K, N, T, F, nf, page, m)
        assert (out[0].tolist(), out[1].tolist(), out[2].tolist()) == (cu, pos, slots)
        assert (lens.tolist(), tables.tolist(), free.tolist(), n_free.item()) == (kv, T, F, nf)
        L = kv
        held = [p for b in range(B) for p in T[b][:-(-L[b] // page)]] + F[:nf]
        assert sorted(held) == list(range(n_pages))


# ---- rows written and read -------------------------------------------------------

def slots_of(m, page, n_pages, seed):
    return torch.randperm(n_pages * page, generator=gen(seed), device="cuda")[:m].to(torch.int32)


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd,kv,page", [(128, 8, 16), (64, 4, 64), (128, 3, 256), (64, 1, 32)])
def test_rows_as_they_are(hd, kv, page, bits, f32):
    """Without a norm and a rotation the pages hold what wq_kv_append writes, byte for byte."""
    m, h, n_pages = 37, kv, 5 if page < 64 else 2
    qkv = randn(m, (h + 2 * kv) * hd, seed=hd + bits, dtype=torch.float32 if f32 else BF)
    qkv[3, h * hd:] = 0  # rows of zeros
    qkv[5, h * hd + 1] = math.nan
    qkv[6, -1] = math.inf
    pool, ref = wq.kv_pool(n_pages, kv, page, hd, bits), wq.kv_pool(n_pages, kv, page, hd, bits)
    slots = slots_of(m, page, n_pages, 7)
    q = wq.qkv_paged(qkv, slots, pool, h, head_norm=False)
    assert torch.equal(q.view(torch.int16), qkv[:, :h * hd].reshape(m, h, hd).to(BF).view(torch.int16))
    # the same rows through the cache's call, a page a sequence
    rows = qkv[:, h * hd:].reshape(m, 2, kv, hd)
    for t in range(m):
        p, at = divmod(slots[t].item(), page)
        one = wq.KVCache(*[x[p:p + 1] for x in (ref.k, ref.v)], *[None if x is None else x[p:p + 1] for x in (ref.k_meta, ref.v_meta)], hd, bits)
        wq.kv_append(one, rows[t, 0].reshape(1, 1, kv, hd), rows[t, 1].reshape(1, 1, kv, hd), i32(at))
    for a, b in ((pool.k, ref.k), (pool.v, ref.v), (pool.k_meta, ref.k_meta), (pool.v_meta, ref.v_meta)):
        if a is not None and bits == 16:  # (a NaN is a NaN, whichever of its bit patterns)
            assert torch.equal(a.isnan(), b.isnan())
            a, b = a.nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf), b.nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf)
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    k, v = wq.paged_read(pool, slots, dtype=torch.float32)
    K, V = pool_values(pool)[:2]
    s = slots.long()
    for got, want in ((k, K), (v, V)):
        want = want[s // page, :, s % page]
        assert torch.equal(got.double().isnan(), want.isnan())
        assert torch.equal(got.double().nan_to_num(), want.nan_to_num())
    kb, vb = wq.paged_read(pool, slots)
    assert torch.equal(kb.nan_to_num(), k.to(BF).nan_to_num()) and torch.equal(vb.nan_to_num(), v.to(BF).nan_to_num())
    assert status() == 0


@pytest.mark.parametrize("m", [1, 2, 33, 300])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("h,kv,hd,d,weights", [(32, 8, 128, 2560, True), (10, 2, 64, 0, True), (5, 5, 128, 72, False), (64, 8, 64, 2880, True)])
def test_normed_and_rotated(h, kv, hd, d, weights, bits, m):
    page, n_pos = 32, 500
    n_pages = -(-m // page) + 1
    qkv = randn(m, (h + 2 * kv) * hd, seed=m) * 1.7
    x = randn(m, d, seed=m + 1, dtype=BF) if d else None
    qw, kw = ((1 + 0.4 * randn(hd, seed=s)).to(BF) if weights else None for s in (3, 4))
    pos = torch.randint(0, n_pos, (m,), generator=gen(9), device="cuda", dtype=torch.int32)
    table = wq.rope_table(n_pos, hd)
    pool, slots = wq.kv_pool(n_pages, kv, page, hd, bits), slots_of(m, page, n_pages, 8)
    q = wq.qkv_paged(qkv, slots, pool, h, positions=pos, table=table, x=x, q_norm=qw, k_norm=kw)
    u = qkv.double()
    if d:
        u = u / torch.sqrt(x.double().pow(2).mean(-1, keepdim=True) + 1e-6)
    u = u.view(m, h + 2 * kv, hd)
    n = u[:, :h + kv]
    n = n / torch.sqrt(n.pow(2).mean(-1, keepdim=True) + 1e-6)
    if weights:
        n = n * torch.cat([qw.double().expand(h, hd), kw.double().expand(kv, hd)])
    cs = table.double()[pos.long()][:, None]
    lo, hi = n[..., :hd // 2], n[..., hd // 2:]
    n = torch.cat([lo * cs[..., 0] - hi * cs[..., 1], hi * cs[..., 0] + lo * cs[..., 1]], -1)
    size = torch.cat([lo.abs() + hi.abs()] * 2, -1)
    # fp32: the sums of squares (hd and d terms, in part one after another), a root, a quotient, five products
    fuzz = (hd / 8 + d / 512 + 16) * 2.0 ** -24
    check(q, n[:, :h], 2.0 ** -8 * (n[:, :h].abs() + fuzz * size[:, :h]) + fuzz * size[:, :h], "q")
    k, v = wq.paged_read(pool, slots, dtype=torch.float32)
    for got, want, off in ((k, n[:, h:], fuzz * size[:, h:]), (v, u[:, h + kv:], fuzz * u[:, h + kv:].abs())):
        if bits == 16:
            check(got, want, 2.0 ** -8 * (want.abs() + off) + off)
        else:
            # a step is the range around zero over 2^bits - 1, as binary16 (2^-11); values are half a step off, those at an
            # end another half (the zero point is rounded too) and what the rounded steps do not reach
            rng = want.amax(-1, keepdim=True).clamp(min=0) - want.amin(-1, keepdim=True).clamp(max=0)
            step = rng / (2 ** bits - 1)
            check(got, want, step * (1.0 + 2.0 ** -10) + rng * 2.0 ** -10 + off + off.amax(-1, keepdim=True))
    # where the codes are not at a border, they are those of the fp64 row
    assert status() == 0


def test_codes_of_equal_rows_are_equal():
    """A row's codes do not hang on its place in the batch or on its head."""
    m, kv, hd = 29, 4, 128
    row = randn(1, hd, seed=1)
    qkv = row.repeat(m, 3 * kv)
    table = wq.rope_table(4, hd)
    pool, slots = wq.kv_pool(2, kv, 16, hd, 4), slots_of(m, 16, 2, 3)
    wq.qkv_paged(qkv, slots, pool, kv, positions=i32(*[2] * m), table=table)
    k, v = wq.paged_read(pool, slots, dtype=torch.float32)
    assert bool((k == k[:1, :1]).all()) and bool((v == v[:1, :1]).all())


def test_slots_that_are_not_kept():
    m, kv, hd, h = 6, 2, 64, 4
    qkv = randn(m, (h + 2 * kv) * hd, seed=2)
    for bits in (16, 8, 4):
        pool = wq.kv_pool(3, kv, 16, hd, bits)
        slots = i32(5, -1, 48, -2, 47, 2 ** 31 - 1)  # two kept, one not asked for, three outside
        q = wq.qkv_paged(qkv, slots, pool, h, head_norm=False)
        assert torch.equal(q, qkv[:, :h * hd].reshape(m, h, hd).to(BF)) and status() == -1 and status() == 0
        K, V = pool_values(pool)[:2]
        kept = torch.zeros(3, 16, dtype=torch.bool, device="cuda")
        kept[0, 5] = kept[2, 15] = True
        there = (K != 0).any(-1).any(1)
        assert torch.equal(there, kept)
        k = torch.full((m, kv, hd), 7.0, dtype=torch.float32, device="cuda")
        v = k.clone()
        wq.paged_read(pool, slots, dtype=torch.float32, k=k, v=v)
        assert status() == -1
        assert bool((k[[2, 3, 5]] == 7).all()) and bool((k[1] == 0).all()) and bool((v[1] == 0).all())
        assert torch.equal(k[0].double(), K[0, :, 5]) and torch.equal(v[4].double(), V[2, :, 15])


def test_positions_outside_the_table():
    m, kv, hd, h = 4, 1, 64, 2
    qkv, table = randn(m, (h + 2 * kv) * hd, seed=3), wq.rope_table(10, hd)
    pool = wq.kv_pool(1, kv, 16, hd, 8)
    q = torch.full((m, h, hd), 9.0, dtype=BF, device="cuda")
    wq.qkv_paged(qkv, i32(0, 1, 2, 3), pool, h, positions=i32(9, 10, -1, 0), table=table, q=q)
    assert status() == -1
    assert bool((q[1:3] == 9).all()) and not bool((q[0] == 9).all())
    k, _ = wq.paged_read(pool, i32(0, 1, 2, 3))
    assert (k != 0).flatten(1).any(1).tolist() == [True, False, False, True]


# ---- attention --------------------------------------------------------------------

def a_pool(n_pages, kv, page, hd, bits, seed=0, loud=True):
    k, v = (randn(n_pages, kv, page, hd, seed=seed + s) for s in (1, 2))
    if loud:
        k[..., 3] *= 5
        v[..., ::17] *= 4
    pool = wq.kv_pool(n_pages, kv, page, hd, bits)
    fill_pool(pool, k.to(BF), v.to(BF))
    return pool


def ragged(nq, lens, page, seed=0, spare=2, max_pages=None):
    """cu, kv_lens, tables of sequences with pages of their own in a drawn order; the pool's pages."""
    cu = [0]
    for n in nq:
        cu.append(cu[-1] + n)
    need = [-(-max(x, 0) // page) for x in lens]
    max_pages = max_pages or max(1, max(need))
    ids = torch.randperm(sum(need) + spare, generator=gen(seed), device="cuda").tolist()
    rows, at = [], 0
    for n in need:
        rows.append(ids[at:at + n] + [0] * (max_pages - n))
        at += n
    return cu, i32(*sum(rows, [])).view(len(nq), max_pages), len(ids)


def run_attn(nq, lens, h, kv, hd, bits, page, seed=0, scale=None, max_q=None, max_pages=None):
    cu, tables, n_pages = ragged(nq, lens, page, seed, max_pages=max_pages)
    pool = a_pool(n_pages, kv, page, hd, bits, seed)
    q = randn(max(1, cu[-1]), h, hd, seed=seed + 9, dtype=BF)
    o = torch.full_like(q, 7.0)
    wq.attn_paged(q, i32(*cu), i32(*lens), tables, pool, max_q=max_q or max(1, max(nq)), scale=scale, o=o)
    ref, bound = attn_ref(q, cu, lens, tables, pool, hd ** -0.5 if scale is None else scale)
    check(o[:cu[-1]], ref[:cu[-1]], bound[:cu[-1]], f"{nq} {lens} {bits}")
    assert bool((o[cu[-1]:] == 7).all())
    assert status() == 0
    return o


HEADS = [(32, 8, 128), (64, 8, 64), (16, 4, 64), (10, 2, 128), (3, 3, 64), (16, 1, 128)]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("h,kv,hd", HEADS)
@pytest.mark.parametrize("lens", [[1], [2, 15, 16, 17], [63, 64, 65, 500], [1000, 1, 129]])
def test_one_token(h, kv, hd, bits, lens):
    for page in (16, 64):
        run_attn([1] * len(lens), lens, h, kv, hd, bits, page, seed=len(lens) + page)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("h,kv,hd", HEADS)
@pytest.mark.parametrize("nq,lens", [([2, 3, 1], [2, 40, 300]), ([5, 0, 7, 1], [5, 9, 70, 129]), ([17], [17]), ([33, 1, 64], [33, 700, 64]),
                                     ([130, 16], [321, 16]), ([1, 200], [90, 1025])])
def test_ragged(h, kv, hd, bits, nq, lens):
    run_attn(nq, lens, h, kv, hd, bits, 32, seed=sum(nq))


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("nq,lens", [([1, 1], [333, 257]), ([3, 100], [259, 515])])
def test_pages(page, bits, nq, lens):
    run_attn(nq, lens, 8, 2, 128, bits, page, seed=page, max_pages=40)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_many_sequences(bits):
    rng = random.Random(bits)
    lens = [rng.randint(1, 90) for _ in range(150)]
    nq = [min(x, rng.choice([0, 1, 1, 1, 2])) for x in lens]
    run_attn(nq, lens, 8, 2, 64, bits, 16, seed=4)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("nq", [1, 4, 60])
def test_long(bits, nq):
    run_attn([nq], [20011], 8, 2, 128, bits, 64, seed=nq)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("h,kv,hd", [(8, 4, 128), (6, 2, 64)])
def test_many_tiles_a_run(h, kv, hd, bits):
    """Runs of tens of tiles, over ends of blocks: short chunks (both streams with the same rows) and longer ones."""
    nq = [9] * 24 + [200, 131, 60, 300]
    run_attn(nq, [4001 + 37 * i for i in range(24)] + [5000, 3000, 4096, 2500], h, kv, hd, bits, 64, seed=3)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-30])
def test_scales(bits, scale):
    run_attn([1, 2, 90], [200, 300, 100], 8, 2, 64, bits, 16, scale=scale, seed=3)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("nq,down", [(1, False), (150, False), (150, True)])
def test_scores_that_rise(nq, down, hd, bits):
    """Scores that grow (or fall) by some 13 powers of two a tile: the maximum is raised, and O rescaled, in every one."""
    h, kv, page, n = 8, 2, 32, 1100
    cu, tables, n_pages = ragged([nq], [n], page, 5)
    k, v = (randn(n_pages, kv, page, hd, seed=s) for s in (1, 2))
    along = torch.sign(randn(hd, seed=3))
    at = torch.arange(n, device="cuda").flip(0) if down else torch.arange(n, device="cuda")
    ids = tables[0].long().repeat_interleave(page)[:n]
    k[ids, :, torch.arange(n, device="cuda") % page] += (at / n * 80 / hd ** 0.5)[:, None, None] * along
    pool = wq.kv_pool(n_pages, kv, page, hd, bits)
    fill_pool(pool, k.to(BF), v.to(BF))
    q = (randn(nq, h, hd, seed=5) + along).to(BF)
    o = wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq)
    ref, bound = attn_ref(q, cu, [n], tables, pool, hd ** -0.5)
    check(o, ref, bound, f"{nq} {hd} {bits}")
    assert status() == 0


def test_max_q_is_a_bound_not_a_shape():
    """The kernels that a larger max_q takes give what the smaller one's do, within the bound."""
    for bits in (16, 8, 4):
        for most in (3, 8, 500):
            run_attn([3, 1, 2] + [1] * 600, [400, 17, 30] + [5] * 600, 8, 2, 64, bits, 16, max_q=most)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("nq", [3, 150])
def test_what_is_not_seen_does_not_count(bits, nq):
    """Infinities and NaN behind a sequence's end, in pages of others, and in newer tokens' rows."""
    h, kv, hd, page, n = 8, 2, 128, 16, 200
    cu, tables, n_pages = ragged([nq], [n], page, 1)
    k, v = (randn(n_pages, kv, page, hd, seed=s) for s in (1, 2))
    at = tables[0].long()
    k.view(-1)[:] = k.view(-1)
    last = at[(n - 1) // page]
    for t, bad in ((k, math.nan), (v, math.inf)):
        t[last, :, n % page:] = bad  # behind the end
        t[last, :, (n - 1) % page] = bad  # the newest token's own row
        others = torch.ones(n_pages, dtype=torch.bool, device="cuda")
        others[at] = False
        t[others] = bad
    pool = wq.kv_pool(n_pages, kv, page, hd, bits)
    fill_pool(pool, k.to(BF), v.to(BF))
    q = randn(nq, h, hd, seed=5, dtype=BF)
    o = wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq)
    assert not bool(o[:-1].isnan().any()) and bool(o[-1].isnan().all())
    # the same without the newest token
    ref, bound = attn_ref(q[:-1], [0, nq - 1], [n - 1], tables, pool, hd ** -0.5)
    check(o[:-1], ref, bound)
    # an infinity of V alone, in a bf16 pool, reaches the rows that see it and its column alone
    if bits == 16:
        k2, v2 = (randn(n_pages, kv, page, hd, seed=s) for s in (1, 2))
        i = n - 2
        v2[at[i // page], 1, i % page, 7] = math.inf
        fill_pool(pool, k2.to(BF), v2.to(BF))
        o = wq.attn_paged(q, i32(*cu), i32(n), tables, pool, max_q=nq)
        inf = torch.zeros_like(o, dtype=torch.bool)
        inf[-2:, h // 2:, 7] = True
        assert torch.equal(o.isinf(), inf) and not bool(o.isnan().any())


def test_not_served_and_out_of_range():
    h, kv, hd, page = 8, 2, 64, 16
    for bits, n in ((8, 1), (4, 1), (16, 40)):
        nq = [n, n, n, n, n]
        cu, tables, n_pages = ragged(nq, [50] * 5, page, 2)
        pool = a_pool(n_pages, kv, page, hd, bits)
        q = randn(cu[-1], h, hd, seed=6, dtype=BF)
        ref, bound = attn_ref(q, cu, [50] * 5, tables, pool, hd ** -0.5)
        o = torch.full_like(q, 7.0)
        lens = [50, -1, n - 1 if n > 1 else 0, 65, 50]  # served, not served, too short, past the table, served
        wq.attn_paged(q, i32(*cu), i32(*lens), tables, pool, max_q=n, o=o)
        assert status() == -1 and status() == 0
        for b in (0, 4):
            check(o[cu[b]:cu[b + 1]], ref[cu[b]:cu[b + 1]], bound[cu[b]:cu[b + 1]])
        assert bool((o[cu[1]:cu[2]] == 0).all()) and bool((o[cu[2]:cu[4]] == 7).all())
        # offsets that do not ascend, or pass m, or are more than max_q apart
        bad = list(cu)
        bad[2], bad[5] = 0, cu[5] + 1
        o.fill_(7.0)
        wq.attn_paged(q, i32(*bad), i32(*[50] * 5), tables, pool, max_q=n, o=o)
        assert status() == -1
        check(o[cu[3]:cu[4]], ref[cu[3]:cu[4]], bound[cu[3]:cu[4]])
        # a page that the pool does not have
        t2 = tables.clone()
        t2[1, 1] = n_pages
        t2[3, 0] = -5
        o.fill_(7.0)
        wq.attn_paged(q, i32(*cu), i32(*[50] * 5), t2, pool, max_q=n, o=o)
        assert status() == -1
        for b in (0, 2, 4):
            check(o[cu[b]:cu[b + 1]], ref[cu[b]:cu[b + 1]], bound[cu[b]:cu[b + 1]])


def test_few_and_many_rows_in_a_batch():
    """Sequences of few rows beside longer ones: each served once, those not served zeros, wrong ones left, rows behind the last left."""
    h, kv, hd, page = 8, 2, 128, 16
    nq = [1, 300, 0, 2, 3, 1, 40, 1, 90, 2, 130, 4]
    lens = [70, 300, 5, 2, 200, -1, 41, 400, -1, 1, 129, 900]  # (the last three: shorter than their rows, twice; a long one)
    for bits in (16, 8, 4):
        cu, tables, n_pages = ragged(nq, [max(x, n, 1) for x, n in zip(lens, nq)], page, 3)
        pool = a_pool(n_pages, kv, page, hd, bits)
        q = randn(cu[-1] + 5, h, hd, seed=6, dtype=BF)
        t2 = tables.clone()
        t2[3, 0], t2[6, 1] = n_pages, -1  # pages that the pool does not have
        o = torch.full_like(q, 7.0)
        wq.attn_paged(q, i32(*cu), i32(*lens), t2, pool, max_q=300, o=o)
        assert status() == -1 and status() == 0
        good = [max(x, n) for x, n in zip(lens, nq)]
        ref, bound = attn_ref(q[:cu[-1]], cu, good, tables, pool, hd ** -0.5)
        for b, (n, length) in enumerate(zip(nq, lens)):
            at = slice(cu[b], cu[b + 1])
            if length < 0:
                assert bool((o[at] == 0).all())
            elif length < n:
                assert bool((o[at] == 7).all())
            elif b not in (3, 6):
                check(o[at], ref[at], bound[at], f"{bits} {b}")
        assert bool((o[cu[-1]:] == 7).all())


def test_shared_pages_and_zero_rows():
    """Two requests over one prefix; a pool of zeros and rows of zeros among others."""
    h, kv, hd, page = 8, 2, 128, 16
    for bits in (16, 8, 4):
        k, v = (randn(6, kv, page, hd, seed=s) for s in (1, 2))
        v[:, :, ::2] = 0
        v[:, :, 1::4] *= 1e-3
        k[2] = 0
        pool = wq.kv_pool(6, kv, page, hd, bits)
        fill_pool(pool, k.to(BF), v.to(BF))
        tables = i32(0, 1, 2, 0, 1, 3).view(2, 3)
        q = randn(2, h, hd, seed=3, dtype=BF)
        o = wq.attn_paged(q, i32(0, 1, 2), i32(40, 48), tables, pool)
        ref, bound = attn_ref(q, [0, 1, 2], [40, 48], tables, pool, hd ** -0.5)
        check(o, ref, bound)
        empty = wq.kv_pool(6, kv, page, hd, bits)
        assert bool((wq.attn_paged(q, i32(0, 1, 2), i32(40, 48), tables, empty) == 0).all())


def test_the_same_twice_and_in_a_graph():
    for bits, nq, lens in ((4, [1] * 9, [700, 3, 64, 65, 1500, 9, 10, 11, 12]), (8, [1, 120, 1], [900, 500, 33]), (16, [150], [600])):
        h, kv, hd, page = 16, 4, 64, 16
        cu, tables, n_pages = ragged(nq, lens, page, 1)
        pool = a_pool(n_pages, kv, page, hd, bits)
        q = randn(cu[-1], h, hd, seed=2, dtype=BF)
        ws = wq.attn_paged_workspace(len(nq), cu[-1], h, kv, hd)
        c, n = i32(*cu), i32(*lens)
        o = wq.attn_paged(q, c, n, tables, pool, max_q=max(nq), ws=ws)
        other = wq.attn_paged(q, c, n, tables, pool, max_q=max(nq))
        assert torch.equal(o, other)
        out = torch.empty_like(o)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            wq.attn_paged(q, c, n, tables, pool, max_q=max(nq), o=out, ws=ws)
        for _ in range(3):
            out.fill_(7.0)
            g.replay()
            assert torch.equal(o, out)
        # other lengths in the same graph
        n.copy_(torch.maximum(n // 2, c[1:] - c[:-1]))
        g.replay()
        ref, bound = attn_ref(q, cu, n.tolist(), tables, pool, hd ** -0.5)
        check(out, ref, bound)


def test_workspace_too_small():
    h, kv, hd = 8, 2, 64
    pool = a_pool(2, kv, 16, hd, 8)
    q = randn(1, h, hd, dtype=BF)
    ws = wq.attn_paged_workspace(1, 1, h, kv, hd)
    with pytest.raises(wq.WQError) as e:
        wq.attn_paged(q, i32(0, 1), i32(5), i32(0).view(1, 1), pool, ws=ws[:ws.numel() - 256])
    assert e.value.status == -7


def test_on_a_stream_of_its_own():
    h, kv, hd, page = 8, 2, 128, 16
    cu, tables, n_pages = ragged([2, 90], [100, 300], page, 1)
    pool = a_pool(n_pages, kv, page, hd, 4)
    q = randn(92, h, hd, seed=1, dtype=BF)
    ref, bound = attn_ref(q, cu, [100, 300], tables, pool, hd ** -0.5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o = wq.attn_paged(q, i32(*cu), i32(100, 300), tables, pool, max_q=90)
    s.synchronize()
    check(o, ref, bound)
