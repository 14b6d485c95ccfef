"""A decoder layer over pages (wq_page_plan, then wq_decoder_paged_forward), run step after step as a continuous
batch: prompts and decode steps in one call, requests that end and are replaced, drafts that are taken back.

Over a bf16 pool against the same tokens through wq_decoder_tree_forward over a contiguous cache; over 8 and 4 bits
against the layer's parts called one by one.  Tolerance: the ways differ by bf16 roundings of q, of the probabilities,
of o, x1 and h, each some 2^-9 / sqrt(3) of its tensor, and what they flip further on; 1e-2 in the 2-norm is
about four times their sum.
"""
import random

import pytest
import torch

from paged_util import i32, status
from paper_2606_04238_gb300 import wq
from test_gpu_tree_decoder import D, H, HD, KV, _layer, _rel

pytestmark = pytest.mark.gpu

PAGE, P, B = 16, 10, 4


class Batch:
    """A pool, its tables and its stack of free pages."""

    def __init__(self, bits, n_pages=34):
        self.pool = wq.kv_pool(n_pages, KV, PAGE, HD, bits)
        self.tables = torch.full((B, P), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(n_pages, device="cuda").to(torch.int32)
        self.n_free = i32(n_pages)
        self.lens = i32(*[0] * B)

    def plan(self, keep, new, m):
        return wq.page_plan(self.lens, i32(*new), self.tables, self.free, self.n_free, PAGE, m, keep=i32(*keep), kv_lens=self.lens)


def _steps(seed):
    """(keep, new) of steps: prompts, decode steps, a request replaced, drafts of which some are taken back."""
    rng = random.Random(seed)
    lens = [0] * B
    for step in range(7):
        if step == 0:
            keep, new = [0] * B, [20, 7, 33, 1]
        else:
            keep = [max(0, n - rng.choice([0, 0, 2])) for n in lens]
            new = [rng.choice([1, 1, 0, 3]) for _ in lens]
            if step == 3:
                keep[1], new[1] = 0, 70  # another request in its place
        yield keep, new
        lens = [k + n for k, n in zip(keep, new)]


@pytest.mark.parametrize("weights", [False, True])
def test_continuous_batch_of_a_bf16_pool(weights):
    layer, batch, table = _layer(wq, 11), Batch(16), wq.rope_table(P * PAGE, HD)
    g = torch.Generator(device="cuda").manual_seed(4)
    caches = [wq.kv_cache(1, KV, P * PAGE, HD, 16) for _ in range(B)]
    ws = wq.decoder_paged_workspace(B, 128, layer)
    ones = torch.ones(HD, dtype=torch.bfloat16, device="cuda") if weights else None
    for keep, new in _steps(1):
        m = sum(new) + 5  # rows behind the last request
        x = torch.randn((m, D), generator=g, device="cuda").to(torch.bfloat16)
        cu, lens, pos, slots = batch.plan(keep, new, m)
        y = wq.decoder_paged_forward(x, cu, lens, pos, slots, layer, batch.pool, batch.tables, table, max_q=max(new), q_norm=ones,
                                     k_norm=ones, ws=ws)
        at = 0
        for b in range(B):
            if new[b] == 0:
                continue
            xb, p = x[None, at:at + new[b]].contiguous(), pos[None, at:at + new[b]].contiguous()
            assert p[0].tolist() == list(range(keep[b], keep[b] + new[b]))
            yb, kn, vn = wq.decoder_tree_forward(xb, i32(keep[b]), p, layer, caches[b], table)
            wq.kv_append(caches[b], kn, vn, i32(keep[b]))
            assert _rel(y[at:at + new[b]], yb[0]) < 1e-2
            at += new[b]
    for b in range(B):  # the pages hold what the caches hold, but for roundings that flip
        n = int(lens[b])
        s = (batch.tables[b].repeat_interleave(PAGE) * PAGE + torch.arange(P * PAGE, device="cuda") % PAGE)[:n].to(torch.int32)
        k, v = wq.paged_read(batch.pool, s)
        for mine, theirs in ((k, caches[b].k), (v, caches[b].v)):
            a, r = mine.float(), theirs[0, :, :n].transpose(0, 1).float()
            tol = r.abs() * 2.0 ** -7 + r.abs().amax(-1, keepdim=True) * 2.0 ** -15
            assert float((a != r).float().mean()) < 0.01 and bool(((a - r).abs() <= tol).all())
    assert status() == 0


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_the_layer_is_its_parts(bits):
    layer, batch, table = _layer(wq, 12), Batch(bits), wq.rope_table(P * PAGE, HD)
    other = Batch(bits)
    g = torch.Generator(device="cuda").manual_seed(5)
    qw, kw = ((1 + 0.2 * torch.randn(HD, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))
    mlp = layer.mlp
    for keep, new in _steps(2):
        m = max(1, sum(new))
        x = torch.randn((m, D), generator=g, device="cuda").to(torch.bfloat16)
        cu, lens, pos, slots = batch.plan(keep, new, m)
        y = wq.decoder_paged_forward(x, cu, lens, pos, slots, layer, batch.pool, batch.tables, table, max_q=max(max(new), 1), q_norm=qw,
                                     k_norm=kw)
        if sum(new) == 0:
            continue
        qkv = wq.down_w4(x, layer.qkv, out_f32=True)
        q = wq.qkv_paged(qkv, slots, other.pool, H, positions=pos, table=table, x=x, q_norm=qw, k_norm=kw)
        o = wq.attn_paged(q, cu, lens, batch.tables, other.pool, max_q=max(new))
        x1 = wq.down_w4(o.view(m, H * HD), layer.o, residual=x)
        h = wq.gateup_w2_lora(x1, mlp.gate, mlp.up, mlp.lora_a, mlp.lora_b_gate, mlp.lora_b_up, mlp.lora_scale, prenorm=True)
        assert _rel(y, wq.down_w4(h, mlp.down, residual=x1)) < 1e-2
    assert torch.equal(batch.pool.k, other.pool.k) and torch.equal(batch.pool.v, other.pool.v)
    assert status() == 0


def test_decode_loop_in_a_graph_and_a_workspace_for_all_sizes():
    """A captured step (plan, layer) replayed; one workspace for prompts and steps of every size."""
    layer, table = _layer(wq, 13), wq.rope_table(P * PAGE, HD)
    g = torch.Generator(device="cuda").manual_seed(6)
    x0 = torch.randn((60, D), generator=g, device="cuda").to(torch.bfloat16)
    xs = torch.randn((20, B, D), generator=g, device="cuda").to(torch.bfloat16)
    torch.manual_seed(1)
    results = []
    for graph in (False, True):
        torch.manual_seed(2)
        torch.cuda.manual_seed(2)
        batch = Batch(4)
        ws = wq.decoder_paged_workspace(B, 60, layer)
        cu, lens, pos, slots = batch.plan([0] * B, [10, 30, 5, 15], 60)
        wq.decoder_paged_forward(x0, cu, lens, pos, slots, layer, batch.pool, batch.tables, table, max_q=30, ws=ws)
        new, x, y = i32(*[1] * B), torch.empty((B, D), dtype=torch.bfloat16, device="cuda"), torch.empty((B, D), dtype=torch.bfloat16, device="cuda")
        out = [torch.empty(s, dtype=torch.int32, device="cuda") for s in (B + 1, B, B)]

        def step():
            cu, lens, pos, slots = wq.page_plan(batch.lens, new, batch.tables, batch.free, batch.n_free, PAGE, B, cu=out[0],
                                                kv_lens=batch.lens, positions=out[1], slots=out[2])
            wq.decoder_paged_forward(x, cu, lens, pos, slots, layer, batch.pool, batch.tables, table, max_q=1, y=y, ws=ws)

        x.copy_(xs[0])
        step()
        ys = [y.clone()]
        if graph:
            cg = torch.cuda.CUDAGraph()
            with torch.cuda.graph(cg):
                step()
        for i in range(1, 20):
            x.copy_(xs[i])
            if graph:
                cg.replay()
            else:
                step()
            ys.append(y.clone())
        results.append(torch.stack(ys))
        assert batch.lens.tolist() == [30, 50, 25, 35] and status() == 0
    assert torch.equal(*results)


def test_a_request_that_is_not_served_leaves_the_others():
    layer, table = _layer(wq, 14), wq.rope_table(P * PAGE, HD)
    batch = Batch(8, n_pages=3)
    x = torch.randn((60, D), device="cuda").to(torch.bfloat16)
    cu, lens, pos, slots = batch.plan([0] * B, [20, 30, 0, 10], 60)  # 2 pages, then 2 of the one left, then 1 behind it
    assert lens.tolist() == [20, -1, 0, -1] and slots[20:].tolist() == [-1] * 40 and batch.n_free.item() == 1
    y = wq.decoder_paged_forward(x, cu, lens, pos, slots, layer, batch.pool, batch.tables, table, max_q=30)
    alone = Batch(8, n_pages=3)
    alone.free.copy_(batch.free)
    c2, l2, p2, s2 = alone.plan([0] * B, [20, 0, 0, 0], 60)
    y2 = wq.decoder_paged_forward(x, c2, l2, p2, s2, layer, alone.pool, alone.tables, table, max_q=20)
    assert _rel(y[:20], y2[:20]) < 1e-2 and status() == 0


def test_layer_refusals():
    layer, table = _layer(wq, 15), wq.rope_table(P * PAGE, HD)
    batch = Batch(8)
    x = torch.zeros((4, D), dtype=torch.bfloat16, device="cuda")
    cu, lens, pos, slots = batch.plan([0] * B, [1] * B, 4)
    call = lambda **kw: wq.decoder_paged_forward(x, cu, lens, pos, slots, layer, kw.pop("pool", batch.pool), batch.tables, table, **kw)  # noqa: E731
    for kw, st in ((dict(pool=wq.kv_pool(4, KV + 1, PAGE, HD, 8)), -2), (dict(max_q=5), -1), (dict(max_q=0), -1),
                   (dict(ws=wq.decoder_paged_workspace(B, 4, layer)[:-256]), -7), (dict(pool=wq.kv_pool(4, KV, 24, HD, 8)), -4)):
        with pytest.raises(wq.WQError) as e:
            call(**kw)
        assert e.value.status == st
    with pytest.raises(AssertionError):
        wq.decoder_paged_forward(x.float(), cu, lens, pos, slots, layer, batch.pool, batch.tables, table)
