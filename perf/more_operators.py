"""The operators of serving from a paged, quantized KV cache, as a serving program calls
them, over the range of sizes it meets.

A case is one of
  plan   the pages, slots, positions and row offsets of one step of a continuous batch from its
         request lengths: one token a request, prompts that take the place of finished requests,
         drafts that were rejected;
  write  query, key and value projections normed a head, rotated, the queries returned and the
         K and V rows quantized to the slots of their tokens, then read back;
  read   K and V rows at a list of slots as bf16 or fp32;
  attn   causal attention of a ragged batch over its pages: one token a request, chunks of
         prompts, both together, whole prompts.
A pool of pages is [pages, kv heads, positions of a page, head], bf16 or packed codes of 8 or 4
bits with a scale and a zero point a row.  Head layouts are those of the package's
configurations (32/8 heads of 128, 40/8 of 128, 64/8 of 64, 16/4 of 64).  Where `own` is false,
the operators are computed in elementary torch operations in 32 bits.
"""
import math
from functools import reduce

import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 1e6


def listed():
    return [
        # one decode step of 32 requests: the smallest plan, all latency
        dict(name="plan_step_b32", kind="plan", b=32, page=16, ctx=4096, prompts=0, prompt=0, drafts=0),
        # 256 requests of which 20 have ended and are replaced by prompts, the others verify up to 5 drafts
        dict(name="plan_mixed_b256", kind="plan", b=256, page=32, ctx=8192, prompts=20, prompt=700, drafts=5),
        # the projections of one decode step of 16 requests, 4B-class heads, 8-bit pool
        dict(name="write_step_m16", kind="write", m=16, heads=32, kv=8, hd=128, d=2560, bits=8, page=16, weights=True, f32=True),
        # 777 tokens of several prompts, heads of 64, a bf16 pool
        dict(name="write_bf16_m777", kind="write", m=777, heads=64, kv=8, hd=64, d=2880, bits=16, page=64, weights=True, f32=True),
        # a chunk of a long prompt to 4 bits, 14B-class heads, bf16 projections
        dict(name="write_chunk_m4093", kind="write", m=4093, heads=40, kv=8, hd=128, d=0, bits=4, page=32, weights=True, f32=False),
        # a short shared prefix handed on in fp32
        dict(name="read_m300", kind="read", m=300, kv=8, hd=128, bits=8, page=16, f32=True),
        # a long one in bf16 from 4 bits
        dict(name="read_m20000", kind="read", m=20000, kv=8, hd=128, bits=4, page=64, f32=False),
        # one token of one request over a short context: all latency
        dict(name="attn_b1", kind="attn", b=1, t=1, chunks=0, chunk=0, heads=32, kv=8, hd=128, bits=8, page=16, ctx=500),
        # a decode step of 64 requests of 4k to 8k positions in 4 bits: the cache's bytes
        dict(name="attn_step_b64", kind="attn", b=64, t=1, chunks=0, chunk=0, heads=32, kv=8, hd=128, bits=4, page=64, ctx=8191),
        # 14 requests decode while two prompts are taken in by chunks of 250, 8 bits, 4B-class heads
        dict(name="attn_mixed_b16", kind="attn", b=14, t=1, chunks=2, chunk=250, heads=32, kv=8, hd=128, bits=8, page=32, ctx=3000),
        # a whole prompt of 4000 tokens over a bf16 pool, 64 query heads of 64
        dict(name="attn_prompt_4000", kind="attn", b=0, t=0, chunks=1, chunk=4000, heads=64, kv=8, hd=64, bits=16, page=16, ctx=4000),
        # 2000 tokens of a long prompt over 14,000 positions in 4 bits, 14B-class heads: the largest call
        dict(name="attn_chunk_2000", kind="attn", b=0, t=0, chunks=1, chunk=2000, heads=40, kv=8, hd=128, bits=4, page=64, ctx=14000),
    ]


HEADS = [(32, 8, 128), (32, 8, 128), (40, 8, 128), (64, 8, 64), (16, 4, 64)]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = work(listed()[-1])
    while True:
        kind = rng.choice(["plan", "write", "write", "read", "attn", "attn", "attn", "attn"])
        h, kv, hd = rng.choice(HEADS)
        bits, page = rng.choice([16, 8, 8, 4, 4]), rng.choice([16, 32, 64, 128, 256])
        if kind == "plan":
            b = _log_int(rng, 1, 1000)
            c = dict(kind=kind, b=b, page=page, ctx=_log_int(rng, 100, 32768), prompts=rng.randint(0, b),
                     prompt=_log_int(rng, 1, 4000), drafts=rng.choice([0, 0, _log_int(rng, 1, 16)]))
            if b * c["drafts"] + c["prompts"] * c["prompt"] + b > 65536 or b * c["ctx"] > 2 ** 23:
                continue
        elif kind == "write":
            f32 = rng.random() < 0.6
            c = dict(kind=kind, m=_log_int(rng, 1, 8192), heads=h, kv=kv, hd=hd, bits=bits, page=page, f32=f32,
                     d=rng.choice([0, 2560, 4096, 5120, 2880]) if bits != 4 else 0, weights=rng.random() < 0.7)
        elif kind == "read":
            c = dict(kind=kind, m=_log_int(rng, 1, 32768), kv=kv, hd=hd, bits=bits, page=page, f32=rng.random() < 0.4)
        else:
            chunks = rng.choice([0, 0, 1, 1, 2, 4])
            b = _log_int(rng, 1, 128) if chunks == 0 else rng.choice([0, _log_int(rng, 1, 32)])
            chunk = _log_int(rng, 2, 4096) if chunks else 0
            c = dict(kind=kind, b=b, t=rng.choice([1, 1, _log_int(rng, 1, 16)]) if b else 0, chunks=chunks, chunk=chunk, heads=h,
                     kv=kv, hd=hd, bits=bits, page=page, ctx=max(chunk, 16) + rng.choice([0, _log_int(rng, 16, 32768)]))
            if (b + chunks) * h * max(c["t"], chunk) * c["ctx"] > 1.2e9 or (b + chunks) * c["ctx"] > 1 << 19:  # the plain form's scores
                continue
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= 4.0e8:
            return c


# ---- inputs -----------------------------------------------------------------

class _Rand:
    """Draws of one case: every tensor has a generator of its own, seeded from the case's seed."""

    def __init__(self, seed):
        self.seed = int(seed)

    def gen(self, key):
        g = torch.Generator(device=DEV)
        g.manual_seed((self.seed * 1_000_003 + key) % (1 << 62))
        return g

    def normal(self, shape, key):
        return torch.randn(shape, generator=self.gen(key), device=DEV, dtype=torch.float32)

    def ints(self, lo, hi, shape, key):
        """int32 values of [lo, hi)."""
        return torch.randint(lo, hi, shape, generator=self.gen(key), device=DEV, dtype=torch.int32)

    def order(self, n, key):
        """A permutation of 0 .. n - 1."""
        return torch.randperm(n, generator=self.gen(key), device=DEV)


def _plan_inputs(c, rnd):
    """A batch in flight: what each request holds, keeps and adds, its table, the stack of free pages."""
    b, page = c["b"], c["page"]
    lens = rnd.ints(max(1, c["ctx"] // 4), c["ctx"] + 1, (b,), 1)
    n_new = torch.ones(b, dtype=torch.int32, device=DEV)
    keep = lens.clone()
    if c["drafts"]:  # some of the last step's drafts were rejected; as many are drafted again
        keep = lens - torch.minimum(rnd.ints(0, c["drafts"] + 1, (b,), 2), lens)
        n_new = rnd.ints(1, c["drafts"] + 2, (b,), 3)
    ended = rnd.order(b, 4)[:c["prompts"]]  # replaced by prompts
    keep[ended] = 0
    n_new[ended] = rnd.ints((c["prompt"] + 1) // 2, c["prompt"] + 1, (c["prompts"],), 5)
    most = c["b"] + c["b"] * c["drafts"] + c["prompts"] * c["prompt"]  # rows of the batch's buffers
    max_pages = -(-(c["ctx"] + c["drafts"] + c["prompt"] + 1) // page)
    n_pages = -(-c["ctx"] // page) * b + b + -(-most // page)
    have = -(-lens.long() // page)
    ids = rnd.order(n_pages, 6).to(torch.int32)
    first = torch.cumsum(have, 0) - have
    at = torch.arange(max_pages, device=DEV)
    tables = torch.where(at < have[:, None], ids[(first[:, None] + at).clamp(max=n_pages - 1)], torch.full_like(ids[:1], -1))
    held = have.sum()
    stack = torch.where(torch.arange(n_pages, device=DEV) < n_pages - held,
                        ids[(torch.arange(n_pages, device=DEV) + held).clamp(max=n_pages - 1)], torch.full_like(ids[:1], -1))
    return dict(lens=lens, keep=keep, n_new=n_new, tables=tables.contiguous(), free=stack, m=most,
                n_free=(n_pages - held).to(torch.int32).view(1), n_free_out=torch.zeros(1, dtype=torch.int32, device=DEV))


def _rows(rnd, shape, key):
    """K or V rows: head-normed values, a few channels of each head larger as in trained models."""
    v = rnd.normal(shape, key)
    loud = torch.rand(shape[-1], generator=rnd.gen(key + 1), device=DEV) < 0.05
    return (v * torch.where(loud, 4.0, 1.0)).to(torch.bfloat16)


def _counts(c, rnd):
    """int32 [sequences]: query tokens of each, in an order of the seed's."""
    n = [c["t"]] * c["b"] + [c["chunk"]] * c["chunks"]
    return torch.tensor(n, dtype=torch.int32, device=DEV)[rnd.order(len(n), 7)]


def _attn_inputs(c, rnd):
    """Queries, row offsets, lengths, tables and the pages' rows of one step."""
    nq, page = _counts(c, rnd), c["page"]
    seqs, hd, kv = nq.numel(), c["hd"], c["kv"]
    low = max(max(c["t"], c["chunk"]), c["ctx"] // 2)
    lens = rnd.ints(low, c["ctx"] + 1, (seqs,), 8) if seqs > 1 else torch.full((1,), c["ctx"], dtype=torch.int32, device=DEV)
    max_pages = -(-c["ctx"] // page)
    n_pages = seqs * max_pages
    cu = torch.zeros(seqs + 1, dtype=torch.int32, device=DEV)
    cu[1:] = torch.cumsum(nq, 0)
    m = c["b"] * c["t"] + c["chunks"] * c["chunk"]
    return dict(q=rnd.normal((m, c["heads"], hd), 9).to(torch.bfloat16), cu=cu, lens=lens,
                tables=rnd.order(n_pages, 10).view(seqs, max_pages).to(torch.int32),
                k=_rows(rnd, (n_pages, kv, page, hd), 20), v=_rows(rnd, (n_pages, kv, page, hd), 30), max_q=max(c["t"], c["chunk"]))


def _write_inputs(c, rnd):
    m, h, kv, hd, page = c["m"], c["heads"], c["kv"], c["hd"], c["page"]
    n_pages = -(-m // page) + 3
    ang = torch.arange(8192, device=DEV, dtype=torch.float64)[:, None] * \
        THETA ** (-2.0 * torch.arange(hd // 2, device=DEV, dtype=torch.float64) / hd)
    weight = lambda key: (1.0 + 0.3 * rnd.normal((hd,), key)).to(torch.bfloat16) if c["weights"] else None  # noqa: E731
    qkv = rnd.normal((m, (h + 2 * kv) * hd), 40) * 1.3
    return dict(qkv=qkv if c["f32"] else qkv.to(torch.bfloat16), pos=rnd.ints(0, 8192, (m,), 41),
                x=(rnd.normal((m, c["d"]), 42) * 0.7).to(torch.bfloat16) if c["d"] else None, qw=weight(43), kw=weight(44),
                table=torch.stack([torch.cos(ang), torch.sin(ang)], -1).to(torch.float32), slots=_slots(c, rnd, n_pages), n_pages=n_pages)


def _slots(c, rnd, n_pages):
    """Whole pages in an order of the seed's, one position after another, as a slot map gives them."""
    at = torch.arange(c["m"], device=DEV) + 5
    return (rnd.order(n_pages, 45)[at // c["page"]] * c["page"] + at % c["page"]).to(torch.int32)


def _inputs(c, seed):
    """The tensors of one case, the same for every implementation."""
    rnd = _Rand(seed)
    if c["kind"] == "plan":
        return _plan_inputs(c, rnd)
    if c["kind"] == "attn":
        return _attn_inputs(c, rnd)
    if c["kind"] == "write":
        return _write_inputs(c, rnd)
    n_pages = -(-c["m"] // c["page"]) + 3
    shape = (n_pages, c["kv"], c["page"], c["hd"])
    return dict(k=_rows(rnd, shape, 20), v=_rows(rnd, shape, 30), slots=_slots(c, rnd, n_pages))


def prepare(case, seed):
    c = case
    s = dict(c=c, **_inputs(c, seed))
    if own:
        from paper_2606_04238_gb300 import wq
        s["wq"] = wq
    if c["kind"] == "plan":
        return s
    if c["kind"] == "write":
        zero = torch.zeros((s["n_pages"], c["kv"], c["page"], c["hd"]), dtype=torch.bfloat16, device=DEV)
        s["pool"] = [_pack(zero, c["bits"]) for _ in "kv"]
    else:
        s["pool"] = [_pack(s.pop(n), c["bits"]) for n in "kv"]
    if own:
        (k, km), (v, vm) = s["pool"]
        s["pool"] = wq.KVCache(k, v, km, vm, c["hd"], c["bits"]) if c["kind"] != "write" else \
            wq.kv_pool(s["n_pages"], c["kv"], c["page"], c["hd"], c["bits"])
        if c["kind"] == "attn":
            s.update(ws=wq.attn_paged_workspace(s["lens"].numel(), s["q"].shape[0], c["heads"], c["kv"], c["hd"]),
                     o=torch.empty_like(s["q"]))
    return s


# ---- how rows are held ----------------------------------------------------------

def _quantize(rows, bits):
    """(codes, scale, zero) of rows [..., hd]: min-max round-to-nearest around zero, every step in 32 bits."""
    r = rows.to(torch.float32)
    qmax = float(2 ** bits - 1)
    lo, hi = r.amin(-1, keepdim=True).clamp(max=0.0), r.amax(-1, keepdim=True).clamp(min=0.0)
    s = ((hi - lo) / qmax).to(torch.float16)
    s = torch.where(s == 0, torch.ones_like(s), s)
    sf = s.to(torch.float32)
    z = torch.round(-lo / sf).clamp(0.0, qmax)
    return (torch.round(r / sf) + z).clamp(0.0, qmax), s, z.to(torch.float16)


def _pack(rows, bits):
    """Rows as a pool holds them: (bf16, None), or (uint8 codes, int32 of scale and zero); 4 bits: value e of
    eight at bits 4 (e / 2) + 16 (e % 2) of a 32-bit word."""
    if bits == 16:
        return rows.to(torch.bfloat16), None
    q, s, z = _quantize(rows, bits)
    meta = (s.view(torch.int16).to(torch.int32) & 0xffff) | (z.view(torch.int16).to(torch.int32) << 16)
    if bits == 8:
        return q.to(torch.uint8).contiguous(), meta.squeeze(-1).contiguous()
    q = q.to(torch.uint8).unflatten(-1, (-1, 2, 2, 2))  # [word, half of the word's eight, pair, even or odd]
    q = (q[..., 0, :] | (q[..., 1, :] << 4)).transpose(-1, -2)  # bytes: even low, even high, odd low, odd high
    return q.flatten(-3).contiguous(), meta.squeeze(-1).contiguous()


def _unpack(held, meta, bits):
    """The fp32 values of held rows."""
    if bits == 16:
        return held.to(torch.float32)
    if bits == 4:
        q = held.unflatten(-1, (-1, 2, 2)).transpose(-1, -2)  # [word, half, even or odd]
        q = torch.stack([q & 15, q >> 4], -2).flatten(-4)
    else:
        q = held
    s = meta.to(torch.int16).view(torch.float16).to(torch.float32)
    z = (meta >> 16).to(torch.int16).view(torch.float16).to(torch.float32)
    return s[..., None] * (q.to(torch.float32) - z[..., None])


# ---- the operators in plain form ----------------------------------------------

def _plain_plan(s):
    c, m = s["c"], s["m"]
    page, b, max_pages = c["page"], c["b"], s["tables"].shape[1]
    lens, keep, new = s["lens"].long(), s["keep"].long(), s["n_new"].long()
    have, need = (lens + page - 1) // page, (keep + new + page - 1) // page
    end = torch.cumsum(new, 0)
    ok = (keep <= lens) & (keep + new <= max_pages * page) & (end <= m)
    want, back = torch.where(ok, need - have, 0).clamp(min=0), torch.where(ok, have - need, 0).clamp(min=0)
    taken, given = torch.cumsum(want, 0), torch.cumsum(back, 0)
    n_free, given_all = s["n_free"].long(), given[-1]
    served = ok & ((want == 0) | (taken <= n_free + given_all))
    taken_all = torch.where(served, want, 0).sum()
    at = torch.arange(max_pages, device=DEV)
    tables, stack = s["tables"], s["free"]
    # pages given back, in order, behind the stack; a place behind the end for what is not
    out = (at >= need[:, None]) & (at < have[:, None]) & (back > 0)[:, None]
    n_pages = stack.numel()
    place = torch.where(out, n_free + (given - back)[:, None] + at - need[:, None], n_pages)
    full = torch.cat([stack, stack[:1]]).scatter(0, place.clamp(max=n_pages).flatten(), tables.flatten())[:-1]
    # pages taken, from the top
    into = (at >= have[:, None]) & (at < need[:, None]) & served[:, None]
    top = n_free + given_all - 1 - ((taken - want)[:, None] + at - have[:, None])
    now = torch.where(into, full[top.clamp(0, n_pages - 1)], tables)
    left = n_free + given_all - taken_all
    slot_of = torch.arange(n_pages, device=DEV)
    stack = torch.where((slot_of >= n_free) & (slot_of < left), full, stack)
    row = torch.arange(m, device=DEV)
    req = torch.searchsorted(end, row, right=True).clamp(max=b - 1)
    there = (row < end[-1]) & served[req]
    pos = torch.where(there, keep[req] + row - (end - new)[req], 0)
    slot = torch.where(there, now[req, pos // page].long() * page + pos % page, -1)
    cu = torch.zeros(b + 1, dtype=torch.int32, device=DEV)
    cu[1:] = end.clamp(max=m)
    i32 = torch.int32
    return [cu, torch.where(served, keep + new, -1).to(i32), pos.to(i32), slot.to(i32), now, stack, left.to(i32).view(1)]


def _sum_squares(u):
    """Sums over the last dimension, pairwise: halves, then eighths of neighbours, then the rest, so that the codes of
    values beside a border do not hang on the order of a sum."""
    fold = lambda v, n: v[..., :n] + v[..., n:]  # noqa: E731
    v = (u * u).unflatten(-1, (2, -1, 8))
    v = reduce(fold, (4, 2, 1), v[..., 0, :, :] + v[..., 1, :, :]).squeeze(-1)
    return reduce(fold, (4, 2, 1)[u.shape[-1] == 64:], v)


def _plain_write(s):
    c = s["c"]
    m, h, kv, hd, bits, page = c["m"], c["heads"], c["kv"], c["hd"], c["bits"], c["page"]
    u = s["qkv"].to(torch.float32)
    if c["d"]:
        x = s["x"].to(torch.float32)
        u = u * (1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS))
    q, k, v = u.view(m, h + 2 * kv, hd).split([h, kv, kv], 1)
    cs = s["table"][s["pos"].long()][:, None]

    def turned(t, weight):
        t = t * (1.0 / torch.sqrt(_sum_squares(t) / hd + EPS))
        if weight is not None:
            t = t * weight.to(torch.float32)
        lo, hi = t[..., :hd // 2], t[..., hd // 2:]
        return torch.cat([lo * cs[..., 0] - hi * cs[..., 1], hi * cs[..., 0] + lo * cs[..., 1]], -1)

    at = s["slots"].long()
    out = [turned(q, s["qw"]).to(torch.bfloat16)]
    for rows, (held, meta) in zip((turned(k, s["kw"]), v), s["pool"]):
        new, new_meta = _pack(rows, bits)
        held[at // page, :, at % page] = new
        if meta is not None:
            meta[at // page, :, at % page] = new_meta
        got = None if meta is None else meta[at // page, :, at % page]
        out.append(_unpack(held[at // page, :, at % page], got, bits).to(torch.bfloat16))
    return out


def _plain_read(s):
    c, at = s["c"], s["slots"].long()
    page, dt = c["page"], torch.float32 if c["f32"] else torch.bfloat16
    return [_unpack(held[at // page, :, at % page], None if meta is None else meta[at // page, :, at % page], c["bits"]).to(dt)
            for held, meta in s["pool"]]


def _plain_attn(s):
    c = s["c"]
    h, kv, hd, page = c["heads"], c["kv"], c["hd"], c["page"]
    rep, seqs, m = h // kv, s["lens"].numel(), s["q"].shape[0]
    cu, lens, most, ctx = s["cu"].long(), s["lens"].long(), s["max_q"], s["tables"].shape[1] * page
    nq = cu[1:] - cu[:-1]
    ids = s["tables"].long()
    k, v = (_unpack(held[ids], None if meta is None else meta[ids], c["bits"]).transpose(1, 2).reshape(seqs, kv, ctx, hd)
            for held, meta in s["pool"])
    i = torch.arange(most, device=DEV)
    row = (cu[:-1, None] + i).clamp(max=m - 1)  # [sequences, most], padded
    q = s["q"][row].to(torch.float32).view(seqs, most, kv, rep, hd).permute(0, 2, 1, 3, 4).reshape(seqs, kv, most * rep, hd)
    x = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(hd)).view(seqs, kv, most, rep, ctx)
    seen = (lens - nq)[:, None] + i + 1  # positions a query sees
    x.masked_fill_((torch.arange(ctx, device=DEV) >= seen[..., None])[:, None, :, None], -math.inf)
    p = x.sub_(x.amax(-1, keepdim=True)).exp_()
    p = p.div_(p.sum(-1, keepdim=True)).view(seqs, kv, most * rep, ctx)
    o = (p @ v).view(seqs, kv, most, rep, hd).permute(0, 2, 1, 3, 4).reshape(seqs, most, h, hd)
    return o[i < nq[:, None]].to(torch.bfloat16)


def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        wq = s["wq"]
        if kind == "plan":
            got = wq.page_plan(s["lens"], s["n_new"], s["tables"], s["free"], s["n_free"], c["page"], s["m"], keep=s["keep"],
                               n_free_out=s["n_free_out"])
            return [*got, s["tables"], s["free"], s["n_free_out"]]
        if kind == "write":
            q = wq.qkv_paged(s["qkv"], s["slots"], s["pool"], c["heads"], positions=s["pos"], table=s["table"], x=s["x"],
                             q_norm=s["qw"], k_norm=s["kw"])
            return [q, *wq.paged_read(s["pool"], s["slots"])]
        if kind == "read":
            return list(wq.paged_read(s["pool"], s["slots"], dtype=torch.float32 if c["f32"] else torch.bfloat16))
        return wq.attn_paged(s["q"], s["cu"], s["lens"], s["tables"], s["pool"], max_q=s["max_q"], o=s["o"], ws=s["ws"])
    return {"plan": _plain_plan, "write": _plain_write, "read": _plain_read, "attn": _plain_attn}[kind](s)


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    c, kind = case, case["kind"]
    if kind == "plan":
        rows = c["b"] * (1 + c["drafts"] / 2) + 0.75 * c["prompts"] * c["prompt"]
        moved = rows / c["page"] + 0.6 * c["prompts"] * c["ctx"] / c["page"]  # pages taken and given back
        return {"bytes": 20.0 * c["b"] + 8.0 * rows + 8.0 * moved, "flops": 4.0 * rows}
    kv, hd, bits = c["kv"], c["hd"], c["bits"]
    held = hd * bits / 8.0 + (0 if bits == 16 else 4)  # bytes of one row of one head
    if kind == "read":
        return {"bytes": c["m"] * (4.0 + 2 * kv * (held + hd * (4 if c["f32"] else 2))), "flops": 2.0 * c["m"] * 2 * kv * hd}
    if kind == "write":
        n = (c["heads"] + 2 * kv) * hd
        out = 2 * c["heads"] * hd + 2 * kv * (held + 2 * hd)  # queries, cached rows and what is read back
        return {"bytes": c["m"] * (n * (4.0 if c["f32"] else 2.0) + 2 * c["d"] + 4 * hd + 8 + out), "flops": 12.0 * c["m"] * n}
    seqs = c["b"] + c["chunks"]
    mean = c["ctx"] if seqs == 1 else (max(max(c["t"], c["chunk"]), c["ctx"] // 2) + c["ctx"]) / 2.0
    m = c["b"] * c["t"] + c["chunks"] * c["chunk"]
    seen = c["b"] * c["t"] * (mean - (c["t"] - 1) / 2.0) + c["chunks"] * c["chunk"] * (mean - (c["chunk"] - 1) / 2.0)
    return {"bytes": seqs * mean * 2.0 * kv * held + 4.0 * m * c["heads"] * hd, "flops": 4.0 * c["heads"] * hd * seen}


# ---- the same in 64 bits ------------------------------------------------------

def _value64(rows, bits):
    """fp64 values of rows [..., hd] after they are held: the quantizer's steps are defined in fp32, so each quotient is
    rounded to fp32 (once: a double quotient of two fp32 numbers rounds to fp32 as the fp32 quotient does)."""
    if bits == 16:
        return rows.bfloat16().double()
    r = rows.float().double()
    top = 2 ** bits - 1
    zero = r.new_zeros(())
    lo, hi = torch.minimum(r.min(-1, keepdim=True)[0], zero), torch.maximum(r.max(-1, keepdim=True)[0], zero)
    scale = ((hi - lo).float().double() / top).float().half().double()
    scale = scale + (scale == 0)
    zero_at = torch.clamp((-lo / scale).float().round().double(), 0, top)
    return (torch.clamp((r / scale).float().round().double() + zero_at, 0, top) - zero_at) * scale


def exact(case, seed):
    c = case
    if c["kind"] == "plan":
        return None
    i, hd, kv, bits = _inputs(c, seed), c["hd"], c["kv"], c["bits"]
    if c["kind"] == "read":
        at = i["slots"].long()
        return [_value64(i[n][at // c["page"], :, at % c["page"]], bits) for n in "kv"]
    h = c["heads"]
    if c["kind"] == "write":
        m = c["m"]
        u = i["qkv"].double().view(m, h + 2 * kv, hd)
        if c["d"]:
            u = u * (i["x"].double().pow(2).mean(1) + EPS).pow(-0.5)[:, None, None]
        turn = torch.view_as_complex(i["table"].double())[i["pos"].long()][:, None]
        n = u[:, :h + kv]
        n = n * (n.pow(2).mean(-1, keepdim=True) + EPS).pow(-0.5)
        if c["weights"]:
            n = torch.cat([n[:, :h] * i["qw"].double(), n[:, h:] * i["kw"].double()], 1)
        n = torch.complex(n[..., :hd // 2].contiguous(), n[..., hd // 2:].contiguous()) * turn
        n = torch.cat([n.real, n.imag], -1)
        return [n[:, :h], _value64(n[:, h:], bits), _value64(u[:, h + kv:], bits)]
    o = torch.zeros((i["q"].shape[0], h, hd), dtype=torch.float64, device=DEV)
    cu, lens = i["cu"].tolist(), i["lens"].tolist()
    for b, n in enumerate(lens):
        t = cu[b + 1] - cu[b]
        pages = i["tables"][b].long()
        sees = torch.arange(n, device=DEV)[None] <= torch.arange(n - t, n, device=DEV)[:, None]
        for g in range(kv):
            keys, vals = (_value64(i[name][pages, g].flatten(0, 1)[:n], bits) for name in "kv")
            for a in range(g * (h // kv), (g + 1) * (h // kv)):
                w = i["q"][cu[b]:cu[b + 1], a].double() @ keys.t() * hd ** -0.5
                o[cu[b]:cu[b + 1], a] = torch.softmax(w.masked_fill_(~sees, -math.inf), -1) @ vals
    return o
