"""The operators of a speculative-decoding step over a quantized KV cache, as a
serving program calls them, over the range of sizes it meets.

A case is one of
  append   new K and V rows quantized into the cache as they are written (8 or 4
           bits, one binary16 scale and whole zero point a row and head, or
           bf16) and read back as the values they stand for: one token a
           sequence, a prompt, or the accepted path of a drafted tree gathered
           by index;
  read     a range of cached positions as bf16 or fp32 rows;
  rope     head norm and rotary positions of the query, key and value
           projections of drafted tokens, each at its own depth;
  tree     attention of a tree of drafted tokens (one token: a decode step) over
           a cache of 16, 8 or 4 bits and the drafts themselves.
Head layouts are those of the package's configurations (32/8 heads of 128, 40/8
of 128, 64/8 of 64, 16/4 of 64).  Where `own` is false, the operators are
computed in elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 1e6


def listed():
    return [
        # one new token of 16 sequences written to an 8-bit cache: the smallest call of a decode step
        dict(name="append_step_b16", kind="append", b=16, t=1, kv=8, hd=128, bits=8, ctx=2048, gather=0, f32=False),
        # the accepted paths (up to 7 of 61 drafts) of 24 sequences, heads of 64
        dict(name="append_accept_b24", kind="append", b=24, t=61, kv=8, hd=64, bits=8, ctx=1024, gather=7, f32=False),
        # a whole prompt of a ragged length written to a 4-bit cache
        dict(name="append_prompt_8191", kind="append", b=1, t=8191, kv=8, hd=128, bits=4, ctx=16384, gather=0, f32=False),
        # eight sequences of different lengths read back from 8 bits (a cache handed to another engine)
        dict(name="read_b8", kind="read", b=8, n=1500, kv=8, hd=128, bits=8, ctx=2048, f32=False),
        # a long context read back from 4 bits in fp32
        dict(name="read_32k", kind="read", b=1, n=32768, kv=8, hd=128, bits=4, ctx=32768, f32=True),
        # five drafted tokens of two sequences, 4B-class heads
        dict(name="rope_m10", kind="rope", m=10, heads=32, kv=8, hd=128, d=2560, ctx=8192),
        # 61 drafted tokens of 20 sequences, 14B-class heads
        dict(name="rope_m1220", kind="rope", m=1220, heads=40, kv=8, hd=128, d=5120, ctx=32768),
        # one token of one sequence, a short context: all latency
        dict(name="tree_b1_t1", kind="tree", b=1, t=1, heads=32, kv=8, hd=128, bits=8, ctx=500, mask="tree"),
        # 16 sequences of 512 to 2048 positions, trees of up to 8 drafts, 8-bit cache
        dict(name="tree_b16_t8", kind="tree", b=16, t=8, heads=32, kv=8, hd=128, bits=8, ctx=2048, mask="tree"),
        # one sequence of 32k positions in 4 bits, 4 drafts
        dict(name="tree_32k_t4", kind="tree", b=1, t=4, heads=32, kv=8, hd=128, bits=4, ctx=32767, mask="tree"),
        # trees of up to 61 drafts over a bf16 cache, 64 query heads of 64
        dict(name="tree_b8_t61", kind="tree", b=8, t=61, heads=64, kv=8, hd=64, bits=16, ctx=4001, mask="tree"),
        # trees of up to 64 drafts over long contexts in 4 bits, 14B-class heads: the largest call
        dict(name="tree_b4_t64", kind="tree", b=4, t=64, heads=40, kv=8, hd=128, bits=4, ctx=16384, mask="tree"),
    ]


HEADS = [(32, 8, 128), (32, 8, 128), (40, 8, 128), (64, 8, 64), (16, 4, 64)]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = work(listed()[-1])
    while True:
        kind = rng.choice(["append", "append", "read", "rope", "tree", "tree", "tree", "tree"])
        h, kv, hd = rng.choice(HEADS)
        bits = rng.choice([16, 8, 8, 4, 4])
        b = _log_int(rng, 1, 32)
        if kind == "append":
            gather = rng.choice([0, 0, _log_int(rng, 1, 9)])
            t = _log_int(rng, max(1, gather), 128) if gather else _log_int(rng, 1, 8192)
            c = dict(kind=kind, b=b, t=t, kv=kv, hd=hd, bits=bits, ctx=t + _log_int(rng, 16, 4096), gather=gather,
                     f32=rng.random() < 0.3)
        elif kind == "read":
            n = _log_int(rng, 1, 32768)
            c = dict(kind=kind, b=b, n=n, kv=kv, hd=hd, bits=bits, ctx=n + rng.randint(0, 500), f32=rng.random() < 0.4)
        elif kind == "rope":
            c = dict(kind=kind, m=_log_int(rng, 1, 2048), heads=h, kv=kv, hd=hd, d=rng.choice([2560, 4096, 5120, 2880]),
                     ctx=_log_int(rng, 256, 32768))
        else:
            c = dict(kind=kind, b=b, t=_log_int(rng, 1, 128), heads=h, kv=kv, hd=hd, bits=bits,
                     ctx=_log_int(rng, 64, 32768), mask=rng.choice(["tree", "tree", "chain"]))
            if c["b"] * c["t"] * h * c["ctx"] > 2 ** 28:  # the plain form's scores
                continue
        if "b" in c and c["b"] * c["ctx"] > 131072:
            continue
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= 3.0e8:
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


def _rows(rnd, shape, key):
    """bf16 K or V rows: head-normed values, a few channels of each head larger as in trained models."""
    v = rnd.normal(shape, key)
    loud = torch.rand(shape[-1], generator=rnd.gen(key + 1), device=DEV) < 0.05
    return (v * torch.where(loud, 4.0, 1.0)).to(torch.bfloat16)


def _lens(rnd, b, ctx, key):
    """A quarter of the context to all of it; one sequence: all of it."""
    if b == 1:
        return torch.full((1,), ctx, dtype=torch.int32, device=DEV)
    return rnd.ints(ctx // 4, ctx + 1, (b,), key)


def _visible(rnd, b, t, mask, key):
    """bool [b, t, t]: draft i sees draft j.  tree: parents drawn among the earlier drafts and the root."""
    if mask == "chain":
        return torch.ones((t, t), dtype=torch.bool, device=DEV).tril().expand(b, t, t).contiguous()
    i = torch.arange(t, device=DEV)
    u = torch.rand((b, t), generator=rnd.gen(key), device=DEV)
    parent = torch.floor(u * (i + 1)).long() - 1  # -1: the context's last token
    vis = torch.zeros((b, t, t + 1), dtype=torch.bool, device=DEV)  # the last column: the root
    rows = torch.arange(b, device=DEV)
    for k in range(t):
        vis[:, k] = vis[rows, parent[:, k]] if k else False
        vis[:, k] &= (parent[:, k] >= 0)[:, None]
        vis[:, k, k] = True
    return vis[:, :, :t].contiguous()


def _words(vis):
    """int32 [b, t, ceil(t / 32)]: bit j % 32 of word j / 32 is column j."""
    b, t, _ = vis.shape
    w = (t + 31) // 32
    pad = torch.zeros((b, t, 32 * w), dtype=torch.int64, device=DEV)
    pad[:, :, :t] = vis
    v = (pad.view(b, t, w, 32) << torch.arange(32, device=DEV)).sum(-1)
    return torch.where(v >= 2 ** 31, v - 2 ** 32, v).to(torch.int32)


def _inputs(c, seed):
    """The tensors of one case, the same for every implementation."""
    rnd, kind = _Rand(seed), c["kind"]
    hd, kv = c["hd"], c["kv"]
    if kind == "rope":
        m, n = c["m"], (c["heads"] + 2 * kv) * hd
        ang = torch.arange(c["ctx"], device=DEV, dtype=torch.float64)[:, None] * \
            THETA ** (-2.0 * torch.arange(hd // 2, device=DEV, dtype=torch.float64) / hd)
        return dict(qkv=rnd.normal((m, n), 1) * 1.3, x=(rnd.normal((m, c["d"]), 2) * 0.7).to(torch.bfloat16),
                    pos=rnd.ints(0, c["ctx"], (m,), 3),
                    table=torch.stack([torch.cos(ang), torch.sin(ang)], -1).to(torch.float32))
    b = c["b"]
    if kind == "append":
        t, n = c["t"], c["gather"] or c["t"]
        i = dict(k=_rows(rnd, (b, t, kv, hd), 10), v=_rows(rnd, (b, t, kv, hd), 20),
                 start=rnd.ints(0, c["ctx"] - n + 1, (b,), 3))
        if c["gather"]:
            i["index"] = torch.argsort(torch.rand((b, t), generator=rnd.gen(4), device=DEV), -1)[:, :n].sort(-1)[0].to(torch.int32)
            i["counts"] = rnd.ints(1, n + 1, (b,), 5)
        return i
    if kind == "read":
        n = c["n"]
        return dict(k=_rows(rnd, (b, c["ctx"], kv, hd), 10), v=_rows(rnd, (b, c["ctx"], kv, hd), 20),
                    start=rnd.ints(0, c["ctx"] - n + 1, (b,), 3))
    t = c["t"]
    return dict(q=rnd.normal((b, t, c["heads"], hd), 1).to(torch.bfloat16), kn=_rows(rnd, (b, t, kv, hd), 30),
                vn=_rows(rnd, (b, t, kv, hd), 40), k=_rows(rnd, (b, c["ctx"], kv, hd), 10),
                v=_rows(rnd, (b, c["ctx"], kv, hd), 20), lens=_lens(rnd, b, c["ctx"], 3),
                counts=torch.full((b,), t, dtype=torch.int32, device=DEV) if b == 1 else rnd.ints((t + 1) // 2, t + 1, (b,), 5),
                vis=_visible(rnd, b, t, c["mask"], 6))


def prepare(case, seed):
    c, i = case, _inputs(case, seed)
    kind, s = c["kind"], dict(c=c)
    if own:
        from paper_2606_04238_gb300 import wq
        s["wq"] = wq
    if kind == "rope":
        s.update(i)
        return s
    b, kv, hd, bits = c["b"], c["kv"], c["hd"], c["bits"]
    if own:
        cache = wq.kv_cache(b, kv, c["ctx"], hd, bits)
        if kind != "append":
            wq.kv_append(cache, i.pop("k"), i.pop("v"), torch.zeros(b, dtype=torch.int32, device=DEV))
        s["cache"] = cache
        if kind == "tree":
            s.update(ws=wq.attn_tree_workspace(b, c["t"], c["heads"], kv, hd, c["ctx"]),
                     o=torch.empty((b, c["t"], c["heads"], hd), dtype=torch.bfloat16, device=DEV))
    elif kind == "append":
        s["cache"] = {n: _store(torch.zeros((b, c["ctx"], kv, hd), dtype=torch.bfloat16, device=DEV), bits) for n in "kv"}
    else:
        s["cache"] = {n: _store(i.pop(n), bits) for n in "kv"}
    if kind == "tree":
        s["mask"] = None if c["mask"] == "chain" else _words(i.pop("vis"))
        i.pop("vis", None)
    s.update(i)
    return s


# ---- the operators in plain form ----------------------------------------------

def _store(rows, bits):
    """Rows [..., hd] as they are cached: bf16, or (codes, scale, zero) of min-max round-to-nearest around zero."""
    if bits == 16:
        return rows.to(torch.bfloat16)
    r = rows.to(torch.float32)
    qmax = float(2 ** bits - 1)
    lo, hi = r.amin(-1, keepdim=True).clamp(max=0.0), r.amax(-1, keepdim=True).clamp(min=0.0)
    s = ((hi - lo) / qmax).to(torch.float16)
    s = torch.where(s == 0, torch.ones_like(s), s)
    sf = s.to(torch.float32)
    z = torch.round(-lo / sf).clamp(0.0, qmax)
    q = (torch.round(r / sf) + z).clamp(0.0, qmax)
    return q.to(torch.uint8), s, z.to(torch.float16)


def _load(held):
    """The fp32 values that cached rows stand for."""
    if torch.is_tensor(held):
        return held.to(torch.float32)
    q, s, z = held
    return s.to(torch.float32) * (q.to(torch.float32) - z.to(torch.float32))


def _put(held, rows, pos, bits):
    """Writes rows [b, n, kv, hd] at positions pos [b, n] (those >= 0) of what is held [b, ctx, kv, hd]."""
    new = _store(rows, bits)
    new, held = ((new,), (held,)) if bits == 16 else (new, held)
    seq = torch.arange(pos.shape[0], device=DEV)[:, None].expand_as(pos)
    at = torch.where(pos < 0, 0, pos)
    for dst, src in zip(held, new):
        keep = (pos < 0).view(*pos.shape, 1, 1)
        dst[seq, at] = torch.where(keep, dst[seq, at], src)


def _pick(held, bits, start, n):
    pos = start.long()[:, None] + torch.arange(n, device=DEV)
    seq = torch.arange(start.shape[0], device=DEV)[:, None]
    return held[seq, pos] if bits == 16 else tuple(t[seq, pos] for t in held)


def _plain_append(s):
    c = s["c"]
    n, dt = c["gather"] or c["t"], torch.float32 if c["f32"] else torch.bfloat16
    step = torch.arange(n, device=DEV)
    pos = s["start"].long()[:, None] + step
    out = []
    for name in "kv":
        rows = s[name]
        if c["gather"]:
            rows = rows[torch.arange(c["b"], device=DEV)[:, None], s["index"].long()]
            inside = step < s["counts"][:, None]
            # a step past the count writes nothing: sent to the last written position's own value
            last = (s["counts"].long() - 1)[:, None]
            take = torch.where(inside, step, last)
            rows = torch.gather(rows, 1, take[:, :, None, None].expand(-1, -1, *rows.shape[2:]))
            _put(s["cache"][name], rows, s["start"].long()[:, None] + take, c["bits"])
            got = _load(_pick(s["cache"][name], c["bits"], s["start"], n))
            got = torch.where(inside[:, :, None, None], got, torch.zeros_like(got))
        else:
            _put(s["cache"][name], rows, pos, c["bits"])
            got = _load(_pick(s["cache"][name], c["bits"], s["start"], n))
        out.append(got.to(dt))
    return out


def _plain_rope(s):
    c = s["c"]
    m, h, kv, hd = c["m"], c["heads"], c["kv"], c["hd"]
    x = s["x"].to(torch.float32)
    qkv = s["qkv"] / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    q, k, v = qkv.view(m, h + 2 * kv, hd).split([h, kv, kv], 1)
    cs = s["table"][s["pos"].long()][:, None]
    out = []
    for u in (q, k):
        u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS)
        lo, hi = u[..., :hd // 2], u[..., hd // 2:]
        out.append(torch.cat([lo * cs[..., 0] - hi * cs[..., 1], hi * cs[..., 0] + lo * cs[..., 1]], -1))
    return [t.to(torch.bfloat16) for t in (*out, v)]


def _plain_tree(s):
    c = s["c"]
    b, t, h, kv, hd = c["b"], c["t"], c["heads"], c["kv"], c["hd"]
    rep = h // kv
    k = torch.cat([_load(s["cache"]["k"]), s["kn"].to(torch.float32)], 1)
    v = torch.cat([_load(s["cache"]["v"]), s["vn"].to(torch.float32)], 1)
    q = s["q"].to(torch.float32).view(b, t, kv, rep, hd).permute(0, 2, 1, 3, 4).reshape(b, kv, t * rep, hd)
    x = q @ k.permute(0, 2, 3, 1) / math.sqrt(hd)  # [b, kv, t rep, ctx + t]
    j = torch.arange(t, device=DEV)
    if s["mask"] is None:
        vis = (j[None] <= j[:, None]).expand(b, t, t)
    else:
        vis = ((s["mask"][:, :, j // 32] >> (j % 32)) & 1).bool()
    there = j < s["counts"][:, None]
    vis = vis & there[:, None, :] & there[:, :, None]
    old = (torch.arange(c["ctx"], device=DEV) < s["lens"][:, None])[:, None].expand(b, t, c["ctx"])
    see = torch.cat([old & there[:, :, None], vis], -1)[:, None, :, None].expand(b, 1, t, rep, c["ctx"] + t)
    see = see.reshape(b, 1, t * rep, c["ctx"] + t)
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    o = p @ v.permute(0, 2, 1, 3) / torch.where(total == 0, torch.ones_like(total), total)
    return o.view(b, kv, t, rep, hd).permute(0, 2, 1, 3, 4).reshape(b, t, h, hd).to(torch.bfloat16)


def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        wq = s["wq"]
        dt = torch.float32 if c.get("f32") else torch.bfloat16
        if kind == "append":
            wq.kv_append(s["cache"], s["k"], s["v"], s["start"], counts=s.get("counts"), index=s.get("index"))
            return list(wq.kv_read(s["cache"], s["start"], c["gather"] or c["t"], counts=s.get("counts"), dtype=dt))
        if kind == "read":
            return list(wq.kv_read(s["cache"], s["start"], c["n"], dtype=dt))
        if kind == "rope":
            return list(wq.qkv_rope(s["qkv"], s["pos"], s["table"], c["heads"], c["kv"], x=s["x"]))
        return wq.attn_tree(s["q"], s["kn"], s["vn"], s["cache"], s["lens"], mask=s["mask"], counts=s["counts"], o=s["o"],
                            ws=s["ws"])
    if kind == "append":
        return _plain_append(s)
    if kind == "read":
        dt = torch.float32 if c["f32"] else torch.bfloat16
        return [_load(_pick(s["cache"][n], c["bits"], s["start"], c["n"])).to(dt) for n in "kv"]
    if kind == "rope":
        return _plain_rope(s)
    return _plain_tree(s)


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    c = case
    hd, kv, kind = c["hd"], c["kv"], c["kind"]
    if kind == "rope":
        n = (c["heads"] + 2 * kv) * hd
        return {"bytes": float(c["m"] * (4 * n + 2 * c["d"] + 2 * n + 8 * (hd // 2) + 4)), "flops": 10.0 * c["m"] * n}
    held = hd * c["bits"] / 8.0 + (0 if c["bits"] == 16 else 4)  # bytes of one cached row of one head
    if kind in ("append", "read"):
        rows = 2.0 * c["b"] * kv * (c["n"] if kind == "read" else c["gather"] or c["t"])
        out = hd * (4 if c["f32"] else 2)
        return {"bytes": rows * (held + out + (0 if kind == "read" else 2 * hd)), "flops": 4.0 * rows * hd}
    mean = c["ctx"] if c["b"] == 1 else 0.625 * c["ctx"]
    t, h = c["t"], c["heads"]
    drafts = t if c["b"] == 1 else 0.75 * t
    return {"bytes": c["b"] * (2.0 * kv * mean * held + drafts * 4.0 * kv * hd + drafts * h * hd * 2 + t * h * hd * 2),
            "flops": 4.0 * c["b"] * drafts * h * hd * (mean + drafts / 2)}


# ---- the same in 64 bits ------------------------------------------------------

def _value64(rows, bits):
    """fp64 values of rows [..., hd] after caching: the quantizer's steps are defined in fp32, so each quotient is
    rounded to fp32 (once: a double quotient of two fp32 numbers rounds to fp32 as the fp32 quotient does)."""
    r = rows.double()
    if bits == 16:
        return r
    top = 2 ** bits - 1
    zero = r.new_zeros(())
    lo, hi = torch.minimum(r.min(-1, keepdim=True)[0], zero), torch.maximum(r.max(-1, keepdim=True)[0], zero)
    scale = ((hi - lo).float().double() / top).float().half().double()
    scale = scale + (scale == 0)
    zero_at = torch.clamp((-lo / scale).float().round().double(), 0, top)
    code = torch.clamp((r / scale).float().round().double() + zero_at, 0, top)
    return (code - zero_at) * scale


def exact(case, seed):
    c, i = case, _inputs(case, seed)
    kind, hd, kv = c["kind"], c["hd"], c["kv"]
    if kind == "rope":
        m, h = c["m"], c["heads"]
        x, pos = i["x"].double(), i["pos"].long()
        u = (i["qkv"].double() * (x.pow(2).mean(1) + EPS).pow(-0.5)[:, None]).view(m, h + 2 * kv, hd)
        turn = torch.view_as_complex(i["table"].double())[pos][:, None]
        n = u[:, :h + kv]
        n = n * (n.pow(2).mean(-1, keepdim=True) + EPS).pow(-0.5)
        n = torch.complex(n[..., :hd // 2].contiguous(), n[..., hd // 2:].contiguous()) * turn
        n = torch.cat([n.real, n.imag], -1)
        return [n[:, :h], n[:, h:], u[:, h + kv:]]
    b, bits = c["b"], c["bits"]
    if kind == "append":
        n, out = c["gather"] or c["t"], []
        for name in "kv":
            r = i[name]
            if c["gather"]:
                r = torch.stack([r[k, i["index"][k].long()] for k in range(b)])
            r = _value64(r, bits)
            for k in range(b if c["gather"] else 0):
                r[k, int(i["counts"][k]):] = 0
            out.append(r)
        return out
    if kind == "read":
        return [torch.stack([_value64(i[name][k, int(i["start"][k]):int(i["start"][k]) + c["n"]], bits)
                             for k in range(b)]) for name in "kv"]
    t, h = c["t"], c["heads"]
    o = torch.zeros((b, t, h, hd), dtype=torch.float64, device=DEV)
    for k in range(b):
        n, m = int(i["lens"][k]), int(i["counts"][k])
        for g in range(kv):
            hs = slice(g * (h // kv), (g + 1) * (h // kv))
            q = i["q"][k, :m, hs].double()
            keys = torch.cat([_value64(i["k"][k, :n, g], bits), i["kn"][k, :m, g].double()])
            vals = torch.cat([_value64(i["v"][k, :n, g], bits), i["vn"][k, :m, g].double()])
            a = torch.einsum("thd,jd->htj", q, keys) * hd ** -0.5
            a[:, :, n:].masked_fill_(~i["vis"][k, :m, :m], -math.inf)
            o[k, :m, hs] = torch.einsum("htj,jd->thd", torch.softmax(a, -1), vals)
    return o
