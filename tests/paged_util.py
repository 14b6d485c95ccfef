"""Plain forms of the operators on pages, in Python and fp64, for their tests."""
import numpy as np
import torch

from paper_2606_04238_gb300 import wq


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def status():
    import ctypes
    s = ctypes.c_int(0)
    assert wq.lib().wq_device_status(ctypes.byref(s)) == 0
    return s.value


def plan_loop(lens, keep, n_new, tables, free, n_free, page, m):
    """wq_page_plan one request after another: (cu, kv_lens, positions, slots, tables, free, n_free, bad)."""
    n_pages, max_pages = len(free), len(tables[0])
    T, F, bad = [list(r) for r in tables], list(free), False
    cu, ok, end = [0], [], 0
    for le, k, n in zip(lens, keep, n_new):
        end += min(max(n, 0), m + 1)
        valid = 0 <= le <= max_pages * page and 0 <= k <= le and n >= 0 and k + n <= max_pages * page and (end <= m or n == 0)
        bad |= not valid
        ok.append(valid)
        cu.append(min(end, m))
    have = [-(-le // page) for le in lens]
    need = [-(-(k + n) // page) for k, n in zip(keep, n_new)]
    stack = F[:n_free]
    for b in range(len(lens)):
        if ok[b]:
            stack += T[b][need[b]:have[b]]
    at, wanted, served = len(stack), 0, []
    pos, slots = [0] * m, [-1] * m
    for b in range(len(lens)):
        want = max(0, need[b] - have[b]) if ok[b] else 0
        wanted += want
        served.append(ok[b] and (want == 0 or wanted <= at))
        if not served[b]:
            continue
        for p in range(have[b], need[b]):
            T[b][p] = stack.pop()
        for j in range(n_new[b]):
            q = keep[b] + j
            pos[cu[b] + j] = q
            slots[cu[b] + j] = T[b][q // page] * page + q % page
    F[n_free:len(stack)] = stack[n_free:]
    assert len(F) == n_pages
    return cu, [k + n if s else -1 for k, n, s in zip(keep, n_new, served)], pos, slots, T, F, len(stack), bad


def fill_pool(pool, k, v):
    """Every page's rows k, v [pages, n_kv, page, hd] (bf16 or fp32) into the pool."""
    wq.kv_append(pool, k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous(),
                 torch.zeros(pool.batch, dtype=torch.int32, device="cuda"))


def pool_values(pool):
    """fp64 (K, V and the sums of the magnitudes that they are differences of; V's scales) [pages, n_kv, page, hd] of a
    pool, from its bytes."""
    out = []
    for held, meta in ((pool.k, pool.k_meta), (pool.v, pool.v_meta)):
        if pool.bits == 16:
            out.append((held.double(), held.double().abs(), held.double()[..., :1] * 0))
            continue
        if pool.bits == 4:
            w = held.view(torch.int32)[..., None].long() & 0xffffffff
            e = torch.arange(8, device="cuda")
            q = ((w >> (4 * (e // 2) + 16 * (e % 2))) & 15).flatten(-2)
        else:
            q = held.long()
        bits = meta.cpu().numpy().view(np.uint32)
        s = torch.from_numpy((bits & 0xffff).astype(np.uint16).view(np.float16).astype(np.float64)).cuda()[..., None]
        z = torch.from_numpy((bits >> 16).astype(np.uint16).view(np.float16).astype(np.float64)).cuda()[..., None]
        out.append((s * (q - z), s * (q + z), s))
    return out[0][0], out[1][0], out[0][1], out[1][1], out[1][2]


def attn_ref(q, cu, kv_lens, tables, pool, scale, own=None):
    """fp64 (o, bound) of wq_attn_paged.  The bound of |got - o|, element by element: each probability off by u of itself
    (its rounding to 16 bits, 2^-11 over a quantized pool, where a kernel may round V once to binary16 too, and 2^-8 over a bf16
    one) and by the error of its score, each fp32 sum
    by n 2^-24 of its terms' magnitudes (codes and zero points are summed apart, so those of code + z), 2^x by 2^-21, and the
    bf16 store by 2^-8.  Over a quantized pool the largest p times V's scale is at least 2^6 where binary16's least step is
    2^-24: what is left of any other code is off by 2^-31 of the largest scale more."""
    kd, vd, ka, va, sv = pool_values(pool)
    m, h, hd = q.shape
    rep = h // pool.n_kv
    u = 2.0 ** -8 if pool.bits == 16 else 2.0 ** -10
    o = torch.zeros((m, h, hd), dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(o)
    for b, n in enumerate(kv_lens):
        t = cu[b + 1] - cu[b]
        if n <= 0 or t <= 0:
            continue
        pages = tables[b, :-(-n // pool.max_len)].long()
        seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - t, n, device="cuda")[:, None]
        for g in range(pool.n_kv):
            K, V, KA, VA, S = (x[pages, g].flatten(0, 1)[:n] for x in (kd, vd, ka, va, sv))
            least = 2.0 ** -31 * S.amax() * (V.abs() / S.clamp(min=2.0 ** -24)).sum(0) if pool.bits != 16 else 0.0
            for a in range(g * rep, (g + 1) * rep):
                Q = q[cu[b]:cu[b + 1], a].double()
                x = (Q @ K.t() * scale).masked_fill(~seen, -torch.inf)
                off = (Q.abs() @ KA.t() * abs(scale)).masked_fill(~seen, 0).amax(-1, keepdim=True) * (hd + 8) * 2.0 ** -24
                p = torch.softmax(x, -1)
                o[cu[b]:cu[b + 1], a] = p @ V
                size = p @ VA
                e = u * (p @ V.abs()) + (2 * off + 2.0 ** -20) * (p @ V.abs()) + (n + 64) * 2.0 ** -24 * size + least
                bound[cu[b]:cu[b + 1], a] = e + 2.0 ** -8 * (o[cu[b]:cu[b + 1], a].abs() + e)
    return o, bound


def check(got, ref, bound, what=""):
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} out of bound, worst {float((err / bound.clamp(min=1e-300)).max()):.3g} x"
