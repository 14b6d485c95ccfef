"""Rows quantized into the KV cache as they are written (wq_kv_append) and read
back (wq_kv_read), and the rotary positions of drafted tokens (wq_qkv_rope).

Codes, scales and zeros are defined in fp32 with round to nearest, so the cache's
contents and what is read back must equal the definition bit for bit (evaluated
here in fp64 with one rounding to fp32 a step, which gives the fp32 results).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wq():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2606_04238_gb300 import wq as mod
    mod.device_status()
    return mod


def _f32(x):
    return x.to(torch.float32).to(torch.float64)


def stored(rows, bits):
    """(fp64 values that rows stand for once cached, codes, scale, zero)."""
    r = rows.double().cpu()
    if bits == 16:
        return r.to(torch.bfloat16).double(), None, None, None
    top = 2 ** bits - 1
    bad = ~torch.isfinite(r).all(-1, keepdim=True)
    r = torch.where(bad, torch.zeros_like(r), r)
    lo, hi = r.amin(-1, keepdim=True).clamp(max=0), r.amax(-1, keepdim=True).clamp(min=0)
    s = _f32(_f32(hi - lo) / top).to(torch.float16).double()
    bad = bad | torch.isinf(s)
    s = torch.where(s == 0, torch.ones_like(s), s)
    z = _f32(-lo / s).round().clamp(0, top)
    q = (_f32(r / s).round() + z).clamp(0, top)
    q, z = (torch.where(bad, torch.zeros_like(t), t) for t in (q, z))
    s = torch.where(bad, torch.full_like(s, math.nan), s)
    return s * (q - z), q, s, z


def _codes(c, which):
    """The cache's codes [b, h, max_len, hd], unpacked as the header describes."""
    t = (c.k if which == "k" else c.v).cpu()
    if c.bits == 8:
        return t.to(torch.int64)
    w = t.contiguous().view(torch.int32).to(torch.int64) & 0xffffffff
    e = torch.arange(8)
    return ((w[..., None] >> (4 * (e // 2) + 16 * (e % 2))) & 15).flatten(-2)


def _meta(c, which):
    m = (c.k_meta if which == "k" else c.v_meta).cpu().view(torch.float16).view(*c.k.shape[:3], 2).double()
    return m[..., :1], m[..., 1:]


def _rows(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * 2.0).to(dtype)


def _same(a, b):
    a, b = a.double().cpu(), b.double().cpu()
    return a.shape == b.shape and bool(((a == b) | (a.isnan() & b.isnan())).all())


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("b,t,h", [(1, 1, 1), (3, 17, 2), (2, 130, 5)])
def test_append_and_read_back(wq, bits, hd, dtype, b, t, h):
    L = t + 9
    k, v = _rows((b, t, h, hd), dtype, 1), _rows((b, t, h, hd), dtype, 2)
    k[0, 0, 0] = 0                       # a row of zeros
    v[0, 0, 0] = v[0, 0, 0].abs() + 1    # of one sign
    v[-1, -1, -1] = -v[-1, -1, -1].abs() - 1
    k[-1, -1, -1, 3] = 300.0             # one large value
    start = torch.arange(b, dtype=torch.int32) * 2 + 5
    c = wq.kv_cache(b, h, L, hd, bits)
    before = [x.clone() for x in (c.k, c.v)]
    wq.kv_append(c, k.cuda(), v.cuda(), start.cuda())
    for out in (torch.float32, torch.bfloat16):
        kr, vr = wq.kv_read(c, start.cuda(), t, dtype=out)
        for got, rows in ((kr, k), (vr, v)):
            assert _same(got, stored(rows, bits)[0].to(out))
    for which, rows, old in (("k", k, before[0]), ("v", v, before[1])):
        if bits != 16:
            _, q, s, z = stored(rows, bits)
            codes, (ms, mz) = _codes(c, which), _meta(c, which)
        held = getattr(c, which).cpu()
        for i in range(b):
            a = int(start[i])
            if bits != 16:
                assert torch.equal(codes[i, :, a:a + t].transpose(0, 1), q[i].to(torch.int64))
                assert _same(ms[i, :, a:a + t].transpose(0, 1), s[i]) and _same(mz[i, :, a:a + t].transpose(0, 1), z[i])
            assert torch.equal(held[i, :, :a], old[i, :, :a].cpu())          # nothing else is written
            assert torch.equal(held[i, :, a + t:], old[i, :, a + t:].cpu())
    assert wq.device_status() == 0


@pytest.mark.parametrize("bits", [8, 4])
def test_rows_at_the_edges_of_the_scale(wq, bits):
    hd = 128
    k = _rows((1, 10, 1, hd), torch.float32, 3)
    k[0, 0] *= 1e-9            # scale underflows to 0: held as 0
    k[0, 1] *= 2e-6            # a subnormal scale
    k[0, 2] *= 3e3 * (2 ** bits - 1)  # large, inside binary16's scales
    k[0, 3] *= 1e9             # scale beyond binary16
    k[0, 4, 0, 7] = math.inf
    k[0, 5, 0, 9] = -math.inf
    k[0, 6, 0, 100] = math.nan
    k[0, 7] = 0.0
    k[0, 7, 0, 1] = 1.0        # one value only
    k[0, 8] = torch.linspace(-1, 1, hd) * (2 ** bits - 1) / 2  # quotients at and near halves
    k[0, 9] = 65504.0
    start = torch.zeros(1, dtype=torch.int32)
    c = wq.kv_cache(1, 1, 10, hd, bits)
    wq.kv_append(c, k.cuda(), k.cuda(), start.cuda())
    kr, vr = wq.kv_read(c, start.cuda(), 10, dtype=torch.float32)
    want = stored(k, bits)[0]
    assert _same(kr, want.float()) and _same(vr, want.float())
    assert torch.isnan(kr[0, 3:7]).all() and torch.isfinite(kr[0, :3]).all() and torch.isfinite(kr[0, 7:]).all()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hd", [64, 128])
def test_quotients_at_and_beside_halves(wq, bits, hd):
    """Values (j + 1/2) s, where v / s is rounded to even, and the fp32 values next to them: codes as the
    fp32 quotient's, scales of binary16 from the smallest on.  A row holds -z s and (top - z) s, exactly in
    fp32 and 19 bits, so that its scale is s and its zero z."""
    top, n = 2 ** bits - 1, 96
    g = torch.Generator().manual_seed(9)
    s = torch.cat([torch.tensor([1.0, 3.0, 1023.0]) * 2.0 ** -24, torch.tensor([1.0, 0.1, 31.0]),
                   2.0 ** (torch.rand(n - 6, generator=g) * 14 - 10)]).to(torch.float16).to(torch.float32)
    z = torch.randint(0, top + 1, (n,), generator=g).float()
    j = torch.floor(torch.rand((n, hd), generator=g) * top) - z[:, None]
    v = (j + 0.5) * s[:, None]
    bits_of = v.view(torch.int32) + torch.randint(-2, 3, (n, hd), generator=g, dtype=torch.int32) * (v != 0)
    v = torch.minimum(torch.maximum(bits_of.view(torch.float32), -(z * s)[:, None]), ((top - z) * s)[:, None])
    v[:, 0], v[:, 1] = -z * s, (top - z) * s
    for dtype in (torch.float32, torch.bfloat16):
        rows = v.to(dtype)[None, :, None]
        c = wq.kv_cache(1, 1, n, hd, bits)
        wq.kv_append(c, rows.cuda(), rows.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"))
        _, q, sc, zc = stored(rows, bits)
        if dtype is torch.float32:
            assert torch.equal(sc.flatten(), s.double()) and torch.equal(zc.flatten(), z.double())
        for which in "kv":
            assert torch.equal(_codes(c, which)[0, 0], q[0, :, 0].to(torch.int64))
            assert _same(_meta(c, which)[0][0, 0], sc[0, :, 0]) and _same(_meta(c, which)[1][0, 0], zc[0, :, 0])


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_accepted_path_and_counts(wq, bits):
    b, t, h, hd, n, L = 4, 37, 3, 64, 9, 50
    k, v = _rows((b, t, h, hd), torch.bfloat16, 5), _rows((b, t, h, hd), torch.bfloat16, 6)
    g = torch.Generator().manual_seed(7)
    index = torch.randint(0, t, (b, n), generator=g, dtype=torch.int32)
    counts = torch.tensor([9, 0, 1, 4], dtype=torch.int32)
    start = torch.tensor([0, 50, 49, 7], dtype=torch.int32)
    c = wq.kv_cache(b, h, L, hd, bits)
    wq.kv_append(c, k.cuda(), v.cuda(), start.cuda(), counts=counts.cuda(), index=index.cuda())
    kr, vr = wq.kv_read(c, start.cuda(), n, counts=counts.cuda(), dtype=torch.float32)
    for got, rows in ((kr, k), (vr, v)):
        want = torch.stack([stored(rows, bits)[0][i][index[i].long()] for i in range(b)])
        for i in range(b):
            want[i, int(counts[i]):] = 0
        assert _same(got, want)
    assert wq.device_status() == 0


def test_strided_rows(wq):
    b, t, hq, h, hd = 2, 11, 6, 2, 128
    qkv = _rows((b, t, hq + 2 * h, hd), torch.bfloat16, 8).cuda()
    k, v = qkv[:, :, hq:hq + h], qkv[:, :, hq + h:]
    start = torch.zeros(b, dtype=torch.int32, device="cuda")
    c = wq.kv_cache(b, h, t, hd, 8)
    wq.kv_append(c, k, v, start)
    kr, vr = wq.kv_read(c, start, t, dtype=torch.float32)
    assert _same(kr, stored(k, 8)[0]) and _same(vr, stored(v, 8)[0])
    heads_first = k.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # [b, h, t, hd] in memory
    c2 = wq.kv_cache(b, h, t, hd, 8)
    wq.kv_append(c2, heads_first, v, start)
    assert torch.equal(c2.k, c.k) and torch.equal(c2.k_meta, c.k_meta)


def test_ranges_are_skipped_and_recorded(wq):
    b, t, h, hd, L = 3, 4, 2, 64, 16
    k = _rows((b, t, h, hd), torch.bfloat16, 9).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for start, counts, index in ((i32(-1, 13, 12), None, None), (i32(0, 0, 0), i32(5, -1, 4), None),
                                 (i32(0, 0, 0), None, i32(0, 1, 2, 3, 0, 1, 4, 3, -1, 1, 2, 3).view(3, 4))):
        c = wq.kv_cache(b, h, L, hd, 8)
        wq.kv_append(c, k, k, start, counts=counts, index=index)
        assert wq.device_status() == -1
        put = (c.k_meta != 0).cpu()
        if index is None:
            assert not put[0].any() and not put[1].any() and put[2].any(0).sum() == 4
        else:
            assert put[:, 0, :4].tolist() == [[True] * 4, [True, True, False, True], [False, True, True, True]]
    c = wq.kv_cache(b, h, L, hd, 8)
    out = torch.full((b, t, h, hd), 7.0, device="cuda")
    wq.kv_read(c, i32(13, 0, -2), t, dtype=torch.float32, k=out, v=out.clone())
    assert wq.device_status() == -1 and wq.device_status() == 0
    assert (out[0] == 7).all() and (out[1] == 0).all() and (out[2] == 7).all()


def test_long_cache_offsets(wq):
    """Row offsets past 2^31 bytes: the last sequence of a cache of 2.2 GB a tensor."""
    b, h, L, hd = 9, 8, 120_001, 128
    c = wq.kv_cache(b, h, L, hd, 16)
    k, v = _rows((b, 2, h, hd), torch.bfloat16, 10).cuda(), _rows((b, 2, h, hd), torch.bfloat16, 11).cuda()
    start = torch.full((b,), L - 2, dtype=torch.int32, device="cuda")
    wq.kv_append(c, k, v, start)
    assert torch.equal(c.k[-1, -1, -2:], k[-1, :, -1]) and torch.equal(c.v[-1, -1, -2:], v[-1, :, -1])
    kr, vr = wq.kv_read(c, start, 2)
    assert torch.equal(kr, k) and torch.equal(vr, v)


# ---- rotary positions ----------------------------------------------------------

def _rope64(qkv, x, pos, table, H, kv, norm):
    m, hd = qkv.shape[0], 2 * table.shape[1]
    u = qkv.double().cpu()
    if x is not None:
        u = u / torch.sqrt((x.double().cpu() ** 2).mean(-1, keepdim=True) + 1e-6)
    u = u.view(m, H + 2 * kv, hd)
    n = u[:, :H + kv]
    if norm:
        n = n / torch.sqrt((n * n).mean(-1, keepdim=True) + 1e-6)
    cs = table.double().cpu()[pos.long().cpu()][:, None]
    lo, hi = n[..., :hd // 2], n[..., hd // 2:]
    n = torch.cat([lo * cs[..., 0] - hi * cs[..., 1], hi * cs[..., 0] + lo * cs[..., 1]], -1)
    return n[:, :H], n[:, H:], u[:, H + kv:]


@pytest.mark.parametrize("H,kv,hd", [(32, 8, 128), (1, 1, 64), (64, 8, 64), (40, 8, 128), (80, 2, 128)])
@pytest.mark.parametrize("m,d,norm", [(1, 8, True), (13, 2560, True), (70, 0, True), (5, 5120, False)])
def test_rope(wq, H, kv, hd, m, d, norm):
    g = torch.Generator().manual_seed(m + H)
    qkv = torch.randn((m, (H + 2 * kv) * hd), generator=g)
    x = (torch.randn((m, d), generator=g) * 3).to(torch.bfloat16) if d else None
    pos = torch.randint(0, 3000, (m,), generator=g, dtype=torch.int32)
    table = wq.rope_table(3000, hd)
    got = wq.qkv_rope(qkv.cuda(), pos.cuda(), table, H, kv, x=None if x is None else x.cuda(), head_norm=norm)
    for a, r in zip(got, _rope64(qkv, x, pos, table, H, kv, norm)):
        # fp32 arithmetic (some 2^-20 of the head's largest value), then half a bf16 ulp of the result
        tol = 2.0 ** -18 * r.abs().amax(-1, keepdim=True) + r.abs() * 2.0 ** -8 * 1.01
        assert a.shape == r.shape and bool(((a.double().cpu() - r).abs() <= tol).all())
    assert wq.device_status() == 0


def test_rope_table_and_positions(wq):
    t = wq.rope_table(40000, 128)
    a = 39999.0 * 1e6 ** (-2.0 * 5 / 128)
    assert abs(float(t[39999, 5, 0]) - math.cos(a)) < 1e-7 and abs(float(t[39999, 5, 1]) - math.sin(a)) < 1e-7
    qkv = torch.randn((3, 3 * 64)).cuda()
    q = torch.full((3, 1, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    pos = torch.tensor([-1, 2, 4], dtype=torch.int32, device="cuda")
    wq.qkv_rope(qkv, pos, wq.rope_table(4, 64), 1, 1, q=q)
    assert wq.device_status() == -1
    assert (q[0] == 5).all() and (q[2] == 5).all() and (q[1] != 5).any()


def test_empty_calls(wq):
    c = wq.kv_cache(2, 1, 4, 64, 8)
    e = torch.empty((2, 0, 1, 64), dtype=torch.bfloat16, device="cuda")
    s = torch.zeros(2, dtype=torch.int32, device="cuda")
    wq.kv_append(c, e, e, s)
    assert wq.kv_read(c, s, 0)[0].shape == (2, 0, 1, 64)
    wq.qkv_rope(torch.empty((0, 192), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"),
                wq.rope_table(4, 64), 1, 1)
    assert wq.device_status() == 0
