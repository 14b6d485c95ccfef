"""Codes, scales and zero points of normed and rotated rows in pages: those of the fp64 row, wherever fp32's errors cannot move
a quotient over the border between two of them."""
import pytest
import torch

from paged_util import status
from paper_2606_04238_gb300 import wq
from test_gpu_paged import BF, gen, randn, slots_of

pytestmark = pytest.mark.gpu


def held(rows, meta, bits):
    """(codes, scales as binary16, zero points) of a pool's K or V."""
    if bits == 4:
        w = rows.view(torch.int32)[..., None].long() & 0xffffffff
        e = torch.arange(8, device="cuda")
        codes = ((w >> (4 * (e // 2) + 16 * (e % 2))) & 15).flatten(-2)
    else:
        codes = rows.long()
    return codes, meta.to(torch.int16).view(torch.float16), (meta >> 16).to(torch.int16).view(torch.float16)


def near_half(x, err):
    return ((x - torch.floor(x)) - 0.5).abs() <= err


def check_row_codes(got, want, off, bits, what):
    """got: codes, scales, zeros [m, kv, ..]; want: fp64 rows, each value of which the kernel has within off."""
    codes, s16, z16 = got
    top = 2 ** bits - 1
    lo, hi = want.amin(-1, keepdim=True).clamp(max=0), want.amax(-1, keepdim=True).clamp(min=0)
    far = off.amax(-1, keepdim=True)
    step = (hi - lo) / top
    by = 2 * far / (hi - lo) + 2.0 ** -22  # relative: both ends, a difference, a quotient
    s = step.half()
    sure = ((step * (1 + by)).half() == s) & ((step * (1 - by)).half() == s)
    sd = s.double()
    z = (-lo / sd).round().clamp(0, top)
    sure_z = sure & ~near_half(-lo / sd, far / sd + (-lo / sd) * 2.0 ** -23)
    assert torch.equal(s16[sure[..., 0]], s[sure]) and torch.equal(z16[sure_z[..., 0]].double(), z[sure_z]), what
    r = want / sd
    sure_c = sure_z & ~near_half(r, off / sd + r.abs() * 2.0 ** -23)
    c = (r.round() + z).clamp(0, top).long()
    assert torch.equal(codes[sure_c], c[sure_c]), f"{what}: {int((codes != c)[sure_c].sum())} of {int(sure_c.sum())} codes"
    # a scale is unsure within `by` (some 2^-17) of a border in steps of 2^-11 to 2^-10, a code within 255 2^-17 of a half: few are
    assert float(sure_c.double().mean()) > 0.9, what


@pytest.mark.parametrize("m", [33, 300])
@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("h,kv,hd,d,weights", [(32, 8, 128, 2560, True), (10, 2, 64, 0, True), (5, 5, 128, 72, False), (64, 8, 64, 2880, True)])
def test_codes_of_normed_and_rotated_rows(h, kv, hd, d, weights, bits, f32, m):
    page, n_pos = 32, 500
    n_pages = -(-m // page) + 1
    qkv = (randn(m, (h + 2 * kv) * hd, seed=m) * 1.7).to(torch.float32 if f32 else BF)
    x = randn(m, d, seed=m + 1, dtype=BF) if d else None
    qw, kw = ((1 + 0.4 * randn(hd, seed=s)).to(BF) if weights else None for s in (3, 4))
    pos = torch.randint(0, n_pos, (m,), generator=gen(9), device="cuda", dtype=torch.int32)
    table = wq.rope_table(n_pos, hd)
    pool, slots = wq.kv_pool(n_pages, kv, page, hd, bits), slots_of(m, page, n_pages, 8)
    wq.qkv_paged(qkv, slots, pool, h, positions=pos, table=table, x=x, q_norm=qw, k_norm=kw)
    u = qkv.double()
    if d:
        u = u / torch.sqrt(x.double().pow(2).mean(-1, keepdim=True) + 1e-6)
    k, v = u.view(m, h + 2 * kv, hd)[:, h:].split(kv, 1)
    k = k / torch.sqrt(k.pow(2).mean(-1, keepdim=True) + 1e-6)
    if weights:
        k = k * kw.double()
    cs = table.double()[pos.long()][:, None]
    lo, hi = k[..., :hd // 2], k[..., hd // 2:]
    k = torch.cat([lo * cs[..., 0] - hi * cs[..., 1], hi * cs[..., 0] + lo * cs[..., 1]], -1)
    # fp32: the sums of squares (hd and d terms, in part one after another), a root, a quotient, five products
    fuzz = (hd / 8 + d / 512 + 16) * 2.0 ** -24
    size = torch.cat([lo.abs() + hi.abs()] * 2, -1)
    s = slots.long()
    for name, rows, meta, want, off in (("K", pool.k, pool.k_meta, k, fuzz * size), ("V", pool.v, pool.v_meta, v, fuzz * v.abs())):
        got = [t[s // page, :, s % page] for t in held(rows, meta, bits)]
        check_row_codes(got, want, off, bits, name)
    assert status() == 0
