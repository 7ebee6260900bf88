"""lsmkv_append_batch on 8-bit pools against its formulas.

A value y is off by the 32-bit arithmetic ahead of its rounding, at most 2^-18 of |a| + |b| (the two
elements that a rotation joins, after the norm; zero without norm and rotation), and by half a step of
e4m3: 2^-4 of the binade of the larger of y and the code, in units of the scale, 2^-10 in the subnormal range. A block's
exponent may be the one of its largest element within the same 2^-18. Everything else is equal bit for bit."""
import numpy as np
import pytest
import torch

from paper_2511_16138_b200 import lsmkv
from pool8 import DEV, exponents, filled, geom8, least_exponent, views
from test_append_gpu import batch, check, formula, rope_table

pytestmark = pytest.mark.gpu

CASES = [
    # dtype, D, rot, interleaved, qn, kn, P, B, hq, hkv, new, history
    (torch.bfloat16, 128, 128, False, False, False, 16, 16, 32, 8, [1] * 9, [0, 1, 15, 16, 17, 31, 100, 5, 1000]),
    (torch.float16, 128, 128, False, True, True, 64, 16, 28, 4, [1, 300, 0, 17, 64], [0, 5, 9, 63, 64]),
    (torch.bfloat16, 64, 64, True, True, False, 16, 1, 8, 8, [40, 1, 1], [0, 16, 3]),
    (torch.float16, 64, 32, False, False, True, 16, 4, 4, 2, [33], [7]),
    (torch.bfloat16, 96, 96, False, True, True, 5, 1, 6, 3, [12, 7], [2, 11]),
    (torch.bfloat16, 96, 48, False, True, True, 24, 8, 6, 3, [12, 7, 60], [2, 11, 21]),
    (torch.float16, 256, 256, False, True, True, 1, 1, 4, 1, [3, 5], [0, 2]),
    (torch.bfloat16, 256, 64, True, False, False, 16, 16, 4, 2, [20], [0]),
    (torch.bfloat16, 256, 16, False, True, True, 32, 16, 4, 2, [70, 3], [0, 17]),
    (torch.bfloat16, 80, 20, False, True, True, 16, 8, 5, 5, [9, 2], [1, 30]),      # element form
    (torch.float16, 80, 20, True, True, False, 16, 16, 5, 1, [9, 2, 40], [1, 30, 9]),  # element form
    (torch.bfloat16, 16, 6, False, False, True, 6, 2, 3, 3, [4, 7], [3, 4]),        # element form
    (torch.float16, 16, 16, True, True, True, 16, 2, 3, 1, [50], [0]),
    (torch.bfloat16, 128, 0, False, True, True, 16, 16, 8, 2, [5, 6], [0, 3]),      # norm alone
    (torch.float16, 128, 0, False, False, False, 16, 4, 8, 2, [5, 6], [0, 3]),      # rounding alone
    (torch.bfloat16, 128, 128, False, True, True, 16, 16, 0, 8, [70, 1], [0, 3]),   # no queries
    (torch.bfloat16, 128, 128, False, False, False, 16, 16, 64, 8, [5000, 3], [3, 0]),
    (torch.float16, 128, 128, False, False, True, 32, 8, 8, 4, [1, 2, 90, 1, 0, 7] * 60, [9, 33, 5, 0, 8, 100] * 60),
]


def stored(pool, before, g, layer, x, size, page, slot, new, kv, table, page_off):
    """K or V of `layer` (buffer number) after an append of rows x [t, heads, D] with error bound size."""
    B, P = g.block_tokens, g.page_tokens
    codes, scales = views(pool, g)
    codes0, scales0 = views(before, g)
    codes, scales, codes0, scales0 = (t[layer] for t in (codes, scales, codes0, scales0))
    blk = slot // B
    e = exponents(scales)[page, :, blk]                                   # [t, heads], after
    # largest element of every block's new tokens, from below and above
    key = page * (P // B) + blk
    lo = torch.zeros(codes.shape[0] * (P // B), x.shape[1], dtype=torch.float64, device=DEV)
    hi = lo.clone()
    at = key[:, None].expand(-1, x.shape[1])
    lo.scatter_reduce_(0, at, (x.abs() - size).clamp_min(0).amax(-1), "amax")
    hi.scatter_reduce_(0, at, (x.abs() + size).amax(-1), "amax")
    lo, hi = least_exponent(lo)[key], least_exponent(hi)[key]
    have = torch.zeros(len(page), dtype=torch.long, device=DEV)           # earlier tokens of the block
    seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).to(DEV)
    first = (torch.tensor(kv) - torch.tensor(new)).to(DEV)[seq]
    pos = first + torch.cat([torch.arange(a) for a in new]).to(DEV)
    have = (first - pos // B * B).clamp_min(0)
    old = exponents(scales0)[page, :, blk]
    lo = torch.where(have[:, None] > 0, torch.maximum(lo, old), lo)
    hi = torch.where(have[:, None] > 0, torch.maximum(hi, old), hi)
    assert ((e >= lo) & (e <= hi)).all()
    # new codes
    y = x * torch.exp2(-e.double())[..., None]
    got = codes[page, slot].double()
    top = torch.maximum(y.abs(), got.abs()).clamp_min(2.0 ** -6)
    half = torch.exp2(torch.floor(torch.log2(top)) - 4)
    tol = half + size * torch.exp2(-e.double())[..., None]
    assert ((got - y).abs() <= tol).all(), float(((got - y).abs() / tol).max())
    if not size.any():
        assert torch.equal(got, y.float().to(torch.float8_e4m3fn).double())
    # earlier tokens of begun blocks follow the scale; nothing else changed
    want, want_s = codes0.clone(), scales0.clone()
    want[page, slot] = codes[page, slot]
    want_s[page, :, blk] = scales[page, :, blk]
    for i, (a, b) in enumerate(zip(new, kv)):
        p0 = b - a
        if a and p0 % B:
            pg, bb = int(table[page_off[i] + p0 // P]), p0 % P // B
            d = exponents(scales0)[pg, :, bb] - exponents(scales)[pg, :, bb]
            assert (d <= 0).all()
            rows = slice(bb * B, p0 % P)
            moved = (codes0[pg, rows].double() * torch.exp2(d.double())[:, None]).float()
            want[pg, rows] = torch.where(d[:, None] == 0, codes0[pg, rows].float(), moved).to(want.dtype)
    assert torch.equal(codes.contiguous().view(torch.uint8), want.view(torch.uint8))
    assert torch.equal(scales.contiguous(), want_s)


def places(new, kv, P, table, page_off):
    pos = torch.cat([torch.arange(b - a, b) for a, b in zip(new, kv)]).to(DEV)
    seq = np.repeat(np.arange(len(new)), new)
    page = torch.tensor(table[page_off[seq] + pos.cpu().numpy() // P], device=DEV)
    return pos, page, pos % P


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_append_equals_its_formulas(case):
    dt, D, rot, inter, qn, kn, P, B, hq, hkv, new, hist = case
    kv = [a + b for a, b in zip(new, hist)]
    seqs, new_off, page_off, table, num = batch(new, kv, P)
    gen = torch.Generator(device=DEV).manual_seed(3)
    n = int(new_off[-1])
    qkv = torch.randn(n, hq + 2 * hkv, D, generator=gen, device=DEV).to(dt)
    # tokens of very different size, so that scales grow, and zeros
    qkv *= torch.exp2(torch.randint(-6, 7, (n, 1, 1), generator=gen, device=DEV).float()).to(dt)
    qkv[n // 2, -1] = 0
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    q_w = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dt) if qn else None
    k_w = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(dt) if kn else None
    tab = rope_table(max(kv), rot) if rot else None
    g = geom8(2, hkv, D, P, B)
    pool = filled(g, num, gen)
    before, layer = pool.clone(), 1
    pos, page, slot = places(new, kv, P, table, page_off)
    with lsmkv.Context(g, 0) as ctx:
        q_out = torch.full((n, hq, D), 7.0, dtype=dt, device=DEV)
        args = (layer, seqs, k, v, lsmkv.pool_table(list(pool)))
        kw = dict(rope=lsmkv.Rope(tab, inter) if rot else None, q_norm=q_w if hq else None, k_norm=k_w, eps=1e-5)
        ctx.append_batch(*args, q=q if hq else None, q_out=q_out if hq else None, **kw)
        assert ctx.last_status()["flags"] == 0
        once = pool.clone()
        # again: the same bytes, and the queries in place
        mine = q.clone()
        ctx.append_batch(*args, q=mine if hq else None, **kw)
        assert ctx.last_status()["flags"] == 0
        assert torch.equal(once, pool)
    if hq:
        assert torch.equal(mine.view(torch.int16), q_out.view(torch.int16))
        check(q_out, *formula(q, q_w, tab, pos, rot, inter, 1e-5), dt)
    x, size = formula(k, k_w, tab, pos, rot, inter, 1e-5)
    size = 2.0 ** -18 * size if rot or kn else torch.zeros_like(size)
    stored(pool, before, g, layer, x, size, page, slot, new, kv, table, page_off)
    stored(pool, before, g, 2 + layer, v.double(), torch.zeros_like(x), page, slot, new, kv, table, page_off)
    other = [0, 2]
    assert torch.equal(pool[other], before[other])


def test_token_by_token_gives_the_scale_of_the_whole_block():
    """A block filled in several calls ends with the exponent of all its tokens; codes of earlier tokens are within
    a step and a half of the last scale's, however often it grew."""
    D, P, B, H, n = 64, 16, 16, 4, 48
    g = geom8(1, H, D, P, B)
    gen = torch.Generator(device=DEV).manual_seed(8)
    k = torch.randn(n, H, D, generator=gen, device=DEV) * torch.exp2(torch.arange(n, device=DEV) % 16 - 8.0)[:, None, None]
    k = k.to(torch.bfloat16)
    pool = torch.full((2, 3, g.page_bytes), 0xFF, dtype=torch.uint8, device=DEV)    # nothing defined
    with lsmkv.Context(g, 0) as ctx:
        for t in range(n):
            seqs, *_ = batch([1], [t + 1], P, spare=0)
            seqs.keep[3].copy_(torch.arange(t // P + 1, dtype=torch.int32))
            ctx.append_batch(0, seqs, k[t:t + 1], k[t:t + 1], lsmkv.pool_table(list(pool)))
        assert ctx.last_status()["flags"] == 0
    codes, scales = views(pool, g)
    amax = k.double().abs().unflatten(0, (3, B)).amax((1, 3))                       # [pages, heads]
    assert torch.equal(exponents(scales)[..., 0], least_exponent(amax).expand(2, -1, -1))
    y = k.double().unflatten(0, (3, P)) * torch.exp2(-least_exponent(amax).double())[:, None, :, None]
    got = codes.double()[0]
    step = torch.exp2(torch.floor(torch.log2(torch.maximum(y.abs(), got.abs()).clamp_min(2.0 ** -6))) - 3)
    assert torch.isfinite(got).all() and ((got - y).abs() <= 1.5 * step).all()


def test_infinities_and_nan_become_nan_and_do_not_move_the_scale():
    D, P, B, H = 32, 16, 8, 2
    g = geom8(1, H, D, P, B)
    for dt in (torch.bfloat16, torch.float16):
        k = torch.ones(16, H, D, dtype=dt, device=DEV)
        k[3, 0, 5], k[4, 1, 6], k[9, 0, 0] = float("inf"), float("nan"), float("-inf")
        k[8:, 1] = float("nan")                                            # a block without a finite element
        v = torch.full_like(k, torch.finfo(dt).max)                        # the largest numbers
        pool = torch.zeros(2, 1, g.page_bytes, dtype=torch.uint8, device=DEV)
        seqs, *_ = batch([16], [16], P, spare=0)
        with lsmkv.Context(g, 0) as ctx:
            ctx.append_batch(0, seqs, k, v, lsmkv.pool_table(list(pool)))
            assert ctx.last_status()["flags"] == 0
        codes, scales = views(pool, g)
        got = codes[0, 0].double()
        assert torch.equal(torch.isnan(got), ~torch.isfinite(k))
        assert (got[torch.isfinite(k)] == 256).all()                       # 256 * 2^-8
        assert exponents(scales)[0, 0].tolist() == [[-8, -8], [-8, -100]]
        e = int(least_exponent(torch.tensor(float(v[0, 0, 0]), dtype=torch.float64)))
        assert (exponents(scales)[1] == e).all()
        if e < 100:
            assert (codes[1].double() * 2.0 ** e - v.double()).abs().max() <= 2.0 ** -4 * float(v[0, 0, 0])
        else:
            assert (codes[1].double() == 448).all()                        # beyond 448 * 2^100


def test_padding_and_left_out_tokens():
    """Padding stores nothing and zeroes its queries; a row of the table that is not there leaves a token out."""
    D, P, B, H, HQ = 64, 16, 16, 2, 4
    g = geom8(1, H, D, P, B)
    new, kv = [5, 3, 2], [2, 0, 40]
    seqs, new_off, page_off, table, num = batch(new, kv, P)
    x = torch.randn(10, HQ + 2 * H, D, device=DEV).to(torch.bfloat16)
    q, k, v = x[:, :HQ], x[:, HQ:HQ + H], x[:, HQ + H:]
    tab = rope_table(40, D)
    pool = torch.zeros(2, num, g.page_bytes, dtype=torch.uint8, device=DEV)
    out = torch.full((10, HQ, D), 3.0, dtype=torch.bfloat16, device=DEV)
    where = torch.tensor([0, 0, 0, 7, 8, 0, 0, 0, 50, 9], dtype=torch.int32, device=DEV)   # 50: none
    with lsmkv.Context(g, 0) as ctx:
        ctx.append_batch(0, seqs, k, v, lsmkv.pool_table(list(pool)), rope=lsmkv.Rope(tab, positions=where), q=q,
                         q_out=out)
        st = ctx.last_status()
    assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 8
    assert not out[:3].any() and not out[5:8].any() and (out[8] == 3.0).all()
    codes, _ = views(pool, g)
    used = codes.float().abs().amax((3, 4)) > 0                            # [2, pages, slots]
    want = torch.zeros_like(used)
    want[:, int(table[page_off[0]]), :2] = True
    want[:, int(table[page_off[2] + 2]), 39 - 32] = True
    assert torch.equal(used, want)
    rows = torch.tensor([3, 4, 9], device=DEV)
    check(out[rows], *formula(q[rows], None, tab, where[rows].long(), D, False, 0), torch.bfloat16)


def test_bad_sequences_and_pages_are_reported_and_left_out():
    D, P, B, H = 64, 16, 8, 2
    g = geom8(1, H, D, P, B)
    new, kv = [4, 20, 3], [9, 40, 3]
    seqs, new_off, page_off, table, num = batch(new, kv, P)
    x = torch.randn(27, 2 * H, D, device=DEV).to(torch.float16)
    k, v = x[:, :H], x[:, H:]
    with lsmkv.Context(g, 0) as ctx:
        def run(s):
            pool = torch.zeros(2, num, g.page_bytes, dtype=torch.uint8, device=DEV)
            ctx.append_batch(0, s, k, v, lsmkv.pool_table(list(pool)))
            return ctx.last_status(), views(pool, g)[0].float().abs().amax((3, 4)) > 0

        st, all_used = run(seqs)
        assert st["flags"] == 0 and int(all_used.sum()) == 2 * 27
        entry = int(page_off[1]) + 2
        seqs.keep[3][entry] = num                                          # the third page of sequence 1
        st, used = run(seqs)
        assert st["flags"] == lsmkv.ST_BAD_PAGE and st["first_bad"] == entry
        want = all_used.clone()
        want[:, int(table[entry])] = False
        assert torch.equal(used, want)
        seqs.keep[3][entry] = int(table[entry])
        seqs.keep[1][1] = 4000                                             # more tokens than pages
        st, used = run(seqs)
        assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 1
        want = all_used.clone()
        want[:, torch.tensor(table[page_off[1]:page_off[2]], device=DEV)] = False
        assert torch.equal(used, want)
        seqs.keep[1][1] = kv[1]
        st, used = run(lsmkv.Seqs(*seqs.keep, 27, 19))                     # a bound that sequence 1 breaks
        assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 1 and torch.equal(used, want)
        pool = torch.zeros(2, num, g.page_bytes, dtype=torch.uint8, device=DEV)
        off = torch.tensor([pool[0].data_ptr() + 8, pool[1].data_ptr()], device=DEV)
        ctx.append_batch(0, seqs, k, v, (off, num - 1))
        assert ctx.last_status()["flags"] == lsmkv.ST_MISALIGNED and not pool.any()
