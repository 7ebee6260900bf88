"""8-bit pools at the ends of their ranges: rows and scales of zero, scales that lie far apart, exponents that grow by the
whole range; against the definitions in 64 bits.

Tolerance of o = sum w v, A = sum w |v|, v = d 2^b (code d, exponent b of its block), all over what the row itself sees:
U |o| for the rounding of the result (half of the type's epsilon) and half the smallest subnormal of float16;
2^-11 A for the weights, which are 16-bit floats of 11 bits; below 2^-14 of the row's largest w 2^b (b taken as -40 at least) they are
subnormal, off by 2^-25 of it, so 2^-25 max(w 2^b) sum |d|; and for the scores, 32-bit sums of products, 2^-12 + 2^-20 times the
largest sum of their magnitudes, of A. A row of the few-row kernel and of the many-row kernel keep the same."""
import math

import pytest
import torch

from paper_2511_16138_b200 import lsmkv
from pool8 import DEV, exponents, filled, geom8, views
from test_append_gpu import U, batch
from test_attend8_gpu import shared_setup

pytestmark = pytest.mark.gpu


def exact(q, pool, g, layer, new_off, kv, page_off, table, scale):
    """o, A, slack of subnormal weights, largest sum of a score's magnitudes, lse; rows without keys are 0 and -inf."""
    n, hq, D = q.shape
    G, B, L = hq // g.n_kv_heads, g.block_tokens, g.n_layers
    codes, scales = views(pool, g)
    o = torch.zeros(n, hq, D, dtype=torch.float64, device=DEV)
    A, slack = torch.zeros_like(o), torch.zeros_like(o)
    size = torch.zeros(n, hq, 1, dtype=torch.float64, device=DEV)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=DEV)
    for i in range(len(kv)):
        a, b = int(new_off[i]), int(new_off[i + 1])
        if a == b or kv[i] == 0:
            continue
        pages = torch.tensor(table[page_off[i]:page_off[i + 1]], device=DEV)

        def rows(buffer):
            c = codes[buffer, pages].double().flatten(0, 1)[:kv[i]]
            e = exponents(scales[buffer, pages]).transpose(1, 2).repeat_interleave(B, 1).flatten(0, 1)[:kv[i]]
            return c.repeat_interleave(G, 1), e.double().repeat_interleave(G, 1)

        kc, ke = rows(layer)
        vc, ve = rows(L + layer)
        k, v = kc * torch.exp2(ke)[..., None], vc * torch.exp2(ve)[..., None]
        s = torch.einsum("thd,jhd->htj", q[a:b].double(), k) * scale
        big = torch.einsum("thd,jhd->htj", q[a:b].double().abs(), k.abs()) * abs(scale)
        p = kv[i] - (b - a) + torch.arange(b - a, device=DEV)
        seen = torch.arange(kv[i], device=DEV)[None] <= p[:, None]
        s = s.masked_fill(~seen, -math.inf)
        lse[a:b] = torch.logsumexp(s, -1).T
        w = torch.exp(s - s.amax(-1, keepdim=True).clamp_min(-1e300))
        w = torch.where(seen.any(-1)[:, None], w / w.sum(-1, keepdim=True), torch.zeros_like(w))
        o[a:b] = torch.einsum("htj,jhd->thd", w, v)
        A[a:b] = torch.einsum("htj,jhd->thd", w, v.abs())
        top = (w * torch.exp2(ve.clamp_min(-40)).T[:, None]).amax(-1)                       # [h, t]
        slack[a:b] = 2.0 ** -25 * top.T[..., None] * torch.einsum("tj,jhd->thd", seen.double(), vc.abs())
        size[a:b, :, 0] = torch.where(seen, big, torch.zeros_like(big)).amax(-1).T
    return o, A, slack, size, lse


def check(out, lse, ref, dt, rows=slice(None)):
    o, A, slack, size, want = (x[rows] for x in ref)
    out = out[rows]
    assert torch.isfinite(out).all()
    scores = 2.0 ** -12 + 2.0 ** -20 * size
    tol = U[dt] * o.abs() + (2.0 ** -11 + scores) * A + slack + (2.0 ** -25 if dt == torch.float16 else 0)
    err = (out.double() - o).abs()
    bad = err > tol
    assert not bad.any(), (int(bad.sum()), float((err / A.clamp_min(1e-300))[bad].max()), bad.nonzero()[:3].tolist())
    if lse is not None:
        lse = lse[rows]
        empty = torch.isinf(want)
        assert torch.equal(torch.isneginf(lse), empty)
        d = ((lse.double() - want).abs() - scores[..., 0] - 2.0 ** -21 * want.abs())[~empty]
        assert not d.numel() or bool((d <= 0).all()), float(d.max())


def attend(g, pool, q, seqs, scale, groups=None, layer=0):
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(g, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        if groups is None:
            ctx.attend_batch(layer, seqs, q, out, pt, scale, lse)
        else:
            ctx.attend_shared_batch(layer, seqs, groups, q, out, pt, scale, lse)
        assert ctx.last_status()["flags"] == 0
    return out, lse


# ---- queries and scales of zero ------------------------------------------------------------------

@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D,B", [(128, 16), (64, 1), (96, 4)])
def test_queries_of_zero_take_the_mean(dt, D, B):
    """Rows of zeros, padding among them, in sequences of few and of many rows."""
    g = geom8(1, 2, D, 16, B)
    new, kv = [40, 1, 300, 70, 33], [70, 100, 900, 7, 0]
    seqs, new_off, page_off, table, num = batch(new, kv, 16)
    gen = torch.Generator(device=DEV).manual_seed(1)
    pool = filled(g, num, gen)
    q = torch.randn(sum(new), 8, D, generator=gen, device=DEV).to(dt)
    q[::3] = 0
    q[:, 5] = 0
    q[new_off[3]:new_off[3] + 63] = 0                       # what an append leaves for padding
    q[new_off[4]:] = 0
    out, lse = attend(g, pool, q, seqs, D ** -0.5)
    check(out, lse, exact(q, pool, g, 0, new_off, kv, page_off, table, D ** -0.5), dt)
    assert not out[new_off[3]:new_off[3] + 63].any() and torch.isneginf(lse[new_off[4]:]).all()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_queries_of_zero_over_shared_prefixes(dt):
    case = (dt, 128, 16, 16, 2, [6, 4], [9, 5], 5, (0, 30))
    g, pool, q, seqs, groups, new_off, kv, page_off, table = shared_setup(case, 16)
    q[::2] = 0
    out, lse = attend(g, pool, q, seqs, 0.1, groups)
    check(out, lse, exact(q, pool, g, 0, new_off, kv, page_off, table, 0.1), dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 100])
def test_a_scale_of_zero(dt, size):
    """Every key weighs the same, whatever the queries."""
    g = geom8(1, 2, 128, 16, 16)
    new, kv = [40, 1, 300], [70, 100, 900]
    seqs, new_off, page_off, table, num = batch(new, kv, 16)
    gen = torch.Generator(device=DEV).manual_seed(2)
    pool = filled(g, num, gen)
    q = torch.randn(sum(new), 8, 128, generator=gen, device=DEV).to(dt)
    if dt == torch.bfloat16:
        q = q * size
    out, lse = attend(g, pool, q, seqs, 0.0)
    check(out, lse, exact(q, pool, g, 0, new_off, kv, page_off, table, 0.0), dt)


def test_append_and_attend_with_padding():
    """What an append leaves of a padded prompt's queries goes through the many-row kernel."""
    D, H, HQ = 128, 2, 8
    g = geom8(1, H, D, 16, 16)
    new, kv = [40, 90], [7, 60]
    seqs, new_off, page_off, table, num = batch(new, kv, 16)
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(sum(new), HQ + 2 * H, D, generator=gen, device=DEV).to(torch.bfloat16)
    q, k, v = x[:, :HQ], x[:, HQ:HQ + H], x[:, HQ + H:]
    pool = torch.zeros(2, num, g.page_bytes, dtype=torch.uint8, device=DEV)
    turned, out = torch.full_like(q, 3.0), torch.full_like(q, 4.0)
    with lsmkv.Context(g, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.append_batch(0, seqs, k, v, pt, q=q, q_out=turned)
        ctx.attend_batch(0, seqs, turned, out, pt, 0.1)
        assert ctx.last_status()["flags"] == 0
    assert not turned[:33].any() and not turned[40:70].any()
    assert not out[:33].any() and not out[40:70].any()
    check(out, None, exact(turned, pool, g, 0, new_off, kv, page_off, table, 0.1), torch.bfloat16)


# ---- exponents that grow by up to the whole range --------------------------------------------------

@pytest.mark.parametrize("rot", [0, 20])                     # 20: element by element
@pytest.mark.parametrize("grow", [126, 127, 128, 129, 160, 200])
@pytest.mark.parametrize("at_once", [False, True])
def test_a_begun_block_whose_exponent_grows_by_the_range(grow, rot, at_once):
    """Tokens of zeros and of the least size, then a large one: the codes of the earlier tokens become zeros."""
    D, H, B, P = 80, 2, 16, 16
    g = geom8(1, H, D, P, B)
    e = grow - 100
    k = torch.zeros(6, H, D, dtype=torch.bfloat16, device=DEV)
    k[1] = 300 * 2.0 ** -100
    k[2] = -448 * 2.0 ** -100
    k[3, 0] = 2.0 ** -105
    k[4] = 448.0 * 2.0 ** e
    k[5] = -3.5 * 2.0 ** (e + 2)
    pool = torch.full((2, 1, g.page_bytes), 0xFF, dtype=torch.uint8, device=DEV)
    tab = torch.cat([torch.ones(P, 10), torch.zeros(P, 10)], 1).to(DEV)          # turns nothing
    with lsmkv.Context(g, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        for a, b in ([(0, 4), (4, 6)] if at_once else [(t, t + 1) for t in range(6)]):
            seqs, *_ = batch([b - a], [b], P, spare=0)
            ctx.append_batch(0, seqs, k[a:b], k[a:b], pt, rope=lsmkv.Rope(tab) if rot else None)
            if b == 4:
                codes, scales = views(pool, g)
                assert (exponents(scales) == -100).all()
                # (300 is not a code; even neighbours lie at 288 and 320)
                want = (k[:4].double() * 2.0 ** 100).float().to(torch.float8_e4m3fn)
                assert torch.equal(codes[:, 0, :4].float(), want.float().expand(2, -1, -1, -1))
        assert ctx.last_status()["flags"] == 0
    codes, scales = views(pool, g)
    assert (exponents(scales) == e).all()
    got = codes[:, 0, :6].float()
    assert not got[:, :4].any()                                                 # (NaN would count)
    assert (got[:, 4] == 448).all() and (got[:, 5] == -14).all()


# ---- scales far apart ----------------------------------------------------------------------------

def raw_codes(pool, g):
    return pool[..., :g.code_bytes].unflatten(-1, (g.page_tokens, g.n_kv_heads, g.head_dim))


def spread_setup(dt, D, B, hq, hkv, new, hist, seed=0):
    kv = [a + b for a, b in zip(new, hist)]
    seqs, new_off, page_off, table, num = batch(new, kv, 16, seed)
    gen = torch.Generator(device=DEV).manual_seed(seed + 7)
    g = geom8(1, hkv, D, 16, B)
    pool = filled(g, num, gen)
    q = torch.randn(sum(new), hq, D, generator=gen, device=DEV).to(dt)
    return g, pool, q, seqs, new_off, kv, page_off, table, gen


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("up", [9, 20, 30, 40])
@pytest.mark.parametrize("new", [4, 5, 90, 300])
def test_rows_do_not_depend_on_tokens_behind_them(dt, up, new):
    """A late token far larger than the others, in its key, its value or both: the rows before it are what they are
    without it, whichever kernel takes them."""
    for B, hq, which in ((1, 8, (0, 1)), (1, 8, (0,)), (16, 8, (1,)), (1, 2, (0, 1))):
        g, pool, q, seqs, new_off, kv, page_off, table, gen = spread_setup(dt, 128, B, hq, 2, [new, 20], [500, 30])
        last = kv[0] - 1
        _, scales = views(pool, g)
        for x in which:
            # (a block of 16 holds tokens that the rows before see)
            scales[x, int(table[last // 16]), :, last % 16 // B] += min(up, 11) if B > 1 and dt == torch.float16 else up
        ref = exact(q, pool, g, 0, new_off, kv, page_off, table, 0.08)
        out, lse = attend(g, pool, q, seqs, 0.08)
        first = new - 1                                     # (the row that sees it has scores of any size)
        rows = [r for r in range(len(q)) if r != first]
        check(out, lse, ref, dt, rows)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("new", [1, 4, 5, 40, 300])
@pytest.mark.parametrize("B", [1, 16])
def test_a_large_value_that_hardly_weighs(dt, new, B):
    """An early token (or block) whose values are 2^23 times the others' and whose weight is nothing: what comes behind it keeps its bits.
    And the other way round, a token that weighs nearly everything and whose values are small."""
    for large in (True, False):
        g, pool, q, seqs, new_off, kv, page_off, table, gen = spread_setup(dt, 128, B, 8, 2, [new, 1], [3000, 300])
        codes, scales = raw_codes(pool, g), views(pool, g)[1]
        q[..., 0] = 16
        codes[0, ..., 0] = 0x66                            # 56
        for i in (0, 1):
            page = int(table[page_off[i]])
            codes[0, page, :B, :, 0] = 0xFE if large else 0x7E                      # 448, less or more than 200 nats away
            scales[0, page, :, 0] += 6
            scales[1, page, :, 0] += 23 if large else -23
        ref = exact(q, pool, g, 0, new_off, kv, page_off, table, 0.08)
        out, lse = attend(g, pool, q, seqs, 0.08)
        check(out, lse, ref, dt)


@pytest.mark.parametrize("case", [
    (torch.bfloat16, 128, 1, 8, 2, [300, 1, 40, 5], [900, 600, 100, 3]),
    (torch.float16, 128, 4, 16, 2, [33, 8, 17], [2000, 40, 129]),
    (torch.bfloat16, 64, 2, 8, 4, [70, 300], [3000, 5]),
    (torch.float16, 96, 1, 12, 4, [128, 30], [700, 0]),
    (torch.float16, 128, 1, 2, 2, [200], [6000]),
    (torch.bfloat16, 80, 8, 56, 8, [37, 90], [64, 700]),
    (torch.bfloat16, 128, 1, 8, 8, [150], [40000]),
], ids=range(7))
@pytest.mark.parametrize("span", [6, 12, 30])
def test_scales_far_apart_everywhere(case, span):
    """A scale drawn for every block, keys and values apart; bad weights or codes of any one key would show."""
    dt, D, B, hq, hkv, new, hist = case
    g, pool, q, seqs, new_off, kv, page_off, table, gen = spread_setup(dt, D, B, hq, hkv, new, hist)
    _, scales = views(pool, g)
    for x, top in ((0, 120), (1, 130)):
        scales[x] = torch.randint(top - span, top + 1, scales[x].shape, generator=gen, device=DEV).to(torch.uint8)
    ref = exact(q, pool, g, 0, new_off, kv, page_off, table, 0.08)
    out, lse = attend(g, pool, q, seqs, 0.08)
    check(out, lse, ref, dt)
    out, _ = attend(g, pool, q, seqs, -0.08)
    check(out, None, exact(q, pool, g, 0, new_off, kv, page_off, table, -0.08), dt)


@pytest.mark.parametrize("B", [1, 16])
def test_scales_far_apart_over_shared_prefixes(B):
    for dt, members, pages, new in ((torch.bfloat16, [6, 4], [9, 5], 5), (torch.float16, [33], [70], 1), (torch.float16, [3, 5], [20, 7], 30)):
        case = (dt, 128, 16, 16, 2, members, pages, new, (0, 30))
        g, pool, q, seqs, groups, new_off, kv, page_off, table = shared_setup(case, B)
        _, scales = views(pool, g)
        gen = torch.Generator(device=DEV).manual_seed(5)
        for x, top in ((0, 119), (1, 130)):
            scales[x] = torch.randint(top - 20, top + 1, scales[x].shape, generator=gen, device=DEV).to(torch.uint8)
        out, lse = attend(g, pool, q, seqs, 0.08, groups)
        check(out, lse, exact(q, pool, g, 0, new_off, kv, page_off, table, 0.08), dt)


def test_nan_beside_scales_far_apart():
    """An undefined value among blocks whose scales lie far apart reaches the rows that see it, and no others."""
    for new in (3, 70, 300):
        g, pool, q, seqs, new_off, kv, page_off, table, gen = spread_setup(torch.bfloat16, 128, 1, 8, 2, [new], [500])
        _, scales = views(pool, g)
        for x, top in ((0, 120), (1, 130)):
            scales[x] = torch.randint(top - 25, top + 1, scales[x].shape, generator=gen, device=DEV).to(torch.uint8)
        ref = exact(q, pool, g, 0, new_off, kv, page_off, table, 0.08)
        p = kv[0] - 2
        raw_codes(pool, g)[1, int(table[p // 16]), p % 16, :, 7] = 0x7F
        out = torch.zeros_like(q)
        with lsmkv.Context(g, 0) as ctx:
            ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08)
        check(out, None, ref, torch.bfloat16, slice(0, new - 2))
        assert torch.isnan(out[new - 2:, :, 7]).all() and torch.isfinite(out[:new - 2]).all()


@pytest.mark.parametrize("up", [5, 30, 45])
@pytest.mark.parametrize("new", [1, 40])
def test_zeros_ahead_of_large_values(new, up):
    """Blocks of zeros have the least exponent; their tokens weigh as much as others', whatever comes behind."""
    g, pool, q, seqs, new_off, kv, page_off, table, gen = spread_setup(torch.bfloat16, 128, 16, 8, 2, [new], [20000])
    codes, scales = raw_codes(pool, g), views(pool, g)[1]
    zero = torch.tensor(table[:1000], device=DEV)
    codes[1, zero] = 0
    scales[1, zero] = 27
    rest = torch.tensor(table[1000:], device=DEV)
    scales[1, rest] += up
    # the first keys fit worse than the others, by six nats
    q[..., 0] = 32
    codes[0, ..., 0] = 0x50                                # 8
    codes[0, torch.tensor(table[:8], device=DEV), :, :, 0] = 0xFA           # -320
    ref = exact(q, pool, g, 0, new_off, kv, page_off, table, 0.08)
    out, lse = attend(g, pool, q, seqs, 0.08)
    check(out, lse, ref, torch.bfloat16)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D,every", [(128, 30), (64, 17), (128, 9)])
def test_short_sequences_ahead_of_longer_ones(dt, D, every):
    """Row tiles that see one key tile give the second half of a CTA's rows nothing to do: it goes ahead to the next one that
    does, and takes that one's scales all the same."""
    n = 1500
    hist = [1000 if i % every == every - 1 else 60 + i % 60 for i in range(n)]
    g, pool, q, seqs, new_off, kv, page_off, table, gen = spread_setup(dt, D, 16, 8, 2, [5] * n, hist)
    _, scales = views(pool, g)
    scales += torch.randint(0, 6, scales.shape, generator=gen, device=DEV).to(torch.uint8)
    out, lse = attend(g, pool, q, seqs, D ** -0.5)
    check(out, lse, exact(q, pool, g, 0, new_off, kv, page_off, table, D ** -0.5), dt)
