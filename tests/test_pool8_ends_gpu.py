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
