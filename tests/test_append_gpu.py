"""lsmkv_append_batch against its formulas in 64 bits.

Tolerance: the kernel computes in 32 bits and rounds once, so a result y made of a and b is off by
at most u |y| (u: half of the type's epsilon, 2^-8 for bfloat16, 2^-11 for float16) for the
rounding, a few 2^-22 of |a| + |b| for the arithmetic (rsqrt and the two products), and half
the smallest subnormal of float16."""
import numpy as np
import pytest
import torch

from paper_2511_16138_b200 import lsmkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {dt: torch.finfo(dt).eps / 2 for dt in (torch.bfloat16, torch.float16)}


def batch(new, kv, P, seed=0, spare=3):
    """Seqs over pages in random order, its pieces on the host, and the number of pages."""
    rng = np.random.default_rng(seed)
    counts = [-(-b // P) for b in kv]
    num = sum(counts) + spare
    table = rng.permutation(num)[:sum(counts)]
    new_off, page_off = np.cumsum([0] + list(new)), np.cumsum([0] + counts)
    t = lambda a, d: torch.tensor(np.asarray(a), dtype=d, device=DEV)  # noqa: E731
    seqs = lsmkv.Seqs(t(new_off, torch.int64), t(kv, torch.int32), t(page_off, torch.int64),
                      t(table if len(table) else [0], torch.int32), int(new_off[-1]),
                      max(list(new) + [1]))
    return seqs, new_off, page_off, table, num


def rope_table(n, rot, seed=1):
    g = torch.Generator().manual_seed(seed)
    ang = torch.rand(n, rot // 2, generator=g, dtype=torch.float64) * 6.3
    return torch.cat([ang.cos(), ang.sin()], 1).float().to(DEV)


def formula(x, w, table, pos, rot, interleaved, eps):
    """(y, |a| + |b|) of rows x [t, heads, D] in 64 bits."""
    x = x.double()
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    size = x.abs()
    if table is None:
        return x, size
    c, s = table.double()[pos, None, :rot // 2], table.double()[pos, None, rot // 2:]
    ia = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    ib = ia + 1 if interleaved else ia + rot // 2
    y, a, b = x.clone(), x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    size = size.clone()
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return y, size


def check(got, want, size, dt):
    tol = U[dt] * want.abs() + 4 * 2.0 ** -22 * size + (2.0 ** -25 if dt == torch.float16 else 0)
    bad = ((got.double() - want).abs() > tol)
    assert not bad.any(), (int(bad.sum()), float((got.double() - want).abs().max()))


CASES = [
    # dtype, D, rot, interleaved, qn, kn, P, hq, hkv, new, extra history
    (torch.bfloat16, 128, 128, False, False, False, 16, 32, 8, [1] * 9, [0, 1, 15, 16, 17, 31, 100, 5, 1000]),
    (torch.float16, 128, 128, False, True, True, 64, 28, 4, [1, 300, 0, 17, 64], [0, 5, 9, 63, 64]),
    (torch.bfloat16, 64, 64, True, True, False, 16, 8, 8, [40, 1, 1], [0, 16, 3]),
    (torch.float16, 64, 32, False, False, True, 16, 4, 2, [33], [7]),
    (torch.bfloat16, 96, 96, False, True, True, 5, 6, 3, [12, 7], [2, 11]),
    (torch.bfloat16, 96, 48, False, True, True, 16, 6, 3, [12, 7], [2, 11]),
    (torch.float16, 256, 256, False, True, True, 1, 4, 1, [3, 5], [0, 2]),
    (torch.bfloat16, 256, 64, True, False, False, 16, 4, 2, [20], [0]),
    (torch.bfloat16, 80, 20, False, True, True, 16, 5, 5, [9, 2], [1, 30]),     # element form
    (torch.float16, 80, 20, True, True, False, 16, 5, 1, [9, 2], [1, 30]),      # element form
    (torch.bfloat16, 72, 72, False, False, False, 16, 3, 3, [4], [3]),          # element form
    (torch.float16, 8, 8, True, True, True, 16, 3, 1, [50], [0]),
    (torch.bfloat16, 8, 2, False, True, True, 16, 3, 1, [50], [0]),
    (torch.bfloat16, 128, 0, False, True, True, 16, 8, 2, [5, 6], [0, 3]),      # norm alone
    (torch.float16, 128, 0, False, False, False, 16, 8, 2, [5, 6], [0, 3]),     # bit copies
    (torch.bfloat16, 128, 128, False, True, True, 16, 0, 8, [70, 1], [0, 3]),   # no queries
    (torch.bfloat16, 128, 128, False, False, False, 16, 64, 8, [5000, 3], [3, 0]),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_equals_its_formulas(case, in_place):
    dt, D, rot, inter, qn, kn, P, hq, hkv, new, hist = case
    kv = [a + b for a, b in zip(new, hist)]
    seqs, new_off, page_off, table, num = batch(new, kv, P)
    g = torch.Generator(device=DEV).manual_seed(3)
    n = int(new_off[-1])
    qkv = torch.randn(n, hq + 2 * hkv, D, generator=g, device=DEV).to(dt)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    q_w = (1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(dt) if qn else None
    k_w = (1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(dt) if kn else None
    tab = rope_table(max(kv), rot) if rot else None
    geom = lsmkv.Geom(2, hkv, D, page_tokens=P, chunk_tokens=P)
    pool = torch.randn(4, num, P, hkv, D, generator=g, device=DEV).to(dt)
    before, q_before = pool.clone(), q.clone()
    layer = 1
    pos = torch.cat([torch.arange(b - a, b) for a, b in zip(new, kv)]).to(DEV)
    with lsmkv.Context(geom, 0) as ctx:
        q_out = q if in_place else torch.full((n, hq, D), 7.0, dtype=dt, device=DEV)
        ctx.append_batch(layer, seqs, k, v, lsmkv.pool_table(list(pool)),
                         rope=lsmkv.Rope(tab, inter) if rot else None, q=q if hq else None,
                         q_out=q_out if hq else None, q_norm=q_w if hq else None, k_norm=k_w,
                         eps=1e-5)
        assert ctx.last_status()["flags"] == 0
    if hq:
        check(q_out, *formula(q_before, q_w, tab, pos, rot, inter, 1e-5), dt)
    seq = np.repeat(np.arange(len(new)), new)
    page = torch.tensor(table[page_off[seq] + pos.cpu().numpy() // P], device=DEV)
    slot = pos % P
    got_k, got_v = pool[layer, page, slot], pool[2 + layer, page, slot]
    if rot or kn:
        check(got_k, *formula(k, k_w, tab, pos, rot, inter, 1e-5), dt)
    else:
        assert torch.equal(got_k.view(torch.int16), k.contiguous().view(torch.int16))
    assert torch.equal(got_v.view(torch.int16), v.contiguous().view(torch.int16))
    # nothing else in the pool changed
    pool[layer, page, slot], pool[2 + layer, page, slot] = before[layer, page, slot], before[2 + layer, page, slot]
    assert torch.equal(pool.view(torch.int16), before.view(torch.int16))


def test_rotation_by_given_positions_padding_and_special_values():
    """Own positions for the angle; padding rows store nothing and zero their queries; values and
    the elements behind the rotation keep infinities, NaN and signed zeros bit for bit."""
    dt, D, rot, P, hq, hkv = torch.bfloat16, 64, 32, 16, 4, 2
    seqs, new_off, page_off, table, num = batch([6, 3], [4, 3], P)      # two padding tokens ahead
    n = 9
    g = torch.Generator(device=DEV).manual_seed(5)
    q, k, v = (torch.randn(n, h, D, generator=g, device=DEV).to(dt) for h in (hq, hkv, hkv))
    odd = torch.tensor([np.inf, -np.inf, np.nan, -0.0], device=DEV, dtype=dt)
    k[..., rot:rot + 4], v[..., :4] = odd, odd
    tab = rope_table(50, rot)
    where = torch.randint(0, 50, (n,), device=DEV, dtype=torch.int32)
    pool = torch.zeros(2, num, P, hkv, D, dtype=dt, device=DEV)
    q_out = torch.full_like(q, 9.0)
    with lsmkv.Context(lsmkv.Geom(1, hkv, D, page_tokens=P, chunk_tokens=P), 0) as ctx:
        ctx.append_batch(0, seqs, k, v, lsmkv.pool_table(list(pool)),
                         rope=lsmkv.Rope(tab, False, where), q=q, q_out=q_out)
        assert ctx.last_status()["flags"] == 0
    assert not q_out[:2].any()
    real = torch.arange(2, 9, device=DEV)
    check(q_out[real], *formula(q[real], None, tab, where[real].long(), rot, False, 0), dt)
    for t in range(2, 9):
        page, slot = (table[0], t - 2) if t < 6 else (table[page_off[1]], t - 6)
        assert torch.equal(pool[1, page, slot].view(torch.int16), v[t].view(torch.int16))
        assert torch.equal(pool[0, page, slot, :, rot:].view(torch.int16), k[t, :, rot:].view(torch.int16))
    assert int((pool[1].view(torch.int16) != 0).any(-1).any(-1).sum()) == 7


def test_append_reports_what_it_leaves_out():
    dt, D, P, hkv = torch.float16, 64, 16, 2
    seqs, new_off, page_off, table, num = batch([2, 2, 2], [2, 20, 40], P)
    k = torch.ones(6, hkv, D, dtype=dt, device=DEV)
    pool = torch.zeros(2, num, P, hkv, D, dtype=dt, device=DEV)
    with lsmkv.Context(lsmkv.Geom(1, hkv, D, page_tokens=P, chunk_tokens=P), 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        seqs.keep[3][int(page_off[1]) + 1] = num                       # page of tokens 18, 19
        ctx.append_batch(0, seqs, k, k, pt)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_PAGE and st["first_bad"] == int(page_off[1]) + 1
        assert int((pool[0, :, :, 0, 0] != 0).sum()) == 4
        pool.zero_()
        seqs.keep[1][2] = 33 + 16                                      # more than its pages hold
        ctx.append_batch(0, seqs, k, k, pt, rope=lsmkv.Rope(rope_table(19, D)))
        st = ctx.last_status()                                         # and token 3 past the table
        assert st["flags"] == lsmkv.ST_BAD_PAGE | lsmkv.ST_BAD_COUNT and st["first_bad"] == 2
        assert int((pool[0, :, :, 0] != 0).any(-1).sum()) == 2
        # a buffer off its boundary: nothing is done
        pool.zero_()
        buf = torch.zeros(pool[0].numel() + 8, dtype=dt, device=DEV)
        off = torch.tensor([buf.data_ptr() + 2, pool[1].data_ptr()], device=DEV)
        ctx.append_batch(0, seqs, k, k, (off, num))
        assert ctx.last_status()["flags"] & lsmkv.ST_MISALIGNED
        assert not buf.any() and not pool.any()


def test_append_refusals():
    dt, D, hkv = torch.bfloat16, 64, 2
    seqs, *_, num = batch([2], [2], 16)
    k = torch.zeros(2, hkv, D, dtype=dt, device=DEV)
    pool = torch.zeros(2, num, 16, hkv, D, dtype=dt, device=DEV)
    pt = lsmkv.pool_table(list(pool))

    def refused(ctx, code=lsmkv.EINVAL, seqs=seqs, layer=0, k=k, **kw):
        with pytest.raises(lsmkv.LsmkvError) as e:
            ctx.append_batch(layer, seqs, k, k, pt, **kw)
        assert e.value.code == code

    with lsmkv.Context(lsmkv.Geom(1, hkv, D, page_tokens=16, chunk_tokens=16), 0) as ctx:
        refused(ctx, layer=1)
        flat = torch.zeros(2 * hkv * D + 8, dtype=dt, device=DEV)
        refused(ctx, k=flat[1:1 + 2 * hkv * D].view(2, hkv, D))                # off a boundary
        refused(ctx, k=torch.zeros(2, hkv, D + 4, dtype=dt, device=DEV)[..., :D])   # odd stride
        refused(ctx, rope=lsmkv.Rope(rope_table(4, D + 2)))
        refused(ctx, k_norm=torch.ones(D, dtype=dt, device=DEV), eps=-1.0)
        for bad in (dict(k=k.float()), dict(k=k[:1]), dict(k=k[:, :1]), dict(k=k[..., ::2]),
                    dict(q=k, q_out=k.half()), dict(k_norm=torch.ones(D - 1, dtype=dt, device=DEV)),
                    dict(rope=lsmkv.Rope(rope_table(4, D), positions=torch.zeros(3, dtype=torch.int32)))):
            with pytest.raises((TypeError, ValueError)):
                a = dict(k=k) | bad
                ctx.append_batch(0, seqs, a.pop("k"), k, pt, **a)
        empty = lsmkv.Seqs(*seqs.keep, 0, 1)
        ctx.append_batch(0, empty, k[:0], k[:0], pt)                            # nothing to do
        assert ctx.last_status()["flags"] == 0 and not pool.any()
    for geom in (lsmkv.Geom(1, hkv, D, elem_bytes=4), lsmkv.Geom(1, hkv, 260), lsmkv.Geom(1, hkv, 264)):
        with lsmkv.Context(geom, 0) as ctx:
            refused(ctx, k=torch.zeros(2, hkv, geom.head_dim, dtype=dt, device=DEV))
