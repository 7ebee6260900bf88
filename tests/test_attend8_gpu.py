"""lsmkv_attend_batch and lsmkv_attend_shared_batch on 8-bit pools against softmax attention in 64 bits
over the values that the codes stand for.

Tolerance of o = sum w v, A = sum w |v|: u |o| for the rounding of the result (2^-8 bfloat16, 2^-11 float16,
half the smallest subnormal more); for the weights, rounded to the type that meets the codes, u A; 2^-12 A for the 32-bit
arithmetic of the scores, as on 16-bit pools. Rounded weights are relative to the largest w * 2^(exponent of the
value's block); below 2^-14 of it they are subnormal, off by 2^-25 each, and the block's largest value is over half of 448 2^exponent:
n 2^-24 max |v| more."""
import math

import numpy as np
import pytest
import torch

from paper_2511_16138_b200 import lsmkv
from pool8 import DEV, filled, geom8, values, views
from test_append_gpu import U, batch
from test_attend_gpu import SHARED, reference

pytestmark = pytest.mark.gpu


def check(out, lse, ref, dt):
    o, A, want_lse, sub = ref                    # sub: n 2^-25 max |v|
    tol = U[dt] * (o.abs() + A) + 2.0 ** -12 * A + 2 * sub
    if dt == torch.float16:
        tol = tol + 2.0 ** -25
    fine = torch.isfinite(o)
    assert torch.equal(fine, torch.isfinite(out))
    err = (out.double() - o).abs()
    bad = (err > tol) & fine
    assert not bad.any(), (int(bad.sum()), float(err[fine].max()), bad.nonzero()[:4].tolist())
    if lse is not None:
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isneginf(lse), empty)
        d = (lse.double() - want_lse).abs()[~empty]
        assert not d.numel() or bool((d <= 2.0 ** -12 + 2.0 ** -21 * want_lse[~empty].abs()).all()), float(d.max())


def garbage_beyond(pool, g, layer, kv, page_off, table):
    """NaN codes and scales of 255 behind every sequence's last token and in unused pages."""
    P, B = g.page_tokens, g.block_tokens
    codes, scales = views(pool, g)
    raw = pool[..., :g.code_bytes].unflatten(-1, codes.shape[2:])
    unused = torch.ones(pool.shape[1], dtype=torch.bool, device=DEV)
    unused[torch.tensor(table, device=DEV).long()] = False
    for b in (layer, g.n_layers + layer):
        pool[b, unused] = 0xFF
        for i, n in enumerate(kv):
            if n % P:
                pg = int(table[page_off[i + 1] - 1])
                raw[b, pg, n % P:] = 0x7F if i % 2 else 0xFF
                scales[b, pg, :, (n % P + B - 1) // B:] = 255


CASES = [
    # dtype, D, P, B, hq, hkv, new, history
    (torch.bfloat16, 128, 16, 16, 32, 8, [1] * 8, [0, 1, 14, 15, 16, 63, 64, 1000]),
    (torch.float16, 128, 64, 1, 28, 4, [1] * 6, [62, 63, 64, 127, 128, 5000]),
    (torch.bfloat16, 64, 16, 4, 4, 4, [1, 2, 3, 16, 17], [0, 3, 500, 40, 99]),
    (torch.float16, 64, 16, 16, 40, 8, [1, 3, 1, 4], [0, 700, 33, 20]),
    (torch.bfloat16, 96, 5, 1, 6, 2, [1, 5, 6, 0, 20], [9, 0, 33, 44, 3]),
    (torch.float16, 96, 24, 8, 6, 2, [1, 5, 6, 0, 20, 300], [9, 0, 33, 44, 3, 50]),
    (torch.bfloat16, 256, 16, 16, 8, 2, [1, 4, 90], [300, 0, 50]),
    (torch.float16, 256, 32, 8, 16, 1, [1, 1, 33], [300, 0, 130]),
    (torch.float16, 208, 16, 2, 3, 3, [1, 40], [100, 100]),
    (torch.bfloat16, 16, 16, 16, 5, 1, [1, 9], [100, 0]),
    (torch.bfloat16, 128, 1, 1, 8, 8, [1, 30], [70, 3]),
    (torch.bfloat16, 128, 16, 16, 16, 1, [1, 1], [3000, 17]),
    (torch.float16, 128, 16, 8, 20, 1, [1, 2], [300, 17]),
    (torch.bfloat16, 128, 16, 16, 64, 1, [1, 2, 70], [300, 17, 1]),
    (torch.bfloat16, 128, 16, 16, 32, 8, [65, 1, 128, 129, 2], [0, 900, 31, 300, 64]),
    (torch.float16, 128, 16, 1, 16, 16, [200, 257], [0, 1]),
    (torch.bfloat16, 128, 16, 16, 56, 8, [37, 300], [64, 700]),
    (torch.float16, 64, 64, 16, 8, 2, [512, 31], [0, 2000]),
    (torch.bfloat16, 128, 24, 4, 8, 2, [100], [4000]),
    (torch.bfloat16, 64, 16, 2, 64, 4, [33, 1], [9, 5]),
    (torch.bfloat16, 128, 16, 16, 4, 1, [1], [40000]),
    (torch.float16, 128, 16, 16, 8, 1, [40], [20000]),
    (torch.bfloat16, 128, 16, 16, 8, 2, [1, 33, 70, 2, 150, 0, 4, 5] * 40, [300, 0, 90, 1000, 40, 7, 16, 31] * 40),
    # heads side by side, eight, four and two at a time; tiles cut by the spans' ends
    (torch.bfloat16, 128, 16, 16, 32, 8, [1] * 60, [1000 + 37 * i for i in range(60)]),
    (torch.float16, 96, 16, 4, 16, 8, [1, 2, 8, 0, 3] * 20, [5, 700, 64, 9, 2000] * 20),
    (torch.bfloat16, 64, 32, 8, 36, 12, [1, 1, 5] * 30, [0, 1500, 33] * 30),
    (torch.float16, 128, 8, 8, 18, 6, [1] * 70, [31 * i for i in range(70)]),
    (torch.bfloat16, 128, 16, 16, 56, 8, [1, 2] * 30, [400, 3000] * 30),
    (torch.bfloat16, 32, 16, 1, 24, 8, [1] * 90, [17 * i for i in range(90)]),
    # one long sequence among many that another kernel takes
    (torch.bfloat16, 128, 16, 16, 32, 8, [1] + [40] * 30, [9000] + [10 * i for i in range(30)]),
    (torch.float16, 48, 16, 8, 12, 4, [20, 1, 300], [77, 800, 0]),
]


def setup(case, seed=0, n_layers=2):
    dt, D, P, B, hq, hkv, new, hist = case
    kv = [a + b for a, b in zip(new, hist)]
    seqs, new_off, page_off, table, num = batch(new, kv, P, seed)
    gen = torch.Generator(device=DEV).manual_seed(seed + 11)
    g = geom8(n_layers, hkv, D, P, B)
    # blocks of different size: exponents differ from token to token
    pool = filled(g, num, gen, torch.exp2(torch.randint(-1, 2, (num, P, 1, 1), generator=gen, device=DEV).float()))
    q = torch.randn(int(new_off[-1]), hq, D, generator=gen, device=DEV).to(dt)
    return g, pool, q, seqs, new_off, kv, page_off, table


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attend_equals_softmax_attention(case):
    dt, D, P = case[:3]
    g, pool, q, seqs, new_off, kv, page_off, table = setup(case)
    layer, scale = 1, D ** -0.5
    garbage_beyond(pool, g, layer, kv, page_off, table)
    ref = reference(q, values(pool, g), layer, 2, new_off, kv, page_off, table, P, scale)
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(g, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.attend_batch(layer, seqs, q, out, pt, scale, lse)
        assert ctx.last_status()["flags"] == 0
        check(out, lse, ref, dt)
        # the same bits again, into the queries' own rows, and without the statistics
        same = q.clone()
        ctx.attend_batch(layer, seqs, same, same, pt, scale)
        assert ctx.last_status()["flags"] == 0
        assert torch.equal(same.view(torch.int16), out.view(torch.int16))
        # a negative scale
        ctx.attend_batch(layer, seqs, q, out, pt, -scale)
        check(out, None, reference(q, values(pool, g), layer, 2, new_off, kv, page_off, table, P, -scale), dt)


def test_padding_rows_and_empty_sequences_are_zero():
    case = (torch.bfloat16, 128, 16, 16, 8, 2, [3, 1, 40, 2, 90], [0] * 5)
    dt, D, P, B, hq, hkv, new, _ = case
    kv = [1, 0, 7, 2, 0]
    seqs, new_off, page_off, table, num = batch(new, kv, P)
    gen = torch.Generator(device=DEV).manual_seed(1)
    g = geom8(1, hkv, D, P, B)
    pool = filled(g, num, gen)
    q = torch.randn(sum(new), hq, D, generator=gen, device=DEV).to(dt)
    out, lse = torch.full_like(q, 3.0), torch.zeros(q.shape[:2], device=DEV)
    with lsmkv.Context(g, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.1, lse)
        assert ctx.last_status()["flags"] == 0
    for i, (a, n) in enumerate(zip(new_off, new)):
        hidden = n - min(kv[i], n)
        assert not out[a:a + hidden].any() and torch.isneginf(lse[a:a + hidden]).all()
    check(out, lse, reference(q, values(pool, g), 0, 1, new_off, kv, page_off, table, P, 0.1), dt)


@pytest.mark.parametrize("new", [2, 3, 4, 70, 300])
@pytest.mark.parametrize("at", [-1, -3, 0])
def test_nan_codes_reach_the_rows_that_see_them(new, at):
    """One new token's value holds a NaN in one element of one head; its key in another head."""
    case = (torch.bfloat16, 128, 16, 16, 8, 2, [new, 2], [50, 30])
    g, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    p = kv[0] + at if at < 0 else kv[0] - new
    raw = pool[..., :g.code_bytes].unflatten(-1, (16, 2, 128))
    raw[1, int(table[p // 16]), p % 16, 0, 4] = 0x7F
    raw[0, int(table[p // 16]), p % 16, 1, 7] = 0xFF
    out = torch.zeros_like(q)
    ref = reference(q, values(pool, g), 0, 1, new_off, kv, page_off, table, 16, 0.08)
    with lsmkv.Context(g, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08)
    first = p - (kv[0] - new)                              # the first row that sees it
    first = max(first, 0)
    clean = torch.ones(len(q), dtype=torch.bool, device=DEV)
    clean[first:new] = False
    check(out[clean], None, tuple(x[clean] for x in ref), torch.bfloat16)
    seen = out[first:new].float()
    assert torch.isnan(seen[:, :4, 4]).all() and torch.isnan(seen[:, 4:]).all()
    rest = torch.cat([seen[:, :4, :4], seen[:, :4, 5:]], -1)
    assert torch.isfinite(rest).all()


def test_scales_of_any_size():
    """Values from 2^-90 to 2^90 beside each other, keys of both sizes, blocks of zeros, large queries."""
    case = (torch.float16, 64, 16, 4, 8, 2, [1, 1, 20, 1], [200, 60, 33, 3])
    g, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    codes, scales = views(pool, g)
    gen = torch.Generator(device=DEV).manual_seed(4)
    scales[1] = torch.randint(127 - 90, 127 + 4, scales[1].shape, generator=gen, device=DEV).to(torch.uint8)
    codes[1, ::3, 4:8] = 0                                  # blocks of zeros, with the least exponent
    scales[1, ::3, :, 1] = 27
    q = q.to(torch.bfloat16) * 2.0 ** 70
    scales[0] = (scales[0].long() - 70).to(torch.uint8)     # scores of ordinary size
    out = torch.zeros_like(q)
    with lsmkv.Context(g, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.125)
        assert ctx.last_status()["flags"] == 0
        ref = reference(q, values(pool, g), 0, 1, new_off, kv, page_off, table, 16, 0.125)
        check(out, None, ref, torch.bfloat16)
        # all values huge
        scales[1] = 127 + 90
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.125)
        ref = reference(q, values(pool, g), 0, 1, new_off, kv, page_off, table, 16, 0.125)
        check(out, None, ref, torch.bfloat16)
        # all values zero
        scales[1] = 27
        codes[1] = 0
        lse = torch.zeros(q.shape[:2], device=DEV)
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.125, lse)
        assert not out.any()
        d = (lse.double() - ref[2]).abs()
        assert bool((d <= 2.0 ** -12 + 2.0 ** -21 * ref[2].abs()).all())


def test_strided_rows_and_streams():
    case = (torch.float16, 64, 16, 16, 8, 4, [1, 50], [200, 100])
    g, pool, q0, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    n = q0.shape[0]
    wide = torch.full((n, 20, 80), 9.0, dtype=torch.float16, device=DEV)
    wide[:, 2:10, 8:72] = q0
    dst = torch.full((8, n, 72), 4.0, dtype=torch.float16, device=DEV)
    q, out = wide[:, 2:10, 8:72], dst.transpose(0, 1)[..., :64]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ref = reference(q, values(pool, g), 0, 1, new_off, kv, page_off, table, 16, 0.125)
    with lsmkv.Context(g, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            ctx.attend_batch(0, seqs, q, out, pt, 0.125, stream=s)
        s.synchronize()
        check(out, None, ref, torch.float16)
        assert (dst[..., 64:] == 4.0).all()


def test_offsets_beyond_32_bits():
    """Pages at the far end of a buffer of more than 2^32 bytes; K and V in one buffer."""
    D, P, B, hkv, hq = 128, 16, 16, 8, 16
    g = geom8(1, hkv, D, P, B)
    num = 2 ** 32 // g.page_bytes + 40
    pool = torch.zeros(1, num, g.page_bytes, dtype=torch.uint8, device=DEV)
    new, kv = [1, 40], [100, 300]
    seqs, new_off, page_off, table, small = batch(new, kv, P)
    gen = torch.Generator(device=DEV).manual_seed(2)
    some = filled(g, small, gen)[:1]
    pool[:, num - small:] = some
    seqs.keep[3].copy_(torch.tensor(table + (num - small), dtype=torch.int32))
    q = torch.randn(41, hq, D, device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(q)
    with lsmkv.Context(g, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table([pool[0], pool[0]]), 0.1)
        assert ctx.last_status()["flags"] == 0
        # and an append there
        rows = torch.randn(41, 2 * hkv, D, device=DEV).to(torch.bfloat16)
        both = pool.expand(2, -1, -1)
        check(out, None, reference(q, values(some.expand(2, -1, -1), g), 0, 1, new_off, kv, page_off, table, P, 0.1),
              torch.bfloat16)
        ctx.append_batch(0, seqs, rows[:, hkv:], rows[:, hkv:], lsmkv.pool_table([pool[0], pool[0]]))
        assert ctx.last_status()["flags"] == 0
    assert both.shape[0] == 2 and not pool[0, :num - small].any()


def test_bad_sequences_and_pages():
    case = (torch.bfloat16, 128, 16, 16, 8, 2, [1, 1, 1, 60], [40, 50, 60, 3])
    g, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    with lsmkv.Context(g, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        for entry in (int(page_off[1]) + 1, int(page_off[3])):
            zero = pool.clone()
            zero[:, int(table[entry]), :g.code_bytes] = 0
            seqs.keep[3][entry] = pool.shape[1]
            out = torch.zeros_like(q)
            ctx.attend_batch(0, seqs, q, out, pt, 0.1)
            st = ctx.last_status()
            assert st["flags"] == lsmkv.ST_BAD_PAGE and st["first_bad"] == entry
            check(out, None, reference(q, values(zero, g), 0, 1, new_off, kv, page_off, table, 16, 0.1), torch.bfloat16)
            seqs.keep[3][entry] = int(table[entry])
        seqs.keep[1][2] = 500
        out = torch.full_like(q, 8.0)
        ctx.attend_batch(0, seqs, q, out, pt, 0.1)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 2 and (out[2] == 8.0).all()
        seqs.keep[1][2] = kv[2]
        ref = reference(q, values(pool, g), 0, 1, new_off, kv, page_off, table, 16, 0.1)
        ok = torch.tensor([r for r in range(len(q)) if r != 2], device=DEV)
        check(out[ok], None, tuple(x[ok] for x in ref), torch.bfloat16)
        off = torch.tensor([pool[0].data_ptr() + 8, pool[1].data_ptr()], device=DEV)
        out.fill_(8.0)
        ctx.attend_batch(0, seqs, q, out, (off, pool.shape[1] - 1), 0.1)
        assert ctx.last_status()["flags"] == lsmkv.ST_MISALIGNED and (out == 8.0).all()


def shared_setup(case, B, seed=0):
    dt, D, P, hq, hkv, members, pages, new, own = case
    rng = np.random.default_rng(seed)
    shared = np.repeat(pages, members)
    n = len(shared)
    kv = [int(s) * P + new + int(rng.integers(own[0], own[1] + 1)) for s in shared]
    seqs, new_off, page_off, table, num = batch([new] * n, kv, P, seed)
    off = np.cumsum([0] + members)
    for k, m in enumerate(members):
        for i in range(off[k] + 1, off[k] + m):
            table[page_off[i]:page_off[i] + pages[k]] = table[page_off[off[k]]:page_off[off[k]] + pages[k]]
    seqs.keep[3].copy_(torch.tensor(table, dtype=torch.int32))
    gen = torch.Generator(device=DEV).manual_seed(seed + 5)
    g = geom8(1, hkv, D, P, B)
    pool = filled(g, num, gen)
    q = (2 * torch.randn(n * new, hq, D, generator=gen, device=DEV)).to(dt)
    groups = lsmkv.Groups(torch.tensor(off, dtype=torch.int32, device=DEV),
                          torch.tensor(pages, dtype=torch.int32, device=DEV))
    return g, pool, q, seqs, groups, new_off, kv, page_off, table


@pytest.mark.parametrize("case", SHARED, ids=[str(i) for i in range(len(SHARED))])
@pytest.mark.parametrize("B", [1, 16])
def test_shared_prefixes(case, B):
    dt, D, P = case[:3]
    g, pool, q, seqs, groups, new_off, kv, page_off, table = shared_setup(case, B)
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(g, 0) as ctx:
        ctx.attend_shared_batch(0, seqs, groups, q, out, lsmkv.pool_table(list(pool)), D ** -0.5, lse)
        assert ctx.last_status()["flags"] == 0
    check(out, lse, reference(q, values(pool, g), 0, 1, new_off, kv, page_off, table, P, D ** -0.5), dt)


def test_captured_calls_replay_over_new_tokens():
    """Append and attend of a step captured once; replays follow the lengths on the device."""
    D, P, B, H, HQ, n = 128, 16, 16, 4, 16, 6
    g = geom8(1, H, D, P, B)
    room = 6
    seqs, new_off, page_off, table, num = batch([1] * n, [room * P] * n, P)
    gen = torch.Generator(device=DEV).manual_seed(6)
    pool = filled(g, num, gen)
    pt = lsmkv.pool_table(list(pool))
    x = torch.zeros(n, HQ + 2 * H, D, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(n, HQ, D, dtype=torch.bfloat16, device=DEV)
    turned = torch.zeros_like(out)
    rope = lsmkv.Rope(torch.cat([torch.ones(room * P, D // 2), torch.zeros(room * P, D // 2)], 1).to(DEV))

    with lsmkv.Context(g, 0) as ctx, lsmkv.Context(g, 0) as other:
        def step(c):
            c.append_batch(0, seqs, x[:, HQ:HQ + H], x[:, HQ + H:], pt, rope=rope, q=x[:, :HQ], q_out=turned)
            c.attend_batch(0, seqs, turned, out, pt, 0.1)

        step(ctx)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
            step(ctx)
        big = batch([1] * 900, [5] * 900, P)[0]                         # the scratch is replaced by a larger one
        ctx.attend_batch(0, big, torch.zeros(900, HQ, D, dtype=torch.bfloat16, device=DEV),
                         torch.zeros(900, HQ, D, dtype=torch.bfloat16, device=DEV), (pt[0], num), 0.1)
        for length in (17, 18, 40, 96):
            seqs.keep[1].fill_(length)
            x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
            before = pool.clone()
            graph.replay()
            torch.cuda.synchronize()
            got, after = out.clone(), pool.clone()
            pool.copy_(before)
            step(other)
            torch.cuda.synchronize()
            assert torch.equal(after, pool) and torch.equal(got, out)
            ref = reference(turned, values(pool, g), 0, 1, new_off, [length] * n, page_off, table, P, 0.1)
            check(out, None, ref, torch.bfloat16)
        ctx.last_status()


def test_a_wait_that_runs_out_is_reported():
    """A key tile of the first CTA never arrives: the many-row kernel gives up after the limit and says so."""
    case = (torch.bfloat16, 128, 16, 16, 16, 2, [200], [4000])
    g, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    out = torch.zeros_like(q)
    with lsmkv.Context(g, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.set_tuning("wait_cycles", 1000000)
        ctx.set_tuning("test_drop_piece", 2)
        ctx.attend_batch(0, seqs, q, out, pt, 0.1)
        assert ctx.last_status()["flags"] == lsmkv.ST_WAIT_EXPIRED
        ctx.set_tuning("test_drop_piece", -1)
        ctx.set_tuning("wait_cycles", 2000000000)
        ctx.attend_batch(0, seqs, q, out, pt, 0.1)
        assert ctx.last_status()["flags"] == 0
    check(out, None, reference(q, values(pool, g), 0, 1, new_off, kv, page_off, table, 16, 0.1), torch.bfloat16)
