"""lsmkv_attend_batch and lsmkv_attend_shared_batch against softmax attention in 64 bits.

Tolerance of an output o = sum w v, per element, with A = sum w |v| (u: half of the type's
epsilon, 2^-8 for bfloat16, 2^-11 for float16): u |o| for the rounding of the result, u A for the
rounding of the weights, and 2^-12 A for the 32-bit arithmetic -- a score is a sum of at most 256
products in 32 bits, off by less than 2^-13 where sum |q k| scale < 2^4, and the weights follow it
to first order. float16 weights below 2^-14 of the largest are subnormal: n 2^-25 max |v| more, and
half the smallest subnormal for the result. A log-sum-exp is off by no more than its scores,
2^-12, and 2^-21 of its size."""
import math

import numpy as np
import pytest
import torch

from paper_2511_16138_b200 import lsmkv
from test_append_gpu import DEV, U, batch

pytestmark = pytest.mark.gpu


def reference(q, pool, layer, n_layers, new_off, kv, page_off, table, P, scale):
    """o, A, lse, weight slack [n, hq, D] in 64 bits; rows without keys are 0 and -inf."""
    n, hq, D = q.shape
    hkv = pool.shape[3]
    o = torch.zeros(n, hq, D, dtype=torch.float64, device=DEV)
    A, sub = torch.zeros_like(o), torch.zeros_like(o)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=DEV)
    for i in range(len(kv)):
        a, b = int(new_off[i]), int(new_off[i + 1])
        if a == b or kv[i] == 0:
            continue
        pages = torch.tensor(table[page_off[i]:page_off[i + 1]], device=DEV)
        k = pool[layer, pages].flatten(0, 1)[:kv[i]].double()
        v = pool[n_layers + layer, pages].flatten(0, 1)[:kv[i]].double()
        k, v = (x.repeat_interleave(hq // hkv, 1) for x in (k, v))
        s = torch.einsum("thd,jhd->htj", q[a:b].double(), k) * scale
        p = kv[i] - (b - a) + torch.arange(b - a, device=DEV)
        hidden = torch.arange(kv[i], device=DEV)[None] > p[:, None]
        s = s.masked_fill(hidden, -math.inf)
        w = torch.exp(s - s.amax(-1, keepdim=True).clamp_min(-1e300))
        total = w.sum(-1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
        # a value that no weight reaches takes no part, whatever it is
        seen = ~hidden
        vv = torch.where(seen.any(0)[:, None, None], v, torch.zeros_like(v))
        if not torch.isfinite(vv).all():
            for t in range(b - a):
                m = seen[t]
                o[a + t] = torch.einsum("hj,jhd->hd", w[:, t, m], v[m])
                A[a + t] = torch.einsum("hj,jhd->hd", w[:, t, m], v[m].abs())
        else:
            o[a:b] = torch.einsum("htj,jhd->thd", w, vv)
            A[a:b] = torch.einsum("htj,jhd->thd", w, vv.abs())
        sub[a:b] = kv[i] * 2.0 ** -25 * vv.nan_to_num(0, 0, 0).abs().amax()
        lse[a:b] = torch.logsumexp(s, -1).T
    return o, A, lse, sub


def check(out, lse, ref, dt):
    o, A, want_lse, sub = ref
    tol = U[dt] * (o.abs() + A) + 2.0 ** -12 * A
    if dt == torch.float16:
        tol = tol + sub + 2.0 ** -25
    err = (out.double() - o).abs()
    fine = torch.isfinite(o)
    assert torch.equal(fine, torch.isfinite(out))
    bad = (err > tol) & fine
    assert not bad.any(), (int(bad.sum()), float(err[fine].max()), bad.nonzero()[:4].tolist())
    if lse is not None:
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isneginf(lse), empty)
        d = (lse.double() - want_lse).abs()[~empty]
        assert not d.numel() or bool((d <= 2.0 ** -12 + 2.0 ** -21 * want_lse[~empty].abs()).all()), float(d.max())


def garbage_beyond(pool, layer, n_layers, kv, page_off, table, P):
    """NaN and infinities in the slots behind every sequence's last token, and in unused pages."""
    used = np.zeros(pool.shape[1], bool)
    used[table] = True
    for half in (layer, n_layers + layer):
        pool[half, torch.tensor(np.flatnonzero(~used), device=DEV)] = math.nan
        for i, n in enumerate(kv):
            if n % P:
                pool[half, int(table[page_off[i + 1] - 1]), n % P:] = math.inf if i % 2 else math.nan


CASES = [
    # dtype, D, P, hq, hkv, new, history
    (torch.bfloat16, 128, 16, 32, 8, [1] * 8, [0, 1, 14, 15, 16, 63, 64, 1000]),
    (torch.float16, 128, 64, 28, 4, [1] * 6, [62, 63, 64, 127, 128, 5000]),
    (torch.bfloat16, 64, 16, 4, 4, [1, 2, 3, 16, 17], [0, 3, 500, 40, 99]),
    (torch.float16, 64, 16, 40, 8, [1, 3, 1, 4], [0, 700, 33, 20]),
    (torch.bfloat16, 96, 5, 6, 2, [1, 5, 6, 0, 20], [9, 0, 33, 44, 3]),
    (torch.bfloat16, 256, 16, 8, 2, [1, 4, 90], [300, 0, 50]),
    (torch.float16, 256, 32, 16, 1, [1, 1, 33], [300, 0, 130]),
    (torch.float16, 200, 16, 3, 3, [1, 40], [100, 100]),
    (torch.bfloat16, 8, 16, 5, 1, [1, 9], [100, 0]),
    (torch.bfloat16, 128, 1, 8, 8, [1, 30], [70, 3]),
    (torch.bfloat16, 128, 16, 16, 1, [1, 1], [3000, 17]),            # 16 heads on one
    (torch.float16, 128, 16, 20, 1, [1, 2], [300, 17]),              # 20 heads on one
    (torch.bfloat16, 128, 16, 64, 1, [1, 2, 70], [300, 17, 1]),      # 64 heads on one
    (torch.bfloat16, 128, 16, 32, 8, [65, 1, 128, 129, 2], [0, 900, 31, 300, 64]),
    (torch.float16, 128, 16, 16, 16, [200, 257], [0, 1]),
    (torch.bfloat16, 128, 16, 56, 8, [37, 300], [64, 700]),          # 7 heads on one
    (torch.float16, 64, 64, 8, 2, [512, 31], [0, 2000]),
    (torch.bfloat16, 128, 24, 8, 2, [100], [4000]),
    (torch.bfloat16, 64, 16, 64, 4, [33, 1], [9, 5]),
    (torch.bfloat16, 128, 16, 4, 1, [1], [40000]),                   # one row tile, many parts
    (torch.float16, 128, 16, 8, 1, [40], [20000]),
    # every CTA goes through many items, of either kernel
    (torch.bfloat16, 128, 16, 8, 2, [1, 33, 70, 2, 150, 0, 4, 5] * 40, [300, 0, 90, 1000, 40, 7, 16, 31] * 40),
]


def setup(case, seed=0, n_layers=2):
    dt, D, P, hq, hkv, new, hist = case
    kv = [a + b for a, b in zip(new, hist)]
    seqs, new_off, page_off, table, num = batch(new, kv, P, seed)
    g = torch.Generator(device=DEV).manual_seed(seed + 11)
    pool = torch.randn(2 * n_layers, num, P, hkv, D, generator=g, device=DEV).to(dt)
    q = (2 * torch.randn(int(new_off[-1]), hq, D, generator=g, device=DEV)).to(dt)
    geom = lsmkv.Geom(n_layers, hkv, D, page_tokens=P, chunk_tokens=P)
    return geom, pool, q, seqs, new_off, kv, page_off, table


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attend_equals_softmax_attention(case):
    dt, D, P = case[:3]
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case)
    layer = 1
    garbage_beyond(pool, layer, 2, kv, page_off, table, P)
    scale = D ** -0.5
    out = torch.full_like(q, 5.0)
    lse = torch.full(q.shape[:2], 5.0, device=DEV)
    ref = reference(q, pool, layer, 2, new_off, kv, page_off, table, P, scale)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.attend_batch(layer, seqs, q, out, pt, scale, lse)
        assert ctx.last_status()["flags"] == 0
        check(out, lse, ref, dt)
        # the same bits again, into the queries' own rows, and without the statistics
        same = q.clone()
        ctx.attend_batch(layer, seqs, same, same, pt, scale)
        assert ctx.last_status()["flags"] == 0
        assert torch.equal(same.view(torch.int16), out.view(torch.int16))


def test_padding_rows_and_empty_sequences_are_zero():
    case = (torch.bfloat16, 128, 16, 8, 2, [3, 1, 40, 2, 90], [0, 0, 0, 0, 0])
    dt, D, P, hq, hkv, new, _ = case
    kv = [1, 0, 7, 2, 0]                                   # fewer tokens than new ones, or none
    seqs, new_off, page_off, table, num = batch(new, kv, P)
    g = torch.Generator(device=DEV).manual_seed(1)
    pool = torch.randn(2, num, P, hkv, D, generator=g, device=DEV).to(dt)
    q = torch.randn(sum(new), hq, D, generator=g, device=DEV).to(dt)
    out, lse = torch.full_like(q, 3.0), torch.zeros(q.shape[:2], device=DEV)
    with lsmkv.Context(lsmkv.Geom(1, hkv, D, page_tokens=P, chunk_tokens=P), 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.1, lse)
        assert ctx.last_status()["flags"] == 0
    for i, (a, n) in enumerate(zip(new_off, new)):
        hidden = n - min(kv[i], n)
        assert not out[a:a + hidden].any() and torch.isneginf(lse[a:a + hidden]).all()
    check(out, lse, reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.1), dt)


@pytest.mark.parametrize("new", [3, 4, 70, 300])
def test_infinities_in_later_tokens_do_not_reach_earlier_rows(new):
    """Key and value of the last two new tokens hold infinities and NaN: rows before them must
    not notice, rows that see them must."""
    case = (torch.bfloat16, 128, 16, 8, 2, [new, 2], [50, 30])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    last = kv[0] - 1
    page = int(table[last // 16])
    pool[1, page, last % 16, :, 3] = math.inf
    pool[1, page, last % 16, :, 4] = math.nan
    prev = int(table[(last - 1) // 16])
    pool[0, prev, (last - 1) % 16, 0, 7] = math.nan
    out = torch.zeros_like(q)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08)
    o, A, lse, sub = ref
    assert torch.isfinite(out[:new - 2]).all() and torch.isfinite(out[new:]).all()
    check(out[:new - 2], None, (o[:new - 2], A[:new - 2], lse, sub[:new - 2]), torch.bfloat16)
    assert torch.isnan(out[new - 1, :4]).all()                      # the undefined key
    assert torch.isinf(out[new - 1, 4:, 3]).all() and torch.isnan(out[new - 1, 4:, 4]).all()


def test_strided_rows_large_scores_and_streams():
    """q and out are slices of wider buffers; scores of thousands; launched on a side stream."""
    case = (torch.float16, 64, 16, 8, 4, [1, 50], [200, 100])
    geom, pool, q0, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    n = q0.shape[0]
    wide = torch.full((n, 20, 80), 9.0, dtype=torch.float16, device=DEV)
    wide[:, 2:10, 8:72] = q0
    dst = torch.full((8, n, 72), 4.0, dtype=torch.float16, device=DEV)
    q, out = wide[:, 2:10, 8:72], dst.transpose(0, 1)[..., :64]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.125)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            ctx.attend_batch(0, seqs, q, out, pt, 0.125, stream=s)
        s.synchronize()
        check(out, None, ref, torch.float16)
        assert (dst[..., 64:] == 4.0).all()
        # one key takes all the weight: the result is its value, whatever the scores' size
        ctx.attend_batch(0, seqs, q, out, pt, 500.0, stream=0)
        torch.cuda.synchronize()
    far = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 500.0)[0]
    near = (out.double() - far).abs().amax(-1) <= 2.0 ** -9 * far.abs().amax(-1)
    assert near.double().mean() > 0.98        # ties within the scores' own rounding aside
    assert torch.isfinite(out).all()


def test_offsets_beyond_32_bits():
    """Pages at the far end of a buffer of more than 2^32 elements; K and V in one buffer."""
    D, P, hkv, hq = 128, 16, 8, 16
    num = 2 ** 32 // (P * hkv * D) + 40
    pool = torch.zeros(1, num, P, hkv, D, dtype=torch.bfloat16, device=DEV)
    new, kv = [1, 40], [100, 300]
    seqs, new_off, page_off, table, small = batch(new, kv, P)
    table = table + (num - small)
    seqs.keep[3].copy_(torch.tensor(table, dtype=torch.int32))
    pool[0, num - small:] = torch.randn(small, P, hkv, D, device=DEV).to(torch.bfloat16)
    q = torch.randn(41, hq, D, device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(q)
    both = pool.expand(2, -1, -1, -1, -1)
    with lsmkv.Context(lsmkv.Geom(1, hkv, D, page_tokens=P, chunk_tokens=P), 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table([pool[0], pool[0]]), 0.1)
        assert ctx.last_status()["flags"] == 0
    check(out, None, reference(q, both, 0, 1, new_off, kv, page_off, table, P, 0.1), torch.bfloat16)


def test_attend_reports_bad_sequences_and_pages():
    case = (torch.bfloat16, 128, 16, 8, 2, [1, 1, 1, 60], [40, 50, 60, 3])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    scale = 0.1
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        # pages as zeros: the same as a page of zeros in the pool
        zero = pool.clone()
        zero[:, int(table[page_off[1] + 1])] = 0
        seqs.keep[3][int(page_off[1]) + 1] = pool.shape[1]
        out = torch.zeros_like(q)
        ctx.attend_batch(0, seqs, q, out, pt, scale)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_PAGE and st["first_bad"] == int(page_off[1]) + 1
        check(out, None, reference(q, zero, 0, 1, new_off, kv, page_off, table, 16, scale), torch.bfloat16)
        seqs.keep[3][int(page_off[1]) + 1] = int(table[page_off[1] + 1])
        # more tokens than pages: that sequence is left out, the others are not
        seqs.keep[1][2] = 500
        out = torch.full_like(q, 8.0)
        ctx.attend_batch(0, seqs, q, out, pt, scale)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 2
        assert (out[2] == 8.0).all()
        seqs.keep[1][2] = kv[2]
        ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, scale)
        ok = torch.tensor([r for r in range(len(q)) if r != 2], device=DEV)
        check(out[ok], None, tuple(x[ok] for x in ref), torch.bfloat16)
        # a bound of new tokens that one sequence breaks
        few = lsmkv.Seqs(*seqs.keep, q.shape[0], 59)
        out = torch.full_like(q, 8.0)
        ctx.attend_batch(0, few, q, out, pt, scale)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 3
        assert (out[3:] == 8.0).all()
        check(out[:3], None, tuple(x[:3] for x in ref), torch.bfloat16)
        off = torch.tensor([pool[0].data_ptr() + 2, pool[1].data_ptr()], device=DEV)
        out.fill_(8.0)
        ctx.attend_batch(0, seqs, q, out, (off, pool.shape[1] - 1), scale)
        assert ctx.last_status()["flags"] == lsmkv.ST_MISALIGNED and (out == 8.0).all()


def test_attend_refusals():
    case = (torch.bfloat16, 64, 16, 4, 2, [2], [3])
    geom, pool, q, seqs, *_ = setup(case, n_layers=1)
    pt = lsmkv.pool_table(list(pool))
    groups = lsmkv.Groups(torch.tensor([0, 1], dtype=torch.int32, device=DEV),
                          torch.zeros(1, dtype=torch.int32, device=DEV))
    two = lsmkv.Groups(torch.tensor([0, 1, 1], dtype=torch.int32, device=DEV),
                       torch.zeros(2, dtype=torch.int32, device=DEV))
    out = torch.zeros_like(q)
    flat = torch.zeros(q.numel() + 8, dtype=q.dtype, device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        for kw in (dict(layer=1), dict(scale=math.inf), dict(scale=math.nan), dict(q=q[:, :3], out=out[:, :3]),
                   dict(out=flat[1:1 + q.numel()].view(q.shape)), dict(pool=(0, 4))):
            a = dict(layer=0, q=q, out=out, pool=pt, scale=0.1) | kw
            for call in (lambda: ctx.attend_batch(a["layer"], seqs, a["q"], a["out"], a["pool"], a["scale"]),
                         lambda: ctx.attend_shared_batch(a["layer"], seqs, groups, a["q"], a["out"],
                                                         a["pool"], a["scale"])):
                with pytest.raises(lsmkv.LsmkvError) as e:
                    call()
                assert e.value.code == lsmkv.EINVAL
        with pytest.raises(lsmkv.LsmkvError):
            ctx.attend_shared_batch(0, seqs, two, q, out, pt, 0.1)             # more groups than sequences
        for a, b, c in ((q, out.half(), None), (q.float(), out.float(), None), (q[:1], out, None),
                        (q, out[:, :2], None), (q, out, torch.zeros(3, device=DEV))):
            with pytest.raises((TypeError, ValueError)):
                ctx.attend_batch(0, seqs, a, b, pt, 0.1, c)
        ctx.attend_batch(0, lsmkv.Seqs(*seqs.keep, 0, 1), q[:0], out[:0], pt, 0.1)
        assert ctx.last_status()["flags"] == 0 and not out.any()


SHARED = [
    # dtype, D, P, hq, hkv, members of every group, shared pages, new tokens a member, own tokens
    (torch.bfloat16, 128, 16, 32, 8, [8], [64], 1, (0, 40)),
    (torch.bfloat16, 128, 16, 32, 8, [1, 2, 3, 40], [5, 1, 0, 30], 1, (0, 100)),
    (torch.float16, 128, 64, 28, 4, [5, 9], [3, 20], 1, (0, 300)),
    (torch.float16, 64, 16, 8, 8, [3, 20, 70], [2, 7, 100], 1, (0, 50)),
    (torch.bfloat16, 128, 16, 16, 2, [6, 4], [9, 4], 5, (0, 30)),
    (torch.bfloat16, 96, 16, 8, 2, [2, 7], [33, 5], 40, (0, 30)),
    (torch.bfloat16, 256, 16, 8, 2, [4, 7], [10, 3], 1, (0, 30)),
    (torch.bfloat16, 128, 16, 64, 8, [33], [700], 1, (0, 200)),
    (torch.bfloat16, 128, 16, 8, 8, [2, 0, 2], [3, 9, 1], 2, (0, 9)),
]


def shared_batch(case, seed=0):
    dt, D, P, hq, hkv, members, pages, new, own = case
    rng = np.random.default_rng(seed)
    shared = np.repeat(pages, members)
    n = len(shared)
    kv = [int(s) * P + new + int(rng.integers(own[0], own[1] + 1)) for s in shared]
    seqs, new_off, page_off, table, num = batch([new] * n, kv, P, seed)
    off = np.cumsum([0] + members)
    for g, (a, b) in enumerate(zip(off, off[1:])):
        for i in range(a + 1, b):
            table[page_off[i]:page_off[i] + pages[g]] = table[page_off[a]:page_off[a] + pages[g]]
    seqs.keep[3].copy_(torch.tensor(table, dtype=torch.int32))
    gen = torch.Generator(device=DEV).manual_seed(seed + 5)
    pool = torch.randn(2, num, P, hkv, D, generator=gen, device=DEV).to(dt)
    q = (2 * torch.randn(n * new, hq, D, generator=gen, device=DEV)).to(dt)
    t = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)  # noqa: E731
    return (lsmkv.Geom(1, hkv, D, page_tokens=P, chunk_tokens=P), pool, q, seqs,
            lsmkv.Groups(t(off), t(pages)), new_off, kv, page_off, table)


@pytest.mark.parametrize("case", SHARED, ids=[str(i) for i in range(len(SHARED))])
def test_shared_prefixes_give_the_same_attention(case):
    dt, D, P = case[:3]
    geom, pool, q, seqs, groups, new_off, kv, page_off, table = shared_batch(case)
    garbage_beyond(pool, 0, 1, kv, page_off, table, P)
    scale = D ** -0.5
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, P, scale)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.attend_shared_batch(0, seqs, groups, q, out, pt, scale, lse)
        assert ctx.last_status()["flags"] == 0
        check(out, lse, ref, dt)
        again = torch.zeros_like(out)
        ctx.attend_shared_batch(0, seqs, groups, q, again, pt, scale)
        assert torch.equal(again.view(torch.int16), out.view(torch.int16))


def test_members_that_do_not_reach_behind_the_common_pages_go_by_themselves():
    """Claimed common pages beyond some members' histories, padding members, and a first member
    with too few pages: same attention for everybody."""
    dt, D, P, hq, hkv = torch.bfloat16, 128, 16, 8, 2
    new = [1, 3, 1, 1, 1, 1, 1]
    kv = [70, 66, 64, 0, 80, 20, 90]                       # groups 0-4 (4 pages) and 5-6 (3 pages)
    seqs, new_off, page_off, table, num = batch(new, kv, P)
    for i in (1, 2, 4):
        k = min(4, -(-kv[i] // P))
        table[page_off[i]:page_off[i] + k] = table[:k]
    seqs.keep[3].copy_(torch.tensor(table, dtype=torch.int32))
    gen = torch.Generator(device=DEV).manual_seed(2)
    pool = torch.randn(2, num, P, hkv, D, generator=gen, device=DEV).to(dt)
    q = torch.randn(sum(new), hq, D, generator=gen, device=DEV).to(dt)
    t = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    groups = lsmkv.Groups(t([0, 5, 7]), t([4, 3]))
    out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device=DEV)
    with lsmkv.Context(lsmkv.Geom(1, hkv, D, page_tokens=P, chunk_tokens=P), 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.attend_shared_batch(0, seqs, groups, q, out, pt, 0.1, lse)
        assert ctx.last_status()["flags"] == 0
        check(out, lse, reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.1), dt)
        ctx.attend_shared_batch(0, seqs, lsmkv.Groups(t([0, 5, 6]), t([4, 3])), q, out, pt, 0.1)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 2
        ctx.attend_shared_batch(0, seqs, lsmkv.Groups(t([0, 8, 7]), t([4, 3])), q, out, pt, 0.1)
        st = ctx.last_status()
        assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 0


def test_a_wait_that_runs_out_is_reported_and_the_context_stays_usable():
    """The many-row kernel with one of its tiles never handed over (the library's test hook) and
    the limit at about a millisecond: every role leaves, the call reports it, and the next call
    of the same context is right."""
    case = (torch.bfloat16, 128, 16, 8, 2, [70, 300], [900, 2000])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    out = torch.zeros_like(q)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.set_tuning("wait_cycles", 2_000_000)
        ctx.set_tuning("test_drop_piece", 3)
        ctx.attend_batch(0, seqs, q, out, pt, 0.08)
        assert ctx.last_status()["flags"] == lsmkv.ST_WAIT_EXPIRED
        ctx.set_tuning("test_drop_piece", -1)
        ctx.set_tuning("wait_cycles", 2_000_000_000)
        ctx.attend_batch(0, seqs, q, out, pt, 0.08)
        assert ctx.last_status()["flags"] == 0
        assert ctx.last_cuda_error() == 0
    check(out, None, reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08), torch.bfloat16)


@pytest.mark.parametrize("case", [
    # more row tiles than CTAs over more keys than the L2 keeps: whole tiles in waves, then spans
    (torch.bfloat16, 128, 16, 64, 8, [600, 333, 20, 1], [9000, 9500, 12000, 500]),
    (torch.float16, 64, 64, 32, 16, [900, 700], [20000, 30000]),
], ids=["128", "64"])
def test_whole_tiles_in_waves(case):
    dt, D, P = case[:3]
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    garbage_beyond(pool, 0, 1, kv, page_off, table, P)
    out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device=DEV)
    assert sum(kv) * pool.shape[3] * D * 4 > 64 << 20
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.attend_batch(0, seqs, q, out, pt, D ** -0.5, lse)
        assert ctx.last_status()["flags"] == 0
        again = torch.zeros_like(out)
        ctx.attend_batch(0, seqs, q, again, pt, D ** -0.5)
        assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    hq, G = q.shape[1], q.shape[1] // pool.shape[3]
    for h in range(pool.shape[3]):                            # head by head: the reference is large
        heads = slice(h * G, (h + 1) * G)
        ref = reference(q[:, heads], pool[:, :, :, h:h + 1], 0, 1, new_off, kv, page_off, table, P, D ** -0.5)
        check(out[:, heads], lse[:, heads], ref, dt)
        torch.cuda.empty_cache()


def test_calls_in_a_cuda_graph_and_one_after_another():
    """Captured and replayed with other inputs; two calls back to back share the scratch."""
    case = (torch.bfloat16, 128, 16, 16, 4, [1, 3, 40, 1], [30, 200, 500, 4000])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    out, out2 = torch.zeros_like(q), torch.zeros_like(q)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.attend_batch(0, seqs, q, out, pt, 0.08)            # scratch is there before the capture
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.attend_batch(0, seqs, q, out, pt, 0.08)
            ctx.attend_batch(0, seqs, out, out2, pt, 0.08)
        q.copy_(torch.randn_like(q))
        pool.copy_(torch.randn_like(pool))
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert ctx.last_status()["flags"] == 0
        del graph
    check(out, None, reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08), torch.bfloat16)
    check(out2, None, reference(out, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08), torch.bfloat16)


def test_negative_and_zero_scale():
    case = (torch.float16, 64, 16, 8, 2, [1, 50], [70, 300])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    with lsmkv.Context(geom, 0) as ctx:
        for scale in (-0.125, 0.0):
            out = torch.zeros_like(q)
            ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), scale)
            assert ctx.last_status()["flags"] == 0
            check(out, None, reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, scale), torch.float16)


@pytest.mark.parametrize("new,history,D", [(3, 50, 128), (70, 50, 128), (300, 4000, 64), (20, 9000, 128), (40, 30, 256)])
def test_infinities_and_output_in_the_queries_own_rows(new, history, D):
    """Undefined values in the last token, output written over the queries: the rows before it are
    what they are without, whole tiles and cut ones."""
    case = (torch.bfloat16, D, 16, 8, 2, [new, 2], [history, 30])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    last = kv[0] - 1
    pool[1, int(table[last // 16]), last % 16] = math.nan
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_batch(0, seqs, q, q, lsmkv.pool_table(list(pool)), 0.08)
        assert ctx.last_status()["flags"] == 0
    keep = [r for r in range(new + 2) if r != new - 1]
    assert torch.isfinite(q[keep]).all() and torch.isnan(q[new - 1]).all()
    check(q[keep], None, (ref[0][keep], ref[1][keep], None, ref[3][keep]), torch.bfloat16)


def test_shared_attend_leaves_out_a_first_member_with_descending_page_offsets():
    """The group shares nothing then and its other members go by themselves. (The table goes on far
    behind the entries that the first member would claim, so that no reading of it leaves it.)"""
    case = (torch.bfloat16, 128, 16, 8, 2, [4, 3], [2, 5], 1, (0, 30))
    geom, pool, q, seqs, groups, new_off, kv, page_off, table = shared_batch(case)
    # sequence 0 now begins behind everything and ends where it did; its claimed pages are no pages
    end = len(table)
    wide = torch.full((end + 64,), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    wide[:end] = seqs.keep[3]
    off = seqs.keep[2].clone()
    off[0] = end
    bad = lsmkv.Seqs(seqs.keep[0], seqs.keep[1], off, wide, seqs.n_new, seqs.max_new)
    out = torch.full_like(q, 5.0)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_shared_batch(0, bad, groups, q, out, lsmkv.pool_table(list(pool)), 0.08)
        st = ctx.last_status()
    assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 0
    assert (out[0] == 5.0).all()
    check(out[1:], None, tuple(x[1:] for x in ref), torch.bfloat16)


def test_shared_attend_names_the_sequence_that_breaks_the_rules():
    """A bad offset between two groups: the item is the first of the two sequences, not a group."""
    case = (torch.bfloat16, 128, 16, 8, 2, [4, 3], [2, 2], 1, (0, 30))
    geom, pool, q, seqs, groups, new_off, kv, page_off, table = shared_batch(case)
    seqs.keep[0][4] = 9999
    out = torch.full_like(q, 5.0)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_shared_batch(0, seqs, groups, q, out, lsmkv.pool_table(list(pool)), 0.08)
        st = ctx.last_status()
    assert st["flags"] == lsmkv.ST_BAD_COUNT and st["first_bad"] == 3
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08)
    ok = torch.tensor([0, 1, 2, 5, 6], device=DEV)
    check(out[ok], None, tuple(x[ok] for x in ref), torch.bfloat16)
    assert (out[3:5] == 5.0).all()


def test_graphs_captured_before_a_larger_call_stay_valid():
    """Small shared and plain steps (one with its output over the queries) are captured, then larger
    batches run, twice as large each time, then the small graphs again over other inputs."""
    small = (torch.bfloat16, 128, 16, 8, 2, [3, 5], [4, 9], 1, (0, 40))
    geom, pool, q, seqs, groups, new_off, kv, page_off, table = shared_batch(small)
    plain = (torch.bfloat16, 128, 16, 8, 2, [40, 1, 70], [100, 30, 0])
    _, pool2, q2, seqs2, new_off2, kv2, page_off2, table2 = setup(plain, n_layers=1)
    out, out2, over = torch.zeros_like(q), torch.zeros_like(q2), q2.clone()
    with lsmkv.Context(geom, 0) as ctx:
        pt, pt2 = lsmkv.pool_table(list(pool)), lsmkv.pool_table(list(pool2))

        def steps():
            ctx.attend_shared_batch(0, seqs, groups, q, out, pt, 0.08)
            ctx.attend_batch(0, seqs2, q2, out2, pt2, 0.08)
            ctx.attend_batch(0, seqs2, over, over, pt2, 0.08)

        steps()                                            # scratch is there before the capture
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            steps()
        for k in range(1, 6):
            large = (torch.bfloat16, 128, 16, 8, 2, [2 ** k * 400, 30], [4, 9], 1, (0, 40))
            _, lpool, lq, lseqs, lgroups, lnew, lkv, lpage, ltable = shared_batch(large, seed=k)
            lout = torch.zeros_like(lq)
            ctx.attend_shared_batch(0, lseqs, lgroups, lq, lout, lsmkv.pool_table(list(lpool)), 0.08)
            wide = (torch.bfloat16, 128, 16, 8, 2, [2 ** k * 100] * 3, [0, 10, 200])
            _, wpool, wq, wseqs, *_ = setup(wide, n_layers=1)
            ctx.attend_batch(0, wseqs, wq, wq, lsmkv.pool_table(list(wpool)), 0.08)
            assert ctx.last_status()["flags"] == 0
        check(lout, None, reference(lq, lpool, 0, 1, lnew, lkv, lpage, ltable, 16, 0.08), torch.bfloat16)
        for x in (q, q2, pool, pool2):
            x.copy_(torch.randn_like(x))
        over.copy_(q2)
        junk = torch.full((64 << 20,), 0xFF, dtype=torch.uint8, device=DEV)    # over memory freed since
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.last_status()["flags"] == 0 and ctx.last_cuda_error() == 0
        del graph, junk
    check(out, None, reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08), torch.bfloat16)
    ref = reference(q2, pool2, 0, 1, new_off2, kv2, page_off2, table2, 16, 0.08)
    check(out2, None, ref, torch.bfloat16)
    check(over, None, ref, torch.bfloat16)


def test_batches_of_more_rows_than_32_bits_number_are_refused():
    """Before anything is launched (rows that repeat one token stand in for memory)."""
    geom = lsmkv.Geom(1, 2, 64, page_tokens=16, chunk_tokens=16)
    case = (torch.bfloat16, 64, 16, 8, 2, [2], [3])
    _, pool, q, seqs, *_ = setup(case, n_layers=1)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        for n in (2 ** 31, 2 ** 30 - 63):
            many = lsmkv.Seqs(*seqs.keep, n, 1)
            rows = q[:1].expand(n, -1, -1)
            with pytest.raises(lsmkv.LsmkvError) as e:
                ctx.attend_batch(0, many, rows, rows, pt, 0.1)
            assert e.value.code == lsmkv.EINVAL


def test_one_token_out_of_a_row_of_any_width():
    """A lone new token whose row has an odd number of elements: the stride is never taken."""
    case = (torch.bfloat16, 64, 16, 8, 2, [1], [100])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    wide = torch.zeros(1, 8 * 64 + 5, dtype=q.dtype, device=DEV)
    wide[:, :512] = q.flatten(1)
    odd, out = wide.as_strided((1, 8, 64), (517, 64, 1)), torch.zeros_like(q)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_batch(0, seqs, odd, out, lsmkv.pool_table(list(pool)), 0.1)
        assert ctx.last_status()["flags"] == 0
    check(out, None, reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.1), torch.bfloat16)


@pytest.mark.parametrize("new", [[1] * 3000, [2, 1, 4, 3] * 300, [70, 1, 200] * 20], ids=["one", "few", "many"])
def test_output_over_the_queries_in_another_layout(new):
    """The queries are every second row of a buffer (and the other way round), the output its first rows;
    output beside the queries in the tokens of one buffer; output over the queries a few tokens on."""
    case = (torch.bfloat16, 128, 16, 8, 2, new, [40] * len(new))
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    n, hq, D = q.shape
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08)
    flat = torch.zeros(2 * n + 3, hq, D, dtype=q.dtype, device=DEV)
    pair = flat[:2 * n].view(n, 2 * hq, D)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        for src, dst in ((flat[:2 * n:2], flat[:n]), (flat[:n], flat[1:2 * n:2]), (pair[:, :hq], pair[:, hq:]),
                         (pair[:, hq:], pair[:, :hq]), (flat[:n], flat[3:n + 3]), (flat[2:n + 2], flat[:n]),
                         (flat[:n].flip(0).contiguous(), flat[:n])):
            src.copy_(q)
            ctx.attend_batch(0, seqs, src, dst, pt, 0.08)
            assert ctx.last_status()["flags"] == 0
            check(dst, None, ref, torch.bfloat16)
