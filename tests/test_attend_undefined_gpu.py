"""Undefined queries, keys and values: the rows that see them come out undefined, and no others,
however a row tile is cut among the CTAs, whatever an earlier kernel left behind, and at a cost
that stays near a clean call's.

Tolerances are those of test_attend_gpu.py."""
import math

import pytest
import torch

from paper_2511_16138_b200 import lsmkv
from test_append_gpu import DEV
from test_attend_gpu import check, garbage_beyond, reference, setup, shared_batch

pytestmark = pytest.mark.gpu


def undefined_exactly(out, lse, ref, lost, dt):
    """Rows (token, head) of `lost` are NaN in every element and in lse, all others as in ref."""
    assert torch.isnan(out[lost]).all() and torch.isnan(lse[lost]).all()
    o, A, want_lse, sub = ref
    check(out[~lost], lse[~lost], (o[~lost], A[~lost], want_lse[~lost], sub[~lost]), dt)


QUERIES = [
    # dtype, D, P, hq, hkv, new, history
    (torch.bfloat16, 128, 16, 32, 8, [1] * 8, [1000, 300, 40, 0, 2000, 700, 128, 129]),   # cut tiles
    (torch.float16, 64, 16, 8, 8, [1] * 200, [5, 20, 130, 0] * 50),                       # mostly whole
    (torch.bfloat16, 256, 16, 8, 2, [1, 2, 1], [900, 300, 20]),
    (torch.bfloat16, 128, 16, 8, 2, [3, 2, 4], [1500, 40, 700]),                          # several tokens
    (torch.bfloat16, 128, 16, 8, 2, [70, 300], [900, 2000]),                              # many rows, cut
    (torch.float16, 64, 16, 16, 16, [200, 257] * 12, [0, 1] * 12),                        # many rows, whole
    (torch.bfloat16, 96, 5, 6, 2, [90], [400]),
]


@pytest.mark.parametrize("case", QUERIES, ids=[str(i) for i in range(len(QUERIES))])
def test_undefined_queries_give_undefined_rows(case):
    dt, D, P, hq = case[:4]
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    lost = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    lost.view(-1)[1::3] = True
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.08)
    q[lost] = math.nan
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08, lse)
        assert ctx.last_status()["flags"] == 0
    undefined_exactly(out, lse, ref, lost, dt)


# The key is alone in its tile of 128 keys for the rows that see no later one. 59 sequences of two KV
# heads and nine key tiles: spans of 148 CTAs begin right before the ninth tile in every fourth.
KEYS = [
    (torch.bfloat16, 128, 16, 8, 2, [1] * 59, [1024] * 59, 1024),
    (torch.float16, 64, 16, 4, 2, [1] * 59, [1024] * 59, 1024),
    (torch.bfloat16, 128, 16, 8, 2, [3] * 59, [1023] * 59, 1024),
    (torch.bfloat16, 128, 16, 8, 2, [40] * 59, [1004] * 59, 1024),
    (torch.float16, 64, 16, 8, 2, [150] * 40, [1004] * 40, 1024),
]


@pytest.mark.parametrize("case", KEYS, ids=[str(i) for i in range(len(KEYS))])
def test_a_lone_undefined_key_reaches_the_rows_that_see_it(case):
    dt, D, P, hq, hkv, new, hist, key = case
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case[:7], n_layers=1)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.08)
    lost = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    for i in range(len(new)):
        pool[0, int(table[page_off[i] + key // P]), key % P] = math.nan
        lost[new_off[i] + max(0, key - hist[i]):new_off[i + 1]] = True
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08, lse)
        assert ctx.last_status()["flags"] == 0
    undefined_exactly(out, lse, ref, lost, dt)


PREFIXES = [
    # as SHARED of test_attend_gpu.py: 65 common pages are eight key tiles and 16 keys
    (torch.bfloat16, 128, 16, 32, 8, [8], [65], 1, (0, 40)),                # few rows
    (torch.bfloat16, 128, 16, 8, 2, [2] * 59, [65] * 59, 1, (0, 40)),       # many rows
    (torch.float16, 64, 16, 8, 2, [2] * 59, [65] * 59, 3, (0, 300)),
]


@pytest.mark.parametrize("what", ["queries", "keys"])
@pytest.mark.parametrize("case", PREFIXES, ids=[str(i) for i in range(len(PREFIXES))])
def test_undefined_rows_over_shared_prefixes(case, what):
    dt, D, P = case[:3]
    geom, pool, q, seqs, groups, new_off, kv, page_off, table = shared_batch(case)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.08)
    lost = torch.zeros(q.shape[:2], dtype=torch.bool, device=DEV)
    if what == "queries":
        lost.view(-1)[1::3] = True
        q[lost] = math.nan
    else:
        members, pages = case[5], case[6]
        first = 0
        for g, n in enumerate(members):
            if g % 3 != 1:                                  # the last common page of the group
                pool[0, int(table[page_off[first] + pages[g] - 1])] = math.nan
                lost[new_off[first]:new_off[first + n]] = True
            first += n
    out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.attend_shared_batch(0, seqs, groups, q, out, lsmkv.pool_table(list(pool)), 0.08, lse)
        assert ctx.last_status()["flags"] == 0
    undefined_exactly(out, lse, ref, lost, dt)


@pytest.mark.parametrize("D", [80, 96])
def test_what_an_earlier_kernel_left_on_chip_does_not_matter(D):
    """A call whose sums are all NaN, then one with narrower heads over long histories, every wait
    limited to about a millisecond: nothing of the first shows in the second, in time either."""
    case = (torch.bfloat16, 128, 16, 32, 8, [2048], [0])
    geom, pool, q, seqs, *_ = setup(case, n_layers=1)
    pool[1] = math.nan
    with lsmkv.Context(geom, 0) as ctx:
        out = torch.zeros_like(q)
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08)
        assert ctx.last_status()["flags"] == 0 and torch.isnan(out).all()
    case = (torch.bfloat16, D, 16, 8, 2, [100] * 100, [20000] + [900] * 99)
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.1)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.set_tuning("wait_cycles", 2_000_000)
        out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device=DEV)
        ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.1, lse)
        assert ctx.last_status()["flags"] == 0
    check(out, lse, ref, torch.bfloat16)


def device_ms(call):
    """Device time of a call, the least of five."""
    best = math.inf
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


LONG = [
    (torch.bfloat16, 128, 16, 64, 8, [1024], [30000]),              # whole tiles in waves, the rest cut
    (torch.float16, 64, 16, 16, 2, [40] * 3, [30000, 20000, 500]),  # cut tiles
    (torch.bfloat16, 128, 16, 8, 2, [4], [30000]),                  # few rows
    (torch.bfloat16, 256, 16, 8, 2, [4, 1, 12], [30000, 30, 700]),
]


@pytest.mark.parametrize("case", LONG, ids=[str(i) for i in range(len(LONG))])
def test_undefined_values_in_long_sequences(case):
    """A NaN value in the first token is every row's own, one in the last token the last row's alone;
    the batch ends in about the time of a clean one, with every wait limited to half a millisecond."""
    dt, D, P, hq, hkv, new, hist = case
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    scale = D ** -0.5
    n0 = new[0]
    # the last (up to) 64 rows of the first sequence, head by head: the reference is large
    tail = min(64, n0)

    def tail_reference(h):
        heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
        return heads, reference(q[n0 - tail:n0, heads], pool[:, :, :, h:h + 1], 0, 1, [0, tail], kv[:1], page_off,
                                table, P, scale)

    out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        ctx.set_tuning("wait_cycles", 1_000_000)
        pt = lsmkv.pool_table(list(pool))

        def call():
            ctx.attend_batch(0, seqs, q, out, pt, scale, lse)

        clean = device_ms(call)
        before = out.clone()
        assert ctx.last_status()["flags"] == 0
        # every row's own
        keep = pool[1, int(table[0]), 0].clone()
        pool[1, int(table[0]), 0] = math.nan
        own = device_ms(call)
        assert ctx.last_status()["flags"] == 0
        assert torch.isnan(out[:n0]).all() and torch.equal(out[n0:], before[n0:])
        assert own < 2 * clean + 0.2, (clean, own)
        pool[1, int(table[0]), 0] = keep
        # the last row's alone, in every second element
        last = kv[0] - 1
        pool[1, int(table[last // P]), last % P, :, ::2] = math.inf
        pool[1, int(table[last // P]), last % P, :, ::4] = math.nan
        hidden = device_ms(call)
        assert ctx.last_status()["flags"] == 0
        assert torch.equal(out[n0:], before[n0:])
        assert hidden < 4 * clean + 1.0, (clean, hidden)
        for h in {0, hkv // 2, hkv - 1}:
            heads, ref = tail_reference(h)
            check(out[n0 - tail:n0, heads], lse[n0 - tail:n0, heads], ref, dt)
        assert torch.isfinite(out[:n0 - 1]).all()


def test_undefined_values_behind_shared_prefixes():
    """Members with several new tokens, of few and of many rows; their own parts hold undefined values
    that only the last row of each sees, and so does what lies behind their last tokens."""
    for new in (3, 40):
        case = (torch.bfloat16, 128, 16, 16, 2, [6, 4], [9, 4], new, (0, 30))
        geom, pool, q, seqs, groups, new_off, kv, page_off, table = shared_batch(case)
        garbage_beyond(pool, 0, 1, kv, page_off, table, 16)
        for i, n in enumerate(kv):
            pool[1, int(table[page_off[i] + (n - 1) // 16]), (n - 1) % 16, :, i % 5::7] = math.nan
        out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device=DEV)
        ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08)
        with lsmkv.Context(geom, 0) as ctx:
            ctx.attend_shared_batch(0, seqs, groups, q, out, lsmkv.pool_table(list(pool)), 0.08, lse)
            assert ctx.last_status()["flags"] == 0
        check(out, lse, ref, torch.bfloat16)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("new", [2, 5, 8, 16])
def test_every_row_of_a_small_tile_sees_its_own_values_alone(dt, new):
    """Each new token's value holds a NaN or an infinity in an element of its own: row t has the
    tokens' 0..t and no others, whole tiles and cut ones, one query head a KV head."""
    for hist in (0, 9, 3000):
        case = (dt, 128, 16, 2, 2, [new, 1], [hist, 5])
        geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
        for t in range(new):
            p = hist + t
            pool[1, int(table[p // 16]), p % 16, :, 3 * t] = math.nan
            pool[1, int(table[p // 16]), p % 16, :, 3 * t + 1] = math.inf
        out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device=DEV)
        ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, 16, 0.08)
        with lsmkv.Context(geom, 0) as ctx:
            ctx.attend_batch(0, seqs, q, out, lsmkv.pool_table(list(pool)), 0.08, lse)
            assert ctx.last_status()["flags"] == 0
        for t in range(new):
            assert torch.isnan(out[t, :, 0:3 * t + 1:3]).all()
            assert not torch.isnan(out[t, :, 3 * (t + 1):]).any()
        check(out, lse, ref, dt)


def test_a_batch_of_undefined_values_costs_little_more():
    """Every value of the first sequence is NaN: its rows are, the other's are not, in about a clean time."""
    case = (torch.bfloat16, 128, 16, 32, 8, [1000, 60], [9000, 500])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device=DEV)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))

        def call():
            ctx.attend_batch(0, seqs, q, out, pt, 0.08, lse)

        clean = device_ms(call)
        before, before_lse = out.clone(), lse.clone()
        pool[1, torch.tensor(table[:page_off[1]], device=DEV)] = math.nan
        undefined = device_ms(call)
        assert ctx.last_status()["flags"] == 0
    assert torch.isnan(out[:1000]).all() and torch.equal(out[1000:], before[1000:])
    assert torch.equal(lse, before_lse)
    assert undefined < 2 * clean + 0.2, (clean, undefined)


@pytest.mark.parametrize("group", [1, 4, 16, 20])
@pytest.mark.parametrize("D,P", [(128, 16), (64, 16), (96, 16), (128, 5), (40, 64)])
def test_every_row_of_a_large_tile_sees_its_own_values_alone(group, D, P):
    """As above with 40 new tokens a sequence, few and many query heads a KV head, short and long
    histories, the output over the queries too."""
    case = (torch.float16, D, P, 2 * group, 2, [40, 3, 40], [9, 200, 5000])
    geom, pool, q, seqs, new_off, kv, page_off, table = setup(case, n_layers=1)
    for i in (0, 2):
        for t in range(40):
            p = kv[i] - 40 + t
            pool[1, int(table[page_off[i] + p // P]), p % P, :, t % D] = math.nan
    out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device=DEV)
    ref = reference(q, pool, 0, 1, new_off, kv, page_off, table, P, 0.08)
    with lsmkv.Context(geom, 0) as ctx:
        pt = lsmkv.pool_table(list(pool))
        ctx.attend_batch(0, seqs, q, out, pt, 0.08, lse)
        assert ctx.last_status()["flags"] == 0
        over = q.clone()
        ctx.attend_batch(0, seqs, over, over, pt, 0.08)
        assert ctx.last_status()["flags"] == 0
    assert torch.equal(out.view(torch.int16), over.view(torch.int16))
    for t in range(40):
        for first in (0, 43):
            assert torch.isnan(out[first + t, :, :min(D, t + 1)]).all()
            assert not torch.isnan(out[first + t, :, t + 1:]).any()
    check(out, lse, ref, torch.float16)
